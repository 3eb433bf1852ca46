// Weight gradients of the experts on the tcgen05 tensor cores,
//   dW_e[m][n] = sum over the rows r of expert e of P[p_row(r)][m] Q[q_row(r)][n]
// (bf16 operands, fp32 accumulation, fp32 result).
//
// The contraction runs over the ragged rows, both operands being read as stored
// (MN-major).  A CTA pair (cta_group::2) owns a 256 x 256 tile of one expert's dW
// and walks the expert's rows in steps of 64; each CTA loads 128 columns of P and
// of Q: by TMA where the rows lie in dispatch order, and gathered in 16-byte pieces
// otherwise, so that neither the tokens nor the outputs' gradient is ever permuted
// in memory.  An expert's last, partial step is gathered on both sides: what lies
// past its end are zeros on both, whatever the next expert's rows hold.  Two accumulators in TMEM let one tile's 256 KB of fp32
// leave while the next tile's products run; an expert without rows gets zeros
// from the epilogue alone.  The result is stored (or added, once per entry) by
// TMA from 32 x 32 blocks.
//
// Warps: 0 TMA, 1 issues the MMAs (first CTA), 2-5 epilogue, 6-11 gather.
#include <cstdint>

#include "experts_mma.cuh"

namespace dol {
namespace {

constexpr int kEpiWarps = 4;
constexpr int kFirstLoader = 2 + kEpiWarps;
constexpr int kThreads = (kFirstLoader + kLoadWarps) * 32;
constexpr int kStep = 64;                       // rows of a step
constexpr uint32_t kBlockBytes = kStep * 128;   // 64 columns of a step
constexpr uint32_t kSide = 2 * kBlockBytes;     // a CTA's 128 columns of one operand
constexpr uint32_t kStage = 2 * kSide;
constexpr int kStages = 6;
constexpr uint32_t kOut = 32 * 128;             // an epilogue warp's 32 x 32 block
constexpr uint32_t kSmem = 1024 + kStages * kStage + kEpiWarps * kOut;
static_assert(kSmem <= 232448 - 2048, "shared memory");
static_assert(kStages >= kLoadWarps, "see kLoadWarps");

struct Tiles {
    const int *offsets;
    int m_tiles, n_tiles;
    int64_t R;
    __device__ void at(int t, int *e, int *m, int *n, int *r0, int *r1) const {
        const int per = m_tiles * n_tiles;
        *e = t / per;
        const int i = t - *e * per;
        *n = i / m_tiles;
        *m = i - *n * m_tiles;
        *r0 = max(0, min(__ldg(offsets + *e), (int)R));
        *r1 = max(*r0, min(__ldg(offsets + *e + 1), (int)R));
    }
};

// One operand as a gathering warp sees it.
struct Side {
    const bf16 *mat;
    const int *rows;
    int64_t count;
    int cols, x;      // columns, and this lane's first one
    uint32_t dst;     // its place in a stage for row lane / 16

    // the matrix rows of routed rows r + lane and r + 32 + lane; -1: none (zeros)
    __device__ int2 ids(int r, int end, int lane, int *status) const {
        int v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = r + 32 * j + lane;
            v[j] = i < end ? (rows ? __ldg(rows + i) : i) : -1;
        }
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool out = v[j] < 0 || v[j] >= count;
            bad |= out && r + 32 * j + lane < end;
            if (out) v[j] = -1;
        }
        if (bad && status) atomicOr(status, kDevBadId);
        return make_int2(v[0], v[1]);
    }
    // Sixteen lanes copy a row's 256 bytes, two rows at a time.
    __device__ void copy(uint32_t stage, int2 id, int lane) const {
        const int row = lane >> 4, piece = lane & 7;
        const bf16 *from = mat + x;
        const bool inside = x < cols;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const int src = __shfl_sync(kFull, j < 16 ? id.x : id.y, (2 * j + row) & 31);
            const bool in = inside && src >= 0;
            cp_async16(stage + dst + j * 256 + ((piece ^ ((2 * j + row) & 7)) << 4),
                       in ? from + (int64_t)src * cols : mat, in);
        }
    }
};

// 128 columns from x on of 64 rows from r on, by TMA.
__device__ __forceinline__ void load_side(unsigned char *dst, const CUtensorMap *map, int cols, int x, int r,
                                          uint32_t bar) {
    if (cols % 64 == 0) {
        pair_load_4d(dst, map, 0, r, x / 64, 0, bar);
    } else {
        pair_load_3d(dst, map, x, r, 0, bar);
        pair_load_3d(dst + kBlockBytes, map, x + 64, r, 0, bar);
    }
}

bool encode_side(CUtensorMap *map, const bf16 *base, int64_t rows, int cols) {
    return cols % 64 == 0 ? encode_mn_pair_map(map, base, 1, (uint64_t)rows, (uint64_t)cols)
                          : encode_tensor_map_3d_bf16(map, base, 1, (uint64_t)rows, (uint64_t)cols, 64, kStep);
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
weight_grad_kernel(const __grid_constant__ CUtensorMap pmap, const __grid_constant__ CUtensorMap qmap,
                   const __grid_constant__ CUtensorMap omap, const WeightGradArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_align<1024>(smem_raw);
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    volatile int *abort = &s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 3);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], 2 * kEpiWarps);
        }
        mbar_init(&drain, 1);
        s_abort = 0;
        fence_barrier_init();
        prefetch_tensormap(&pmap);
        prefetch_tensormap(&qmap);
        prefetch_tensormap(&omap);
    }
    if (warp == 1) pair_tmem_alloc(&tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const Tiles sched{a.offsets, (a.M + 255) / 256, (a.N + 255) / 256, a.R};
    const int tiles = a.E * sched.m_tiles * sched.n_tiles;
    const int pairs = (int)(gridDim.x >> 1), pair = (int)(blockIdx.x >> 1);
    int e, m, n, r0, r1;
    if (warp == 0) {
        // ---------------------------------------------------------- TMA
        if (lane == 0) {
            const uint32_t bar0 = map_to_rank(&full[0], 0);
            const uint32_t whole = (a.p_rows ? 0u : 2u * kSide) + (a.q_rows ? 0u : 2u * kSide);
            int it = 0;
            bool good = true;
            for (int t = pair; good && t < tiles; t += pairs) {
                sched.at(t, &e, &m, &n, &r0, &r1);
                const int px = m * 256 + (int)rank * 128, qx = n * 256 + (int)rank * 128;
                for (int r = r0; r < r1; r += kStep, ++it) {
                    const int s = it % kStages;
                    if (it >= kStages) {
                        good = pair_wait(&empty[s], (uint32_t)(it / kStages - 1) & 1u, a.status, abort);
                        if (!good) break;
                    }
                    const bool tail = r + kStep > r1 || whole == 0;
                    if (rank == 0) {
                        if (tail) mbar_arrive(&full[s]);
                        else mbar_arrive_expect_tx(&full[s], whole);
                    }
                    if (tail) continue;
                    unsigned char *st = smem + (size_t)s * kStage;
                    const uint32_t bar = bar0 + 8u * (uint32_t)s;
                    if (!a.p_rows) load_side(st, &pmap, a.M, px, r, bar);
                    if (!a.q_rows) load_side(st + kSide, &qmap, a.N, qx, r, bar);
                }
            }
            if (!good && rank == 0)
                for (int i = it > kStages ? it - kStages : 0; i < it; ++i)
                    mbar_wait(&full[i % kStages], (uint32_t)(i / kStages) & 1u, a.status);
        }
        __syncwarp();
    } else if (warp >= kFirstLoader) {
        // ---------------------------------------------------------- gather
        const uint32_t place = (uint32_t)(((lane >> 3) & 1) * kBlockBytes + (lane >> 4) * 128);
        const uint32_t base = smem_u32(smem), full0 = map_to_rank(&full[0], 0);
        int it = 0, mine = warp - kFirstLoader;  // steps so far, this warp's next one
        bool good = true;
        for (int t = pair; good && t < tiles; t += pairs) {
            sched.at(t, &e, &m, &n, &r0, &r1);
            const int c = (int)rank * 128 + 8 * (lane & 15);
            const Side sp{a.P, a.p_rows, a.p_count, a.M, m * 256 + c, place};
            const Side sq{a.Q, a.q_rows, a.q_count, a.N, n * 256 + c, place + kSide};
            const int end = it + (r1 - r0 + kStep - 1) / kStep;
            for (; mine < end; mine += kLoadWarps) {
                const int s = mine % kStages, r = r0 + (mine - it) * kStep;
                const bool tail = r + kStep > r1, do_p = a.p_rows || tail, do_q = a.q_rows || tail;
                int2 pi, qi;
                if (do_p) pi = sp.ids(r, r1, lane, a.status);
                if (do_q) qi = sq.ids(r, r1, lane, a.status);
                if (mine >= kStages) {
                    good = pair_wait_warp(&empty[s], (uint32_t)(mine / kStages - 1) & 1u, a.status, abort, lane);
                    if (!good) break;
                }
                if (do_p) sp.copy(base + (uint32_t)s * kStage, pi, lane);
                if (do_q) sq.copy(base + (uint32_t)s * kStage, qi, lane);
                gathered(full0 + 8u * (uint32_t)s, lane);
            }
            it = end;
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------- MMA issuer
        if (rank == 0 && lane == 0) {
            const uint32_t idesc = pair_idesc(256, true, true);
            const uint32_t base = smem_u32(smem);
            int it = 0, done = 0;  // done: tiles with rows
            bool good = true;
            for (int t = pair; good && t < tiles; t += pairs) {
                sched.at(t, &e, &m, &n, &r0, &r1);
                if (r0 == r1) continue;
                const int buf = done & 1;
                if (done >= 2) good = pair_wait(&acc_empty[buf], (uint32_t)((done >> 1) - 1) & 1u, a.status, abort);
                if (!good) break;
                tc_fence_after();
                for (int r = r0; r < r1; r += kStep, ++it) {
                    const int s = it % kStages;
                    good = pair_wait(&full[s], (uint32_t)(it / kStages) & 1u, a.status, abort);
                    if (!good) break;
                    tc_fence_after();
                    const uint32_t sp = base + (uint32_t)s * kStage, sq = sp + kSide;
#pragma unroll
                    for (int kk = 0; kk < kStep / 16; ++kk)
                        pair_mma(tmem + (uint32_t)(buf * 256), desc_mn_sw128(sp + kk * 2048, kBlockBytes),
                                 desc_mn_sw128(sq + kk * 2048, kBlockBytes), idesc, (r > r0 || kk > 0) ? 1u : 0u);
                    pair_commit(&empty[s]);
                }
                if (good) pair_commit(&acc_full[buf]);
                ++done;
            }
            if (!good) {  // the tensor cores are done with shared memory before the CTA ends
                pair_commit(&drain);
                mbar_wait(&drain, 0u, a.status);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------- epilogue
        const int quad = warp & 3, part = (warp - 2) >> 2;
        unsigned char *mine = smem + kStages * kStage + (warp - 2) * kOut;
        const uint32_t empty_addr = map_to_rank(&acc_empty[0], 0);
        int done = 0;
        for (int t = pair; t < tiles; t += pairs) {
            sched.at(t, &e, &m, &n, &r0, &r1);
            const bool any = r1 > r0;
            if (!any && a.accumulate) continue;
            const int buf = done & 1;
            if (any) {
                const bool good = pair_wait_warp(&acc_full[buf], (uint32_t)(done >> 1) & 1u, a.status, abort, lane);
                if (!good) break;
                tc_fence_after();
            }
            const int m0 = m * 256 + (int)rank * 128 + 32 * quad;
            const uint32_t col = tmem + ((uint32_t)(32 * quad) << 16) + (uint32_t)(buf * 256);
            for (int c = 32 * part; c < 256; c += 8 * kEpiWarps) {
                const int n0 = n * 256 + c;
                if (n0 >= a.N || m0 >= a.M) break;
                uint32_t r[32];
                if (any) {
                    tmem_ld32(col + (uint32_t)c, r);
                    tmem_wait_ld();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) r[i] = 0u;
                }
                if (lane == 0) bulk_wait_read<0>();  // the last block has left
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<uint4 *>(mine + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                        make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (a.accumulate) tma_reduce_add_3d(&omap, mine, n0, m0, e);
                    else tma_store_3d(&omap, mine, n0, m0, e);
                    bulk_commit_group();
                }
            }
            if (any) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(empty_addr + 8u * (uint32_t)buf);
                ++done;
            }
        }
        if (lane == 0) bulk_wait_all<0>();
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    if (warp == 1) pair_tmem_dealloc(tmem, 512);
}

}  // namespace

cudaError_t launch_weight_grad(const WeightGradArgs &a, cudaStream_t s) {
    CUtensorMap pmap, qmap, omap;
    if (!encode_side(&pmap, a.P, a.p_count, a.M) || !encode_side(&qmap, a.Q, a.q_count, a.N) ||
        !encode_tensor_map_3d_f32(&omap, a.dW, (uint64_t)a.E, (uint64_t)a.M, (uint64_t)a.N, 32))
        return cudaErrorInvalidValue;
    cudaError_t e = ensure_smem_limit<weight_grad_kernel>(kSmem);
    if (e != cudaSuccess) return e;
    int dev = 0, sms = 0;
    e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const int64_t tiles = (int64_t)a.E * ((a.M + 255) / 256) * ((a.N + 255) / 256);
    const int64_t pairs = min64(tiles, sms / 2);
    weight_grad_kernel<<<dim3((unsigned)(2 * pairs)), kThreads, kSmem, s>>>(pmap, qmap, omap, a);
    return cudaGetLastError();
}

}  // namespace dol
