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
// Warps: 0 TMA, 1 issues the MMAs (first CTA), 2-5 epilogue, 6-9 gather, 10
// announces their steps.
#include <cstdint>

#include "experts_mma.cuh"

namespace dol {
namespace {

constexpr int kEpiWarps = 4;
constexpr int kFirstLoader = 2 + kEpiWarps;
constexpr int kThreads = (kFirstLoader + kLoadWarps + 1) * 32;
constexpr int kStep = 64;                       // rows of a step
constexpr uint32_t kBlockBytes = kStep * 128;   // 64 columns of a step
constexpr uint32_t kSide = 2 * kBlockBytes;     // a CTA's 128 columns of one operand
constexpr uint32_t kStage = 2 * kSide;
constexpr int kStages = 6;
constexpr uint32_t kOut = 32 * 128;             // an epilogue warp's 32 x 32 block
constexpr uint32_t kSmem = 1024 + kStages * kStage + kEpiWarps * kOut;
static_assert(kSmem <= 232448 - 2048, "shared memory");

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

// A gathering thread's share of one operand's step: 16 bytes of 8 of the 64 rows.
struct Side {
    const bf16 *mat;
    const int *rows;
    int64_t count;
    int cols, x;      // columns, and this thread's first one
    uint32_t dst;     // its place in a stage for row 0 of its eight (8 rows apart)

    // the matrix rows of routed rows r, r + 8, ..., r + 56; -1: none (zeros)
    __device__ void ids(int r, int end, int *status, int (&id)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = r + 8 * j;
            id[j] = -1;
            if (i < end) {
                const int src = rows ? __ldg(rows + i) : i;
                if (src >= 0 && src < count) id[j] = src;
                else if (status) atomicOr(status, kDevBadId);
            }
        }
    }
    __device__ void copy(uint32_t stage, const int (&id)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = id[j] >= 0 && x < cols;
            cp_async16(stage + dst + j * 1024, mat + (in ? (int64_t)id[j] * cols + x : 0), in);
        }
    }
};

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
weight_grad_kernel(const __grid_constant__ CUtensorMap pmap, const __grid_constant__ CUtensorMap qmap,
                   const __grid_constant__ CUtensorMap omap, const WeightGradArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_align<1024>(smem_raw);
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], landed[kStages], acc_full[2], acc_empty[2], drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort;
    volatile int *abort = &s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&full[i], 3);
            mbar_init(&landed[i], 32 * kLoadWarps);
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
                    for (int b = 0; b < 2; ++b) {
                        if (!a.p_rows) pair_load_3d(st + b * kBlockBytes, &pmap, px + 64 * b, r, 0, bar);
                        if (!a.q_rows) pair_load_3d(st + kSide + b * kBlockBytes, &qmap, qx + 64 * b, r, 0, bar);
                    }
                }
            }
            if (!good && rank == 0)
                for (int i = it > kStages ? it - kStages : 0; i < it; ++i)
                    mbar_wait(&full[i % kStages], (uint32_t)(i / kStages) & 1u, a.status);
        }
        __syncwarp();
    } else if (warp == kFirstLoader + kLoadWarps) {
        // ---------------------------------------------------------- announce
        if (lane == 0) {
            const uint32_t full0 = map_to_rank(&full[0], 0);
            int it = 0;
            bool good = true;
            for (int t = pair; good && t < tiles; t += pairs) {
                sched.at(t, &e, &m, &n, &r0, &r1);
                for (int r = r0; good && r < r1; r += kStep, ++it) {
                    const int s = it % kStages;
                    good = announce(&landed[s], (uint32_t)(it / kStages) & 1u, full0 + 8u * (uint32_t)s, a.status, abort);
                }
            }
        }
        __syncwarp();
    } else if (warp >= kFirstLoader) {
        // ---------------------------------------------------------- gather
        // Sixteen lanes copy a row's 256 bytes of one operand, a pass takes 8 rows.
        const int i = (int)threadIdx.x - kFirstLoader * 32, piece = i & 15, row = i >> 4;
        const uint32_t place = (uint32_t)((piece >> 3) * kBlockBytes + row * 128 + (((piece & 7) ^ row) << 4));
        const uint32_t base = smem_u32(smem);
        int it = 0;
        bool good = true;
        for (int t = pair; good && t < tiles; t += pairs) {
            sched.at(t, &e, &m, &n, &r0, &r1);
            const int c = (int)rank * 128 + 8 * piece;
            const Side sp{a.P, a.p_rows, a.p_count, a.M, m * 256 + c, place};
            const Side sq{a.Q, a.q_rows, a.q_count, a.N, n * 256 + c, place + kSide};
            int pi[8], qi[8];  // of the step, read under the wait for the one before
            if (a.p_rows || r0 + kStep > r1) sp.ids(r0 + row, r1, a.status, pi);
            if (a.q_rows || r0 + kStep > r1) sq.ids(r0 + row, r1, a.status, qi);
            for (int r = r0; r < r1; r += kStep, ++it) {
                const int s = it % kStages;
                if (it >= kStages) {
                    good = pair_wait(&empty[s], (uint32_t)(it / kStages - 1) & 1u, a.status, abort);
                    good = __all_sync(kFull, good);
                    if (!good) break;
                }
                const bool tail = r + kStep > r1, tail_next = r + 2 * kStep > r1;
                if (a.p_rows || tail) sp.copy(base + (uint32_t)s * kStage, pi);
                if (a.q_rows || tail) sq.copy(base + (uint32_t)s * kStage, qi);
                cp_async_arrive(&landed[s]);
                if (a.p_rows || tail_next) sp.ids(r + kStep + row, r1, a.status, pi);
                if (a.q_rows || tail_next) sq.ids(r + kStep + row, r1, a.status, qi);
            }
        }
        cp_async_wait_all();
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
                const bool good = __all_sync(kFull, pair_wait(&acc_full[buf], (uint32_t)(done >> 1) & 1u, a.status, abort));
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
    if (!encode_tensor_map_3d_bf16(&pmap, a.P, 1, (uint64_t)a.p_count, (uint64_t)a.M, 64, kStep) ||
        !encode_tensor_map_3d_bf16(&qmap, a.Q, 1, (uint64_t)a.q_count, (uint64_t)a.N, 64, kStep) ||
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
