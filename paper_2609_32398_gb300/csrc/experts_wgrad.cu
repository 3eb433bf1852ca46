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
// past its end are zeros on both, whatever the next expert's rows hold.  Two
// accumulators in TMEM let one's 256 KB of fp32 leave while the next one's products
// run; an expert without rows gets zeros from the epilogue alone.  The result is
// stored by TMA from 32 x 32 blocks.
//
// The tensor cores cut off what an addition to an accumulator shifts out, so that its
// error grows with the additions.  An accumulator therefore takes kSpan rows at
// most: a tile's first one is stored (or added to dW), and the others, in order and each after
// the one before has been written, are added to it in memory, where the fp32 sum is rounded.
//
// Warps: 0 TMA, 1 issues the MMAs (first CTA), 2-5 epilogue, 6-11 gather.
//
// What bounds it: at 16384 tokens (1024 rows an expert, H = 2048, 2F = 1536) 628 us, 1.31
// PFLOP/s; the products and TMA copies alone run at 1.7, the gathering beside them costs
// 90 us and the 1.6 GB of results another 100.  With few rows the results are all of it:
// 201 MB in 37 us.
#include <cstdint>

#include "experts_mma.cuh"

namespace dol {
namespace {

constexpr int kEpiWarps = 4;
constexpr int kFirstLoader = 2 + kEpiWarps;
constexpr int kThreads = (kFirstLoader + kLoadWarps) * 32;
constexpr int kStep = 64;                       // rows of a step
// Rows of an accumulator at most.  Error of dW by its norm, normal rows and, in brackets, all
// terms positive: 2.1e-6 (5.6e-6) for any number of rows, against 1.5e-4 (8.2e-4) for 131072
// in one accumulator.  With 1024 it is 1.0e-6 (2.2e-6) and dW1 of 16384 tokens takes 670 us
// instead of 643 (632 in one accumulator each), that of 49152 tokens 1990 instead of 1925 (1784);
// with 4096 4.4e-6 (1.4e-5).
constexpr int kSpan = 2048;
constexpr uint32_t kBlockBytes = kStep * 128;   // 64 columns of a step
constexpr uint32_t kSide = 2 * kBlockBytes;     // a CTA's 128 columns of one operand
constexpr uint32_t kStage = 2 * kSide;
constexpr int kStages = 6;
constexpr uint32_t kOut = 32 * 128;             // an epilogue warp's 32 x 32 block
// Shared memory: ring, the epilogue's blocks (two a warp where the table leaves the room:
// one is filled while the other leaves), the experts' first rows [E + 1].
constexpr uint32_t kSmemLimit = 232448 - 512;  // the barriers are not dynamic
constexpr uint32_t smem_with(int E, int blocks) {
    return 1024 + kStages * kStage + kEpiWarps * blocks * kOut + 4u * ((uint32_t)E + 1u);
}
constexpr int out_blocks(int E) { return smem_with(E, 2) <= kSmemLimit ? 2 : 1; }
constexpr uint32_t smem_bytes(int E) { return smem_with(E, out_blocks(E)); }
static_assert(smem_bytes(1024) <= kSmemLimit && out_blocks(256) == 2, "shared memory");
static_assert(kStages == kLoadWarps, "a gathering warp has one stage of its own");

// The tiles of a pair in turn: t = pair, pair + pairs, ...
struct Walk {
    const int *start;        // shared, [E + 1]
    int E, m_tiles, per;     // per: tiles of an expert
    uint32_t m_magic;
    int step_e, step_i;      // pairs in experts and tiles
    int e, i;                // expert, and tile of it
    int m, n, r0, r1;

    __device__ __forceinline__ bool find() {
        if (e >= E) return false;
        n = divide_by(i, m_magic);
        m = i - n * m_tiles;
        r0 = start[e];
        r1 = max(r0, start[e + 1]);
        return true;
    }
    __device__ __forceinline__ bool next() {
        e += step_e;
        i += step_i;
        if (i >= per) {
            i -= per;
            ++e;
        }
        return find();
    }
};

// A tile's rows, n of them, are added up in accumulators of span_of(n) rows each, whole steps
// and all but the last equal.
__device__ __forceinline__ int span_of(int n) {
    const int parts = (n + kSpan - 1) / kSpan;
    return parts > 1 ? ((n + parts - 1) / parts + kStep - 1) / kStep * kStep : n;
}

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
__device__ __forceinline__ void load_side(uint32_t dst, const CUtensorMap *map, int cols, int x, int r,
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
            mbar_init(&full[i], 4);  // each CTA's TMA warp and its gathering warp of the step
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
    pdl_wait();
    // not before: the kernel before may share this SM and still have to take its own
    if (warp == 1) pair_tmem_alloc(&tmem_slot, 512);
    const int blocks = out_blocks(a.E);
    int *start = reinterpret_cast<int *>(smem + kStages * kStage + kEpiWarps * blocks * kOut);
    for (int i = threadIdx.x; i <= a.E; i += kThreads) start[i] = max(0, min(__ldg(a.offsets + i), (int)a.R));
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int m_tiles = (a.M + 255) / 256, per = m_tiles * ((a.N + 255) / 256);
    const int pairs = (int)(gridDim.x >> 1), pair = (int)(blockIdx.x >> 1);
    Walk w{start, a.E, m_tiles, per, a.m_magic, pairs / per, pairs % per, pair / per, pair % per, 0, 0, 0, 0};
    const uint32_t ring = smem_u32(smem), full0 = smem_u32(full), empty0 = smem_u32(empty);
    const uint32_t full_pair = map_to_rank(full, 0);  // the first CTA's
    if (warp == 0) {
        // ---------------------------------------------------------- TMA
        const bool one = elect_one();
        const uint32_t whole = (a.p_rows ? 0u : 2u * kSide) + (a.q_rows ? 0u : 2u * kSide);
        Ring at{0, 0};
        int it = 0;
        bool good = true;
        for (bool any = w.find(); good && any; any = w.next()) {
            const int px = w.m * 256 + (int)rank * 128, qx = w.n * 256 + (int)rank * 128;
            for (int r = w.r0; r < w.r1; r += kStep, ++it) {
                good = pair_wait_all(empty0 + 8 * at.s, at.phase ^ 1u, a.status, abort);
                if (!good) break;
                const bool tail = r + kStep > w.r1 || whole == 0;
                if (one) {
                    // the second CTA's warp arrives too: a step that has nothing to load by
                    // TMA must not leave it a phase behind, which its parity could not tell
                    if (rank == 0 && !tail) mbar_expect_tx_addr(full0 + 8 * at.s, whole);
                    else mbar_arrive_cluster(full_pair + 8 * at.s);
                    if (!tail) {
                        const uint32_t st = ring + at.s * kStage, bar = full_pair + 8 * at.s;
                        if (!a.p_rows) load_side(st, &pmap, a.M, px, r, bar);
                        if (!a.q_rows) load_side(st + kSide, &qmap, a.N, qx, r, bar);
                    }
                }
                __syncwarp();
                at.next(kStages);
            }
        }
        if (!good && rank == 0 && lane == 0)
            for (int i = it > kStages ? it - kStages : 0; i < it; ++i)
                mbar_wait(&full[i % kStages], (uint32_t)(i / kStages) & 1u, a.status);
        __syncwarp();
    } else if (warp >= kFirstLoader) {
        // ---------------------------------------------------------- gather
        const uint32_t place = (uint32_t)(((lane >> 3) & 1) * kBlockBytes + (lane >> 4) * 128);
        const int s = warp - kFirstLoader;  // this warp's stage of the ring
        const int c = (int)rank * 128 + 8 * (lane & 15);
        const uint32_t st = ring + (uint32_t)s * kStage;
        int k = s, steps = 0, lap = 0;  // the next step of the tile, the tile's steps
        bool good = true, do_p = false, do_q = false;
        int2 pi, qi;
        Side sp{a.P, a.p_rows, a.p_count, a.M, 0, place}, sq{a.Q, a.q_rows, a.q_count, a.N, 0, place + kSide};
        // moves on to this warp's next step and reads its row ids
        auto seek = [&](bool any) {
            while (any) {
                steps = (w.r1 - w.r0 + kStep - 1) / kStep;
                if (k < steps) break;
                k -= steps;
                any = w.next();
            }
            if (any) {
                const int r = w.r0 + k * kStep;
                const bool tail = r + kStep > w.r1;
                do_p = a.p_rows || tail;
                do_q = a.q_rows || tail;
                sp.x = w.m * 256 + c;
                sq.x = w.n * 256 + c;
                if (do_p) pi = sp.ids(r, w.r1, lane, a.status);
                if (do_q) qi = sq.ids(r, w.r1, lane, a.status);
            }
            return any;
        };
        for (bool any = seek(w.find()); any; ++lap) {
            if (lap > 0) {
                good = pair_wait_warp(empty0 + 8 * s, (uint32_t)(lap - 1) & 1u, a.status, abort, lane);
                if (!good) break;
            }
            if (do_p) sp.copy(st, pi, lane);
            if (do_q) sq.copy(st, qi, lane);
            k += kLoadWarps;
            any = seek(any);  // under the copies
            gathered(full_pair + 8 * s, lane);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------- MMA issuer
        if (rank == 0) {
            const bool one = elect_one();
            constexpr uint32_t idesc = pair_idesc(256, true, true);
            const uint64_t pd0 = desc_mn_sw128(ring, kBlockBytes), qd0 = desc_mn_sw128(ring + kSide, kBlockBytes);
            const uint32_t acc_full0 = smem_u32(acc_full), acc_empty0 = smem_u32(acc_empty);
            Ring at{0, 0};
            int done = 0;  // accumulators
            bool good = true;
            for (bool any = w.find(); good && any; any = w.next()) {
                const int span = span_of(w.r1 - w.r0);
                for (int r = w.r0; good && r < w.r1; ++done) {
                    const uint32_t buf = done & 1, turns = (uint32_t)done >> 1;
                    good = pair_wait_all(acc_empty0 + 8 * buf, (turns & 1u) ^ 1u, a.status, abort);
                    if (!good) break;
                    tc_fence_after();
                    const uint32_t d = tmem + buf * 256;
                    uint32_t more = 0;
                    for (const int end = r + min(span, w.r1 - r); r < end; r += kStep) {
                        good = pair_wait_all(full0 + 8 * at.s, at.phase, a.status, abort);
                        if (!good) break;
                        tc_fence_after();
                        const uint32_t off = at.s * (kStage / 16);
                        if (one) {
#pragma unroll
                            for (int kk = 0; kk < kStep / 16; ++kk)
                                pair_mma(d, desc_at(pd0, off + kk * (2048 / 16)), desc_at(qd0, off + kk * (2048 / 16)),
                                         idesc, kk > 0 ? 1u : more);
                            pair_commit(empty0 + 8 * at.s);
                        }
                        __syncwarp();
                        more = 1;
                        at.next(kStages);
                    }
                    if (good && one) pair_commit(acc_full0 + 8 * buf);
                    __syncwarp();
                }
            }
            if (!good && one) {  // the tensor cores are done with shared memory before the CTA ends
                pair_commit(smem_u32(&drain));
                mbar_wait(&drain, 0u, a.status);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------- epilogue
        const int quad = warp & 3, part = (warp - 2) >> 2;
        unsigned char *places = smem + kStages * kStage + (warp - 2) * blocks * kOut;
        int turn = 0;  // the place of the next block
        const uint32_t empty_addr = map_to_rank(&acc_empty[0], 0);
        int done = 0, left = 0, span = 0;  // of the tile: rows not yet accumulated, rows of an accumulator
        bool first = true, more = w.find();
        for (; more; first = left <= 0, more = first ? w.next() : true) {
            if (first) {
                left = w.r1 - w.r0;
                span = span_of(left);
            }
            const bool any = left > 0;
            if (!any && a.accumulate) continue;
            const int buf = done & 1;
            if (any) {
                const bool good = pair_wait_warp(smem_u32(&acc_full[buf]), (uint32_t)(done >> 1) & 1u, a.status, abort, lane);
                if (!good) break;
                tc_fence_after();
                left -= span;
            }
            // an accumulator is added to what the ones before it left, which has been written then
            const bool add = a.accumulate || !first;
            if (!first) {
                if (lane == 0) bulk_wait_all<0>();
                __syncwarp();
            }
            const int m0 = w.m * 256 + (int)rank * 128 + 32 * quad;
            const uint32_t col = tmem + ((uint32_t)(32 * quad) << 16) + (uint32_t)(buf * 256);
            for (int c = 32 * part; c < 256; c += 8 * kEpiWarps) {
                const int n0 = w.n * 256 + c;
                if (n0 >= a.N || m0 >= a.M) break;
                uint32_t r[32];
                if (any) {
                    tmem_ld32(col + (uint32_t)c, r);
                    tmem_wait_ld();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) r[i] = 0u;
                }
                unsigned char *mine = places + turn * kOut;
                if (blocks == 2) {
                    turn ^= 1;
                    if (lane == 0) bulk_wait_read<1>();  // what was in it has left
                } else if (lane == 0) {
                    bulk_wait_read<0>();
                }
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<uint4 *>(mine + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                        make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (add) tma_reduce_add_3d(&omap, mine, n0, m0, w.e);
                    else tma_store_3d(&omap, mine, n0, m0, w.e);
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
    pdl_trigger();  // this CTA's work is done: the next kernel may begin to arrive
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
    cudaError_t e = ensure_smem_limit<weight_grad_kernel>(kSmemLimit);
    if (e != cudaSuccess) return e;
    int dev = 0, sms = 0;
    e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    WeightGradArgs b = a;
    b.m_magic = divide_magic((uint32_t)(a.M + 255) / 256);
    const int64_t tiles = (int64_t)a.E * ((a.M + 255) / 256) * ((a.N + 255) / 256);
    const int64_t pairs = min64(tiles, sms / 2);
    return launch_after(weight_grad_kernel, dim3((unsigned)(2 * pairs)), kThreads, smem_bytes(a.E), s, pmap, qmap, omap, b);
}

}  // namespace dol
