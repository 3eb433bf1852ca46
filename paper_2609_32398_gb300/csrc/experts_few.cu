// The expert products for a handful of routed rows (a decode step of one or a few
// tokens): the weights are read once per routed row and everything else is small,
// so these kernels stream weight rows through the ALUs, one warp per result or a few,
// with as many loads in flight as its registers hold.  The work is R N results of equal size,
// spread evenly over the GPU; the tensor-core kernels' tiles of 256 weight rows
// leave a part of it idle then (8 routed rows of E = 128 experts, H = 2048, F = 768:
// 96 CTAs of 152).  Rows that share an expert read its weights again, from the L2:
// kFewRows is where that starts to cost more than the idle part saves.  Bound by memory
// and the latency of two dependent loads (the group ends, then the weights): the up
// projection of those 8 rows takes 10.1 us for 50 MB, 7.4 at the copy rate.
//
// Sums are fp32, lane by lane in order and then over the lanes.
#include "experts.cuh"
#include "tma.cuh"

namespace dol {
namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ float dot8(uint4 a, uint4 b, float s) {
    const unsigned x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), s);
        s = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), s);
    }
    return s;
}

// How many of the E groups end at or before each of n routed rows: the rows' experts
// (E: none has it; nor has any a row before the first group).  Four loads of 32 group ends
// at a time.
template <int n>
__device__ __forceinline__ void experts_of(const int *offsets, int E, const int (&row)[n], int lane, int (&e)[n]) {
    const int lo = __ldg(offsets);
#pragma unroll
    for (int q = 0; q < n; ++q) e[q] = 0;
    for (int base = 0; base < E; base += 128) {
        int end[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = base + 32 * j + lane;
            end[j] = i < E ? __ldg(offsets + i + 1) : 0x7fffffff;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int q = 0; q < n; ++q) e[q] += __popc(__ballot_sync(kFull, end[j] <= row[q] && end[j] != 0x7fffffff));
    }
#pragma unroll
    for (int q = 0; q < n; ++q)
        if (row[q] < lo) e[q] = E;
}

// A warp takes kCols result columns of one routed row at a time, kPieces 16-byte
// pieces of each weight row a lane and all of them in flight: sixteen where the sizes
// allow.  Plain: Y[r][n]; up: act[r][f] from two weight rows.
template <bool kUp, int kCols, int kPieces>
__global__ void __launch_bounds__(kWarps * 32)
few_product_kernel(const ProductArgs p, int cols) {
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r[1] = {(int)blockIdx.y};
    int e[1];
    int src = p.rows ? __ldg(p.rows + r[0]) : r[0];
    experts_of(p.offsets, p.E, r, lane, e);
    if (e[0] >= p.E) return;
    const bool in = src >= 0 && src < p.a_rows;
    if (!in && threadIdx.x == 0 && blockIdx.x == 0 && p.status) atomicOr(p.status, kDevBadId);
    if (!in) src = 0;
    const int pieces = p.K / 8;
    const uint4 *a = reinterpret_cast<const uint4 *>(p.A + (int64_t)src * p.K);
    const uint4 *weights = reinterpret_cast<const uint4 *>(p.W + (int64_t)e[0] * p.N * p.K);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int n = ((int)blockIdx.x * kWarps + warp) * kCols; n < cols; n += (int)gridDim.x * kWarps * kCols) {
        float sw[kCols] = {}, su[kCols] = {};
        for (int c0 = lane; c0 < pieces && in; c0 += kPieces * 32) {
            uint4 av[kPieces], wv[kCols][kPieces], uv[kCols][kPieces];
#pragma unroll
            for (int i = 0; i < kCols; ++i)
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    const int c = c0 + 32 * j;
                    const bool have = c < pieces && n + i < cols;
                    wv[i][j] = have ? __ldg(weights + (int64_t)(n + i) * pieces + c) : zero;
                    if (kUp) uv[i][j] = have ? __ldg(weights + (int64_t)(cols + n + i) * pieces + c) : zero;
                }
#pragma unroll
            for (int j = 0; j < kPieces; ++j) av[j] = c0 + 32 * j < pieces ? __ldg(a + c0 + 32 * j) : zero;
#pragma unroll
            for (int i = 0; i < kCols; ++i)
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    if (c0 + 32 * j >= pieces) continue;
                    sw[i] = dot8(av[j], wv[i][j], sw[i]);
                    if (kUp) su[i] = dot8(av[j], uv[i][j], su[i]);
                }
        }
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            sw[i] = warp_sum(sw[i]);
            if (kUp) su[i] = warp_sum(su[i]);
            const float v = kUp ? sw[i] * sigmoid_f(sw[i]) * su[i] : sw[i];
            if (lane == i && n + i < cols) p.out[(int64_t)r[0] * cols + n + i] = __float2bfloat16_rn(v);
        }
    }
}

// kSplit warps per (token, result column), each with a share of the token's k rows, four
// of them at a time: 24 pieces of weights and values, of which the 52 to 56 registers that
// the compiler takes hold a half at once.  fp32 sums, joined in order through shared memory.
template <int kSplit, int kPieces>
__global__ void __launch_bounds__(kWarps * 32)
few_join_kernel(const ProductArgs p, const int *__restrict__ pos, const float *__restrict__ weights, int k) {
    __shared__ float part[kWarps];
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t = blockIdx.y, n = blockIdx.x * (kWarps / kSplit) + warp / kSplit;
    const int pieces = p.K / 8;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    float sum = 0.0f;
    for (int q0 = 4 * (warp % kSplit); q0 < k && n < p.N; q0 += 4 * kSplit) {
        int row[4], e[4];
        float scale[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            row[q] = q0 + q < k ? __ldg(pos + t * k + q0 + q) : -1;
            scale[q] = weights && q0 + q < k ? __ldg(weights + t * k + q0 + q) : 1.0f;
        }
        experts_of(p.offsets, p.E, row, lane, e);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool out = row[q] < 0 || row[q] >= p.R || e[q] >= p.E;
            if (out && q0 + q < k && lane == 0 && n == 0 && p.status) atomicOr(p.status, kDevBadId);
            if (out) row[q] = -1;
        }
        for (int c0 = lane; c0 < pieces; c0 += kPieces * 32) {
            uint4 wv[4][kPieces], av[4][kPieces];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 *w = reinterpret_cast<const uint4 *>(p.W + ((int64_t)e[q] * p.N + n) * p.K);
                const uint4 *a = reinterpret_cast<const uint4 *>(p.A + (int64_t)row[q] * p.K);
#pragma unroll
                for (int j = 0; j < kPieces; ++j) {
                    const bool in = row[q] >= 0 && c0 + 32 * j < pieces;
                    wv[q][j] = in ? __ldg(w + c0 + 32 * j) : zero;
                    av[q][j] = in ? __ldg(a + c0 + 32 * j) : zero;
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < kPieces; ++j) s = dot8(av[q][j], wv[q][j], s);
                if (row[q] >= 0) sum = fmaf(scale[q], s, sum);
            }
        }
    }
    sum = warp_sum(sum);
    if (kSplit > 1) {
        if (lane == 0) part[warp] = sum;
        __syncthreads();
        if (warp % kSplit == 0)
#pragma unroll
            for (int i = 1; i < kSplit; ++i) sum += part[warp + i];
    }
    if (warp % kSplit == 0 && lane == 0 && n < p.N) p.out[(int64_t)t * p.N + n] = __float2bfloat16_rn(sum);
}

template <bool kUp, int kCols, int kPieces>
cudaError_t launch_columns(const ProductArgs &a, int cols, cudaStream_t s) {
    // as many blocks as are resident at two an SM, and no warp with one turn more than
    // the others where that can be had
    const int64_t turns = (cols + kWarps * kCols - 1) / (kWarps * kCols);
    const int64_t most = min64(turns, (2 * 152 + a.R - 1) / a.R);
    const int64_t laps = (turns + most - 1) / most;
    return launch_after(few_product_kernel<kUp, kCols, kPieces>, dim3((unsigned)((turns + laps - 1) / laps), (unsigned)a.R),
                        kWarps * 32, 0, s, a, cols);
}

}  // namespace

cudaError_t launch_few_product(ProductMode mode, const ProductArgs &a, cudaStream_t s) {
    const int cols = mode == kProductUp ? a.N / 2 : a.N;
    if (mode == kProductUp) {
        if (a.K <= 512) return launch_columns<true, 4, 2>(a, cols, s);
        if (a.K <= 1024) return launch_columns<true, 2, 4>(a, cols, s);
        return launch_columns<true, 1, 8>(a, cols, s);
    }
    if (a.K <= 512) return launch_columns<false, 8, 2>(a, cols, s);
    if (a.K <= 1024) return launch_columns<false, 4, 4>(a, cols, s);
    return launch_columns<false, 2, 8>(a, cols, s);
}

cudaError_t launch_few_join(const ProductArgs &a, const int *pos, const float *weights, int64_t T, int k,
                            cudaStream_t s) {
    const int split = k > 8 ? 4 : k > 4 ? 2 : 1, per = kWarps / split;
    const dim3 grid((unsigned)((a.N + per - 1) / per), (unsigned)T);
    if (split == 4) return launch_after(few_join_kernel<4, 3>, grid, kWarps * 32, 0, s, a, pos, weights, k);
    if (split == 2) return launch_after(few_join_kernel<2, 3>, grid, kWarps * 32, 0, s, a, pos, weights, k);
    return launch_after(few_join_kernel<1, 3>, grid, kWarps * 32, 0, s, a, pos, weights, k);
}

}  // namespace dol
