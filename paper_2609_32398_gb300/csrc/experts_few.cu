// The expert products for a handful of routed rows (a decode step of one or a few
// tokens): the weights are read once per routed row and everything else is small,
// so these kernels stream weight rows through the ALUs, one warp per result, with
// every load of a result in flight at once.  The work is R N results of equal size,
// spread evenly over the GPU; the tensor-core kernels' tiles of 256 weight rows
// leave a part of it idle then (8 routed rows of E = 128 experts, H = 2048, F = 768:
// 96 CTAs of 152).  Rows that share an expert read its weights again, from the L2:
// kFewRows is where that starts to cost more than the idle part saves.
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

// The expert of routed row r: how many groups end at or before it (E: none has it).
__device__ __forceinline__ int expert_of(const int *offsets, int E, int r, int lane) {
    int e = 0;
    for (int base = 0; base < E; base += 32) {
        const bool past = base + lane < E && __ldg(offsets + base + lane + 1) <= r;
        e += __popc(__ballot_sync(kFull, past));
    }
    return e;
}

// One warp per (routed row, result column): plain, Y[r][n]; up, act[r][f] from two
// weight rows.
template <bool kUp>
__global__ void __launch_bounds__(kWarps * 32)
few_product_kernel(const ProductArgs p, int cols) {
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = blockIdx.y, n = blockIdx.x * kWarps + warp;
    if (n >= cols) return;
    const int e = expert_of(p.offsets, p.E, r, lane);
    int src = p.rows ? __ldg(p.rows + r) : r;
    if (e >= p.E) return;
    bool in = src >= 0 && src < p.a_rows;
    if (!in && lane == 0 && p.status) atomicOr(p.status, kDevBadId);
    if (!in) src = 0;
    const int pieces = p.K / 8;
    const uint4 *a = reinterpret_cast<const uint4 *>(p.A + (int64_t)src * p.K);
    const uint4 *w = reinterpret_cast<const uint4 *>(p.W + ((int64_t)e * p.N + n) * p.K);
    const uint4 *u = reinterpret_cast<const uint4 *>(p.W + ((int64_t)e * p.N + cols + n) * p.K);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    float sw = 0.0f, su = 0.0f;
    for (int c0 = lane; c0 < pieces; c0 += 8 * 32) {
        uint4 av[8], wv[8], uv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = c0 + 32 * j;
            wv[j] = c < pieces ? __ldg(w + c) : zero;
            if (kUp) uv[j] = c < pieces ? __ldg(u + c) : zero;
            av[j] = c < pieces && in ? __ldg(a + c) : zero;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (c0 + 32 * j >= pieces || !in) continue;  // a row of zeros is one whatever the weights hold
            sw = dot8(av[j], wv[j], sw);
            if (kUp) su = dot8(av[j], uv[j], su);
        }
    }
    sw = warp_sum(sw);
    if (kUp) su = warp_sum(su);
    if (lane == 0) {
        const float v = kUp ? sw * sigmoid_f(sw) * su : sw;
        p.out[(int64_t)r * cols + n] = __float2bfloat16_rn(v);
    }
}

// One warp per (token, result column): its k rows' products summed in fp32.
__global__ void __launch_bounds__(kWarps * 32)
few_join_kernel(const ProductArgs p, const int *__restrict__ pos, const float *__restrict__ weights, int k) {
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t = blockIdx.y, n = blockIdx.x * kWarps + warp;
    if (n >= p.N) return;
    const int pieces = p.K / 8;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    float sum = 0.0f;
    for (int q0 = 0; q0 < k; q0 += 4) {
        int row[4], e[4] = {0, 0, 0, 0};
        float scale[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            row[q] = q0 + q < k ? __ldg(pos + t * k + q0 + q) : -1;
            scale[q] = weights && q0 + q < k ? __ldg(weights + t * k + q0 + q) : 1.0f;
        }
        for (int base = 0; base < p.E; base += 32) {
            const int end = base + lane < p.E ? __ldg(p.offsets + base + lane + 1) : 0x7fffffff;
#pragma unroll
            for (int q = 0; q < 4; ++q) e[q] += __popc(__ballot_sync(kFull, base + lane < p.E && end <= row[q]));
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool out = row[q] < 0 || row[q] >= p.R || e[q] >= p.E;
            if (out && q0 + q < k && lane == 0 && p.status) atomicOr(p.status, kDevBadId);
            if (out) row[q] = -1;
        }
        for (int c0 = lane; c0 < pieces; c0 += 3 * 32) {
            uint4 av[4][3], wv[4][3];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 *a = reinterpret_cast<const uint4 *>(p.A + (int64_t)row[q] * p.K);
                const uint4 *w = reinterpret_cast<const uint4 *>(p.W + ((int64_t)e[q] * p.N + n) * p.K);
#pragma unroll
                for (int j = 0; j < 3; ++j) {
                    const bool in = row[q] >= 0 && c0 + 32 * j < pieces;
                    wv[q][j] = in ? __ldg(w + c0 + 32 * j) : zero;
                    av[q][j] = in ? __ldg(a + c0 + 32 * j) : zero;
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float s = 0.0f;
#pragma unroll
                for (int j = 0; j < 3; ++j) s = dot8(av[q][j], wv[q][j], s);
                if (row[q] >= 0) sum = fmaf(scale[q], s, sum);
            }
        }
    }
    sum = warp_sum(sum);
    if (lane == 0) p.out[(int64_t)t * p.N + n] = __float2bfloat16_rn(sum);
}

}  // namespace

cudaError_t launch_few_product(ProductMode mode, const ProductArgs &a, cudaStream_t s) {
    const int cols = mode == kProductUp ? a.N / 2 : a.N;
    const dim3 grid((unsigned)((cols + kWarps - 1) / kWarps), (unsigned)a.R);
    if (mode == kProductUp) return launch_after(few_product_kernel<true>, grid, kWarps * 32, 0, s, a, cols);
    return launch_after(few_product_kernel<false>, grid, kWarps * 32, 0, s, a, cols);
}

cudaError_t launch_few_join(const ProductArgs &a, const int *pos, const float *weights, int64_t T, int k,
                            cudaStream_t s) {
    return launch_after(few_join_kernel, dim3((unsigned)((a.N + kWarps - 1) / kWarps), (unsigned)T), kWarps * 32, 0, s, a,
                        pos, weights, k);
}

}  // namespace dol
