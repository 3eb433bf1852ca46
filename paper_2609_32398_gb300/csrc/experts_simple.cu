// First kernels of the expert operators: 64 x 64 tiles in shared memory, fp32
// arithmetic on the ALU.
#include "experts.cuh"

namespace dol {
namespace {

constexpr int kT = 64;   // tile rows and columns
constexpr int kKs = 16;  // contraction step

// The expert and first row of row tile `tile`; false past the last one.
__device__ bool find_tile(const int *offsets, int E, int64_t R, int tile, int *e_out, int *r0, int *r1) {
    int left = tile;
    for (int e = 0; e < E; ++e) {
        const int a = max(0, min(offsets[e], (int)R)), b = max(a, min(offsets[e + 1], (int)R));
        const int n = (b - a + kT - 1) / kT;
        if (left < n) {
            *e_out = e;
            *r0 = a + left * kT;
            *r1 = min(b, *r0 + kT);
            return true;
        }
        left -= n;
    }
    return false;
}

template <int kMode>
__global__ void __launch_bounds__(256) product_simple_kernel(const ProductArgs a) {
    __shared__ int s_e, s_r0, s_r1, s_ok;
    __shared__ float sa[kT][kKs + 1], sw[kT][kKs + 1], sz[kT][kT + 1];
    if (threadIdx.x == 0) s_ok = find_tile(a.offsets, a.E, a.R, blockIdx.y, &s_e, &s_r0, &s_r1);
    __syncthreads();
    if (!s_ok) return;
    const int e = s_e, r0 = s_r0, nr = s_r1 - s_r0, F = a.N / 2;
    // up: 32 gate rows of W, then the 32 up rows of the same columns
    const int n0 = blockIdx.x * (kMode == kProductUp ? kT / 2 : kT);
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < a.K; k0 += kKs) {
        for (int i = threadIdx.x; i < kT * kKs; i += 256) {
            const int row = i / kKs, k = k0 + i % kKs;
            float v = 0.0f;
            if (row < nr && k < a.K) {
                const int src = a.rows ? a.rows[r0 + row] : r0 + row;
                if (src >= 0 && src < a.a_rows) v = __bfloat162float(a.A[(int64_t)src * a.K + k]);
                else if (a.status) atomicOr(a.status, kDevBadId);
            }
            sa[row][i % kKs] = v;
            int n = n0 + row;
            if (kMode == kProductUp) n = row < 32 ? n0 + row : F + n0 + row - 32;
            const bool in = kMode == kProductUp ? n0 + (row & 31) < F : n < a.N;
            float w = 0.0f;
            if (in && k < a.K)
                w = __bfloat162float(a.transposed ? a.W[((int64_t)e * a.K + k) * a.N + n]
                                                  : a.W[((int64_t)e * a.N + n) * a.K + k]);
            sw[row][i % kKs] = w;
        }
        __syncthreads();
        for (int k = 0; k < kKs; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[ty + 16 * i][k], sw[tx + 16 * j][k], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) sz[ty + 16 * i][tx + 16 * j] = acc[i][j];
    __syncthreads();
    if (kMode == kProductPlain) {
        for (int i = threadIdx.x; i < kT * kT; i += 256) {
            const int row = i / kT, n = n0 + i % kT;
            if (row < nr && n < a.N) a.out[(int64_t)(r0 + row) * a.N + n] = __float2bfloat16_rn(sz[row][i % kT]);
        }
    } else if (kMode == kProductUp) {
        for (int i = threadIdx.x; i < kT * 32; i += 256) {
            const int row = i / 32, f = n0 + i % 32;
            if (row >= nr || f >= F) continue;
            const float g = sz[row][i % 32];
            a.out[(int64_t)(r0 + row) * F + f] = __float2bfloat16_rn(g * sigmoid_f(g) * sz[row][32 + i % 32]);
        }
        // 8-bit blocks: [64 rows][4 blocks of 16]; columns 0-31 gate, 32-63 up
        for (int i = threadIdx.x; a.codes && i < kT * 4; i += 256) {
            const int row = i / 4, c = (i % 4) * kQBlock;
            const int f = n0 + (c & 31);
            if (row >= nr || f >= F) continue;
            const int col = (c < 32 ? 0 : F) + f;
            unsigned top = 0;  // the bits of |v| order as the values do, NaN above infinity
            for (int j = 0; j < kQBlock; ++j) top = max(top, __float_as_uint(sz[row][c + j]) & 0x7fffffffu);
            const int ex = q8_exponent(__uint_as_float(top));
            const float inv = q8_inverse(ex);
            const int64_t at = (int64_t)(r0 + row) * a.N + col;
            for (int j = 0; j < kQBlock; ++j) a.codes[at + j] = ex == 255 ? 0 : (int8_t)q8_code(sz[row][c + j], inv);
            a.exponents[at / kQBlock] = (uint8_t)ex;
        }
    } else {
        // N = F columns; 8 strips... two strips of 32 columns a tile
        const int lane = threadIdx.x & 31;
        for (int i = threadIdx.x; i < kT * kT; i += 256) {
            const int row = i / kT, f = n0 + i % kT;
            float part = 0.0f;
            if (row < nr && f < a.N) {
                const int64_t r = r0 + row;
                const int64_t cg = r * 2 * a.N + f, cu = cg + a.N;
                const float zg = a.codes[cg] * q8_scale(a.exponents[cg / kQBlock]);
                const float zu = a.codes[cu] * q8_scale(a.exponents[cu / kQBlock]);
                const float s = sigmoid_f(zg), w = a.row_weight[r], g = sz[row][i % kT];
                const float act = zg * s * zu;
                a.dz[cg] = __float2bfloat16_rn(g * w * zu * (s * (1.0f + zg * (1.0f - s))));
                a.dz[cu] = __float2bfloat16_rn(g * w * zg * s);
                a.out[r * a.N + f] = __float2bfloat16_rn(act * w);
                part = g * act;
            }
            part = warp_sum(part);
            const int strip = (n0 + (i % kT)) / 32;
            if (lane == 0 && row < nr && strip * 32 < a.N) a.strips[(int64_t)strip * a.R + r0 + row] = part;
        }
    }
}

__global__ void __launch_bounds__(256) weight_grad_simple_kernel(const WeightGradArgs a) {
    __shared__ float sp[kKs][kT + 1], sq[kKs][kT + 1];
    const int e = blockIdx.z, m0 = blockIdx.y * kT, n0 = blockIdx.x * kT;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int r0 = max(0, min(a.offsets[e], (int)a.R)), r1 = max(r0, min(a.offsets[e + 1], (int)a.R));
    float acc[4][4] = {};
    for (int k0 = r0; k0 < r1; k0 += kKs) {
        for (int i = threadIdx.x; i < kT * kKs; i += 256) {
            const int kk = i / kT, c = i % kT, r = k0 + kk;
            float p = 0.0f, q = 0.0f;
            if (r < r1) {
                const int rp = a.p_rows ? a.p_rows[r] : r, rq = a.q_rows ? a.q_rows[r] : r;
                if (rp < 0 || rp >= a.p_count || rq < 0 || rq >= a.q_count) {
                    if (a.status) atomicOr(a.status, kDevBadId);
                }
                if (rp >= 0 && rp < a.p_count && m0 + c < a.M) p = __bfloat162float(a.P[(int64_t)rp * a.M + m0 + c]);
                if (rq >= 0 && rq < a.q_count && n0 + c < a.N) q = __bfloat162float(a.Q[(int64_t)rq * a.N + n0 + c]);
            }
            sp[kk][c] = p;
            sq[kk][c] = q;
        }
        __syncthreads();
        for (int k = 0; k < kKs; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sp[k][ty + 16 * i], sq[k][tx + 16 * j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
            if (m < a.M && n < a.N) {
                float *d = a.dW + ((int64_t)e * a.M + m) * a.N + n;
                *d = acc[i][j] + (a.accumulate ? *d : 0.0f);
            }
        }
}

}  // namespace

cudaError_t launch_product(ProductMode mode, const ProductArgs &a, cudaStream_t s) {
    const int cols = mode == kProductUp ? a.N / 2 : a.N, per = mode == kProductUp ? kT / 2 : kT;
    const int64_t tiles = min64(a.R, (a.R + kT - 1) / kT + a.E);
    const dim3 grid((cols + per - 1) / per, (unsigned)tiles);
    if (mode == kProductPlain) product_simple_kernel<kProductPlain><<<grid, 256, 0, s>>>(a);
    else if (mode == kProductUp) product_simple_kernel<kProductUp><<<grid, 256, 0, s>>>(a);
    else product_simple_kernel<kProductUpGrad><<<grid, 256, 0, s>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_weight_grad(const WeightGradArgs &a, cudaStream_t s) {
    weight_grad_simple_kernel<<<dim3((a.N + kT - 1) / kT, (a.M + kT - 1) / kT, a.E), 256, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace dol
