// To and from blocks of 128 in e4m3: rows (1 x 128), weights (128 x 128) and the values
// that codes stand for.  Every value is read once and nothing is computed twice, so that the
// memory bounds all three.  The power of two makes the scaling exact; the one rounding is
// the code's (half a step of 2^-3 of its binade).
#include <climits>

#include "experts8.cuh"
#include "tma.cuh"

namespace dol {
namespace {

// Sixteen lanes hold a block of a row, eight values each; a thread takes kTurns blocks with
// their loads in flight together.
constexpr int kTurns = 4;

__global__ void __launch_bounds__(256)
quantise_rows_kernel(const uint4 *__restrict__ x, int64_t M, int K, uint2 *__restrict__ codes,
                     uint8_t *__restrict__ exponents) {
    pdl_wait();
    const int nb = blocks8(K), pieces = K / 8, piece = threadIdx.x & 15;
    const int64_t n = M * nb, i0 = (int64_t)blockIdx.x * (16 * kTurns) + (threadIdx.x >> 4);
    // one division a thread, in 32 bits where that does
    int64_t row = n <= INT_MAX ? (int64_t)((unsigned)i0 / (unsigned)nb) : i0 / nb;
    int block = (int)(i0 - row * nb);
    uint4 v[kTurns];
    int64_t at[kTurns];
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        const int c = block * 16 + piece;
        at[u] = row < M && c < pieces ? row * pieces + c : -1;
        v[u] = at[u] >= 0 ? __ldg(x + at[u]) : make_uint4(0, 0, 0, 0);
        for (block += 16; block >= nb; block -= nb) ++row;
    }
#pragma unroll
    for (int u = 0; u < kTurns; ++u) {
        unsigned top = abs_max2(abs_max2(abs_max2(abs_max2(0u, v[u].x), v[u].y), v[u].z), v[u].w);
#pragma unroll
        for (int o = 1; o < 16; o *= 2) top = max(top, __shfl_xor_sync(kFull, top, o));
        const int e = e8_exponent(top);
        if (at[u] >= 0) codes[at[u]] = e8_codes8(v[u], e8_inverse(e));
        if (piece == 0 && i0 + 16 * u < n) exponents[i0 + 16 * u] = (uint8_t)e;
    }
}

// A CTA has one block: 16 rows of 16 pieces at a time, all of it in registers between the
// largest value and the codes.
__global__ void __launch_bounds__(256)
quantise_weights_kernel(const uint4 *__restrict__ w, int N, int K, uint2 *__restrict__ codes,
                        uint8_t *__restrict__ exponents) {
    __shared__ unsigned s_top[8];
    pdl_wait();
    const int pieces = K / 8, nb = blocks8(K), kb = blockIdx.x % nb, mb = blockIdx.x / nb;
    const int c = kb * 16 + (threadIdx.x & 15), r0 = mb * kBlock8 + (threadIdx.x >> 4);
    const int64_t plane = (int64_t)blockIdx.y * N;
    uint4 v[8];
    unsigned top = 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const bool in = c < pieces && r0 + 16 * u < N;
        v[u] = in ? __ldg(w + (plane + r0 + 16 * u) * pieces + c) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) top = abs_max2(abs_max2(abs_max2(abs_max2(top, v[u].x), v[u].y), v[u].z), v[u].w);
    top = __reduce_max_sync(kFull, top);
    if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, s_top[i]);
    const int e = e8_exponent(top);
    const float inv = e8_inverse(e);
#pragma unroll
    for (int u = 0; u < 8; ++u)
        if (c < pieces && r0 + 16 * u < N) codes[(plane + r0 + 16 * u) * pieces + c] = e8_codes8(v[u], inv);
    if (threadIdx.x == 0) exponents[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = (uint8_t)e;
}

// A thread has 16 codes at a time: 16 bytes in, 32 out.  `block_rows` rows share exponents.
__global__ void __launch_bounds__(256)
block_values_kernel(const uint4 *__restrict__ codes, const uint8_t *__restrict__ exponents, int64_t n, int64_t N, int K,
                    int block_rows, bf16 *__restrict__ values) {
    pdl_wait();
    const int64_t i0 = (int64_t)blockIdx.x * 512 + threadIdx.x;
    const int pieces = K / 16, nb = blocks8(K);
    const int64_t mb = (N + block_rows - 1) / block_rows;
    uint4 c[2];
    int e[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int64_t i = i0 + 256 * u;
        c[u] = make_uint4(0, 0, 0, 0);
        e[u] = 3;
        if (i < n) {
            const int64_t row = i / pieces;
            int64_t at = row;
            if (block_rows > 1) at = row / N * mb + row % N / block_rows;
            c[u] = __ldg(codes + i);
            e[u] = __ldg(exponents + at * nb + (int)(i - row * pieces) / 8);
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int64_t i = i0 + 256 * u;
        if (i >= n) break;
        const float scale = e8_scale(e[u]);
        const unsigned w[4] = {c[u].x, c[u].y, c[u].z, c[u].w};
        float v[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j / 2] >> (16 * (j & 1))), __NV_E4M3);
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
            v[2 * j] = f.x * scale;
            v[2 * j + 1] = f.y * scale;
        }
        store16(values + 16 * i, v);
    }
}

}  // namespace

cudaError_t launch_quantise_rows(const bf16 *x, int64_t M, int K, uint8_t *codes, uint8_t *exponents, cudaStream_t s) {
    const int64_t n = M * blocks8(K);
    return launch_after(quantise_rows_kernel, dim3((unsigned)((n + 16 * kTurns - 1) / (16 * kTurns))), 256, 0, s,
                        reinterpret_cast<const uint4 *>(x), M, K, reinterpret_cast<uint2 *>(codes), exponents);
}

cudaError_t launch_quantise_weights(const bf16 *w, int64_t planes, int N, int K, uint8_t *codes, uint8_t *exponents,
                                    cudaStream_t s) {
    return launch_after(quantise_weights_kernel, dim3((unsigned)(blocks8(N) * blocks8(K)), (unsigned)planes), 256, 0, s,
                        reinterpret_cast<const uint4 *>(w), N, K, reinterpret_cast<uint2 *>(codes), exponents);
}

cudaError_t launch_block_values(const uint8_t *codes, const uint8_t *exponents, int64_t planes, int64_t N, int K,
                                int block_rows, bf16 *values, cudaStream_t s) {
    const int64_t n = planes * N * (K / 16);
    return launch_after(block_values_kernel, dim3((unsigned)((n + 511) / 512)), 256, 0, s,
                        reinterpret_cast<const uint4 *>(codes), exponents, n, N, K, block_rows, values);
}

}  // namespace dol
