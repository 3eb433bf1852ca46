// Internal declarations of the 8-bit expert operators (experts8.cu holds their C ABI):
// blocks of 128 values in e4m3 with one power of two, and products of such matrices.
//
// The value of a code c in a block of exponent byte e is c 2^(e - 127); e = 255 makes the
// block NaN.  Rows [M][K] have blocks of 1 x 128 and exponents [M][ceil(K / 128)],
// weights [E][N][K] blocks of 128 x 128 and exponents [E][ceil(N / 128)][ceil(K / 128)]; gate
// and up rows of W1 [E][2 F][H] are blocked apart: exponents [E][2][ceil(F / 128)][ceil(H / 128)].
#pragma once

#include <cuda_fp8.h>

#include "experts.cuh"

namespace dol {

constexpr int kBlock8 = 128;
__host__ __device__ inline int blocks8(int n) { return (n + kBlock8 - 1) / kBlock8; }

enum Product8Mode {
    kProduct8Plain = 0,  // Y[r][n] = sum_k A[r][k] W[n][k]
    kProduct8Up = 1,     // act[r][f] = silu(z[f]) z[F + f], in blocks of 1 x 128
};

struct Product8Args {
    const uint8_t *A;      // codes [a_rows][K]
    const uint8_t *ax;     // their exponents
    int64_t a_rows;
    const int *rows;       // [R] or null: row r reads A[rows[r]] or A[r]
    const uint8_t *W;      // codes [E][N][K]
    const uint8_t *wx;
    const int *offsets;    // [E + 1]; null: E = 1 and all R rows
    int64_t R;
    int K, N, E;           // kProduct8Up: N = 2 F weight rows
    bf16 *out;             // plain: Y [R][N]
    float *wide;           // plain: Y [R][N] in fp32 instead of out (may be null)
    uint8_t *codes;        // up: [R][F]
    uint8_t *exponents;    //     [R][ceil(F / 128)]
    int align;             // of rows of exponents in bytes: 4, 2 or 1, set by the launch
    int *status;
};

cudaError_t launch_product8(Product8Mode mode, const Product8Args &a, cudaStream_t s);

cudaError_t launch_quantise_rows(const bf16 *x, int64_t M, int K, uint8_t *codes, uint8_t *exponents, cudaStream_t s);
// planes of [N][K], each blocked by itself
cudaError_t launch_quantise_weights(const bf16 *w, int64_t planes, int N, int K, uint8_t *codes, uint8_t *exponents,
                                    cudaStream_t s);
// bf16 values of planes [N][K] with blocks of `block_rows` (1 or 128) x 128
cudaError_t launch_block_values(const uint8_t *codes, const uint8_t *exponents, int64_t planes, int64_t N, int K,
                                int block_rows, bf16 *values, cudaStream_t s);

// ---------------------------------------------------------------- device helpers

// The exponent byte of a block whose largest magnitude has the float bits b: the least e >=
// 3 with max |v| <= 448 2^(e - 127), at most 247.  With max |v| = m 2^x, m in [1, 2): x - 8
// where m <= 1.75 and x - 7 otherwise, which the addition carries out on the float's bits.
// From 3 on every value of a code, down to 2^-9 of the scale, is a bf16 number (2^-133 is
// the least).  255: the block holds a NaN or an infinity.
__device__ __forceinline__ int e8_exponent(unsigned b) {
    if (b >= 0x7f800000u) return 255;
    const int e = (int)((b + 0x1fffffu) >> 23) - 8;
    return e < 3 ? 3 : e;
}
// 2^(127 - e), a normal number for 3 <= e <= 247; e = 255: NaN, so that its codes are too.
__device__ __forceinline__ float e8_inverse(int e) {
    return __uint_as_float(e == 255 ? 0x7fc00000u : (unsigned)(254 - e) << 23);
}
__device__ __forceinline__ float e8_scale(int e) {
    return __uint_as_float(e == 255 ? 0x7fc00000u : e == 0 ? 0x00400000u : (unsigned)e << 23);
}
// Four values, scaled, as four codes (round to nearest even; none is over 448).
__device__ __forceinline__ unsigned e8_codes4(float a, float b, float c, float d, float inv) {
    const unsigned lo = __nv_cvt_float2_to_fp8x2(make_float2(a * inv, b * inv), __NV_SATFINITE, __NV_E4M3);
    const unsigned hi = __nv_cvt_float2_to_fp8x2(make_float2(c * inv, d * inv), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}
__device__ __forceinline__ unsigned abs_max(unsigned top, float v) {
    return max(top, __float_as_uint(v) & 0x7fffffffu);
}
// The larger of the magnitudes of a word's two bf16 values with `top` (bits of a float).
__device__ __forceinline__ unsigned abs_max2(unsigned top, unsigned w) {
    return max(max(top, (w << 16) & 0x7fffffffu), w & 0x7fff0000u);
}
__device__ __forceinline__ uint2 e8_codes8(uint4 v, float inv) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    unsigned out[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        out[i] = e8_codes4(__uint_as_float(w[2 * i] << 16), __uint_as_float(w[2 * i] & 0xffff0000u),
                           __uint_as_float(w[2 * i + 1] << 16), __uint_as_float(w[2 * i + 1] & 0xffff0000u), inv);
    return make_uint2(out[0], out[1]);
}

}  // namespace dol
