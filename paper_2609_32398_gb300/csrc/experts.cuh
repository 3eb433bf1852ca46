// Internal declarations of the expert operators (experts.cu holds their C ABI):
// the products of an MoE layer's experts on the router's dispatch order.
//
// Routed rows r = 0 .. R-1 are grouped by expert, offsets[e] .. offsets[e+1]
// belonging to expert e; the matrix rows they read are rows[r] (gathered) or r.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "dol_internal.cuh"

namespace dol {

typedef __nv_bfloat16 bf16;

// Values that share one exponent byte in an 8-bit checkpoint.
constexpr int kQBlock = 16;

// Columns of a partial sum of the combine weights' gradient.
constexpr int kStrip = 128;

enum ProductMode {
    kProductPlain = 0,   // Y[r][n] = sum_k A[r][k] W[n][k]
    kProductUp = 1,      // act[r][f] = silu(z[f]) z[F + f], and z in 8 bits
    kProductUpGrad = 2,  // the gradient of kProductUp through W2 (its values in 8 bits)
};

struct ProductArgs {
    const bf16 *A;         // [a_rows][K]
    int64_t a_rows;
    const int *rows;       // [R] or null: row r reads A[rows[r]] or A[r]
    const bf16 *W;         // [E][N][K], or [E][K][N] when transposed
    const int *offsets;    // [E + 1]
    int64_t R;
    int K, N, E;           // kProductUp: N = 2 F weight rows
    bool transposed;
    bf16 *out;             // plain: Y [R][N]; up: act [R][F]; up_grad: w act [R][F]
    float *wide;           // plain: Y [R][N] in fp32 instead of out (may be null)
    int8_t *codes;         // up: written (may be null); up_grad: read  [R][2 F]
    uint8_t *exponents;    //                                           [R][2 F / 16]
    bf16 *dz;              // up_grad: [R][2 F]
    const float *row_weight;  // up_grad: [R]
    float *strips;         // up_grad: [ceil(F / kStrip)][R], sums of g act over kStrip columns
    int *status;
};

cudaError_t launch_product(ProductMode mode, const ProductArgs &a, cudaStream_t s);

// The products of at most kFewRows routed rows without checkpoint, weights as they
// are (not transposed), and the joined ones of at most kFewTokens tokens of them, where
// out is [T][N] (experts_few.cu).  Measured on both sides (us in a graph, weights from
// memory; F = 768, 128 experts; few rows against tensor cores), for rows of different
// experts and, in brackets, all of one expert.  H = 2048, up: R = 2 4.9 and 11.5 (4.2 and
// 11.3), 8 10.1 and 14.5 (7.2 and 11.3), 16 17.3 and 24.2 (12.1 and 11.4), 24 23.5 and 27.3,
// 32 39 and 36; down: 3.7 and 8.1 (3.3 and 8.0), 6.4 and 9.8 (5.4 and 8.0), 11.1 and 14.1
// (8.4 and 8.1), 19.3 and 17.0, 25 and 19.  Joined, T k rows: 1 x 8 9.9 and 12.0 (6.0 and
// 10.5), 2 x 2 7.2 and 10.9 (5.7 and 10.2), 2 x 4 10.0 and 11.8 (6.0 and 10.3), 2 x 8 17.8
// and 16.6 (10.0 and 10.6), 16 x 1 15.5 and 10.6; H = 512: 2 x 8 5.7 and 11.6 (4.6 and 9.7).
// So sixteen rows of one expert, and two tokens of eight experts each at H = 2048, are 3 to
// 7 % slower than the other side; all else up to the limits is faster.
constexpr int64_t kFewRows = 16;
constexpr int64_t kFewTokens = 2;
cudaError_t launch_few_product(ProductMode mode, const ProductArgs &a, cudaStream_t s);
cudaError_t launch_few_join(const ProductArgs &a, const int *pos, const float *weights, int64_t T, int k,
                            cudaStream_t s);

struct WeightGradArgs {
    const bf16 *P;  // [p_count][M]
    const bf16 *Q;  // [q_count][N]
    int64_t p_count, q_count;
    const int *p_rows, *q_rows;  // [R] or null
    const int *offsets;
    int64_t R;
    int M, N, E;
    bool accumulate;
    float *dW;  // [E][M][N]
    int *status;
    uint32_t m_magic;  // of the tiles along M, set by the launch
};

cudaError_t launch_weight_grad(const WeightGradArgs &a, cudaStream_t s);

// out[t][n] = sum_q weights[t][q] Y[pos[t][q]][n] (weights null: all one) in fp32,
// rounded once.  A pos outside [offsets[0], offsets[E]) is left out and recorded.
// Y is fp32 where `wide`, else bf16.
cudaError_t launch_join(const void *Y, bool wide, const int *pos, const float *weights, const int *offsets,
                        int64_t T, int k, int N, int E, bf16 *out, int *status, cudaStream_t s);
// row_weight[r] = combine[t][q] with t = rows[r] and pos[t][q] = r; 0 for a row that no
// choice of its token names.  A pos outside [offsets[0], offsets[E]) is recorded.
cudaError_t launch_row_weights(const float *combine, const int *rows, const int *pos, const int *offsets, int E,
                               int64_t T, int k, float *row_weight, int *status, cudaStream_t s);
// dcombine[t][q] = sum over the strips of strips[.][pos[t][q]], in order; 0 for a pos
// outside [offsets[0], offsets[E])
cudaError_t launch_strip_sums(const float *strips, int n_strips, const int *pos, const int *offsets,
                              int E, int64_t R, float *dcombine, cudaStream_t s);
cudaError_t launch_checkpoint_values(const int8_t *codes, const uint8_t *exponents, int64_t rows,
                                     int cols, bf16 *values, cudaStream_t s);

// Launch as a programmatic dependent of the kernel before on `s`: the kernel calls
// griddepcontrol.wait before it touches global memory.
template <class... P, class... A>
inline cudaError_t launch_after(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// ---------------------------------------------------------------- device helpers

// The routed rows that groups hold, offsets[0] .. offsets[E] clipped to [0, R]: the others
// are written by no product, so that nothing may read what their places hold.
__device__ __forceinline__ int2 rows_of_groups(const int *offsets, int E, int64_t R) {
    const int lo = __ldg(offsets), hi = __ldg(offsets + E);
    return make_int2(max(lo, 0), (int)min64(max(hi, 0), R));
}

// 8-bit checkpoint of a block of 16 values: codes in [-127, 127] times 2^(e - 127),
// e the exponent byte.  e is the least >= 1 with max |v| <= 127 * 2^(e - 127), at most 249:
// for max |v| = m 2^x with m in [1, 2) that is x - 6 where m <= 127/64 and x - 5
// otherwise, which the addition carries out on the float's bits.  A block with a NaN
// or an infinity has e = 255 and stands for 16 NaNs.
__device__ __forceinline__ int q8_exponent(float amax) {
    const unsigned b = __float_as_uint(amax);
    if (b >= 0x7f800000u) return 255;
    const int e = (int)((b + 0x1ffffu) >> 23) - 6;
    return e < 1 ? 1 : e;
}
// 2^(127 - e) and 2^(e - 127), both normal for 1 <= e <= 249; e = 255: 0 and NaN.
__device__ __forceinline__ float q8_inverse(int e) {
    return e == 255 ? 0.0f : __uint_as_float((unsigned)(254 - e) << 23);
}
__device__ __forceinline__ float q8_scale(int e) {
    return __uint_as_float(e == 255 ? 0x7fc00000u : (unsigned)e << 23);
}
// round(v * inv), ties to even, as a byte: |v * inv| <= 127, so the sum with 1.5 * 2^23
// holds the integer in its low bits.
__device__ __forceinline__ unsigned q8_code(float v, float inv) {
    return __float_as_uint(fmaf(v, inv, 12582912.0f)) & 0xffu;
}
// Two fp32 values that one instruction works on (the epilogues are bound by how many
// instructions they issue).
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair2(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split2(f32x2 v, float &lo, float &hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// sigma(z) = 1 / (1 + 2^(-z log2 e)) of both: 2^x overflows to infinity below z = -88
// and gives 0.
__device__ __forceinline__ f32x2 sigmoid2(f32x2 z) {
    float a, b;
    split2(mul2(z, pair2(-1.44269504f, -1.44269504f)), a, b);
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    split2(add2(pair2(a, b), pair2(1.0f, 1.0f)), a, b);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    return pair2(a, b);
}

__device__ __forceinline__ float sigmoid_f(float z) {
    float a, b;
    split2(sigmoid2(pair2(z, z)), a, b);
    return a;
}

// The codes of bytes b and b + 1 of a word, sign bits turned over beforehand (word ^
// 0x80808080), times the block's scale: such a byte below the exponent of 2^23 is
// 2^23 + 128 + code.  (The conversion instruction shares its pipe with sigma's
// exponential and division.)
__device__ __forceinline__ f32x2 q8_values(unsigned word, int b, f32x2 scale) {
    const float lo = __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7440u + (unsigned)b));
    const float hi = __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7440u + (unsigned)b + 1u));
    return mul2(add2(pair2(lo, hi), pair2(-8388736.0f, -8388736.0f)), scale);
}

__device__ __forceinline__ unsigned pack2(float lo, float hi) {
    __nv_bfloat162 p = __float22bfloat162_rn(make_float2(lo, hi));
    return *reinterpret_cast<unsigned *>(&p);
}

// 16 values rounded to bf16: 32 bytes, one whole sector in one store where dst is
// aligned to it (a half sector a store costs the L2 twice the writes).
__device__ __forceinline__ void store16(bf16 *dst, const float *v) {
    unsigned w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = pack2(v[2 * i], v[2 * i + 1]);
    if ((reinterpret_cast<uintptr_t>(dst) & 31u) == 0) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(w[0]), "r"(w[1]),
                     "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4 *>(dst)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(dst)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

}  // namespace dol
