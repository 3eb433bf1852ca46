// The small kernels of the expert operators: the weighted join of a token's k
// routed rows, the combine weights by row, their gradient from the strip sums,
// and the values of an 8-bit checkpoint.  All are bound by memory (the join and
// the values) or by their launch (the other two).
#include "experts.cuh"
#include "tma.cuh"

namespace dol {
namespace {

__device__ __forceinline__ void add8(float (&acc)[8], uint4 v, float w) {
    const unsigned u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        acc[2 * i] = fmaf(w, __uint_as_float(u[i] << 16), acc[2 * i]);
        acc[2 * i + 1] = fmaf(w, __uint_as_float(u[i] & 0xffff0000u), acc[2 * i + 1]);
    }
}

// The pieces of a token's rows that a thread reads: up to eight choices at a time.
struct Picks {
    int row[8];   // -1: left out
    float w[8];
};
__device__ __forceinline__ Picks read_picks(const int *pos, const float *weights, int64_t t, int k, int q0,
                                            int2 in, int *status) {
    Picks p;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        p.row[q] = q0 + q < k ? __ldg(pos + t * k + q0 + q) : -1;
        p.w[q] = weights && q0 + q < k ? __ldg(weights + t * k + q0 + q) : 1.0f;
    }
    bool bad = false;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const bool out = p.row[q] < in.x || p.row[q] >= in.y;
        bad |= out && q0 + q < k;
        if (out) p.row[q] = -1;
    }
    if (bad && status) atomicOr(status, kDevBadId);
    return p;
}

// A thread has 8 columns and walks over tokens; a token's rows are read as 16-byte
// pieces, eight in flight a thread and 24 warps an SM.  A choice that is left out adds
// nothing (its row is not read).  Bound by memory: T = 16384, k = 8, N = 2048 moves 604 MB
// in about 110 us.  (The next token's positions read ahead cost the third block an SM:
// 383 against 376 us for the products and the join.)
template <typename Y>
__global__ void __launch_bounds__(256, sizeof(Y) == 2 ? 3 : 2)
join_kernel(const Y *__restrict__ y, const int *__restrict__ pos, const float *__restrict__ weights,
            const int *__restrict__ offsets, int64_t T, int k, int N, int E, int cx, bf16 *__restrict__ out,
            int *status) {
    pdl_wait();
    const int2 in = rows_of_groups(offsets, E, T * k);
    const int c = (int)blockIdx.y * 256 + (int)threadIdx.x % cx, per = 256 / cx;
    const int64_t step = (int64_t)gridDim.x * per;
    int64_t t = (int64_t)blockIdx.x * per + (int)threadIdx.x / cx;
    if (c >= N / 8 || t >= T) return;
    Picks now = read_picks(pos, weights, t, k, 0, in, status);
    for (; t < T; t += step) {
        float acc[8] = {};
        for (int q0 = 0; q0 < k; q0 += 8) {
            if constexpr (sizeof(Y) == 2) {
                uint4 v[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    v[q] = make_uint4(0, 0, 0, 0);
                    if (now.row[q] >= 0) v[q] = __ldg(reinterpret_cast<const uint4 *>(y + (int64_t)now.row[q] * N) + c);
                }
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (now.row[q] >= 0) add8(acc, v[q], now.w[q]);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float4 v[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        v[q] = make_float4(0, 0, 0, 0);
                        if (now.row[q] >= 0)
                            v[q] = __ldg(reinterpret_cast<const float4 *>(y + (int64_t)now.row[q] * N) + 2 * c + h);
                    }
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        if (now.row[q] < 0) continue;
                        acc[4 * h] = fmaf(now.w[q], v[q].x, acc[4 * h]);
                        acc[4 * h + 1] = fmaf(now.w[q], v[q].y, acc[4 * h + 1]);
                        acc[4 * h + 2] = fmaf(now.w[q], v[q].z, acc[4 * h + 2]);
                        acc[4 * h + 3] = fmaf(now.w[q], v[q].w, acc[4 * h + 3]);
                    }
                }
            }
            if (q0 + 8 < k) now = read_picks(pos, weights, t, k, q0 + 8, in, status);
            else if (t + step < T) now = read_picks(pos, weights, t + step, k, 0, in, status);
        }
        reinterpret_cast<uint4 *>(out + t * N)[c] = make_uint4(pack2(acc[0], acc[1]), pack2(acc[2], acc[3]),
                                                               pack2(acc[4], acc[5]), pack2(acc[6], acc[7]));
    }
}

// A routed row looks its choice up among its token's k (and is not told by the choice): every
// row then has a weight, also one that no choice names.
__global__ void row_weights_kernel(const float *__restrict__ combine, const int *__restrict__ rows,
                                   const int *__restrict__ pos, const int *__restrict__ offsets, int E, int64_t T,
                                   int k, float *__restrict__ row_weight, int *status) {
    pdl_wait();
    const int64_t R = T * k, r = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (r >= R) return;
    const int t = __ldg(rows + r), p = __ldg(pos + r);
    const int2 in = rows_of_groups(offsets, E, R);
    float w = 0.0f;
    if (t >= 0 && t < T) {
        const int64_t at = (int64_t)t * k;
        for (int q0 = 0; q0 < k; q0 += 8) {  // positions and weights in flight together
            int named[8];
            float c[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                named[q] = q0 + q < k ? __ldg(pos + at + q0 + q) : -1;
                c[q] = q0 + q < k ? __ldg(combine + at + q0 + q) : 0.0f;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (named[q] == r) w = c[q];
        }
    }
    row_weight[r] = w;
    if ((p < in.x || p >= in.y) && status) atomicOr(status, kDevBadId);
}

__global__ void strip_sums_kernel(const float *__restrict__ strips, int n, const int *__restrict__ pos,
                                  const int *__restrict__ offsets, int E, int64_t R, float *__restrict__ dcombine) {
    pdl_wait();
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= R) return;
    const int p = pos[i];
    const int2 in = rows_of_groups(offsets, E, R);
    float s = 0.0f;
    if (p >= in.x && p < in.y)
#pragma unroll 8
        for (int j = 0; j < n; ++j) s += strips[(int64_t)j * R + p];
    dcombine[i] = s;
}

// A thread takes two blocks of 16 codes, their loads in flight together: 16 bytes and an
// exponent in, 32 bytes out each.  131072 x 1536 values: 90.5 us, 6.8 TB/s (one block a
// thread 104.5, four 90.5).
__global__ void __launch_bounds__(256)
checkpoint_values_kernel(const uint4 *__restrict__ codes, const uint8_t *__restrict__ exponents, int64_t blocks,
                         uint4 *__restrict__ values) {
    pdl_wait();
    const int64_t i0 = (int64_t)blockIdx.x * 512 + threadIdx.x;
    uint4 c[2];
    int e[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int64_t i = i0 + 256 * u;
        c[u] = i < blocks ? __ldg(codes + i) : make_uint4(0, 0, 0, 0);
        e[u] = i < blocks ? __ldg(exponents + i) : 1;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int64_t i = i0 + 256 * u;
        if (i >= blocks) break;
        const float scale = q8_scale(e[u]);
        const f32x2 s = pair2(scale, scale);
        const unsigned w[4] = {c[u].x ^ 0x80808080u, c[u].y ^ 0x80808080u, c[u].z ^ 0x80808080u, c[u].w ^ 0x80808080u};
        float v[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) split2(q8_values(w[j / 2], 2 * (j & 1), s), v[2 * j], v[2 * j + 1]);
        store16(reinterpret_cast<bf16 *>(values + 2 * i), v);
    }
}

}  // namespace

cudaError_t launch_join(const void *Y, bool wide, const int *pos, const float *weights, const int *offsets,
                        int64_t T, int k, int N, int E, bf16 *out, int *status, cudaStream_t s) {
    int cx = 1;  // threads side by side on a token
    while (cx < 256 && cx < N / 8) cx *= 2;
    const int64_t need = (T + 256 / cx - 1) / (256 / cx);
    const unsigned gy = (unsigned)((N / 8 + 255) / 256);
    // four times what is resident at once: the last blocks even out (382 against 391 us for
    // the products and the join of 16384 tokens, H = 2048)
    const unsigned gx = (unsigned)min64(need, (12 * 152 + gy - 1) / gy);
    if (wide)
        return launch_after(join_kernel<float>, dim3(gx, gy), 256, 0, s, static_cast<const float *>(Y), pos, weights,
                            offsets, T, k, N, E, cx, out, status);
    return launch_after(join_kernel<bf16>, dim3(gx, gy), 256, 0, s, static_cast<const bf16 *>(Y), pos, weights, offsets,
                        T, k, N, E, cx, out, status);
}

cudaError_t launch_row_weights(const float *combine, const int *rows, const int *pos, const int *offsets, int E,
                               int64_t T, int k, float *row_weight, int *status, cudaStream_t s) {
    return launch_after(row_weights_kernel, dim3((unsigned)((T * k + 255) / 256)), 256, 0, s, combine, rows, pos, offsets,
                        E, T, k, row_weight, status);
}

cudaError_t launch_strip_sums(const float *strips, int n_strips, const int *pos, const int *offsets, int E,
                              int64_t R, float *dcombine, cudaStream_t s) {
    return launch_after(strip_sums_kernel, dim3((unsigned)((R + 255) / 256)), 256, 0, s, strips, n_strips, pos, offsets,
                        E, R, dcombine);
}

cudaError_t launch_checkpoint_values(const int8_t *codes, const uint8_t *exponents, int64_t rows, int cols,
                                     bf16 *values, cudaStream_t s) {
    const int64_t n = rows * (cols / kQBlock);
    return launch_after(checkpoint_values_kernel, dim3((unsigned)((n + 511) / 512)), 256, 0, s,
                        reinterpret_cast<const uint4 *>(codes), exponents, n, reinterpret_cast<uint4 *>(values));
}

}  // namespace dol
