// C ABI of the expert operators (include/doloss.h): argument checks and launches.
#include "experts_abi.cuh"
#include "experts_mma.cuh"

namespace dol {
namespace {

// Whether the up projection's tiles of one expert (at most 256 rows each; narrower ones only
// where there are few) are divided exactly by its weight tiles of 128 columns.  Of the
// other products, with at most 512 weight tiles, all that fit the memory are.
do_status check_up_tiles(int64_t R, int32_t F) {
    const int tiles = (F + 127) / 128;
    return (uint64_t)((R + 255) / 256) * tiles > divide_limit((uint32_t)tiles) ? DO_ERR_UNSUPPORTED : DO_OK;
}

cudaError_t product(ProductMode mode, const ProductArgs &a, cudaStream_t s) {
    if (a.R <= kFewRows && !a.transposed && !a.codes) return launch_few_product(mode, a, s);
    return launch_product(mode, a, s);
}

// a.out: [T][N]; workspace: join_bytes (not used by the few-row kernel).
cudaError_t product_join(ProductArgs a, const int *pos, const float *weights, int64_t T, int k, void *workspace,
                         cudaStream_t s) {
    if (a.R <= kFewRows && T <= kFewTokens && !a.transposed) return launch_few_join(a, pos, weights, T, k, s);
    bf16 *out = a.out;
    const bool wide = join_wide(a.R, a.N);
    a.wide = wide ? static_cast<float *>(workspace) : nullptr;
    a.out = static_cast<bf16 *>(workspace);
    const cudaError_t e = launch_product(kProductPlain, a, s);
    return e != cudaSuccess ? e : launch_join(workspace, wide, pos, weights, a.offsets, T, k, a.N, a.E, out, a.status, s);
}

ProductArgs product_args(const void *A, int64_t a_rows, const int32_t *rows, const void *W, const int32_t *offsets,
                         int64_t R, int32_t K, int32_t N, int32_t E, bool transposed, void *out, int32_t *status) {
    ProductArgs a = {};
    a.A = static_cast<const bf16 *>(A);
    a.a_rows = a_rows;
    a.rows = rows;
    a.W = static_cast<const bf16 *>(W);
    a.offsets = offsets;
    a.R = R;
    a.K = K;
    a.N = N;
    a.E = E;
    a.transposed = transposed;
    a.out = static_cast<bf16 *>(out);
    a.status = status;
    return a;
}

}  // namespace
}  // namespace dol

using dol::off;

extern "C" {

do_status do_expert_up(const void *X, const void *W1, const int32_t *rows, const int32_t *offsets, int64_t T,
                       int32_t H, int32_t F, int32_t E, int64_t R, void *act, void *codes, void *exponents,
                       int32_t *status_flags, void *stream) {
    do_status st = dol::check_sizes(R, E, H, F, 8, dol::kQBlock);
    if (st != DO_OK) return st;
    if (!X || !W1 || !offsets || !act || T < 1 || (!codes) != (!exponents)) return DO_ERR_INVALID_ARG;
    if (!rows && T < R) return DO_ERR_INVALID_ARG;
    if (off(X, 16) || off(W1, 16) || off(act, 16) || off(codes, 16) || off(offsets, 4) || off(rows, 4) ||
        off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    if (T > INT32_MAX - 256) return DO_ERR_UNSUPPORTED;
    st = dol::check_up_tiles(R, F);
    if (st != DO_OK) return st;
    dol::ProductArgs a = dol::product_args(X, T, rows, W1, offsets, R, H, 2 * F, E, false, act, status_flags);
    a.codes = static_cast<int8_t *>(codes);
    a.exponents = static_cast<uint8_t *>(exponents);
    return dol::of(dol::product(dol::kProductUp, a, static_cast<cudaStream_t>(stream)));
}

do_status do_checkpoint_values(const void *codes, const void *exponents, int64_t rows, int32_t cols, void *values,
                               void *stream) {
    if (!codes || !exponents || !values || rows < 1 || cols < 1) return DO_ERR_INVALID_ARG;
    if (off(codes, 16) || off(values, 16)) return DO_ERR_INVALID_ARG;
    if (cols % dol::kQBlock) return DO_ERR_UNSUPPORTED;
    return dol::of(dol::launch_checkpoint_values(static_cast<const int8_t *>(codes),
                                                 static_cast<const uint8_t *>(exponents), rows, cols,
                                                 static_cast<dol::bf16 *>(values), static_cast<cudaStream_t>(stream)));
}

do_status do_grouped_matmul(const void *A, const void *W, const int32_t *rows, const int32_t *offsets, int64_t T,
                            int32_t K, int32_t N, int32_t E, int64_t R, int32_t transposed, void *Y,
                            int32_t *status_flags, void *stream) {
    do_status st = dol::check_sizes(R, E, K, N, 8, 8);
    if (st != DO_OK) return st;
    if (!A || !W || !offsets || !Y || T < 1 || (transposed != 0 && transposed != 1)) return DO_ERR_INVALID_ARG;
    if (!rows && T < R) return DO_ERR_INVALID_ARG;
    if (off(A, 16) || off(W, 16) || off(Y, 16) || off(offsets, 4) || off(rows, 4) || off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    if (T > INT32_MAX - 256) return DO_ERR_UNSUPPORTED;
    return dol::of(dol::product(dol::kProductPlain,
                                dol::product_args(A, T, rows, W, offsets, R, K, N, E, transposed != 0, Y, status_flags),
                                static_cast<cudaStream_t>(stream)));
}

size_t do_grouped_matmul_join_workspace_size(int64_t T, int32_t k, int32_t N) {
    if (T < 1 || k < 1 || N < 1 || T > INT32_MAX / k) return 0;
    return dol::join_bytes((int64_t)T * k, N);
}

do_status do_grouped_matmul_join(const void *A, const void *W, const int32_t *offsets, const int32_t *pos,
                                 const float *weights, int64_t T, int32_t k, int32_t K, int32_t N, int32_t E,
                                 int32_t transposed, void *out, int32_t *status_flags, void *workspace,
                                 size_t workspace_bytes, void *stream) {
    if (T < 1 || k < 1) return DO_ERR_INVALID_ARG;
    if (T > INT32_MAX / k) return DO_ERR_UNSUPPORTED;
    const int64_t R = T * k;
    do_status st = dol::check_sizes(R, E, K, N, 8, 8);
    if (st != DO_OK) return st;
    if (!A || !W || !offsets || !pos || !out || (transposed != 0 && transposed != 1)) return DO_ERR_INVALID_ARG;
    if (off(A, 16) || off(W, 16) || off(out, 16) || off(offsets, 4) || off(pos, 4) || off(weights, 4) ||
        off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    if (!workspace || off(workspace, 256) || workspace_bytes < do_grouped_matmul_join_workspace_size(T, k, N))
        return DO_ERR_WORKSPACE;
    return dol::of(dol::product_join(
        dol::product_args(A, R, nullptr, W, offsets, R, K, N, E, transposed != 0, out, status_flags), pos, weights, T, k,
        workspace, static_cast<cudaStream_t>(stream)));
}

size_t do_expert_ffn_workspace_size(int64_t T, int32_t k, int32_t H, int32_t F) {
    if (T < 1 || k < 1 || H < 1 || F < 1 || T > INT32_MAX / k) return 0;
    return dol::round256(sizeof(dol::bf16) * (size_t)T * k * F) + dol::join_bytes((int64_t)T * k, H);
}

do_status do_expert_ffn(const void *X, const void *W1, const void *W2, const float *combine, const int32_t *rows,
                        const int32_t *offsets, const int32_t *pos, int64_t T, int32_t k, int32_t H, int32_t F,
                        int32_t E, void *out, int32_t *status_flags, void *workspace, size_t workspace_bytes,
                        void *stream) {
    if (T < 1 || k < 1) return DO_ERR_INVALID_ARG;
    if (T > INT32_MAX / k) return DO_ERR_UNSUPPORTED;
    const int64_t R = T * k;
    do_status st = dol::check_sizes(R, E, H, F, 8, dol::kQBlock);
    if (st != DO_OK) return st;
    if (!X || !W1 || !W2 || !combine || !rows || !offsets || !pos || !out) return DO_ERR_INVALID_ARG;
    if (off(X, 16) || off(W1, 16) || off(W2, 16) || off(out, 16) || off(combine, 4) || off(rows, 4) ||
        off(offsets, 4) || off(pos, 4) || off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    st = dol::check_up_tiles(R, F);
    if (st != DO_OK) return st;
    if (!workspace || off(workspace, 256) || workspace_bytes < do_expert_ffn_workspace_size(T, k, H, F))
        return DO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // between the products the activations are bf16, the tensor cores' operand type
    void *y = static_cast<char *>(workspace) + dol::round256(sizeof(dol::bf16) * (size_t)R * F);
    cudaError_t e = dol::product(
        dol::kProductUp, dol::product_args(X, T, rows, W1, offsets, R, H, 2 * F, E, false, workspace, status_flags), s);
    if (e == cudaSuccess)
        e = dol::product_join(
            dol::product_args(workspace, R, nullptr, W2, offsets, R, F, H, E, false, out, status_flags), pos, combine, T,
            k, y, s);
    return dol::of(e);
}

size_t do_expert_up_backward_workspace_size(int64_t T, int32_t k, int32_t F) {
    if (T < 1 || k < 1 || F < 1 || T > INT32_MAX / k) return 0;
    return dol::round256(sizeof(float) * (size_t)T * k * (1 + (size_t)(F + dol::kStrip - 1) / dol::kStrip));
}

do_status do_expert_up_backward(const void *dout, const void *W2, const void *codes, const void *exponents,
                                const float *combine, const int32_t *rows, const int32_t *offsets,
                                const int32_t *pos, int64_t T, int32_t k, int32_t H, int32_t F, int32_t E, void *dz,
                                void *act, float *dcombine, int32_t *status_flags, void *workspace,
                                size_t workspace_bytes, void *stream) {
    if (T < 1 || k < 1) return DO_ERR_INVALID_ARG;
    if (T > INT32_MAX / k) return DO_ERR_UNSUPPORTED;
    const int64_t R = T * k;
    do_status st = dol::check_sizes(R, E, H, F, 8, dol::kQBlock);
    if (st != DO_OK) return st;
    if (!dout || !W2 || !codes || !exponents || !combine || !rows || !offsets || !pos || !dz || !act || !dcombine)
        return DO_ERR_INVALID_ARG;
    if (off(dout, 16) || off(W2, 16) || off(codes, 16) || off(dz, 16) || off(act, 16) || off(combine, 4) ||
        off(rows, 4) || off(offsets, 4) || off(pos, 4) || off(dcombine, 4) || off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    if (!workspace || off(workspace, 256) || workspace_bytes < do_expert_up_backward_workspace_size(T, k, F))
        return DO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    float *row_weight = static_cast<float *>(workspace);
    dol::ProductArgs a = dol::product_args(dout, T, rows, W2, offsets, R, H, F, E, true, act, status_flags);
    a.codes = const_cast<int8_t *>(static_cast<const int8_t *>(codes));
    a.exponents = const_cast<uint8_t *>(static_cast<const uint8_t *>(exponents));
    a.dz = static_cast<dol::bf16 *>(dz);
    a.row_weight = row_weight;
    a.strips = row_weight + R;
    cudaError_t e = dol::launch_row_weights(combine, rows, pos, offsets, E, T, k, row_weight, status_flags, s);
    if (e == cudaSuccess) e = dol::launch_product(dol::kProductUpGrad, a, s);
    if (e == cudaSuccess) e = dol::launch_strip_sums(a.strips, (F + dol::kStrip - 1) / dol::kStrip, pos, offsets, E, R, dcombine, s);
    return dol::of(e);
}

do_status do_grouped_weight_grad(const void *P, const void *Q, const int32_t *p_rows, const int32_t *q_rows,
                                 const int32_t *offsets, int64_t Tp, int64_t Tq, int32_t M, int32_t N, int32_t E,
                                 int64_t R, int32_t accumulate, float *dW, int32_t *status_flags, void *stream) {
    do_status st = dol::check_sizes(R, E, M, N, 8, 8);
    if (st != DO_OK) return st;
    if (!P || !Q || !offsets || !dW || Tp < 1 || Tq < 1 || (accumulate != 0 && accumulate != 1))
        return DO_ERR_INVALID_ARG;
    if ((!p_rows && Tp < R) || (!q_rows && Tq < R)) return DO_ERR_INVALID_ARG;
    if (off(P, 16) || off(Q, 16) || off(dW, 16) || off(p_rows, 4) || off(q_rows, 4) || off(offsets, 4) ||
        off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    if (Tp > INT32_MAX - 256 || Tq > INT32_MAX - 256) return DO_ERR_UNSUPPORTED;
    dol::WeightGradArgs a = {};
    a.P = static_cast<const dol::bf16 *>(P);
    a.Q = static_cast<const dol::bf16 *>(Q);
    a.p_count = Tp;
    a.q_count = Tq;
    a.p_rows = p_rows;
    a.q_rows = q_rows;
    a.offsets = offsets;
    a.R = R;
    a.M = M;
    a.N = N;
    a.E = E;
    a.accumulate = accumulate != 0;
    a.dW = dW;
    a.status = status_flags;
    return dol::of(dol::launch_weight_grad(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
