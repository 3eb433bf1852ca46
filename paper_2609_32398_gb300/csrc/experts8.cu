// C ABI of the 8-bit expert operators (include/doloss.h): argument checks and launches.
#include "experts8.cuh"
#include "experts_abi.cuh"
#include "experts_mma.cuh"

namespace dol {
namespace {

// Whether the tiles of one expert (at most 240 rows each; narrower ones only where there
// are few) are divided exactly by its weight tiles.
do_status check_tiles8(int64_t R, int32_t m_tiles) {
    return (uint64_t)((R + 239) / 240) * m_tiles > divide_limit((uint32_t)m_tiles) ? DO_ERR_UNSUPPORTED : DO_OK;
}

Product8Args product8_args(const void *A, const void *ax, int64_t a_rows, const int32_t *rows, const void *W,
                           const void *wx, const int32_t *offsets, int64_t R, int32_t K, int32_t N, int32_t E,
                           int32_t *status) {
    Product8Args a = {};
    a.A = static_cast<const uint8_t *>(A);
    a.ax = static_cast<const uint8_t *>(ax);
    a.a_rows = a_rows;
    a.rows = rows;
    a.W = static_cast<const uint8_t *>(W);
    a.wx = static_cast<const uint8_t *>(wx);
    a.offsets = offsets;
    a.R = R;
    a.K = K;
    a.N = N;
    a.E = E;
    a.status = status;
    return a;
}

// Workspace of do_expert_ffn8: the quantised tokens and activations, and what a join takes.
struct FfnRoom {
    size_t x, xe, act, acte, y, all;
};
FfnRoom ffn_room(int64_t T, int32_t k, int32_t H, int32_t F) {
    FfnRoom r = {};
    const size_t R = (size_t)T * k;
    r.xe = r.x + round256((size_t)T * H);
    r.act = r.xe + round256((size_t)T * blocks8(H));
    r.acte = r.act + round256(R * F);
    r.y = r.acte + round256(R * blocks8(F));
    r.all = r.y + join_bytes((int64_t)R, H);
    return r;
}

}  // namespace
}  // namespace dol

using dol::off;

extern "C" {

do_status do_quantise_rows(const void *X, int64_t M, int32_t K, void *codes, void *exponents, void *stream) {
    if (!X || !codes || !exponents || M < 1 || K < 1 || off(X, 16) || off(codes, 16)) return DO_ERR_INVALID_ARG;
    if (K % 16 || K > (1 << 17) || M > INT32_MAX - 256) return DO_ERR_UNSUPPORTED;
    return dol::of(dol::launch_quantise_rows(static_cast<const dol::bf16 *>(X), M, K, static_cast<uint8_t *>(codes),
                                             static_cast<uint8_t *>(exponents), static_cast<cudaStream_t>(stream)));
}

do_status do_quantise_weights(const void *W, int32_t E, int32_t N, int32_t K, int32_t gated, void *codes,
                              void *exponents, void *stream) {
    if (!W || !codes || !exponents || E < 1 || N < 1 || K < 1 || off(W, 16) || off(codes, 16) ||
        (gated != 0 && gated != 1) || (gated && N % 2))
        return DO_ERR_INVALID_ARG;
    if (E > 1024 || K % 16 || K > (1 << 17) || N > (1 << 18)) return DO_ERR_UNSUPPORTED;
    return dol::of(dol::launch_quantise_weights(static_cast<const dol::bf16 *>(W), gated ? 2 * E : E, gated ? N / 2 : N, K,
                                                static_cast<uint8_t *>(codes), static_cast<uint8_t *>(exponents),
                                                static_cast<cudaStream_t>(stream)));
}

do_status do_block_values(const void *codes, const void *exponents, int64_t planes, int64_t N, int32_t K,
                          int32_t block_rows, void *values, void *stream) {
    if (!codes || !exponents || !values || planes < 1 || N < 1 || K < 1 || off(codes, 16) || off(values, 16) ||
        (block_rows != 1 && block_rows != dol::kBlock8))
        return DO_ERR_INVALID_ARG;
    if (K % 16 || K > (1 << 17) || planes > INT32_MAX || N > INT32_MAX ||
        planes * N > (int64_t)512 * INT32_MAX / (K / 16))
        return DO_ERR_UNSUPPORTED;
    return dol::of(dol::launch_block_values(static_cast<const uint8_t *>(codes), static_cast<const uint8_t *>(exponents),
                                            planes, N, K, block_rows, static_cast<dol::bf16 *>(values),
                                            static_cast<cudaStream_t>(stream)));
}

do_status do_grouped_matmul8(const void *A, const void *A_exponents, const void *W, const void *W_exponents,
                             const int32_t *rows, const int32_t *offsets, int64_t T, int32_t K, int32_t N, int32_t E,
                             int64_t R, void *Y, int32_t *status_flags, void *stream) {
    do_status st = dol::check_sizes(R, E, K, N, 16, 8);
    if (st != DO_OK) return st;
    if (!A || !A_exponents || !W || !W_exponents || !Y || T < 1 || (!offsets && E != 1)) return DO_ERR_INVALID_ARG;
    if (!rows && T < R) return DO_ERR_INVALID_ARG;
    if (off(A, 16) || off(W, 16) || off(Y, 16) || off(offsets, 4) || off(rows, 4) || off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    if (T > INT32_MAX - 256) return DO_ERR_UNSUPPORTED;
    st = dol::check_tiles8(R, (N + 255) / 256);
    if (st != DO_OK) return st;
    dol::Product8Args a =
        dol::product8_args(A, A_exponents, T, rows, W, W_exponents, offsets, R, K, N, E, status_flags);
    a.out = static_cast<dol::bf16 *>(Y);
    return dol::of(dol::launch_product8(dol::kProduct8Plain, a, static_cast<cudaStream_t>(stream)));
}

do_status do_expert_up8(const void *X, const void *X_exponents, const void *W1, const void *W1_exponents,
                        const int32_t *rows, const int32_t *offsets, int64_t T, int32_t H, int32_t F, int32_t E,
                        int64_t R, void *act, void *act_exponents, int32_t *status_flags, void *stream) {
    do_status st = dol::check_sizes(R, E, H, F, 16, 16);
    if (st != DO_OK) return st;
    if (!X || !X_exponents || !W1 || !W1_exponents || !offsets || !act || !act_exponents || T < 1)
        return DO_ERR_INVALID_ARG;
    if (!rows && T < R) return DO_ERR_INVALID_ARG;
    if (off(X, 16) || off(W1, 16) || off(act, 16) || off(offsets, 4) || off(rows, 4) || off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    if (T > INT32_MAX - 256) return DO_ERR_UNSUPPORTED;
    st = dol::check_tiles8(R, (F + 127) / 128);
    if (st != DO_OK) return st;
    dol::Product8Args a =
        dol::product8_args(X, X_exponents, T, rows, W1, W1_exponents, offsets, R, H, 2 * F, E, status_flags);
    a.codes = static_cast<uint8_t *>(act);
    a.exponents = static_cast<uint8_t *>(act_exponents);
    return dol::of(dol::launch_product8(dol::kProduct8Up, a, static_cast<cudaStream_t>(stream)));
}

size_t do_expert_ffn8_workspace_size(int64_t T, int32_t k, int32_t H, int32_t F) {
    if (T < 1 || k < 1 || H < 1 || F < 1 || T > INT32_MAX / k) return 0;
    return dol::ffn_room(T, k, H, F).all;
}

do_status do_expert_ffn8(const void *X, const void *W1, const void *W1_exponents, const void *W2,
                         const void *W2_exponents, const float *combine, const int32_t *rows, const int32_t *offsets,
                         const int32_t *pos, int64_t T, int32_t k, int32_t H, int32_t F, int32_t E, void *out,
                         int32_t *status_flags, void *workspace, size_t workspace_bytes, void *stream) {
    if (T < 1 || k < 1) return DO_ERR_INVALID_ARG;
    if (T > INT32_MAX / k) return DO_ERR_UNSUPPORTED;
    const int64_t R = T * k;
    do_status st = dol::check_sizes(R, E, H, F, 16, 16);
    if (st != DO_OK) return st;
    if (!X || !W1 || !W1_exponents || !W2 || !W2_exponents || !combine || !rows || !offsets || !pos || !out)
        return DO_ERR_INVALID_ARG;
    if (off(X, 16) || off(W1, 16) || off(W2, 16) || off(out, 16) || off(combine, 4) || off(rows, 4) ||
        off(offsets, 4) || off(pos, 4) || off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    st = dol::check_tiles8(R, (F + 127) / 128);
    if (st == DO_OK) st = dol::check_tiles8(R, (H + 255) / 256);
    if (st != DO_OK) return st;
    const dol::FfnRoom room = dol::ffn_room(T, k, H, F);
    if (!workspace || off(workspace, 256) || workspace_bytes < room.all) return DO_ERR_WORKSPACE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    cudaError_t e =
        dol::launch_quantise_rows(static_cast<const dol::bf16 *>(X), T, H, ws + room.x, ws + room.xe, s);
    if (e != cudaSuccess) return dol::of(e);
    dol::Product8Args a = dol::product8_args(ws + room.x, ws + room.xe, T, rows, W1, W1_exponents, offsets, R, H, 2 * F,
                                             E, status_flags);
    a.codes = ws + room.act;
    a.exponents = ws + room.acte;
    e = dol::launch_product8(dol::kProduct8Up, a, s);
    if (e != cudaSuccess) return dol::of(e);
    const bool wide = dol::join_wide(R, H);
    a = dol::product8_args(ws + room.act, ws + room.acte, R, nullptr, W2, W2_exponents, offsets, R, F, H, E,
                           status_flags);
    a.wide = wide ? reinterpret_cast<float *>(ws + room.y) : nullptr;
    a.out = reinterpret_cast<dol::bf16 *>(ws + room.y);
    e = dol::launch_product8(dol::kProduct8Plain, a, s);
    if (e != cudaSuccess) return dol::of(e);
    return dol::of(dol::launch_join(ws + room.y, wide, pos, combine, offsets, T, k, H, E, static_cast<dol::bf16 *>(out),
                                    status_flags, s));
}

}  // extern "C"
