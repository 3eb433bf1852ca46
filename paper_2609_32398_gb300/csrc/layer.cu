// C ABI of the whole MoE layer for a few tokens (include/doloss.h): argument checks, and which kernels.
#include "layer.cuh"
#include "experts_abi.cuh"
#include "experts_tiles.cuh"

namespace dol {
namespace {

// Of the two kernels for a few tokens: counters, activations, results; of the grouped products: the
// dispatch order and what do_expert_ffn takes.  Both begin at 0: the second part's offsets are written after
// the router has cleared the counters, which nothing reads then.
struct LayerRoom {
    size_t counters, act, y, offsets, rows, pos, ffn, all;
};
LayerRoom layer_room(int64_t T, int32_t k, int32_t H, int32_t F) {
    LayerRoom r = {};
    const size_t R = (size_t)T * k;
    r.act = r.counters + round256(sizeof(unsigned) * kLayerCounters);
    r.y = r.act + round256(sizeof(float) * R * F);
    r.rows = r.offsets + round256(sizeof(int) * (kLayerExperts + 1));
    r.pos = r.rows + round256(sizeof(int) * R);
    r.ffn = r.pos + round256(sizeof(int) * R);
    const size_t few = r.y + round256(sizeof(float) * R * H), grouped = r.ffn + do_expert_ffn_workspace_size(T, k, H, F);
    r.all = few > grouped ? few : grouped;
    return r;
}

// bf16 weights whose experts have many tokens each go through the grouped products on tcgen05 (router,
// order, up, down, join: five kernels), which do not repeat a step for every eight tokens and every
// tile for every 32.  Measured on both sides (us in a graph; two kernels against five), H = 2048, F = 768: 64
// tokens of 8 of 8 experts 80.2 and 35.8, of 5 of 40 92.9 and 85.1, of 8 of 128 (four tokens an expert) 205 and
// 198; 16 of 8 of 8 34.6 and 32.2.  Smaller layers: H = 1024, F = 512, 64 of 4 of 16 35.4 and 27.5; H = 512, F = 256,
// 64 of 8 of 8 26.7 and 21.6, of 2 of 8 19.5 and 20.0, of 3 of 24 19.8 and 20.7, of 8 of 64 26.1 and 30.2.
bool layer_grouped(const LayerArgs &a) {
    const int64_t R = (int64_t)a.T * a.k, bytes = (int64_t)a.E * 3 * a.F * a.H * 2;
    return R >= 16 * a.E || (R >= 8 * a.E && bytes >= (64 << 20));
}

}  // namespace
}  // namespace dol

using dol::off;

extern "C" {

size_t do_moe_layer_workspace_size(int64_t T, int32_t k, int32_t H, int32_t F) {
    if (T < 1 || k < 1 || H < 1 || F < 1 || T > dol::kLayerTokens || k > dol::kLayerChoices) return 0;
    return dol::layer_room(T, k, H, F).all;
}

do_status do_moe_layer(const void *X, const void *Wr, const void *W1, const void *W1_exponents, const void *W2,
                       const void *W2_exponents, int64_t T, int32_t H, int32_t F, int32_t E, int32_t k, int32_t gate,
                       void *out, int32_t *expert_ids, float *combine, int32_t *status_flags, void *workspace,
                       size_t workspace_bytes, void *stream) {
    if (!X || !Wr || !W1 || !W2 || !out || !expert_ids || !combine || (!W1_exponents) != (!W2_exponents))
        return DO_ERR_INVALID_ARG;
    if (T < 1 || H < 1 || F < 1 || E < 1 || k < 1 || k > E || (gate != DO_GATE_SIGMOID_NORM && gate != DO_GATE_SOFTMAX))
        return DO_ERR_INVALID_ARG;
    if (off(X, 16) || off(Wr, 16) || off(W1, 16) || off(W2, 16) || off(out, 16) || off(expert_ids, 4) ||
        off(combine, 4) || off(status_flags, 4))
        return DO_ERR_INVALID_ARG;
    const bool eight = W1_exponents != nullptr;
    const int widest = dol::kLayerUnits * (eight ? 128 : 64);
    if (T > dol::kLayerTokens || k > dol::kLayerChoices || E > dol::kLayerExperts || H > widest || F > widest ||
        H % (eight ? 16 : 8) || F % 16)
        return DO_ERR_UNSUPPORTED;
    if (!workspace || off(workspace, 256) || workspace_bytes < do_moe_layer_workspace_size(T, k, H, F))
        return DO_ERR_WORKSPACE;
    const int sms = dol::sm_count();
    if (sms < 8 || sms > dol::kLayerRanges) return DO_ERR_CUDA;
    const dol::LayerRoom room = dol::layer_room(T, k, H, F);
    char *ws = static_cast<char *>(workspace);
    dol::LayerArgs a = {};
    a.x = static_cast<const dol::bf16 *>(X);
    a.router = static_cast<const dol::bf16 *>(Wr);
    a.w1 = W1;
    a.w2 = W2;
    a.w1x = static_cast<const uint8_t *>(W1_exponents);
    a.w2x = static_cast<const uint8_t *>(W2_exponents);
    a.T = (int)T;
    a.H = H;
    a.F = F;
    a.E = E;
    a.k = k;
    a.gate = gate;
    a.out = static_cast<dol::bf16 *>(out);
    a.ids = expert_ids;
    a.combine = combine;
    a.counters = reinterpret_cast<unsigned *>(ws + room.counters);
    a.act = ws + room.act;
    a.y = reinterpret_cast<float *>(ws + room.y);
    a.status = status_flags;
    a.ranges = sms;
    a.blocks = H < sms ? H : sms;
    const bool few = dol::layer_few(a, eight);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dol::launch_layer_route(a, s);
    if (e != cudaSuccess) return dol::of(e);
    if (!eight && !few && dol::layer_grouped(a)) {
        int *offsets = reinterpret_cast<int *>(ws + room.offsets), *rows = reinterpret_cast<int *>(ws + room.rows);
        int *pos = reinterpret_cast<int *>(ws + room.pos);
        const cudaError_t o = dol::launch_layer_order(a, offsets, rows, pos, s);
        if (o != cudaSuccess) return dol::of(o);
        return do_expert_ffn(X, W1, W2, combine, rows, offsets, pos, T, k, H, F, E, out, status_flags, ws + room.ffn,
                             room.all - room.ffn, stream);
    }
    return dol::of(few ? dol::launch_layer_few(a, eight, sms, s) : dol::launch_layer_experts(a, eight, sms, s));
}

}  // extern "C"
