// C ABI of the whole MoE layer for a few tokens (include/doloss.h): argument checks and launches.
#include "layer.cuh"
#include "experts_abi.cuh"
#include "experts_tiles.cuh"

namespace dol {
namespace {

struct LayerRoom {
    size_t counters, act, y, all;
};
LayerRoom layer_room(int64_t R, int32_t H, int32_t F) {
    LayerRoom r = {};
    r.act = r.counters + round256(sizeof(unsigned) * kLayerCounters);
    r.y = r.act + round256(sizeof(bf16) * (size_t)R * F);
    r.all = r.y + round256(sizeof(float) * (size_t)R * H);
    return r;
}

}  // namespace
}  // namespace dol

using dol::off;

extern "C" {

size_t do_moe_layer_workspace_size(int64_t T, int32_t k, int32_t H, int32_t F) {
    if (T < 1 || k < 1 || H < 1 || F < 1 || T > dol::kLayerTokens || k > dol::kLayerChoices) return 0;
    return dol::layer_room(T * k, H, F).all;
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
    const dol::LayerRoom room = dol::layer_room(T * k, H, F);
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
    a.act = reinterpret_cast<dol::bf16 *>(ws + room.act);
    a.y = reinterpret_cast<float *>(ws + room.y);
    a.status = status_flags;
    a.ranges = sms;
    a.blocks = H < sms ? H : sms;
    const bool few = dol::layer_few(a, eight);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dol::launch_layer_route(a, s);
    if (e != cudaSuccess) return dol::of(e);
    return dol::of(few ? dol::launch_layer_few(a, eight, sms, s) : dol::launch_layer_experts(a, eight, sms, s));
}

}  // extern "C"
