// Internal declarations of the whole MoE layer for a few tokens (layer.cu holds its C ABI):
// two kernels, the router (layer_route.cu) and the experts with their join
// (layer_experts.cu).
#pragma once

#include "experts8.cuh"

namespace dol {

constexpr int kLayerTokens = 64;    // T at most
constexpr int kLayerChoices = 32;   // k at most
constexpr int kLayerExperts = 1024; // E at most
constexpr int kLayerUnits = 64;     // 128-byte pieces of a weight row at most

struct LayerArgs {
    const bf16 *x;         // [T][H]
    const bf16 *router;    // [E][H]
    const void *w1, *w2;   // bf16 [E][2 F][H] and [E][H][F], or codes
    const uint8_t *w1x, *w2x;  // the codes' exponents
    int T, H, F, E, k, gate;
    bf16 *out;             // [T][H]
    int *ids;              // [T][k]
    float *combine;        // [T][k]
    bf16 *act;             // [T k][F]
    float *y;              // [T k][H]
    unsigned *counters;    // tickets, up ranges done, arrivals at each block of out's columns
    int *status;
    int ranges;            // of the up projection
    int blocks, subsets;   // of out's columns, and of the experts for each of them
    int stage_bytes;       // shared memory for the products' rows
};

size_t layer_counters(const LayerArgs &a);
// The split of both projections' work, for `sms` SMs.
void layer_split(LayerArgs *a, int sms);
cudaError_t launch_layer_route(const LayerArgs &a, cudaStream_t s);
cudaError_t launch_layer_experts(LayerArgs a, bool eight, int sms, cudaStream_t s);

}  // namespace dol
