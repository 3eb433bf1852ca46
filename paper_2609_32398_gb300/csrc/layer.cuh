// Internal declarations of the whole MoE layer for a few tokens (layer.cu holds its C ABI): the router
// (layer_route.cu), then the experts with their join, in one kernel for few routed rows (layer_few.cu) or
// more (layer_experts.cu); or, where bf16 experts have many tokens each, the dispatch order
// (layer_order.cu) and the grouped products.
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
    void *act;             // [T k][F]: bf16, or fp32 with codes
    float *y;              // [T k][H]
    unsigned *counters;    // kLayerCounters: tickets, ranges done, and one for each range
    int *status;
    int ranges;            // that the rows of all used weights are divided into
    int blocks;            // of out's columns (few routed rows)
    int stage_bytes;       // shared memory for the products' rows
};

constexpr int kLayerFewRows = 40;

constexpr int kLayerRanges = 200;   // at most
constexpr int kLayerCounters = 2 + kLayerRanges;

// Whether the kernel for few routed rows takes it.
bool layer_few(const LayerArgs &a, bool eight);
cudaError_t launch_layer_few(const LayerArgs &a, bool eight, int sms, cudaStream_t s);
cudaError_t launch_layer_route(const LayerArgs &a, cudaStream_t s);
// offsets [E + 1], rows [T k] and pos [T][k] of the choices in a.ids.
cudaError_t launch_layer_order(const LayerArgs &a, int *offsets, int *rows, int *pos, cudaStream_t s);
cudaError_t launch_layer_experts(LayerArgs a, bool eight, int sms, cudaStream_t s);

}  // namespace dol
