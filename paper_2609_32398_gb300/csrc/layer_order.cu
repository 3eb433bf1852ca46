// The dispatch order of a few tokens' choices, by one CTA: for the layer's path on the grouped
// products, where an expert has many tokens (see layer.cu).  The order within a group is of no
// consequence: a row's products do not depend on its column, and the join goes by pos.
#include "layer_device.cuh"

namespace dol {
namespace {

constexpr int kThreads = 512, kEach = kLayerExperts / kThreads, kRoutes = kLayerTokens * kLayerChoices / kThreads;

__global__ void __launch_bounds__(kThreads) layer_order_kernel(const LayerArgs p, int *offsets, int *rows, int *pos) {
    __shared__ int count[kLayerExperts], part[kThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, R = p.T * p.k;
    for (int e = threadIdx.x; e < kLayerExperts; e += kThreads) count[e] = 0;
    pdl_wait();
    __syncthreads();
    int id[kRoutes], rank[kRoutes];
#pragma unroll
    for (int i = 0; i < kRoutes; ++i) {
        const int r = (int)threadIdx.x + i * kThreads;
        id[i] = r < R ? __ldcg(p.ids + r) : -1;
        if (id[i] >= 0) rank[i] = atomicAdd(&count[id[i]], 1);
    }
    __syncthreads();
    int c[kEach], mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) mine += c[i] = count[kEach * threadIdx.x + i];
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(kFull, sum, o);
        if (lane >= o) sum += v;
    }
    if (lane == 31) part[warp] = sum;
    __syncthreads();
    int before = sum - mine;
    for (int w = 0; w < warp; ++w) before += part[w];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int e = kEach * (int)threadIdx.x + i;
        count[e] = before;
        if (e < p.E) offsets[e] = before;
        before += c[i];
    }
    if (threadIdx.x == 0) offsets[p.E] = R;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRoutes; ++i) {
        const int r = (int)threadIdx.x + i * kThreads;
        if (id[i] < 0) continue;
        const int at = count[id[i]] + rank[i];
        rows[at] = r / p.k;
        pos[r] = at;
    }
    pdl_trigger();
}

}  // namespace

cudaError_t launch_layer_order(const LayerArgs &a, int *offsets, int *rows, int *pos, cudaStream_t s) {
    return launch_after(layer_order_kernel, dim3(1), kThreads, 0, s, a, offsets, rows, pos);
}

}  // namespace dol
