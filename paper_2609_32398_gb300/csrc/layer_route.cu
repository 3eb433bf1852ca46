// The router of a few tokens: logits z = x Wr^T, the k largest of each token and its
// combine weights, in one kernel.
//
// A cluster of eight CTAs has one token (or four or five, where there are more than eight tokens: Wr
// is then read from the L2 a quarter as often); each CTA takes an eighth of the experts,
// and the logits go through distributed shared memory to the CTA that selects for the token.
//
// The order of two experts should not hang on how a sum was split: products of two bf16
// values are exact in fp32, and their sums are kept as a pair of floats, the running sum s
// and the sum of its rounding errors.  With s' = fl(a b + s) and b' = fl(s' - s), the error is (s -
// fl(s' - b')) + (a b - b'), exact whichever of s and a b is the larger (Knuth's two-sum; a b -
// (s' - s) alone, three packed operations cheaper, is off where the product is: experts of the same
// columns in another order then differed by up to 2^-26 of the largest logit).  That costs seven
// packed operations for two products.  The pairs are what is compared, equal ones in favour of the lower
// expert.  With n = 4 ceil(H / 256) + 6 additions on a product's way, U = 2^-24 and A the sum of the
// products' magnitudes, the errors' sum is at most n U A: what its own roundings lose is at
// most 2^-38 A (H = 2048) to 2^-34 A (8192), and nothing where all products are multiples of a g
// >= n A 2^-48.
//
// Bound by latency: a token's 0.5 MB of Wr (E = 128, H = 2048) come from the L2 in a
// microsecond.  They come by asynchronous copies to shared memory, 4 KB of each row at a time, all
// on their way together (loads to registers the compiler spread over the sums, which cost one
// token's call 2 us of 26 and that of 48 tokens 3 of 109).
#include "doloss.h"
#include "experts_mma.cuh"
#include "layer_device.cuh"

namespace dol {
namespace {

constexpr int kCluster = 8, kChunk = 256, kThreads = 512, kWarps = kThreads / 32;
typedef unsigned long long u64;

// (s, c) += (s2, c2): s exact with its error in c
__device__ __forceinline__ void add_pair(float &s, float &c, float s2, float c2) {
    const float t = s + s2, z = t - s, e = (s - (t - z)) + (s2 - z);
    c = (c + c2) + e;
    s = t;
}

// Larger for a larger value, never 0: the value rounded to fp32, then what that leaves (both zeros
// are one value; fp64 would order the same and takes 60 cycles an instruction).  NaNs are one value above
// all others, whatever their bits, so that a token that holds one still has k different experts.
__device__ __forceinline__ unsigned order_of(float v) {
    const unsigned b = __float_as_uint(v + 0.0f);
    return v != v ? 0xffffffffu : (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned o) { return __uint_as_float((o >> 31) ? o ^ 0x80000000u : ~o); }
__device__ __forceinline__ u64 order_key(float s, float c) {
    const float z = s + c, d = z - s, rest = (s - (z - d)) + (c - d);
    return (u64)order_of(z) << 32 | order_of(rest);
}

__device__ __forceinline__ void store_remote(uint32_t addr, u64 v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}

// The k largest keys of one token, by the whole CTA: chosen[q] and top[q]; keys are in its shared
// memory.  Up to 256 experts each key counts the ones before it, a few threads a key (k rounds of
// a maximum over a warp took 2.4 us for k = 8); with more a warp takes the rounds.
__device__ __forceinline__ void select(u64 *keys, int E, int k, int *chosen, u64 *top) {
    const int lane = threadIdx.x & 31;
    if (E <= 256) {
        // threads a key: as many as there are
        const int shift = E <= 32 ? 4 : E <= 64 ? 3 : E <= 128 ? 2 : 1, share = 1 << shift;
        for (int base = 0; base < E << shift; base += kThreads) {
            const int i = base + (int)threadIdx.x, e = i >> shift, from = i & (share - 1);
            const u64 mine = e < E ? keys[e] : 0;
            int before = 0;
#pragma unroll 8
            for (int j = from; j < E; j += share) {
                const u64 other = keys[j];
                before += other > mine || (other == mine && j < e);
            }
            for (int o = 1; o < share; o *= 2) before += __shfl_xor_sync(kFull, before, o);
            if (e < E && (i & (share - 1)) == 0 && before < k) {
                chosen[before] = e;
                top[before] = mine;
            }
        }
    } else if (threadIdx.x < 32) {  // a lane owns experts lane, lane + 32, ...
        u64 best = 0;
        int best_e = 0x7fffffff;
        auto scan = [&]() {
            best = 0;
            best_e = 0x7fffffff;
            for (int e = lane; e < E; e += 32) {
                const u64 v = keys[e];
                if (v > best) {
                    best = v;
                    best_e = e;
                }
            }
        };
        scan();
        for (int q = 0; q < k; ++q) {
            const unsigned hi = (unsigned)(best >> 32), high = __reduce_max_sync(kFull, hi);
            const unsigned lo = hi == high ? (unsigned)best : 0u, low = __reduce_max_sync(kFull, lo);
            const unsigned e = __reduce_min_sync(kFull, hi == high && lo == low ? (unsigned)best_e : 0x7fffffffu);
            if ((unsigned)best_e == e) {
                chosen[q] = (int)e;
                top[q] = best;
                keys[e] = 0;
                scan();
            }
        }
    }
    __syncthreads();
}

// A token's choice and its weights, by one warp; the sigmoids over a common factor where they
// could all underflow.
__device__ __forceinline__ void write_choice(const int *chosen, const u64 *top, const LayerArgs &p, int t, int lane) {
    const bool in = lane < p.k;
    const float zf = in ? value_of((unsigned)(top[lane] >> 32)) : 0.0f, rest = in ? value_of((unsigned)top[lane]) : 0.0f;
    const float first = __shfl_sync(kFull, zf, 0), d = (zf - first) + (rest - __shfl_sync(kFull, rest, 0));
    float w;
    if (p.gate == DO_GATE_SOFTMAX) w = expf(d);
    else if (first >= 0.0f) w = 1.0f / (1.0f + expf(-zf));
    else w = expf(d) / (1.0f + expf(zf));
    const float sum = warp_sum(in ? w : 0.0f);
    if (in) {
        const int at = t * p.k + lane;
        p.ids[at] = chosen[lane];
        p.combine[at] = w / sum;
    }
}

// A warp takes one of the CTA's experts for kTokens tokens at a time.
template <int kTokens>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads, 1)
layer_route_kernel(const LayerArgs p) {
    __shared__ u64 keys[kLayerExperts];
    pdl_wait();
    pdl_trigger();  // the experts' CTAs come up meanwhile, read the tokens and wait for this kernel's end
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank(), t0 = (int)(blockIdx.x / kCluster) * kTokens;
    if (blockIdx.x == 0 && threadIdx.x < kLayerCounters) p.counters[threadIdx.x] = 0;
    const int per = (p.E + kCluster - 1) / kCluster, e1 = min(p.E, (rank + 1) * per), pieces = p.H / 8;
    const uint4 *x = reinterpret_cast<const uint4 *>(p.x), *wr = reinterpret_cast<const uint4 *>(p.router);
    const uint32_t keys_at = smem_u32(keys);
    const f32x2 minus = pair2(-1.0f, -1.0f);
    // tokens [kTokens], then each warp's expert, kChunk pieces of 8 columns of them at a time
    extern __shared__ __align__(16) uint4 rows[];
    uint4 *mine = rows + (kTokens + warp) * kChunk;
    cluster_sync_all();  // every CTA of the cluster has begun: its shared memory may be written
    for (int first = rank * per; first < e1; first += kWarps) {
        const int e = first + warp;
        f32x2 s[kTokens], c[kTokens];
#pragma unroll
        for (int t = 0; t < kTokens; ++t) s[t] = c[t] = pair2(0.0f, 0.0f);
        for (int from = 0; from < pieces; from += kChunk) {
            const int n = min(kChunk, pieces - from);
            __syncthreads();  // the chunk before has been read
            if (e < e1)
                for (int at = lane; at < n; at += 32) cp_async16(smem_u32(mine + at), wr + (int64_t)e * pieces + from + at, true);
#pragma unroll
            for (int t = 0; t < kTokens; ++t)
                for (int at = threadIdx.x; at < n; at += kThreads)
                    cp_async16(smem_u32(rows + t * kChunk + at), x + (int64_t)min(t0 + t, p.T - 1) * pieces + from + at, true);
            copies_sent();
            wait_copies<0>();
            __syncthreads();
            if (e < e1) {
#pragma unroll 2
                for (int at = lane; at < n; at += 32) {
                    const uint4 wv = mine[at];
                    uint4 xv[kTokens];
#pragma unroll
                    for (int t = 0; t < kTokens; ++t) xv[t] = rows[t * kChunk + at];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f32x2 w2 = unpack2(word(wv, j));
#pragma unroll
                        for (int t = 0; t < kTokens; ++t) {
                            const f32x2 v = unpack2(word(xv[t], j));
                            const f32x2 sum = fma2(w2, v, s[t]), back = fma2(sum, minus, s[t]);  // -b'
                            const f32x2 of_s = fma2(add2(sum, back), minus, s[t]), of_ab = fma2(w2, v, back);
                            c[t] = add2(c[t], add2(of_s, of_ab));
                            s[t] = sum;
                        }
                    }
                }
            }
        }
        // over the two halves and the lanes: while there are several values, half of the lanes
        // go on with half of them
        constexpr int kValues = kTokens == 1 ? 1 : kTokens <= 4 ? 4 : 8;  // zeros past kTokens
        static_assert(kTokens <= kCluster, "");
        float vs[kValues] = {}, vc[kValues] = {};
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
            float s_hi, c_hi;
            split2(s[t], vs[t], s_hi);
            split2(c[t], vc[t], c_hi);
            add_pair(vs[t], vc[t], s_hi, c_hi);
        }
        int token = 0, o = 16;
#pragma unroll
        for (int n = kValues / 2; n >= 1; n >>= 1, o >>= 1) {
            const bool up = lane & o;
            token += up ? n : 0;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float other_s = __shfl_xor_sync(kFull, up ? vs[i] : vs[i + n], o);
                const float other_c = __shfl_xor_sync(kFull, up ? vc[i] : vc[i + n], o);
                vs[i] = up ? vs[i + n] : vs[i];
                vc[i] = up ? vc[i + n] : vc[i];
                add_pair(vs[i], vc[i], other_s, other_c);
            }
        }
        const int whole = 2 * o - 1;  // lanes that end with the same value
        for (; o >= 1; o >>= 1) {
            const float other_s = __shfl_xor_sync(kFull, vs[0], o), other_c = __shfl_xor_sync(kFull, vc[0], o);
            add_pair(vs[0], vc[0], other_s, other_c);
        }
        if ((lane & whole) == 0 && token < kTokens && e < e1) {
            uint32_t to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(keys_at + 8u * (uint32_t)e), "r"(token));
            store_remote(to, order_key(vs[0], vc[0]));
        }
    }
    cluster_sync_all();
    if (rank < kTokens && t0 + rank < p.T) {
        __shared__ int chosen[kLayerChoices];
        __shared__ u64 top[kLayerChoices];
        select(keys, p.E, p.k, chosen, top);
        if (warp == 0) write_choice(chosen, top, p, t0 + rank, lane);
    }
}

// A CTA asks for more than half of an SM's shared memory and has it to itself: with room for two, a
// cluster's eight share four SMs.  Fifteen clusters fit that way, so that more than 60 tokens go by fives.
// The layer's call in a graph, H = 2048, F = 768, 8 of 128 experts, bf16 (us): CTAs alone against two to an
// SM, 8 tokens 87.6 and 89.9, 48 tokens 193.8 and 198.8; 64 tokens by fives 204.1, by fours alone, whose
// sixteenth cluster waits for another's end, 210.0, by fours two to an SM 207.6.
constexpr size_t kAlone = 116 * 1024;

template <int kTokens>
cudaError_t launch(const LayerArgs &a, cudaStream_t s) {
    constexpr auto kernel = layer_route_kernel<kTokens>;
    static_assert((kTokens + kWarps) * kChunk * sizeof(uint4) <= kAlone, "");
    const cudaError_t e = ensure_smem_limit<kernel>(kAlone);
    if (e != cudaSuccess) return e;
    return launch_after(kernel, dim3((unsigned)(kCluster * ((a.T + kTokens - 1) / kTokens))), kThreads, kAlone, s, a);
}

}  // namespace

cudaError_t launch_layer_route(const LayerArgs &a, cudaStream_t s) {
    return a.T <= 8 ? launch<1>(a, s) : a.T <= 60 ? launch<4>(a, s) : launch<5>(a, s);
}

}  // namespace dol
