// What the product kernels share beside their PTX: the tiles of ragged groups, the
// epilogues' turned blocks and their barriers.
#pragma once

#include "experts_mma.cuh"

namespace dol {

struct Tile {
    int e, m, r0, n, width;  // expert, weight tile, first routed row, rows, MMA width
};

// The tiles of a pair in turn: t = pair, pair + pairs, ..., the expert found by going on
// from the last one's.
struct Walk {
    const int *first, *start, *width;  // shared
    int tiles, pairs, m_tiles;
    uint32_t m_magic;
    int t, e;
    Tile tile;

    __device__ __forceinline__ bool find() {
        if (t >= tiles) return false;
        while (first[e + 1] <= t) ++e;
        const int i = t - first[e], j = divide_by(i, m_magic), w = width[e], a = start[e];
        tile.e = e;
        tile.m = i - j * m_tiles;
        tile.r0 = a + j * w;
        tile.n = min(w, start[e + 1] - tile.r0);
        tile.width = (tile.n + 15) & ~15;
        return true;
    }
    __device__ __forceinline__ bool next() {
        t += pairs;
        return find();
    }
};

__device__ __forceinline__ int next_cap(int cap) { return cap > 128 ? 128 : 64; }

// The first tile of each expert: a scan of ceil(n / cap) m_tiles over the experts.  Tiles are
// kCap rows at most, or 128 or 64 while that leaves half of the pairs without one (all of them
// multiples of 16: a width is rounded up to one, and past its cap the last tile would be empty):
// a tile's time is mostly its epilogue then, which narrower tiles divide.  bf16, T = 1000, H =
// 512, F = 256, E = 8, k = 2, against 256 rows always: the gradient 17.9 to 13.4 us, up 9.7 to 8.4,
// a plain product 8.8 to 8.4; T = 1000, H = 2048, F = 768 (48 tiles, not divided) 20.6 either way.
// Called by all kThreads threads of the CTA; returns the number of tiles, of which first[E]
// is left to the caller.  offsets null: one group of R rows.
template <int kCap, int kThreads>
__device__ __forceinline__ int tile_table(const int *offsets, int E, int64_t R, int m_tiles, int pairs, int *first,
                                          int *start, int *width, int *part) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto bound = [&](int e) {
        return offsets ? max(0, min(__ldg(offsets + e), (int)R)) : e == 0 ? 0 : (int)R;
    };
    static_assert(kCap % 16 == 0 && kCap > 128 && kCap <= 256, "");
    int carry;
    for (int cap = kCap;; cap = next_cap(cap)) {
        carry = 0;
        int wide = 0;  // some group could be divided further
        for (int base = 0; base <= E; base += kThreads) {
            const int e = base + (int)threadIdx.x;
            int c = 0, n = 0;
            if (e <= E) start[e] = bound(e);
            if (e < E) {
                n = max(0, bound(e + 1) - start[e]);
                const int nt = (n + cap - 1) / cap;
                width[e] = nt > 0 ? ((n + nt - 1) / nt + 15) & ~15 : 0;
                c = nt * m_tiles;
            }
            int x = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(kFull, x, o);
                if (lane >= o) x += y;
            }
            if (lane == 31) part[warp] = x;
            wide |= __syncthreads_or(n > next_cap(cap));
            int before = carry, all = 0;
            for (int i = 0; i < kThreads / 32; ++i) {
                if (i < warp) before += part[i];
                all += part[i];
            }
            if (e < E) first[e] = before + x - c;
            carry += all;
            __syncthreads();
        }
        if (!wide || cap == 64 || 2 * carry > pairs) break;
    }
    return carry;
}

// Named barriers of a group of four epilogue warps.
__device__ __forceinline__ void group_sync(int id) {
    asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory");
}
__device__ __forceinline__ int group_and(int id, int ok) {
    int all;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.s32 q, %1, 0;\n\t"
        "bar.red.and.pred p, %2, 128, q;\n\t"
        "selp.s32 %0, 1, 0, p;\n\t}"
        : "=r"(all)
        : "r"(ok), "r"(id)
        : "memory");
    return all;
}

// Where 16-byte piece j of row i of warp q's block lies in its 128 bytes.
__device__ __forceinline__ int turn_slot(int j, int i, int q) { return (j ^ q ^ ((i & 1) << 2)) << 4; }

__device__ __forceinline__ void load4(float *v, const unsigned char *from) {
    const float4 f = *reinterpret_cast<const float4 *>(from);
    v[0] = f.x;
    v[1] = f.y;
    v[2] = f.z;
    v[3] = f.w;
}

inline int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 0;
    return n;
}

}  // namespace dol
