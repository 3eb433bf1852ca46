// The experts of a few tokens and their join in one kernel:
//
//   out[t] = sum_q combine[t][q] W2_e (silu(W1g_e x[t]) * W1u_e x[t]),  e = ids[t][q]
//
// The weights of the experts that are used are read once, everything else is small, so that
// the memory is what bounds it and the whole design is for keeping reads in flight:
//
//  - One CTA an SM.  The rows of all used experts' W1 form one list that is divided evenly,
//    to the row: range i of n has its i-th n-th part.  For W2 each CTA has a block of out's
//    columns, for all used experts or (many tokens) for a quarter of them.
//  - A warp's part of a tile is 16 weight rows x 512 bytes at most, straight from global
//    memory to registers in the layout of the tensor cores' first operand, 64 registers a
//    thread: 128 KB in flight an SM.  (The order of k within a 16-byte piece is the same for
//    both operands, and free otherwise.)  As soon as a tile's products have read them
//    the next tile's loads leave, also over the seam between the projections, where W2's
//    do not wait for the activations.
//  - The rows, at most a few dozen a CTA, lie in shared memory: they are the tensor
//    cores' second operand (mma.sync m16n8k16: a tile of 16 x 512 bytes is 16 or 32 instructions for
//    eight tokens, a tenth of the time that its bytes take from memory, so that the larger
//    tiles of tcgen05 would have nothing to give).
//  - Warps that share a tile's k join their sums in shared memory, in order.
//
// 8-bit weights: codes are exact in fp16, and so are the rows' values times a power of two for
// each 128 of a row that puts the largest just below fp16's range (what falls below
// 2^-40 of that is lost, far below the sums' fp32).  Each block's sum is scaled by both powers
// in fp32.
//
// Order.  CTAs take tickets: first the ranges of W1, then the blocks of W2.  A block's CTA
// waits until all ranges are done, and those were all taken before, by CTAs that run: none waits
// for one that may not have been started, whatever else the GPU runs.  A block's last
// CTA joins it.  All sums have a fixed order; the wait is bounded.
#include <cuda_fp16.h>

#include "layer.cuh"
#include "tma.cuh"

namespace dol {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kPieces = 8;                     // 128-byte pieces of a row that a warp holds
constexpr int kStride = 10;                    // of a row of 8 sums: no bank conflicts either way
constexpr int kSums = 16 * kStride;
constexpr int kRoutes = kLayerTokens * kLayerChoices;
constexpr uint32_t kSmemLimit = 232448;

struct Lists {
    alignas(16) float sums[2][kWarps][kSums];  // written in pairs
    int count[kLayerExperts];  // then the first row of each expert
    int start[kLayerExperts + 1];  // of each used expert
    unsigned short expert[kLayerExperts], row[kRoutes];
    int part[kWarps];
    int ticket, good, last;
};

__device__ __forceinline__ uint4 load_weights(const unsigned char *p, bool in) {
    uint4 v;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.s32 p, %5, 0;\n\t"
        "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
        "@p ld.global.nc.L1::no_allocate.L2::256B.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
        : "l"(p), "r"((int)in));
    return v;
}

template <bool kHalf>
__device__ __forceinline__ void mma16(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0,
                                      unsigned b1) {
    if constexpr (kHalf)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two codes of a word (the lower or the upper ones) as fp16.
template <int kUpper>
__device__ __forceinline__ unsigned codes_half2(unsigned w) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * kUpper)), __NV_E4M3);
    return (unsigned)h.x | (unsigned)h.y << 16;
}
__device__ __forceinline__ unsigned word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

__device__ __forceinline__ void warps_sync(int id, int warps) {
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory");
}

// The slots [from, to) whose rows [r0, r1) are in shared memory at a time.
struct Batch {
    int from, to, r0, r1;
};
struct Place {
    int slot, tile;
    bool valid;
};

// One projection on this CTA's share: up, the rows [lo, hi) of the list of all used experts'
// pairs of gate and up rows; down, the columns [lo, hi) of out for the slots [s0, s1).
template <bool kUp, bool k8>
struct Phase {
    const LayerArgs &p;
    Lists &s;
    unsigned char *stage;
    int lo, hi, s0, s1;
    int warp, lane, K, row_bytes, pieces, warps, group, groups, u0, nu, stride, room;
    unsigned turn;

    __device__ __forceinline__ Phase(const LayerArgs &p_, Lists &s_, unsigned char *stage_, int lo_, int hi_, int s0_, int s1_,
                     unsigned turn_)
        : p(p_), s(s_), stage(stage_), lo(lo_), hi(hi_), s0(s0_), s1(s1_), turn(turn_) {
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        K = kUp ? p.H : p.F;
        row_bytes = K * (k8 ? 1 : 2);
        pieces = (row_bytes + 127) / 128;
        warps = (pieces + kPieces - 1) / kPieces;  // that share a tile
        groups = kWarps / warps;
        group = warp / warps;
        const int each = (pieces + warps - 1) / warps;
        u0 = warp % warps * each;
        nu = max(0, min(each, pieces - u0));
        stride = pieces * (k8 ? 256 : 128) + 64;
        room = p.stage_bytes / (stride + (k8 ? 8 * pieces : 0)) & ~7;
    }

    // up: the pairs of slot that are in this range; down: its columns
    __device__ __forceinline__ int2 bounds(int slot) const {
        if (!kUp) return make_int2(lo, hi);
        return make_int2(max(lo - slot * p.F, 0), min(hi - slot * p.F, p.F));
    }
    __device__ __forceinline__ int tiles(int slot) const {
        const int2 b = bounds(slot);
        return kUp ? (b.y - b.x + 7) / 8 : (b.y - b.x + 15) / 16;
    }
    __device__ __forceinline__ int2 tile_rows(int slot, int tile) const {
        const int2 b = bounds(slot);
        const int n = tiles(slot), len = b.y - b.x;
        return make_int2(b.x + tile * len / n, b.x + (tile + 1) * len / n);
    }
    __device__ __forceinline__ void settle(Place &at, const Batch &b) const {
        at.valid = group < groups && b.r0 < b.r1;
        while (at.valid) {
            const int n = tiles(at.slot);
            if (at.tile < n) return;
            at.tile -= n;
            if (++at.slot >= b.to) at.valid = false;
        }
    }
    __device__ __forceinline__ Place first(const Batch &b) const {
        Place at{b.from, group, true};
        settle(at, b);
        return at;
    }
    // The next slots from row r0 of slot `from` on whose rows fit, or as many rows of that one.
    __device__ __forceinline__ Batch batch(int from, int r0) const {
        const int end = s.start[s1];
        if (r0 >= end) return Batch{s1, s1, end, end};
        if (s.start[from + 1] - r0 > room) return Batch{from, from + 1, r0, r0 + room};
        int a = from + 1, b = s1;  // the last slot bound that fits
        while (a < b) {
            const int m = (a + b + 1) / 2;
            if (s.start[m] - r0 <= room) a = m;
            else b = m - 1;
        }
        return Batch{from, a, r0, s.start[a]};
    }
    __device__ __forceinline__ Batch after(const Batch &b) const {
        const int from = b.r1 >= s.start[b.to] ? b.to : b.to - 1;
        return from >= s1 ? Batch{s1, s1, b.r1, b.r1} : batch(from, b.r1);
    }

    // Rows r0 .. r1 to shared memory: the columns that the weights' pieces reach, zeros past
    // K.  Sixteen lanes have 128 values.
    __device__ __forceinline__ void bring(const Batch &b) const {
        const int blocks = k8 ? pieces : (pieces + 1) / 2, n = (b.r1 - b.r0) * blocks, piece = threadIdx.x & 15;
#pragma unroll 2
        for (int base = 0; base < n; base += kThreads / 16) {
            const int i = base + (int)(threadIdx.x >> 4);
            const int r = i / blocks, c = (i - r * blocks) * 16 + piece;  // 8-value piece of the row
            uint4 v = make_uint4(0, 0, 0, 0);
            if (i < n && 8 * c < K) {
                const int from = s.row[b.r0 + r];
                if (kUp) v = __ldg(reinterpret_cast<const uint4 *>(p.x + (int64_t)(from / p.k) * K) + c);
                else v = __ldcg(reinterpret_cast<const uint4 *>(p.act + (int64_t)from * K) + c);
            }
            if constexpr (k8) {
                unsigned top = abs_max2(abs_max2(abs_max2(abs_max2(0u, v.x), v.y), v.z), v.w);
#pragma unroll
                for (int o = 1; o < 16; o *= 2) top = max(top, __shfl_xor_sync(kFull, top, o));
                // the largest value, 2^(x - 127) and more, to 2^14 and more
                const int x = (int)(top >> 23);
                const int up = x == 255 ? 127 : min(254, 268 - x);   // exponent byte of the factor
                const float f = __uint_as_float((unsigned)up << 23);
                uint4 h;
                unsigned *hw = reinterpret_cast<unsigned *>(&h);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned w = word(v, j);
                    const __half2 two = __floats2half2_rn(__uint_as_float(w << 16) * f, __uint_as_float(w & 0xffff0000u) * f);
                    hw[j] = *reinterpret_cast<const unsigned *>(&two);
                }
                if (i < n) {
                    // 16 values a lane of the tensor cores, in two halves 64 bytes apart
                    const int slot = (c >> 3) * 8 + (c & 1) * 4 + ((c >> 1) & 3);
                    *reinterpret_cast<uint4 *>(stage + r * stride + slot * 16) = h;
                    // back by 2^(127 - up), in two factors: the first one keeps a block's sum (below
                    // 2^31) in range, the second one follows the weights' scale
                    const int back = 254 - up, far = back > 127 ? 64 : 0;
                    const int e = back - far;
                    if (piece == 0)
                        *reinterpret_cast<float2 *>(stage + room * stride + 8 * (r * pieces + i - r * blocks)) =
                            make_float2(__uint_as_float(e > 0 ? (unsigned)e << 23 : 0x00400000u),
                                        __uint_as_float((unsigned)(127 + far) << 23));
                }
            } else if (i < n && 8 * c < 64 * pieces) {
                *reinterpret_cast<uint4 *>(stage + r * stride + c * 16) = v;
            }
        }
    }

    // Where a lane finds its weights of a tile: rows g and g + 8 (up: a gate row and its up row).
    struct Source {
        const unsigned char *w[2];
        const uint8_t *x[2];
        bool in[2];
    };
    __device__ __forceinline__ Source source(const Place &at) const {
        Source f = {};
        if (!at.valid) return f;
        const int2 rows = tile_rows(at.slot, at.tile);
        const int e = s.expert[at.slot], g = lane >> 2, n = rows.y - rows.x;
        f.in[0] = g < n;
        f.in[1] = kUp ? g < n : g + 8 < n;
        const unsigned char *w = static_cast<const unsigned char *>(kUp ? p.w1 : p.w2) + u0 * 128 + (lane & 3) * 16;
        const int64_t row = kUp ? (int64_t)e * 2 * p.F + rows.x + g : (int64_t)e * p.H + rows.x + g;
        f.w[0] = w + row * row_bytes;
        f.w[1] = w + (row + (kUp ? p.F : 8)) * row_bytes;
        if constexpr (k8) {
            const uint8_t *wx = kUp ? p.w1x : p.w2x;
            const int m0 = rows.x + min(g, n - 1), m1 = kUp ? m0 : rows.x + min(g + 8, n - 1);
            const int rb = kUp ? blocks8(p.F) : blocks8(p.H);
            f.x[0] = wx + ((int64_t)(kUp ? 2 * e : e) * rb + m0 / kBlock8) * pieces + u0;
            f.x[1] = wx + ((int64_t)(kUp ? 2 * e + 1 : e) * rb + m1 / kBlock8) * pieces + u0;
        }
        return f;
    }
    // Piece u of it, as registers [64-byte half][row].
    __device__ __forceinline__ void load(const Source &f, int u, uint4 (&a)[2][2], int (&x)[2]) const {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const bool in = u < nu && (u0 + u) * 128 + j * 64 + (lane & 3) * 16 < row_bytes;
#pragma unroll
            for (int i = 0; i < 2; ++i) a[j][i] = load_weights(f.w[i] + u * 128 + j * 64, in && f.in[i]);
        }
        if constexpr (k8) {
#pragma unroll
            for (int i = 0; i < 2; ++i) x[i] = u < nu && f.x[i] ? (int)__ldg(f.x[i] + u) : 127;
        }
    }

    // Sums of the tile with the eight rows from r on (of those in shared memory; past `last` the
    // last one again, whose results nobody reads).  With kRefill each piece's registers take the
    // next tile's weights as soon as they have been used.
    template <bool kRefill>
    __device__ __forceinline__ void products(uint4 (&a)[kPieces][2][2], int (&x)[kPieces][2], int r, int last, float (&d)[4],
                                             const Source &next) const {
        const int g = lane >> 2, t = lane & 3;
        const unsigned char *b = stage + min(r + g, last) * stride + t * 16 + u0 * (k8 ? 256 : 128);
        float even[4] = {0.0f, 0.0f, 0.0f, 0.0f}, odd[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int u = 0; u < kPieces; ++u) {
            if (u >= nu) break;
            if constexpr (!k8) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(b + u * 128 + j * 64);
                    const uint4 &w0 = a[u][j][0], &w1 = a[u][j][1];
                    mma16<false>(even, w0.x, w1.x, w0.y, w1.y, v.x, v.y);
                    mma16<false>(odd, w0.z, w1.z, w0.w, w1.w, v.z, v.w);
                }
            } else {
                float sum[2][4] = {};
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(b + u * 256 + j * 128 + h * 64);
                        const unsigned c0 = word(a[u][j][0], 2 * h), c1 = word(a[u][j][1], 2 * h);
                        const unsigned e0 = word(a[u][j][0], 2 * h + 1), e1 = word(a[u][j][1], 2 * h + 1);
                        mma16<true>(sum[0], codes_half2<0>(c0), codes_half2<0>(c1), codes_half2<1>(c0),
                                    codes_half2<1>(c1), v.x, v.y);
                        mma16<true>(sum[1], codes_half2<0>(e0), codes_half2<0>(e1), codes_half2<1>(e0),
                                    codes_half2<1>(e1), v.z, v.w);
                    }
                const float w0 = e8_scale(x[u][0]), w1 = e8_scale(x[u][1]);
                const unsigned char *f = stage + room * stride + 8 * (u0 + u);
                const float2 f0 = *reinterpret_cast<const float2 *>(f + 8 * pieces * min(r + 2 * t, last));
                const float2 f1 = *reinterpret_cast<const float2 *>(f + 8 * pieces * min(r + 2 * t + 1, last));
                even[0] += (sum[0][0] + sum[1][0]) * f0.x * w0 * f0.y;
                even[1] += (sum[0][1] + sum[1][1]) * f1.x * w0 * f1.y;
                even[2] += (sum[0][2] + sum[1][2]) * f0.x * w1 * f0.y;
                even[3] += (sum[0][3] + sum[1][3]) * f1.x * w1 * f1.y;
            }
            if constexpr (kRefill) load(next, u, a[u], x[u]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = even[i] + odd[i];
    }

    // The tile's sums over the warps that share it, and what becomes of them.  rows: of the list.
    __device__ __forceinline__ void finish(const float (&d)[4], int2 tile, int r0, int n) {
        float *mine = s.sums[turn & 1][warp] + (lane >> 2) * kStride + 2 * (lane & 3);
        *reinterpret_cast<float2 *>(mine) = make_float2(d[0], d[1]);
        *reinterpret_cast<float2 *>(mine + 8 * kStride) = make_float2(d[2], d[3]);
        warps_sync(1 + group, warps);
        // (the other half of the sums may be written meanwhile; this one after the next barrier)
        const float *all = s.sums[turn & 1][group * warps];
        ++turn;
        const int me = threadIdx.x - group * warps * 32;
        if constexpr (kUp) {
            for (int o = me; o < 64; o += warps * 32) {
                const int i = o & 7, col = o >> 3;
                float gate = 0.0f, up = 0.0f;
                for (int w = 0; w < warps; ++w) {
                    gate += all[w * kSums + i * kStride + col];
                    up += all[w * kSums + (i + 8) * kStride + col];
                }
                if (tile.x + i < tile.y && col < n)
                    p.act[(int64_t)s.row[r0 + col] * p.F + tile.x + i] = __float2bfloat16_rn(gate * sigmoid_f(gate) * up);
            }
        } else {
            for (int o = me; o < 128; o += warps * 32) {
                const int i = o & 15, col = o >> 4;
                float y = 0.0f;
                for (int w = 0; w < warps; ++w) y += all[w * kSums + i * kStride + col];
                if (tile.x + i < tile.y && col < n) p.y[(int64_t)s.row[r0 + col] * p.H + tile.x + i] = y;
            }
        }
    }

    template <class Ready>
    __device__ __forceinline__ bool run(const Ready &ready) {
        Batch now = s0 < s1 ? batch(s0, s.start[s0]) : Batch{s1, s1, 0, 0};
        Place at = first(now);
        uint4 a[kPieces][2][2];
        int x[kPieces][2];
        {
            const Source f = source(at);
#pragma unroll
            for (int u = 0; u < kPieces; ++u) load(f, u, a[u], x[u]);
        }
        if (!ready()) return false;
        while (now.r0 < now.r1) {
            __syncthreads();
            bring(now);
            __syncthreads();
            const Batch next = after(now);
            bool more = at.valid;
            while (more) {
                const int2 tile = tile_rows(at.slot, at.tile);
                const int r0 = max(s.start[at.slot], now.r0), r1 = min(s.start[at.slot + 1], now.r1), last = r1 - now.r0 - 1;
                float d[4];
                int r = r0;
                for (; r + 8 < r1; r += 8) {
                    products<false>(a, x, r - now.r0, last, d, Source{});
                    finish(d, tile, r, 8);
                }
                at.tile += groups;
                settle(at, now);
                more = at.valid;
                if (!more) at = first(next);
                products<true>(a, x, r - now.r0, last, d, source(at));
                finish(d, tile, r, r1 - r);
            }
            now = next;
        }
        __syncthreads();
        return true;
    }
};

// The used experts in ascending order, and the rows t k + q of each.
__device__ __forceinline__ int make_lists(const LayerArgs &p, Lists &s) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, R = p.T * p.k;
    int id[kRoutes / kThreads], rank[kRoutes / kThreads];
#pragma unroll
    for (int i = 0; i < kRoutes / kThreads; ++i) {
        const int r = (int)threadIdx.x + i * kThreads;
        id[i] = r < R ? __ldcg(p.ids + r) : -1;
    }
    for (int e = threadIdx.x; e < kLayerExperts; e += kThreads) s.count[e] = 0;
    __syncthreads();
    // (the order of an expert's rows is of no consequence: each has a column of its own)
#pragma unroll
    for (int i = 0; i < kRoutes / kThreads; ++i)
        if (id[i] >= 0) rank[i] = atomicAdd(&s.count[id[i]], 1);
    __syncthreads();
    constexpr int kEach = kLayerExperts / kThreads;
    int c[kEach], mine = 0;  // used experts in the upper half, rows in the lower
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        c[i] = s.count[kEach * threadIdx.x + i];
        mine += c[i] ? 0x10000 + c[i] : 0;
    }
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(kFull, sum, o);
        if (lane >= o) sum += v;
    }
    if (lane == 31) s.part[warp] = sum;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += s.part[w];
        all += s.part[w];
    }
    before += sum - mine;
    const int slots = all >> 16;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int e = kEach * (int)threadIdx.x + i;
        if (c[i]) {
            s.expert[before >> 16] = (unsigned short)e;
            s.start[before >> 16] = before & 0xffff;
            s.count[e] = before & 0xffff;
            before += 0x10000 + c[i];
        }
    }
    if (threadIdx.x == 0) s.start[slots] = R;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRoutes / kThreads; ++i)
        if (id[i] >= 0) s.row[s.count[id[i]] + rank[i]] = (unsigned short)(threadIdx.x + i * kThreads);
    __syncthreads();
    return slots;
}

__device__ __forceinline__ unsigned load_acquire(const unsigned *p) {
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

template <bool k8>
__global__ void __launch_bounds__(kThreads, 1) layer_experts_kernel(const LayerArgs p) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_align<128>(smem_raw);
    Lists &s = *reinterpret_cast<Lists *>(smem);
    unsigned char *stage = smem + (sizeof(Lists) + 127) / 128 * 128;
    unsigned *tickets = p.counters, *done = p.counters + 1, *arrived = p.counters + 2;
    pdl_wait();
    if (threadIdx.x == 0) s.ticket = (int)atomicAdd(tickets, 1u);
    const int slots = make_lists(p, s);
    const int pairs = slots * p.F;
    int ticket = s.ticket;
    for (;;) {
        __syncthreads();
        if (threadIdx.x == 0) s.ticket = (int)atomicAdd(tickets, 1u);  // the next one, taken while this one runs
        if (ticket < p.ranges) {
            const int lo = (int)((int64_t)pairs * ticket / p.ranges), hi = (int)((int64_t)pairs * (ticket + 1) / p.ranges);
            const int first = lo / p.F, end = lo < hi ? (hi - 1) / p.F + 1 : first;
            Phase<true, k8> up(p, s, stage, lo, hi, first, end, 0u);
            up.run([] { return true; });
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) atomicAdd(done, 1u);
        } else if (ticket < p.ranges + p.blocks * p.subsets) {
            const int i = ticket - p.ranges, block = i / p.subsets, part = i - block * p.subsets;
            const int lo = (int)((int64_t)p.H * block / p.blocks), hi = (int)((int64_t)p.H * (block + 1) / p.blocks);
            Phase<false, k8> down(p, s, stage, lo, hi, slots * part / p.subsets, slots * (part + 1) / p.subsets, 0u);
            const bool good = down.run([&] {
                if (threadIdx.x == 0) {
                    int ok = 1;
                    unsigned long long t0 = 0;
                    for (unsigned it = 1; load_acquire(done) < (unsigned)p.ranges; ++it) {
                        if (it & 255u) continue;
                        const unsigned long long t = global_ns();
                        if (t0 == 0) t0 = t;
                        if (t - t0 > kWaitLimitNs) {
                            if (p.status) atomicOr(p.status, kDevTimeout);
                            ok = 0;
                            break;
                        }
                    }
                    s.good = ok;
                }
                __syncthreads();
                return s.good != 0;
            });
            if (!good) return;
            if (p.subsets > 1) {
                __threadfence();
                __syncthreads();
                if (threadIdx.x == 0) s.last = atomicAdd(arrived + block, 1u) + 1 == (unsigned)p.subsets;
                __syncthreads();
                __threadfence();
            }
            if (p.subsets == 1 || s.last) {
                const int n = hi - lo;
                for (int j = threadIdx.x; j < n * p.T; j += kThreads) {
                    const int t = j / n, h = lo + j - t * n;
                    float sum = 0.0f;
#pragma unroll 8
                    for (int q = 0; q < p.k; ++q)
                        sum = fmaf(__ldcg(p.combine + t * p.k + q), __ldcg(p.y + (int64_t)(t * p.k + q) * p.H + h), sum);
                    p.out[(int64_t)t * p.H + h] = __float2bfloat16_rn(sum);
                }
            }
        } else {
            break;
        }
        __syncthreads();
        ticket = s.ticket;
    }
    pdl_trigger();
}

}  // namespace

size_t layer_counters(const LayerArgs &a) { return 2 + (size_t)a.blocks; }

void layer_split(LayerArgs *a, int sms) {
    a->ranges = sms;
    // one block of columns an SM, or a half or a quarter as many that share its experts: each
    // reads all rows of its experts' activations, which many tokens make as much as the weights
    const int R = a->T * a->k;
    a->subsets = R <= 32 ? 1 : R <= 128 ? 2 : 4;
    a->blocks = sms / a->subsets;
    if (a->blocks > a->H) a->blocks = a->H;
}

cudaError_t launch_layer_experts(LayerArgs a, bool eight, int sms, cudaStream_t s) {
    constexpr uint32_t fixed = 128 + (sizeof(Lists) + 127) / 128 * 128;
    a.stage_bytes = (int)(kSmemLimit - fixed);
    cudaError_t e = eight ? ensure_smem_limit<layer_experts_kernel<true>>(kSmemLimit)
                          : ensure_smem_limit<layer_experts_kernel<false>>(kSmemLimit);
    if (e != cudaSuccess) return e;
    return launch_after(eight ? layer_experts_kernel<true> : layer_experts_kernel<false>, dim3((unsigned)sms), kThreads,
                        kSmemLimit, s, a);
}

}  // namespace dol
