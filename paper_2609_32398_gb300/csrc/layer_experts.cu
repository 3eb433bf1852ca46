// The experts of a few tokens and their join in one kernel:
//
//   out[t] = sum_q combine[t][q] W2_e (silu(W1g_e x[t]) * W1u_e x[t]),  e = ids[t][q]
//
// The weights of the experts that are used are read once, everything else is small, so that
// the memory is what bounds it and the whole design is for keeping reads in flight:
//
//  - One CTA an SM.  The rows of all used experts' W1 form one list that is divided evenly,
//    to the tile: range i of n has its i-th n-th part; so do those of W2, and the elements of out.
//    A range meets the tokens of one or two experts.  (With a block of out's columns for each
//    CTA no results would pass through memory, but every CTA would read the activations of all
//    tokens, as much as the weights for 64 tokens.)
//  - Each warp takes tiles of its own, 16 weight rows (up: eight gate rows and their up rows)
//    over the whole k, and has a ring of two steps of 256 bytes of each row, filled by
//    asynchronous copies: 128 KB in flight an SM and no register held by them.  (Straight
//    to registers, the wait for one tile took in the loads of the next, and what there was to
//    compute between them doubled the time.)  The next step's copies leave as soon as the
//    products have read a step, also over the seam between the projections, where W2's do not
//    wait for the activations.  No sum crosses warps.
//  - The rows, at most a few dozen a CTA, lie in shared memory: they are the tensor
//    cores' second operand (mma.sync m16n8k16: a step is 8 or 16 instructions for eight
//    tokens, a tenth of the time that its bytes take from memory, so that the larger tiles of
//    tcgen05 would have nothing to give).
//
// 8-bit weights: codes are exact in fp16, and so are the tokens' values times a power of two for
// each 128 of a row that puts the largest just below fp16's range (what falls below
// 2^-40 of that is lost, far below the sums' fp32).  Activations, kept in fp32, are rounded to fp16's 11
// bits there: 1.66e-3 of the result's norm for 64 tokens, 1.65e-3 being the result's own rounding, and 2.34e-3
// by way of bf16.  Each block's sum is scaled by both powers in fp32.
//
// Order.  CTAs take tickets for the ranges of W1 until there are none left, and then go on with
// the same ranges of W2 and of out.  A range of W2 waits for those of W1 that have its experts'
// activations, its neighbours, and out for all.  All of W1 were taken before anybody waits, by
// CTAs that run: none waits for one that may not have been started, whatever else the GPU runs.
// All sums have a fixed order; the waits are bounded.
#include <cuda_fp16.h>

#include "layer_device.cuh"

namespace dol {
namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32;
constexpr int kRing = 2;                       // steps in a warp's ring
constexpr int kPieces = 2;                     // 128-byte pieces of a row in a step
constexpr int kRowStride = kPieces * 128 + 16; // of a row in the ring: no bank conflicts
constexpr int kStepBytes = 16 * kRowStride;
constexpr int kRoutes = kLayerTokens * kLayerChoices;
constexpr uint32_t kSmemLimit = 232448;

// What a warp does with a tile: rows [row, row + n) of the weights of one expert (down: columns) with
// the tokens [r, end) of the list, which are in shared memory from r0 on; n = 0: no more.
struct Tile {
    int slot, row, n, r, end, r0;
};
constexpr int kAhead = 4;  // tiles that a warp remembers; its copies are two ahead of its products at most

struct Lists {
    Tile tile[kWarps][kAhead];
    int count[kLayerExperts];  // then the first row of each expert
    int start[kLayerExperts + 1];  // of each used expert
    unsigned short expert[kLayerExperts], row[kRoutes];
    int part[kWarps];
    int ticket, queue, mine;
    unsigned short range[kLayerRanges];  // that this CTA took
};

__device__ __forceinline__ void load_matrices(uint32_t (&v)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(addr)
                 : "memory");
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

// The slots [from, to) whose rows [r0, r1) are in shared memory at a time.
struct Batch {
    int from, to, r0, r1;
};
// Where a warp's copies are: a tile (of a batch whose first one has number `before` in the CTA's queue)
// and a step of its k.
struct Place {
    Batch in;
    int before, slot, row, n, r, end, step;
    bool valid;
};

// A warp's ring in shared memory, the step to be used and the one to be filled.
struct StepRing {
    uint32_t data, out, in;
};

// One projection on this CTA's share, a range of the tiles of all used experts' rows of W2 (up: of
// pairs of gate and up rows).  The warps take its tiles in turn, from a queue: a fixed share each
// left some of them a tile, a fifth of the time, behind the others.
template <bool kUp, bool k8>
struct Phase {
    static constexpr int kTile = kUp ? 8 : 16;  // rows of a tile
    static constexpr int kCols = k8 ? 2 : 4;    // eights of tokens that share a step (registers)
    const LayerArgs &p;
    Lists &s;
    unsigned char *stage;
    StepRing &ring;
    int lo, hi, s0, s1;  // tiles, and their slots
    int warp, lane, K, N, per, row_bytes, pieces, steps, stride, room;
    Place ahead;         // of the copies
    unsigned begun;      // tiles that they have begun
    const unsigned char *source;  // of the lane's copies at `ahead`
    int2 scales;         // the next tile's exponents (see exponents)

    __device__ __forceinline__ Phase(const LayerArgs &p_, Lists &s_, unsigned char *stage_, StepRing &ring_, int slots, int range)
        : p(p_), s(s_), stage(stage_), ring(ring_) {
        warp = threadIdx.x >> 5;
        lane = threadIdx.x & 31;
        K = kUp ? p.H : p.F;
        N = kUp ? p.F : p.H;
        per = (N + kTile - 1) / kTile;
        row_bytes = K * (k8 ? 1 : 2);
        pieces = (row_bytes + 127) / 128;
        steps = (pieces + kPieces - 1) / kPieces;
        stride = pieces * (k8 ? 256 : 128) + 16;
        room = p.stage_bytes / (stride + (k8 ? 8 * pieces : 0));
        if (room >= 8) room &= ~7;
        const int all = slots * per;
        lo = (int)((int64_t)all * range / p.ranges);
        hi = (int)((int64_t)all * (range + 1) / p.ranges);
        s0 = lo / per;
        s1 = lo < hi ? (hi - 1) / per + 1 : s0;
        ahead = Place{};
        ahead.in = first_batch();
        take_tile(ahead);
        begun = 0;
        begin_tile();
        if (k8 && ahead.valid) scales = exponents(ahead.slot, ahead.row);
        fill();
        move_ahead();
        fill();
    }

    __device__ __forceinline__ Batch first_batch() const {
        return s0 < s1 ? batch(s0, s.start[s0]) : Batch{s1, s1, 0, 0};
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

    // The next tile of the queue.  It counts the tiles of one batch after the other.
    __device__ __forceinline__ void take_tile(Place &w) const {
        int i = 0;
        if (lane == 0) i = atomicAdd(&s.queue, 1);
        i = __shfl_sync(kFull, i, 0);
        for (;;) {
            if (w.in.r0 >= w.in.r1) {
                w.valid = false;
                return;
            }
            const int first = max(lo, w.in.from * per), n = min(hi, w.in.to * per) - first;
            if (i - w.before < n) {
                const int tile = first + i - w.before;
                w.slot = max(w.slot, w.in.from);
                while (tile >= (w.slot + 1) * per) ++w.slot;
                w.row = (tile - w.slot * per) * kTile;
                w.n = min(N - w.row, kTile);
                break;
            }
            w.before += n;
            w.in = after(w.in);
            w.slot = w.in.from;
        }
        w.r = max(s.start[w.slot], w.in.r0);
        w.end = min(s.start[w.slot + 1], w.in.r1);
        w.step = 0;
        w.valid = true;
    }
    // The next tokens of the tile, or the next tile.
    __device__ __forceinline__ void next_tile(Place &w) const {
        w.step = 0;
        w.r += 8 * kCols;
        if (w.r >= w.end) take_tile(w);
    }
    __device__ __forceinline__ void move_ahead() {
        source += kPieces * 128;
        if (!ahead.valid || ++ahead.step < steps) return;
        next_tile(ahead);
        begin_tile();
        // (with one step a tile the copies are two tiles ahead: see run)
        if (k8 && steps > 1 && ahead.valid) scales = exponents(ahead.slot, ahead.row);
    }
    // Exponents of a tile's weights, lane l those of pieces l and 32 + l: of its rows, or of its gate
    // rows and of its up rows.
    __device__ __forceinline__ int2 exponents(int slot, int row) const {
        const int e = s.expert[slot], blocks = blocks8(N);
        const uint8_t *x = (kUp ? p.w1x + (int64_t)2 * e * blocks * pieces : p.w2x + (int64_t)e * blocks * pieces) +
                           row / kBlock8 * pieces;
        int2 v = make_int2(0, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (32 * i + lane >= pieces) continue;
            v.x |= __ldg(x + 32 * i + lane) << (8 * i);
            if (kUp) v.y |= __ldg(x + blocks * pieces + 32 * i + lane) << (8 * i);
        }
        return v;
    }

    // Half a warp copies 256 bytes of a row at a time: up, a gate row and its up row; down, two
    // rows that follow each other.
    __device__ __forceinline__ void begin_tile() {
        if (lane == 0)
            s.tile[warp][begun % kAhead] = Tile{ahead.slot, ahead.row, ahead.valid ? ahead.n : 0, ahead.r, min(ahead.end, ahead.r + 8 * kCols), ahead.in.r0};
        ++begun;
        if (!ahead.valid) return;
        const int e = s.expert[ahead.slot], half = lane >> 4;
        const unsigned char *w = static_cast<const unsigned char *>(kUp ? p.w1 : p.w2) + (lane & 15) * 16;
        const int64_t row = (int64_t)e * (kUp ? 2 * p.F : p.H) + ahead.row + (kUp ? half * p.F : half);
        source = w + row * row_bytes;
    }
    // Copies of the step at `ahead` into the ring (up: gate rows, up rows from 8 on), zeros where a row's
    // last piece is not full.  One group of copies, empty ones too.
    __device__ __forceinline__ void fill() {
        __syncwarp();  // the products have read what was there
        if (ahead.valid) {
            const int half = lane >> 4, c = (lane & 15) * 16;
            const int left = row_bytes - ahead.step * (kPieces * 128);  // bytes of the row from this step on
            uint32_t to = ring.data + ring.in * kStepBytes + (kUp ? 8 * half : half) * kRowStride + c;
            const bool in = c < left;
            const unsigned char *w = in ? source : source - c;  // an address of this row
            const int n = kUp ? ahead.n : (ahead.n - half + 1) / 2, jump = kUp ? row_bytes : 2 * row_bytes;
            if (c < ((left + 127) & ~127)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i < n) cp_async16(to + i * (kUp ? kRowStride : 2 * kRowStride), w, in);
                    w += jump;
                }
            }
            ring.in ^= 1u;
        }
        copies_sent();
    }

    // Rows r0 .. r1 to shared memory: the columns that the weights' pieces reach, zeros past K.
    // Sixteen lanes have 128 values, four loads a lane are in flight together.
    __device__ __forceinline__ void bring(const Batch &b) const {
        constexpr bool kWide = k8 && !kUp;  // activations in fp32
        constexpr int kWords = kWide ? 2 : 1, kFlight = 4 / kWords, kStep = kThreads / 16;
        const int blocks = k8 ? pieces : (pieces + 1) / 2, n = (b.r1 - b.r0) * blocks, piece = threadIdx.x & 15;
        const float inv = 1.0f / (float)blocks;
        for (int base = threadIdx.x >> 4; __any_sync(kFull, base < n); base += kFlight * kStep) {
            uint4 v[kFlight][kWords];
#pragma unroll
            for (int j = 0; j < kFlight; ++j) {
                const int i = base + j * kStep, r = (int)(((float)i + 0.5f) * inv), c = (i - r * blocks) * 16 + piece;  // i < 2^14: exact
#pragma unroll
                for (int q = 0; q < kWords; ++q) v[j][q] = make_uint4(0, 0, 0, 0);
                if (i < n && 8 * c < K) {
                    const int from = s.row[b.r0 + r];
                    const uint4 *src = kUp ? reinterpret_cast<const uint4 *>(p.x) + (int64_t)(from / p.k) * (K / 8)
                                           : static_cast<const uint4 *>(p.act) + (int64_t)from * (K / 8 * kWords);
#pragma unroll
                    for (int q = 0; q < kWords; ++q) v[j][q] = __ldcg(src + kWords * c + q);
                }
            }
#pragma unroll
            for (int j = 0; j < kFlight; ++j) {
                const int i = base + j * kStep, r = (int)(((float)i + 0.5f) * inv), block = i - r * blocks;
                if constexpr (!k8) {
                    if (i < n && 8 * (block * 16 + piece) < 64 * pieces)
                        *reinterpret_cast<uint4 *>(stage + r * stride + (block * 16 + piece) * 16) = v[j][0];
                } else {
                    unsigned w[8], top = 0;  // eight values
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        if constexpr (kWide) w[q] = word(v[j][q / 4], q & 3);
                        else w[q] = q & 1 ? word(v[j][0], q / 2) & 0xffff0000u : word(v[j][0], q / 2) << 16;
                        top = max(top, w[q] & 0x7fffffffu);
                    }
#pragma unroll
                    for (int o = 1; o < 16; o *= 2) top = max(top, __shfl_xor_sync(kFull, top, o));
                    // the largest value, 2^(x - 127) and more, to 2^14 and more
                    const int x = (int)(top >> 23);
                    const int up = x == 255 ? 127 : min(254, 268 - x);   // exponent byte of the factor
                    const float f = __uint_as_float((unsigned)up << 23);
                    unsigned hw[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const __half2 two = __floats2half2_rn(__uint_as_float(w[2 * q]) * f, __uint_as_float(w[2 * q + 1]) * f);
                        hw[q] = *reinterpret_cast<const unsigned *>(&two);
                    }
                    if (i >= n) continue;
                    // codes come from shared memory four a lane, so that a lane's values 4 t .. 4 t + 3 go
                    // where the tensor cores want its 2 t, 2 t + 1, 8 + 2 t and 9 + 2 t
                    unsigned char *at16 = stage + r * stride + (block * 8 + (piece >> 1)) * 32;  // of sixteen values
                    *reinterpret_cast<uint2 *>(at16 + 8 * (piece & 1)) = make_uint2(hw[0], hw[2]);
                    *reinterpret_cast<uint2 *>(at16 + 16 + 8 * (piece & 1)) = make_uint2(hw[1], hw[3]);
                    // back by 2^(127 - up), in two factors: the first one keeps a block's sum (below
                    // 2^31) in range, the second one follows the weights' scale
                    const int back = 254 - up, far = back > 127 ? 64 : 0;
                    const int e = back - far;
                    if (piece == 0)
                        *reinterpret_cast<float2 *>(stage + room * stride + 8 * (r * pieces + block)) =
                            make_float2(__uint_as_float(e > 0 ? (unsigned)e << 23 : 0x00400000u),
                                        __uint_as_float((unsigned)(127 + far) << 23));
                }
            }
        }
    }

    // The sums of a step with the tokens' rows r on in shared memory (past `last` the last one again,
    // whose results nobody reads).
    __device__ __forceinline__ void products(const Tile &at, int step, int2 x, float (&d)[kCols][4]) const {
        const int t = lane & 3, u0 = step * kPieces, r = at.r - at.r0, last = at.end - at.r0 - 1;
        const bool two = u0 + 1 < pieces;
        const uint32_t a = ring.data + ring.out * kStepBytes + (lane & 15) * kRowStride + (lane >> 4) * 16;
        const uint32_t b = smem_u32(stage) + u0 * (k8 ? 256 : 128) + (lane >> 3) * 16;
        if constexpr (!k8) {
#pragma unroll
            for (int u = 0; u < kPieces; ++u) {
                if (u > 0 && !two) break;
                uint32_t w[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) load_matrices(w[j], a + u * 128 + j * 32);
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    if (c > 0 && r + 8 * c > last) break;
                    const uint32_t row = b + min(r + 8 * c + (lane & 7), last) * stride + u * 128;
                    uint32_t v[2][4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) load_matrices(v[j], row + j * 64);
                    float odd[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        mma16<false>(d[c], w[2 * j][0], w[2 * j][1], w[2 * j][2], w[2 * j][3], v[j][0], v[j][1]);
                        mma16<false>(odd, w[2 * j + 1][0], w[2 * j + 1][1], w[2 * j + 1][2], w[2 * j + 1][3], v[j][2], v[j][3]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[c][i] += odd[i];
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < kPieces; ++u) {
                if (u > 0 && !two) break;
                uint32_t w[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) load_matrices(w[j], a + u * 128 + j * 32);
                const int q = u0 + u, shift = q >> 5 << 3;
                const float w0 = e8_scale(__shfl_sync(kFull, x.x, q & 31) >> shift & 255);
                const float w1 = kUp ? e8_scale(__shfl_sync(kFull, x.y, q & 31) >> shift & 255) : w0;
                const unsigned char *f = stage + room * stride + 8 * q;
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    if (c > 0 && r + 8 * c > last) break;
                    const uint32_t row = b + min(r + 8 * c + (lane & 7), last) * stride + u * 256;
                    const float2 f0 = *reinterpret_cast<const float2 *>(f + 8 * pieces * min(r + 8 * c + 2 * t, last));
                    const float2 f1 = *reinterpret_cast<const float2 *>(f + 8 * pieces * min(r + 8 * c + 2 * t + 1, last));
                    uint32_t v[4][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) load_matrices(v[j], row + j * 64);
                    float sum[2][4] = {};
                    // (the codes are turned into fp16 again for every eight tokens, of which few experts have
                    // more: held for all they would not fit the registers)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t *q4 = w[j];
                        mma16<true>(sum[0], codes_half2<0>(q4[0]), codes_half2<0>(q4[1]), codes_half2<1>(q4[0]),
                                    codes_half2<1>(q4[1]), v[j][0], v[j][1]);
                        mma16<true>(sum[1], codes_half2<0>(q4[2]), codes_half2<0>(q4[3]), codes_half2<1>(q4[2]),
                                    codes_half2<1>(q4[3]), v[j][2], v[j][3]);
                    }
                    d[c][0] += (sum[0][0] + sum[1][0]) * f0.x * w0 * f0.y;
                    d[c][1] += (sum[0][1] + sum[1][1]) * f1.x * w0 * f1.y;
                    d[c][2] += (sum[0][2] + sum[1][2]) * f0.x * w1 * f0.y;
                    d[c][3] += (sum[0][3] + sum[1][3]) * f1.x * w1 * f1.y;
                }
            }
        }
    }

    // What becomes of a tile's sums: rows g and g + 8, tokens 2 t and 2 t + 1 of eight.
    __device__ __forceinline__ void finish(const Tile &at, const float (&d)[kCols][4]) const {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            if (at.r + 8 * c >= at.end) break;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = at.r + 8 * c + 2 * t + i;
                if (r >= at.end) break;
                const int64_t to = s.row[r];
                if constexpr (kUp) {
                    const float gate = d[c][i];
                    const float act = gate * sigmoid_f(gate) * d[c][2 + i];
                    if (g >= at.n) continue;
                    // (bf16 weights: bf16 is what the tensor cores take beside them)
                    if constexpr (k8) static_cast<float *>(p.act)[to * p.F + at.row + g] = act;
                    else static_cast<bf16 *>(p.act)[to * p.F + at.row + g] = __float2bfloat16_rn(act);
                } else {
                    if (g < at.n) p.y[to * p.H + at.row + g] = d[c][i];
                    if (g + 8 < at.n) p.y[to * p.H + at.row + g + 8] = d[c][2 + i];
                }
            }
        }
    }

    // The share, once `ready` says that the rows may be read (the first steps are on their way
    // since the constructor).
    template <class Ready>
    __device__ __forceinline__ bool run(const Ready &ready) {
        if (!ready()) return false;
        Batch now = first_batch();
        __syncwarp();
        unsigned done = 0;
        Tile at = s.tile[warp][0];
        while (now.r0 < now.r1) {
            __syncthreads();
            bring(now);
            __syncthreads();
            for (; at.n > 0 && at.r0 == now.r0; at = s.tile[warp][++done % kAhead]) {
                float d[kCols][4] = {};
                int2 x = make_int2(0, 0);
                if constexpr (k8) x = steps > 1 ? scales : exponents(at.slot, at.row);
                for (int step = 0; step < steps; ++step) {
                    wait_copies<kRing - 1>();
                    __syncwarp();
                    products(at, step, x, d);
                    ring.out ^= 1u;
                    move_ahead();
                    fill();
                }
                finish(at, d);
            }
            now = after(now);
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

// The range that has tile i of n (range r: those from n r / ranges on).
__device__ __forceinline__ int range_of(int i, int n, int ranges) {
    return (int)((((int64_t)i + 1) * ranges - 1) / n);
}

template <bool k8>
__global__ void __launch_bounds__(kThreads, 1) layer_experts_kernel(const LayerArgs p) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_align<128>(smem_raw);
    Lists &s = *reinterpret_cast<Lists *>(smem);
    unsigned char *stage = smem + (sizeof(Lists) + 127) / 128 * 128;
    unsigned *tickets = p.counters, *down_done = p.counters + 1, *up_done = p.counters + 2;
    const int warp = threadIdx.x >> 5;
    StepRing ring{smem_u32(stage) + warp * (kRing * kStepBytes), 0u, 0u};
    stage += kWarps * kRing * kStepBytes;
    pdl_wait();
    if (threadIdx.x == 0) {
        s.ticket = (int)atomicAdd(tickets, 1u);
        s.mine = 0;
    }
    const int slots = make_lists(p, s);
    for (;;) {
        __syncthreads();
        const int range = s.ticket;
        if (range >= p.ranges) break;
        __syncthreads();
        if (threadIdx.x == 0) {
            s.range[s.mine++] = (unsigned short)range;
            s.queue = 0;
            s.ticket = (int)atomicAdd(tickets, 1u);
        }
        __syncthreads();
        Phase<true, k8> up(p, s, stage, ring, slots, range);
        up.run([] { return true; });
        __threadfence();  // what this range wrote may be read
        __syncthreads();
        if (threadIdx.x == 0) atomicExch(up_done + range, 1u);
    }
    const int mine = s.mine;
    for (int i = 0; i < mine; ++i) {
        __syncthreads();
        if (threadIdx.x == 0) s.queue = 0;
        __syncthreads();
        Phase<false, k8> down(p, s, stage, ring, slots, s.range[i]);
        const bool good = down.run([&] {
            // the ranges of W1's tiles of the slots
            const int per = (p.F + 7) / 8, from = range_of(down.s0 * per, slots * per, p.ranges);
            const int to = down.s0 < down.s1 ? range_of(down.s1 * per - 1, slots * per, p.ranges) : from - 1;
            int ok = 1;
            if (from + (int)threadIdx.x <= to) ok = wait_count(up_done + from + threadIdx.x, 1u, p.status);
            return __syncthreads_and(ok) != 0;
        });
        if (!good) {
            wait_copies<0>();
            return;
        }
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) atomicAdd(down_done, 1u);
    }
    int ok = 1;
    if (mine && threadIdx.x == 0) ok = wait_count(down_done, (unsigned)p.ranges, p.status);
    if (!__syncthreads_and(ok)) return;
    for (int j = 0; j < mine; ++j) {
        const int n = p.T * p.H, lo = (int)((int64_t)n * s.range[j] / p.ranges), hi = (int)((int64_t)n * (s.range[j] + 1) / p.ranges);
        for (int i = lo + (int)threadIdx.x; i < hi; i += kThreads) {
            const int t = i / p.H, h = i - t * p.H;
            float sum = 0.0f;
#pragma unroll 8
            for (int q = 0; q < p.k; ++q)
                sum = fmaf(__ldcg(p.combine + t * p.k + q), __ldcg(p.y + (int64_t)(t * p.k + q) * p.H + h), sum);
            p.out[i] = __float2bfloat16_rn(sum);
        }
    }
    pdl_trigger();
}

}  // namespace

cudaError_t launch_layer_experts(LayerArgs a, bool eight, int sms, cudaStream_t s) {
    constexpr uint32_t fixed = 128 + (sizeof(Lists) + 127) / 128 * 128 + kWarps * kRing * kStepBytes;
    a.stage_bytes = (int)(kSmemLimit - fixed);
    cudaError_t e = eight ? ensure_smem_limit<layer_experts_kernel<true>>(kSmemLimit)
                          : ensure_smem_limit<layer_experts_kernel<false>>(kSmemLimit);
    if (e != cudaSuccess) return e;
    return launch_after(eight ? layer_experts_kernel<true> : layer_experts_kernel<false>, dim3((unsigned)sms), kThreads,
                        kSmemLimit, s, a);
}

}  // namespace dol
