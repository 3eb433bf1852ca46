// Products of each expert's weights with its routed rows on the tcgen05 tensor
// cores (kind::f16: bf16 operands, fp32 accumulation):
//
//   D[m][r] = sum_k W_e[m][k] A[row(r)][k]          m: weight rows, r: routed rows
//
// with three epilogues: the rows as they are, the SwiGLU activation with its 8-bit
// checkpoint, and the gradient of that.  The weights are the M side: their sizes
// are fixed and fill tiles of 256, while the ragged side, the rows of an expert,
// is the N side, whose width may be any multiple of 16.  An expert's n rows are
// ceil(n / 256) tiles of equal width, so that a ragged group wastes at most 15
// columns a tile (a fixed 256-row tile would waste 128 rows an expert on average)
// and a decode step's groups of one or two rows take tiles 16 wide.  Where that is too
// few tiles for half of the pairs, 128 or 64 rows are the most instead.
//
// A persistent CTA pair (cta_group::2, 256 weight rows x up to 256 routed rows in
// 2 x 256 TMEM columns, so that one tile's epilogue runs under the next tile's
// products) takes tiles in a fixed order.  Per 64-wide step of k each CTA loads
// its 128 weight rows by TMA (one box, or two where the weights are read through
// their other side) and half of the routed rows: in one box where they lie in
// dispatch order, and gathered four at a time by their row ids otherwise, so that no
// permuted copy of the tokens exists.  What a tile holds past its group's end ends
// in accumulator columns that nobody reads.
//
// Warps: 0 weights by TMA, 1 issues the MMAs (first CTA), then the epilogue's, then
// those that gather rows or one that loads them in boxes.  A TMEM lane is a
// weight row and a register a routed row; the four epilogue warps of a group turn
// blocks of 16 routed rows x 128 columns (up: 32 x 64 of the gate and their up
// values) in shared memory and deal the rows out among them, 16 columns a thread
// and a row's columns over neighbouring threads: whole 128-byte lines are then read
// and written where a warp's own 32 columns would be 64 bytes of each of 16 rows
// (four times the passes through the SM's load-store pipe, which bound the gradient's
// epilogue), and the activation and a block's exponent need no other thread.  The
// 16-byte pieces are xor-swizzled: no bank conflicts either way.
//
// What bounds it: the tensor cores, once a tile has a few tens of steps.  131072 rows of
// one expert, 2048 x 1536: 429 us, 1.92 PFLOP/s (of 1.94 measured); the up projection of
// 16384 tokens over 128 experts (H = 2048, F = 768) 479 us, 1.72 PFLOP/s, with its
// checkpoint 505; the gradient through W2 and the activation 362 us, of which the
// products alone 280: its epilogue moves 820 MB.  Short contractions (768 to 1024) pay
// one to two microseconds a tile, few tiles the rounding up to whole rounds of 76 pairs,
// few rows the reading of the weights (16 tokens: 76 us of 81).
//
// Every wait is bounded; one that runs out records kDevTimeout.
#include <cstdint>

#include "experts_mma.cuh"

namespace dol {
namespace {

constexpr int kTileN = 256;               // routed rows of a tile at most
// The epilogue's blocks take 16 KB in every mode, so that the ring has six stages of
// 32 KB: one group of four warps with 32 routed rows at a time, or, where a thread can
// do with 16 of a row's 32 values, two groups with 16 (the gate and up values of a
// column are 16 TMEM lanes apart and want one thread).
__host__ __device__ constexpr int epi_warps(int mode) { return mode == kProductUp ? 4 : 8; }
__host__ __device__ constexpr int first_loader(int mode) { return 2 + epi_warps(mode); }
// Gathering warps: load_split of them share a step, kLoadSteps steps are filled at a time
// (see pair_gather4).  The gradient's epilogue leaves registers for six.
constexpr int kLoadSteps = 3;
__host__ __device__ constexpr int load_split(int mode) { return mode == kProductUpGrad ? 2 : 4; }
__host__ __device__ constexpr int load_warps(int mode) { return kLoadSteps * load_split(mode); }
__host__ __device__ constexpr int threads_of(int mode, bool gather) {
    return (first_loader(mode) + (gather ? load_warps(mode) : 1)) * 32;
}
constexpr uint32_t kTurnAll = 16384;
constexpr uint32_t kABytes = 128 * 128;   // a CTA's weight rows of one step
constexpr int kMaxStages = 12;
constexpr uint32_t kSmemLimit = 232448;

struct PairArgs {
    ProductArgs p;
    int m_tiles;    // tiles of 256 weight rows (up: of 128 gate rows and their up rows)
    uint32_t m_magic;  // divide_magic(m_tiles)
    int stages;     // of the ring
    uint32_t b_bytes;  // room for a CTA's routed rows of one step
    bool paired;    // transposed weights with N a multiple of 64: one box a step
};

// Shared memory: ring [stages][weights | rows], turn blocks [16 KB], and for each
// expert its first tile [E + 1], first row [E + 1] and the width of its tiles [E + 1].
__host__ __device__ inline uint32_t table_bytes(int E) { return 4u * 3u * ((uint32_t)E + 1u); }
__host__ __device__ inline uint32_t off_turn(int stages, uint32_t b_bytes) { return stages * (kABytes + b_bytes); }

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

// 16 values to their codes and exponent.
__device__ __forceinline__ uint4 quantise16(const float *v, int *exponent) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    const int e = q8_exponent(__uint_as_float(top));
    const float inv = q8_inverse(e);
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
        w[j] = q8_code(v[4 * j], inv) | q8_code(v[4 * j + 1], inv) << 8 | q8_code(v[4 * j + 2], inv) << 16 |
               q8_code(v[4 * j + 3], inv) << 24;
    if (e == 255) w[0] = w[1] = w[2] = w[3] = 0u;
    *exponent = e;
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// One routed row's values of the tile: up, 16 of the gate from column c0 on and their
// 16 of the up side; otherwise 16 columns from c0 on.
__device__ __forceinline__ void finish_plain(const ProductArgs &p, int64_t r, int c0, const float (&v)[16]) {
    if (p.wide) {
        float4 *to = reinterpret_cast<float4 *>(p.wide + r * p.N + c0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c0 + 4 * j < p.N) to[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        return;
    }
    bf16 *dst = p.out + r * p.N + c0;
    if (c0 + 16 <= p.N) store16(dst, v);
    else if (c0 < p.N)  // N is a multiple of 8
        *reinterpret_cast<uint4 *>(dst) =
            make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
}

__device__ __forceinline__ void finish_up(const ProductArgs &p, int64_t r, int c0, float (&v)[32]) {
    const int F = p.N / 2;
    if (c0 >= F) return;
    if (p.codes) {
        int eg, eu;
        const uint4 g = quantise16(v, &eg), u = quantise16(v + 16, &eu);
        const int64_t at = r * p.N + c0;
        *reinterpret_cast<uint4 *>(p.codes + at) = g;
        *reinterpret_cast<uint4 *>(p.codes + at + F) = u;
        p.exponents[at / kQBlock] = (uint8_t)eg;
        p.exponents[(at + F) / kQBlock] = (uint8_t)eu;
    }
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const f32x2 g = pair2(v[i], v[i + 1]);
        split2(mul2(mul2(g, sigmoid2(g)), pair2(v[16 + i], v[17 + i])), v[i], v[i + 1]);
    }
    store16(p.out + r * F + c0, v);
}

// What finish_grad reads of its row, as it lies in memory: nothing waits for these loads
// before finish_grad does.
struct Kept {
    uint4 gate, up;
    unsigned gate_exponent, up_exponent;
    float weight;
};
__device__ __forceinline__ Kept read_kept(const ProductArgs &p, int64_t r, int c0) {
    Kept k = {};
    if (c0 < p.N) {
        const int64_t cg = r * 2 * p.N + c0, cu = cg + p.N;
        k.gate = __ldg(reinterpret_cast<const uint4 *>(p.codes + cg));
        k.up = __ldg(reinterpret_cast<const uint4 *>(p.codes + cu));
        k.gate_exponent = __ldg(p.exponents + cg / kQBlock);
        k.up_exponent = __ldg(p.exponents + cu / kQBlock);
        k.weight = __ldg(p.row_weight + r);
    }
    return k;
}
// Returns the sum of g act over the 16 columns.
__device__ __forceinline__ float finish_grad(const ProductArgs &p, int64_t r, int c0, const float (&v)[16],
                                             const Kept &k) {
    const int F = p.N;
    if (c0 >= F) return 0.0f;
    const unsigned flip = 0x80808080u;
    const unsigned ug[4] = {k.gate.x ^ flip, k.gate.y ^ flip, k.gate.z ^ flip, k.gate.w ^ flip};
    const unsigned uu[4] = {k.up.x ^ flip, k.up.y ^ flip, k.up.z ^ flip, k.up.w ^ flip};
    const float gate_scale = q8_scale((int)k.gate_exponent), up_scale = q8_scale((int)k.up_exponent);
    const f32x2 sg = pair2(gate_scale, gate_scale), su = pair2(up_scale, up_scale);
    const f32x2 w = pair2(k.weight, k.weight), one = pair2(1.0f, 1.0f), minus = pair2(-1.0f, -1.0f);
    f32x2 sum = pair2(0.0f, 0.0f);
    float dg[16], du[16], act[16];
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
        const f32x2 zg = q8_values(ug[i / 4], i & 3, sg), zu = q8_values(uu[i / 4], i & 3, su);
        const f32x2 s = sigmoid2(zg), g = pair2(v[i], v[i + 1]);
        const f32x2 silu = mul2(zg, s), a = mul2(silu, zu), gw = mul2(g, w);
        sum = fma2(g, a, sum);
        split2(mul2(gw, silu), du[i], du[i + 1]);
        split2(mul2(mul2(gw, zu), fma2(silu, fma2(s, minus, one), s)), dg[i], dg[i + 1]);
        split2(mul2(a, w), act[i], act[i + 1]);
    }
    bf16 *dz = p.dz + r * 2 * F + c0, *out = p.out + r * F + c0;
    store16(dz, dg);
    store16(dz + F, du);
    store16(out, act);
    float lo, hi;
    split2(sum, lo, hi);
    return lo + hi;
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

template <int kMode, bool kGather, bool kTransposed>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(threads_of(kMode, kGather), 1)
product_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap amap, const PairArgs a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_align<1024>(smem_raw);
    constexpr int kEpiWarps = epi_warps(kMode), kFirstLoader = first_loader(kMode);
    constexpr int kThreads = threads_of(kMode, kGather);
    const ProductArgs &p = a.p;
    const int E = p.E, stages = a.stages;
    const uint32_t stage_bytes = kABytes + a.b_bytes;
    unsigned char *turn = smem + off_turn(stages, a.b_bytes);
    int *first = reinterpret_cast<int *>(turn + kTurnAll), *start = first + E + 1, *width = start + E + 1;
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drain;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort, s_part[kThreads / 32];
    volatile int *abort = &s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(&full[i], kGather ? 1 + 2 * load_split(kMode) : 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], 2 * kEpiWarps);
        }
        mbar_init(&drain, 1);
        s_abort = 0;
        fence_barrier_init();
        prefetch_tensormap(&wmap);
        prefetch_tensormap(&amap);
    }
    pdl_wait();
    // not before: the kernel before may share this SM and still have to take its own
    if (warp == 1) pair_tmem_alloc(&tmem_slot, 512);
    // The first tile of each expert: a scan of ceil(n / cap) m_tiles over the experts.  Tiles
    // are 256 rows at most, or 128 or 64 while that leaves half of the pairs without one:
    // a tile's time is mostly its epilogue then, which narrower tiles divide.  T = 1000, H = 512,
    // F = 256, E = 8, k = 2, against 256 always: the gradient 17.9 to 13.4 us, up 9.7 to 8.4, a
    // plain product 8.8 to 8.4; T = 1000, H = 2048, F = 768 (48 tiles, not divided) 20.6 either way.
    const int pairs = (int)(gridDim.x >> 1);
    int carry;
    for (int cap = kTileN;; cap /= 2) {
        carry = 0;
        int wide = 0;  // some group could be divided further
        for (int base = 0; base <= E; base += kThreads) {
            const int e = base + (int)threadIdx.x;
            int c = 0, n = 0;
            if (e <= E) start[e] = max(0, min(__ldg(p.offsets + e), (int)p.R));
            if (e < E) {
                n = max(0, max(0, min(__ldg(p.offsets + e + 1), (int)p.R)) - start[e]);
                const int nt = (n + cap - 1) / cap;
                width[e] = nt > 0 ? ((n + nt - 1) / nt + 15) & ~15 : 0;
                c = nt * a.m_tiles;
            }
            int x = c;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(kFull, x, o);
                if (lane >= o) x += y;
            }
            if (lane == 31) s_part[warp] = x;
            wide |= __syncthreads_or(n > cap / 2);
            int before = carry, all = 0;
            for (int i = 0; i < kThreads / 32; ++i) {
                if (i < warp) before += s_part[i];
                all += s_part[i];
            }
            if (e < E) first[e] = before + x - c;
            carry += all;
            __syncthreads();
        }
        if (!wide || cap == 64 || 2 * carry > pairs) break;
    }
    if (threadIdx.x == 0) first[E] = carry;
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int steps = (p.K + 63) / 64;
    Walk walk{first, start, width, carry, pairs, a.m_tiles, a.m_magic, (int)(blockIdx.x >> 1), 0, {}};
    const Tile &tl = walk.tile;
    const uint32_t ring = smem_u32(smem), full0 = smem_u32(full), empty0 = smem_u32(empty);
    const uint32_t full_pair = map_to_rank(full, 0);  // the first CTA's
    if (warp == 0) {
        // ---------------------------------------------------------- weights
        const bool one = elect_one();
        Ring at{0, 0};
        bool good = true;
        int it = 0;
        for (bool any = walk.find(); good && any; any = walk.next()) {
            const int m0 = tl.m * 256 + (int)rank * 128, mb = tl.m * 8 + (int)rank * 4;
            const uint32_t bytes = 2u * (kABytes + (kGather ? (uint32_t)tl.width * 64u : a.b_bytes));
            for (int k = 0; k < p.K; k += 64, ++it) {
                good = pair_wait_all(empty0 + 8 * at.s, at.phase ^ 1u, p.status, abort);
                if (!good) break;
                const uint32_t st = ring + at.s * stage_bytes, bar = full_pair + 8 * at.s;
                if (one) {
                    if (rank == 0) mbar_expect_tx_addr(full0 + 8 * at.s, bytes);
                    if constexpr (kMode == kProductUp) {
                        pair_load_5d(st, &wmap, k, 0, 0, mb, tl.e, bar);
                    } else if constexpr (!kTransposed) {
                        pair_load_3d(st, &wmap, k, m0, tl.e, bar);
                    } else if (a.paired) {
                        pair_load_4d(st, &wmap, 0, k, m0 / 64, tl.e, bar);
                    } else {
                        pair_load_3d(st, &wmap, m0, k, tl.e, bar);
                        pair_load_3d(st + kABytes / 2, &wmap, m0 + 64, k, tl.e, bar);
                    }
                }
                __syncwarp();
                at.next(stages);
            }
        }
        // a run that gave up: the loads in flight complete before the CTA ends (in the
        // usual case the MMAs waited for them)
        if (!good && rank == 0 && lane == 0)
            for (int i = it > stages ? it - stages : 0; i < it; ++i)
                mbar_wait(&full[i % stages], (uint32_t)(i / stages) & 1u, p.status);
        __syncwarp();
    } else if (!kGather && warp == kFirstLoader) {
        // ---------------------------------------------------------- rows in dispatch order
        // One box as high as the widest tile's half: what it holds past this tile's half
        // is not used.
        const bool one = elect_one();
        Ring at{0, 0};
        bool good = true;
        for (bool any = walk.find(); good && any; any = walk.next()) {
            const int r = tl.r0 + (int)rank * (tl.width / 2);
            for (int k = 0; k < p.K; k += 64) {
                good = pair_wait_all(empty0 + 8 * at.s, at.phase ^ 1u, p.status, abort);
                if (!good) break;
                if (one)
                    pair_load_3d(ring + at.s * stage_bytes + kABytes, &amap, k, r, 0, full_pair + 8 * at.s);
                __syncwarp();
                at.next(stages);
            }
        }
        __syncwarp();
    } else if (kGather && warp >= kFirstLoader) {
        // ---------------------------------------------------------- gather
        // Of the kSplit warps that share a step, lane l of the w-th copies this CTA's
        // routed rows 4 (l kSplit + w) .. + 3 of the tile.
        constexpr int kSplit = load_split(kMode);
        const int loader = warp - kFirstLoader, mine4 = 4 * (lane * kSplit + loader % kSplit);
        const int none = (int)p.a_rows;
        int4 ids;
        auto read_ids = [&]() {
            const int half = tl.width / 2;
            int v[4];
            bool bad = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = (int)rank * half + mine4 + j;
                v[j] = mine4 < half && n < tl.n ? __ldg(p.rows + tl.r0 + n) : none;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = (int)rank * half + mine4 + j;
                const bool out = v[j] < 0 || v[j] >= none;
                bad |= out && mine4 < half && n < tl.n;
                if (out) v[j] = none;
            }
            if (bad && p.status) atomicOr(p.status, kDevBadId);
            ids = make_int4(v[0], v[1], v[2], v[3]);
        };
        int it = 0, mine = loader / kSplit;  // steps so far, this warp's next one
        bool good = true, any = walk.find();
        if (any) read_ids();
        while (good && any) {
            const int half = tl.width / 2, end = it + steps;
            for (; mine < end; mine += kLoadSteps) {
                const int s = mine % stages;
                if (mine >= stages) {
                    good = pair_wait_warp(empty0 + 8 * s, (uint32_t)(mine / stages - 1) & 1u, p.status, abort, lane);
                    if (!good) break;
                }
                if (mine4 < half)
                    pair_gather4(ring + (uint32_t)s * stage_bytes + kABytes + mine4 * 128, &amap, 64 * (mine - it), ids,
                                 full_pair + 8 * s);
                __syncwarp();
                // a step waits for each of its warps, with copies or (a narrow tile) without:
                // none may fall a phase behind
                if (lane == 0) mbar_arrive_cluster(full_pair + 8 * s);
            }
            any = walk.next();
            if (any) read_ids();
            it = end;
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------- MMA issuer
        if (rank == 0) {
            const bool one = elect_one();
            Ring at{0, 0};
            int done = 0;
            bool good = true;
            // descriptors of stage 0: a step along k is 32 bytes in a K-major row, 16 rows
            // of 128 bytes in an MN-major block
            const uint64_t ad0 = kTransposed ? desc_mn_sw128(ring, kABytes / 2) : umma_desc_sw128(ring);
            const uint64_t bd0 = umma_desc_sw128(ring + kABytes);
            constexpr uint32_t kAStep = kTransposed ? 2048 / 16 : 32 / 16, kBStep = 32 / 16;
            const uint32_t acc_full0 = smem_u32(acc_full), acc_empty0 = smem_u32(acc_empty);
            for (bool any = walk.find(); good && any; any = walk.next(), ++done) {
                const uint32_t buf = done & 1, turns = (uint32_t)done >> 1;
                good = pair_wait_all(acc_empty0 + 8 * buf, (turns & 1u) ^ 1u, p.status, abort);
                if (!good) break;
                tc_fence_after();
                const uint32_t d = tmem + buf * 256;
                const uint32_t idesc = pair_idesc(tl.width, kTransposed, false);
                uint32_t more = 0;
                for (int k = 0; k < steps; ++k) {
                    good = pair_wait_all(full0 + 8 * at.s, at.phase, p.status, abort);
                    if (!good) break;
                    tc_fence_after();
                    const uint32_t off = at.s * (stage_bytes / 16);
                    if (one) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            pair_mma(d, desc_at(ad0, off + kk * kAStep), desc_at(bd0, off + kk * kBStep), idesc,
                                     kk > 0 ? 1u : more);
                        pair_commit(empty0 + 8 * at.s);
                    }
                    __syncwarp();
                    more = 1;
                    at.next(stages);
                }
                if (good && one) pair_commit(acc_full0 + 8 * buf);
                __syncwarp();
            }
            if (!good && one) {  // the tensor cores are done with shared memory before the CTA ends
                pair_commit(smem_u32(&drain));
                mbar_wait(&drain, 0u, p.status);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------- epilogue
        constexpr int kRows = kMode == kProductUp ? 32 : 16, kGroups = kEpiWarps / 4;
        const int quad = warp & 3, group = (warp - 2) >> 2;
        unsigned char *blocks = turn + group * (kTurnAll / kGroups);  // [4 warps][kRows][128 B]
        const uint32_t empty_addr = map_to_rank(&acc_empty[0], 0);
        // this lane's routed row of a block and its 16 columns
        const int row = kMode == kProductUp ? 8 * quad + (lane >> 2) : 4 * quad + (lane >> 3);
        const int piece = kMode == kProductUp ? lane & 3 : lane & 7;
        int done = 0;
        for (bool any = walk.find(); any; any = walk.next(), ++done) {
            const int buf = done & 1;
            const int c0 = kMode == kProductUp ? tl.m * 128 + (int)rank * 64 + 16 * piece
                                               : tl.m * 256 + (int)rank * 128 + 16 * piece;
            // up_grad: what the first two rows want of the checkpoint comes under the
            // products (fetching the next tile's whole checkpoint to the L2 here read a
            // part of it twice: 372 us against 362)
            Kept kept[2] = {};
            if constexpr (kMode == kProductUpGrad) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (16 * group + 32 * i + row < tl.n) kept[i] = read_kept(p, tl.r0 + 16 * group + 32 * i + row, c0);
            }
            int ok = pair_wait_warp(smem_u32(&acc_full[buf]), (uint32_t)(done >> 1) & 1u, p.status, abort, lane);
            ok = group_and(1 + group, ok);  // the group's warps go on, or give up, together
            if (!ok) break;
            tc_fence_after();
            const uint32_t col = tmem + ((uint32_t)(32 * quad) << 16) + (uint32_t)(buf * 256);
            for (int n0 = kRows * group; n0 < tl.n; n0 += kRows * kGroups) {
                uint32_t r[kRows];
                if constexpr (kMode == kProductUp) tmem_ld32(col + (uint32_t)n0, r);
                else tmem_ld16(col + (uint32_t)n0, r);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < kRows; ++i)
                    *reinterpret_cast<uint32_t *>(blocks + (quad * kRows + i) * 128 + turn_slot(lane >> 2, i, quad) +
                                                  (lane & 3) * 4) = r[i];
                group_sync(1 + group);
                const int n = n0 + row;
                const int64_t at = tl.r0 + n;
                if constexpr (kMode == kProductUp) {
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        load4(v + 4 * j, blocks + (piece * kRows + row) * 128 + turn_slot(j, row, piece));
                    group_sync(1 + group);  // the blocks may be written again
                    if (n < tl.n) finish_up(p, at, c0, v);
                } else {
                    float v[16];
                    const int from = piece >> 1, h = piece & 1;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        load4(v + 4 * j, blocks + (from * kRows + row) * 128 + turn_slot(4 * h + j, row, from));
                    group_sync(1 + group);
                    if constexpr (kMode == kProductPlain) {
                        if (n < tl.n) finish_plain(p, at, c0, v);
                    } else {
                        Kept later = {};
                        if (n + 64 < tl.n) later = read_kept(p, at + 64, c0);
                        float sum = n < tl.n ? finish_grad(p, at, c0, v, kept[0]) : 0.0f;
#pragma unroll
                        for (int o = 1; o < 8; o *= 2) sum += __shfl_xor_sync(kFull, sum, o);
                        if (n < tl.n && piece == 0 && c0 < p.N) p.strips[(int64_t)(c0 / kStrip) * p.R + at] = sum;
                        kept[0] = kept[1];
                        kept[1] = later;
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(empty_addr + 8u * (uint32_t)buf);
        }
    }
    pdl_trigger();  // this CTA's work is done: the next kernel may begin to arrive
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    if (warp == 1) pair_tmem_dealloc(tmem, 512);
}

int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return 0;
    return n;
}

template <int kMode, bool kGather, bool kTransposed>
cudaError_t launch(const ProductArgs &p, cudaStream_t s) {
    PairArgs a = {};
    a.p = p;
    CUtensorMap wmap, amap;
    const uint64_t E = p.E, N = p.N, K = p.K;
    bool ok;
    a.m_tiles = kMode == kProductUp ? (p.N / 2 + 127) / 128 : (p.N + 255) / 256;
    a.m_magic = divide_magic((uint32_t)a.m_tiles);
    if (kMode == kProductUp) {
        ok = encode_gate_up_map(&wmap, p.W, E, N / 2, K);
    } else if (!kTransposed) {
        ok = encode_tensor_map_3d_bf16(&wmap, p.W, E, N, K, 64, 128);
    } else {
        a.paired = N % 64 == 0;
        ok = a.paired ? encode_mn_pair_map(&wmap, p.W, E, K, N) : encode_tensor_map_3d_bf16(&wmap, p.W, E, K, N, 64, 64);
    }
    // a group has at most R rows, so that a step's routed rows fit a narrower ring
    // (and more of it) in small calls
    const uint32_t half = (uint32_t)(p.R < kTileN ? (p.R + 15) / 16 * 16 : kTileN) / 2;
    a.b_bytes = half * 128;
    ok = ok && (kGather ? encode_gather_map(&amap, p.A, (uint64_t)p.a_rows, K)
                        : encode_tensor_map_3d_bf16(&amap, p.A, 1, (uint64_t)p.a_rows, K, 64, half));
    const int sms = sm_count();
    if (!ok || sms < 2) return cudaErrorInvalidValue;
    const uint32_t fixed = 1024 + kTurnAll + table_bytes(p.E) + 2048;
    a.stages = (int)((kSmemLimit - fixed) / (kABytes + a.b_bytes));
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    if (a.stages < kLoadSteps + 1) return cudaErrorInvalidConfiguration;
    const uint32_t smem = 1024 + off_turn(a.stages, a.b_bytes) + kTurnAll + table_bytes(p.E);
    constexpr auto kernel = product_kernel<kMode, kGather, kTransposed>;
    cudaError_t e = ensure_smem_limit<kernel>(kSmemLimit - 2048);
    if (e != cudaSuccess) return e;
    // at most R groups have rows, and a group of n rows has n / 64 + 1 tiles at most
    const int64_t most = (p.R / 64 + min64(p.R, p.E)) * a.m_tiles;
    const int64_t pairs = min64(most, sms / 2);
    return launch_after(kernel, dim3((unsigned)(2 * pairs)), threads_of(kMode, kGather), smem, s, wmap, amap, a);
}

template <bool kGather>
cudaError_t launch_mode(ProductMode mode, const ProductArgs &a, cudaStream_t s) {
    if (mode == kProductUp) return launch<kProductUp, kGather, false>(a, s);
    return a.transposed ? launch<kProductPlain, kGather, true>(a, s) : launch<kProductPlain, kGather, false>(a, s);
}

}  // namespace

cudaError_t launch_product(ProductMode mode, const ProductArgs &a, cudaStream_t s) {
    if (mode == kProductUpGrad) return launch<kProductUpGrad, true, true>(a, s);
    return a.rows ? launch_mode<true>(mode, a, s) : launch_mode<false>(mode, a, s);
}

}  // namespace dol
