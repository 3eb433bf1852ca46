// Products of 8-bit weights with 8-bit rows on the tcgen05 tensor cores, their blocks'
// powers of two applied by the tensor cores themselves (kind::mxf8f6f4 with block scales:
// e4m3 operands, fp32 accumulation, one exponent byte per row and 32 columns):
//
//   D[m][r] = sum_b 2^(ew[m / 128][b] + ea[row(r)][b] - 254) sum_{k in block b} W_e[m][k] A[row(r)][k]
//
// Tiles, roles and rings are those of the bf16 products (experts_product.cu): the weights
// are the M side, 256 rows over a CTA pair; the ragged rows are the N side in equal
// tiles of at most 240; a step of the ring is 128 columns of k, one block, so that a
// step has one exponent per weight block and per routed row.  240 and not 256: two
// accumulators leave 32 TMEM columns, of which two groups of four steps' exponents take 24.
//
// Exponents.  The instruction wants a word of four bytes for every row, 32 rows to a TMEM
// column, and takes the byte that its descriptor names: a word is a row's exponents of four
// steps, as they lie in memory.  Warps of each CTA write those of its 128 weight rows and of
// all the tile's routed rows to one of four places in shared memory, running ahead of the ring, and the
// MMA's thread has them copied to TMEM before the four steps' products, in order with them.
// (Written for every step, four equal bytes a word, that warp was the bound of short
// contractions: 379 us for 131072 rows of 768 to 2048 columns, of which 195 without it.)
//
// Epilogues: the rows as they are (bf16, or fp32 for a join), and SwiGLU with its result
// in blocks of 1 x 128 again.  A pair's tile is 128 gate rows and their up rows, 64 of each a
// CTA, so that a block's largest value is the larger of the two CTAs': each sends its own
// to the other (st.async into the other's shared memory, counted by a barrier of the
// receiving warp) and finishes the block before while the answer is on its way.
//
// Every wait is bounded; one that runs out records kDevTimeout.
#include <cstdint>

#include "experts8.cuh"
#include "experts_tiles.cuh"

namespace dol {
namespace {

constexpr int kTileN = 240;               // routed rows of a tile at most
constexpr int kEpiWarps = 8;
constexpr int kGroups = kEpiWarps / 4;
constexpr int kScaleWarp = 2 + kEpiWarps;
// Warps that write exponents take the groups of four steps in turn, a place each: a group waits
// for its rows' ids and then for their exponents, 1 to 2 us each under load, and a short contraction
// has a tile of two groups every 2 us (131072 rows of 768: 323 us with one such warp).  Where rows
// are gathered, the loaders leave registers for two.
__host__ __device__ constexpr int scale_warps(bool gather) { return gather ? 2 : 4; }
__host__ __device__ constexpr int first_loader(bool gather) { return kScaleWarp + scale_warps(gather); }
// Gathering warps, as in the bf16 products: load_split of them share a step, kLoadSteps steps
// are filled at a time.
constexpr int kLoadSteps = 3;
__host__ __device__ constexpr int load_split(int mode) { return mode == kProduct8Up ? 2 : 4; }
__host__ __device__ constexpr int load_warps(int mode) { return kLoadSteps * load_split(mode); }
__host__ __device__ constexpr int threads_of(int mode, bool gather) {
    return (first_loader(gather) + (gather ? load_warps(mode) : 1)) * 32;
}
// The epilogue's blocks of 32 (up) or 16 routed rows x 128 values.
__host__ __device__ constexpr int block_rows(int mode) { return mode == kProduct8Up ? 32 : 16; }
__host__ __device__ constexpr uint32_t turn_bytes(int mode) { return kGroups * 4 * block_rows(mode) * 128; }
constexpr uint32_t kABytes = 128 * 128;       // a CTA's weight rows of one step
constexpr uint32_t kScaleBytes = 512 + 1024;  // a CTA's exponents of four steps: weights, routed rows
constexpr int kScalePlaces = 4;
constexpr int kMaxStages = 12;
constexpr uint32_t kSmemLimit = 232448;
constexpr uint32_t kScaleColumn = 2 * kTileN;  // TMEM: 4 columns of weights, 8 of routed rows, twice
constexpr int kUpBlocks = (kTileN + 31) / 32;  // of 32 routed rows in a tile

struct PairArgs8 {
    Product8Args p;
    int m_tiles;       // tiles of 256 weight rows (up: of 128 gate rows and their up rows)
    uint32_t m_magic;  // divide_magic(m_tiles)
    int stages;        // of the ring
    uint32_t b_bytes;  // room for a CTA's routed rows of one step
};

// Shared memory: ring [stages][weights | rows], exponents [places][weights | rows], turn
// blocks, and for each expert its first tile, first row and the width of its tiles [E + 1].
__host__ __device__ inline uint32_t table_bytes(int E) { return 4u * 3u * ((uint32_t)E + 1u); }
__host__ __device__ inline uint32_t off_scales(int stages, uint32_t b_bytes) { return stages * (kABytes + b_bytes); }
__host__ __device__ inline uint32_t off_turn(int stages, uint32_t b_bytes) {
    return off_scales(stages, b_bytes) + kScalePlaces * kScaleBytes;
}

// D (+)= A B with block scales at the TMEM addresses sa and sb.
__device__ __forceinline__ void pair_mma8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                          uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb)
        : "memory");
}
// 32 rows of 16 bytes from shared memory to four TMEM columns, in all four quarters of the
// lanes and in both CTAs, each from its own memory.
__device__ __forceinline__ void pair_copy_scales(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Descriptor of those rows: no swizzle, groups of 8 rows 128 bytes apart.
__device__ __forceinline__ uint64_t desc_scales(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(128 >> 4) << 32) |
           ((uint64_t)1 << 46);
}
// Instruction descriptor: e4m3 A and B, both K-major, exponent bytes as scales, M = 256 over
// the pair, N = n (a multiple of 16), byte j of the exponents' words.
__host__ __device__ constexpr uint32_t pair_idesc8(int n, int j) {
    return ((uint32_t)(n / 8) << 17) | (1u << 23) | ((uint32_t)(256 / 16) << 24) | ((uint32_t)j << 4) | ((uint32_t)j << 29);
}
// A value into the other CTA's shared memory, its four bytes counted on a barrier there.
__device__ __forceinline__ void send_word(uint32_t to, unsigned v, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(to), "r"(v), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void finish_plain(const Product8Args &p, int64_t r, int c0, const float (&v)[16]) {
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

// 16 values of the activation, kept until the other CTA's largest value is there.
struct Waiting {
    float act[16];
    unsigned top;  // bits of this CTA's largest magnitude of the row
    int n;         // the row in its tile; -1: none is waiting
};

template <int kMode, bool kGather>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(threads_of(kMode, kGather), 1)
product8_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap amap, const PairArgs8 a) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_align<1024>(smem_raw);
    constexpr int kThreads = threads_of(kMode, kGather), kFirstLoader = first_loader(kGather);
    const Product8Args &p = a.p;
    const int E = p.E, stages = a.stages;
    const uint32_t stage_bytes = kABytes + a.b_bytes;
    unsigned char *scales = smem + off_scales(stages, a.b_bytes), *turn = smem + off_turn(stages, a.b_bytes);
    int *first = reinterpret_cast<int *>(turn + turn_bytes(kMode)), *start = first + E + 1, *width = start + E + 1;
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drain;
    __shared__ __align__(8) uint64_t scales_full[kScalePlaces], scales_empty[kScalePlaces];
    __shared__ __align__(8) uint64_t top_here[2][kUpBlocks][4];  // up: the other CTA's values are here
    __shared__ unsigned top_of[2][kUpBlocks * 32];
    __shared__ uint32_t tmem_slot;
    __shared__ int s_abort, s_part[kThreads / 32];
    volatile int *abort = &s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(&full[i], 1 + (kGather ? 2 * load_split(kMode) : 0));
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < kScalePlaces; ++i) {
            mbar_init(&scales_full[i], 2);
            mbar_init(&scales_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], 2 * kEpiWarps);
        }
        if (kMode == kProduct8Up)
            for (int i = 0; i < 2 * kUpBlocks * 4; ++i) mbar_init(&top_here[0][0][0] + i, 1);
        mbar_init(&drain, 1);
        s_abort = 0;
        fence_barrier_init();
        prefetch_tensormap(&wmap);
        prefetch_tensormap(&amap);
    }
    pdl_wait();
    // not before: the kernel before may share this SM and still have to take its own
    if (warp == 1) pair_tmem_alloc(&tmem_slot, 512);
    const int pairs = (int)(gridDim.x >> 1);
    const int carry = tile_table<kTileN, kThreads>(p.offsets, E, p.R, a.m_tiles, pairs, first, start, width, s_part);
    if (threadIdx.x == 0) first[E] = carry;
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int steps = blocks8(p.K);
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
            for (int k = 0; k < p.K; k += 128, ++it) {
                good = pair_wait_all(empty0 + 8 * at.s, at.phase ^ 1u, p.status, abort);
                if (!good) break;
                const uint32_t st = ring + at.s * stage_bytes, bar = full_pair + 8 * at.s;
                if (one) {
                    if (rank == 0) mbar_expect_tx_addr(full0 + 8 * at.s, bytes);
                    if constexpr (kMode == kProduct8Up) pair_load_5d(st, &wmap, k, 0, 0, mb, tl.e, bar);
                    else pair_load_3d(st, &wmap, k, m0, tl.e, bar);
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
    } else if (warp >= kScaleWarp && warp < kFirstLoader) {
        // ---------------------------------------------------------- exponents
        // Lane l has rows l, 32 + l, ... of the weights (all of a block share one; up: 16 gate
        // rows and 16 up rows in turn) and of the tile.
        Ring at{0, 0};
        bool good = true;
        const int none = (int)p.a_rows;
        const int nb = kMode == kProduct8Up ? blocks8(p.N / 2) : blocks8(p.N);
        const unsigned unit = 0x7f7f7f7fu;  // scale 1, for what nobody reads
        const uint32_t empty_addr = smem_u32(scales_empty), full_addr = map_to_rank(scales_full, 0);
        constexpr int kTurns = scale_warps(kGather);
        int turn = 0;  // whose the next group is
        auto four = [&](const uint8_t *row, int k) -> unsigned {  // of steps k .. k + 3, k a multiple of 4
            if (!row) return unit;
            if (p.align == 4) return __ldg(reinterpret_cast<const unsigned *>(row + k));
            unsigned w = 0;
            if (p.align == 2) {
                w = __ldg(reinterpret_cast<const unsigned short *>(row + k));
                if (k + 2 < steps) w |= (unsigned)__ldg(reinterpret_cast<const unsigned short *>(row + k + 2)) << 16;
                return w;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k + j < steps) w |= (unsigned)__ldg(row + k + j) << (8 * j);
            return w;
        };
        for (bool any = walk.find(); good && any; any = walk.next()) {
            const uint8_t *row[8], *weight = nullptr;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const int n = 32 * c + lane;
                int id = n < tl.n ? tl.r0 + n : none;
                if (kGather && n < tl.n) id = __ldg(p.rows + tl.r0 + n);
                row[c] = id >= 0 && id < none ? p.ax + (int64_t)id * steps : nullptr;
            }
            if (kMode == kProduct8Up) {
                const int plane = 2 * tl.e + (lane >> 4);
                weight = p.wx + ((int64_t)plane * nb + tl.m) * steps;
            } else if (2 * tl.m + (int)rank < nb) {
                weight = p.wx + ((int64_t)tl.e * nb + 2 * tl.m + (int)rank) * steps;
            }
            for (int k = 0; good && k < steps; k += 4, at.next(kScalePlaces), turn = turn + 1 == kTurns ? 0 : turn + 1) {
                if (turn != warp - kScaleWarp) continue;
                unsigned now[9];
#pragma unroll
                for (int c = 0; c < 8; ++c) now[c] = four(row[c], k);
                now[8] = four(weight, k);
                good = pair_wait_warp(empty_addr + 8 * at.s, at.phase ^ 1u, p.status, abort, lane);
                if (!good) break;
                uint4 *to = reinterpret_cast<uint4 *>(scales + at.s * kScaleBytes) + lane;
                to[0] = make_uint4(now[8], now[8], now[8], now[8]);
                to[32] = make_uint4(now[0], now[1], now[2], now[3]);
                to[64] = make_uint4(now[4], now[5], now[6], now[7]);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(full_addr + 8 * at.s);
            }
        }
        __syncwarp();
    } else if (!kGather && warp == kFirstLoader) {
        // ---------------------------------------------------------- rows in dispatch order
        const bool one = elect_one();
        Ring at{0, 0};
        bool good = true;
        for (bool any = walk.find(); good && any; any = walk.next()) {
            const int r = tl.r0 + (int)rank * (tl.width / 2);
            for (int k = 0; k < p.K; k += 128) {
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
                    pair_gather4(ring + (uint32_t)s * stage_bytes + kABytes + mine4 * 128, &amap, 128 * (mine - it), ids,
                                 full_pair + 8 * s);
                __syncwarp();
                // a step waits for each of its warps, with copies or (a narrow tile) without
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
            Ring at{0, 0}, place{0, 0};
            int done = 0;
            bool good = true;
            const uint64_t ad0 = umma_desc_sw128(ring), bd0 = umma_desc_sw128(ring + kABytes);
            const uint64_t sd0 = desc_scales(smem_u32(scales));
            const uint32_t acc_full0 = smem_u32(acc_full), acc_empty0 = smem_u32(acc_empty);
            const uint32_t scales_full0 = smem_u32(scales_full), scales_empty0 = smem_u32(scales_empty);
            uint32_t sa = tmem + kScaleColumn;
            for (bool any = walk.find(); good && any; any = walk.next(), ++done) {
                const uint32_t buf = done & 1, turns = (uint32_t)done >> 1;
                good = pair_wait_all(acc_empty0 + 8 * buf, (turns & 1u) ^ 1u, p.status, abort);
                if (!good) break;
                tc_fence_after();
                const uint32_t d = tmem + buf * kTileN;
                const uint32_t idesc = pair_idesc8(tl.width, 0);
                uint32_t more = 0;
                for (int k = 0; k < steps; ++k) {
                    if ((k & 3) == 0) {
                        good = pair_wait_all(scales_full0 + 8 * place.s, place.phase, p.status, abort);
                        if (!good) break;
                        tc_fence_after();
                        sa = (tmem + kScaleColumn) + (tmem + kScaleColumn + 12 - sa);  // the other place
                        const uint32_t off = place.s * (kScaleBytes / 16);
                        if (one) {
                            pair_copy_scales(sa, desc_at(sd0, off));
                            pair_copy_scales(sa + 4, desc_at(sd0, off + 512 / 16));
                            pair_copy_scales(sa + 8, desc_at(sd0, off + 1024 / 16));
                            pair_commit(scales_empty0 + 8 * place.s);
                        }
                        __syncwarp();
                        place.next(kScalePlaces);
                    }
                    good = pair_wait_all(full0 + 8 * at.s, at.phase, p.status, abort);
                    if (!good) break;
                    tc_fence_after();
                    const uint32_t off = at.s * (stage_bytes / 16), pick = (uint32_t)(k & 3) * ((1u << 4) | (1u << 29));
                    if (one) {
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            pair_mma8(d, desc_at(ad0, off + kk * (32 / 16)), desc_at(bd0, off + kk * (32 / 16)), idesc | pick, sa,
                                      sa + 4, kk > 0 ? 1u : more);
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
        constexpr int kRows = block_rows(kMode);
        const int quad = warp & 3, group = (warp - 2) >> 2;
        unsigned char *blocks = turn + group * (turn_bytes(kMode) / kGroups);  // [4 warps][kRows][128 B]
        const uint32_t empty_addr = map_to_rank(&acc_empty[0], 0);
        // this lane's routed row of a block and its 16 columns
        const int row = kMode == kProduct8Up ? 8 * quad + (lane >> 2) : 4 * quad + (lane >> 3);
        const int piece = kMode == kProduct8Up ? lane & 3 : lane & 7;
        const uint32_t there = map_to_rank(&top_of[0][0], rank ^ 1u), there_bar = map_to_rank(&top_here[0][0][0], rank ^ 1u);
        uint32_t waits[2] = {0u, 0u};  // phase of this warp's barrier of each block
        int done = 0;
        for (bool any = walk.find(); any; any = walk.next(), ++done) {
            const int buf = done & 1;
            const int c0 = kMode == kProduct8Up ? tl.m * 128 + (int)rank * 64 + 16 * piece
                                                : tl.m * 256 + (int)rank * 128 + 16 * piece;
            int ok = pair_wait_warp(smem_u32(&acc_full[buf]), (uint32_t)(done >> 1) & 1u, p.status, abort, lane);
            ok = group_and(1 + group, ok);  // the group's warps go on, or give up, together
            if (!ok) break;
            tc_fence_after();
            const uint32_t col = tmem + ((uint32_t)(32 * quad) << 16) + (uint32_t)(buf * kTileN);
            Waiting held;
            held.n = -1;
            auto finish_up = [&]() {
                // the other CTA's largest value of each row of the block has come
                const int blk = held.n >> 5;
                uint32_t &phase = waits[buf];
                // (every lane waits for itself: what one lane has acquired, the others may read too early)
                pair_wait_all(smem_u32(&top_here[buf][blk][quad]), phase >> blk & 1u, p.status, abort);
                phase ^= 1u << blk;
                const unsigned top = max(held.top, *reinterpret_cast<volatile unsigned *>(&top_of[buf][held.n]));
                const int e = e8_exponent(top);
                const float inv = e8_inverse(e);
                const int F = p.N / 2;
                if (held.n >= tl.n || c0 >= F) return;
                const int64_t at = tl.r0 + held.n;
                const float *v = held.act;
                *reinterpret_cast<uint4 *>(p.codes + at * F + c0) =
                    make_uint4(e8_codes4(v[0], v[1], v[2], v[3], inv), e8_codes4(v[4], v[5], v[6], v[7], inv),
                               e8_codes4(v[8], v[9], v[10], v[11], inv), e8_codes4(v[12], v[13], v[14], v[15], inv));
                if (rank == 0 && piece == 0) p.exponents[at * blocks8(F) + tl.m] = (uint8_t)e;
            };
            for (int n0 = kRows * group; n0 < tl.n; n0 += kRows * kGroups) {
                uint32_t r[kRows];
                if constexpr (kMode == kProduct8Up) tmem_ld32(col + (uint32_t)n0, r);
                else tmem_ld16(col + (uint32_t)n0, r);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < kRows; ++i)
                    *reinterpret_cast<uint32_t *>(blocks + (quad * kRows + i) * 128 + turn_slot(lane >> 2, i, quad) +
                                                  (lane & 3) * 4) = r[i];
                group_sync(1 + group);
                const int n = n0 + row;
                if constexpr (kMode == kProduct8Up) {
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        load4(v + 4 * j, blocks + (piece * kRows + row) * 128 + turn_slot(j, row, piece));
                    group_sync(1 + group);  // the blocks may be written again
                    unsigned top = 0;
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        const f32x2 g = pair2(v[i], v[i + 1]);
                        split2(mul2(mul2(g, sigmoid2(g)), pair2(v[16 + i], v[17 + i])), v[i], v[i + 1]);
                        top = abs_max(abs_max(top, v[i]), v[i + 1]);
                    }
                    top = max(top, __shfl_xor_sync(kFull, top, 1));
                    top = max(top, __shfl_xor_sync(kFull, top, 2));
                    const int bar = (buf * kUpBlocks + (n0 >> 5)) * 4 + quad;
                    if (lane == 0) mbar_expect_tx_addr(smem_u32(&top_here[0][0][0] + bar), 32u);
                    if (piece == 0) send_word(there + 4u * (uint32_t)(buf * kUpBlocks * 32 + n), top, there_bar + 8u * (uint32_t)bar);
                    if (held.n >= 0) finish_up();
#pragma unroll
                    for (int i = 0; i < 16; ++i) held.act[i] = v[i];
                    held.top = top;
                    held.n = n;
                } else {
                    float v[16];
                    const int from = piece >> 1, h = piece & 1;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        load4(v + 4 * j, blocks + (from * kRows + row) * 128 + turn_slot(4 * h + j, row, from));
                    group_sync(1 + group);
                    if (n < tl.n) finish_plain(p, tl.r0 + n, c0, v);
                }
            }
            // before this buffer is given back: the other CTA may send its next tile's values then
            if (kMode == kProduct8Up && held.n >= 0) finish_up();
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

template <int kMode, bool kGather>
cudaError_t launch(const Product8Args &p, cudaStream_t s) {
    PairArgs8 a = {};
    a.p = p;
    const uintptr_t lowest = reinterpret_cast<uintptr_t>(p.ax) | reinterpret_cast<uintptr_t>(p.wx) | (uintptr_t)blocks8(p.K);
    a.p.align = lowest % 4 == 0 ? 4 : lowest % 2 == 0 ? 2 : 1;
    CUtensorMap wmap, amap;
    const uint64_t E = p.E, N = p.N, K = p.K;
    a.m_tiles = kMode == kProduct8Up ? (p.N / 2 + 127) / 128 : (p.N + 255) / 256;
    a.m_magic = divide_magic((uint32_t)a.m_tiles);
    bool ok = kMode == kProduct8Up ? encode_gate_up_map_u8(&wmap, p.W, E, N / 2, K)
                                   : encode_tensor_map_3d_u8(&wmap, p.W, E, N, K, 128, 128);
    // a group has at most R rows, so that a step's routed rows fit a narrower ring
    // (and more of it) in small calls
    const uint32_t half = (uint32_t)(p.R < kTileN ? (p.R + 15) / 16 * 16 : kTileN) / 2;
    a.b_bytes = half * 128;
    ok = ok && (kGather ? encode_gather_map_u8(&amap, p.A, (uint64_t)p.a_rows, K)
                        : encode_tensor_map_3d_u8(&amap, p.A, 1, (uint64_t)p.a_rows, K, 128, half));
    const int sms = sm_count();
    if (!ok || sms < 2) return cudaErrorInvalidValue;
    const uint32_t fixed = 1024 + kScalePlaces * kScaleBytes + turn_bytes(kMode) + table_bytes(p.E) + 4096;
    a.stages = (int)((kSmemLimit - fixed) / (kABytes + a.b_bytes));
    if (a.stages > kMaxStages) a.stages = kMaxStages;
    if (a.stages < kLoadSteps + 1) return cudaErrorInvalidConfiguration;
    const uint32_t smem = 1024 + off_turn(a.stages, a.b_bytes) + turn_bytes(kMode) + table_bytes(p.E);
    constexpr auto kernel = product8_kernel<kMode, kGather>;
    cudaError_t e = ensure_smem_limit<kernel>(kSmemLimit - 4096);
    if (e != cudaSuccess) return e;
    // at most R groups have rows, and a group of n rows has n / 64 + 1 tiles at most
    const int64_t most = (p.R / 64 + min64(p.R, p.E)) * a.m_tiles;
    const int64_t pairs = min64(most, sms / 2);
    return launch_after(kernel, dim3((unsigned)(2 * pairs)), threads_of(kMode, kGather), smem, s, wmap, amap, a);
}

}  // namespace

cudaError_t launch_product8(Product8Mode mode, const Product8Args &a, cudaStream_t s) {
    if (mode == kProduct8Up) return a.rows ? launch<kProduct8Up, true>(a, s) : launch<kProduct8Up, false>(a, s);
    return a.rows ? launch<kProduct8Plain, true>(a, s) : launch<kProduct8Plain, false>(a, s);
}

}  // namespace dol
