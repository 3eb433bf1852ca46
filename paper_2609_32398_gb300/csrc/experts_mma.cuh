// PTX of the CTA-pair kernels of the expert operators: thread-block clusters of
// two, tcgen05 with cta_group::2 (one accumulator of 256 rows over two SMs) and
// row-gathering TMA loads.
#pragma once

#include "experts.cuh"
#include "tma.cuh"

namespace dol {

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Address, in the cluster's shared window, of this CTA's `p` as CTA `rank` has it.
__device__ __forceinline__ uint32_t map_to_rank(const void *p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}

// Arrive on a barrier of either CTA of the pair.  What the arrival stands for lies in
// this CTA's shared memory or TMEM and has been completed and fenced by the caller
// (a proxy fence after the copies' wait, or tcgen05.wait and its fence), and the tensor
// core that uses it next is this SM's own, so that the arrival need not be a release
// over the cluster: that one waits for every access of the thread in flight, and made a
// step of a ring of copies cost 690 ns instead of 270.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}

__device__ __forceinline__ bool mbar_try_wait_addr(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Bounded wait (as mbar_wait) with cluster scope on the barrier at a shared address;
// gives up when the CTA has given up elsewhere.  The clock is read every 1024 tries
// only, as reading it takes longer than most waits.
__device__ __forceinline__ bool pair_wait_slow(uint32_t bar, uint32_t parity, int *status, volatile int *abort) {
    unsigned long long t0 = 0;
    for (uint32_t it = 1;; ++it) {
        if (mbar_try_wait_addr(bar, parity)) return true;
        if ((it & 1023u) == 0u) {
            const unsigned long long t = global_ns();
            if (t0 == 0) t0 = t;
            if (*abort || t - t0 > kWaitLimitNs) {
                if (status) atomicOr(status, kDevTimeout);
                *abort = 1;
                return false;
            }
        }
    }
}
__device__ __forceinline__ bool pair_wait(uint32_t bar, uint32_t parity, int *status, volatile int *abort) {
    if (mbar_try_wait_addr(bar, parity)) return true;
    return pair_wait_slow(bar, parity, status, abort);
}

// The wait of a warp that issues copies or MMAs.  Such a warp walks its loop as a whole
// and lets one lane issue: the operands of these instructions are then in the uniform
// registers that they are read from, where a loop of a single lane moves each of them
// there first (a plain product of 131072 x 2048 x 1536 took 486 us with one lane, 431 with
// the warp).  All lanes leave with the same answer.
__device__ __forceinline__ bool pair_wait_all(uint32_t bar, uint32_t parity, int *status, volatile int *abort) {
    unsigned long long t0 = 0;
    for (uint32_t it = 1;; ++it) {
        if (__all_sync(kFull, mbar_try_wait_addr(bar, parity))) return true;
        if ((it & 1023u) == 0u) {
            const unsigned long long t = global_ns();
            if (t0 == 0) t0 = t;
            if (__any_sync(kFull, *abort || t - t0 > kWaitLimitNs)) {
                if (status) atomicOr(status, kDevTimeout);
                *abort = 1;
                return false;
            }
        }
    }
}

// One lane of a converged warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(one));
    return one != 0;
}

// The same by a whole warp: one lane polls (32 lanes polling cost the shared memory
// that the tensor cores read from), the others follow it.
__device__ __forceinline__ bool pair_wait_warp(uint32_t bar, uint32_t parity, int *status, volatile int *abort,
                                               int lane) {
    int ok = 1;
    if (lane == 0) ok = pair_wait(bar, parity, status, abort);
    return __shfl_sync(kFull, ok, 0) != 0;
}

__device__ __forceinline__ void mbar_expect_tx_addr(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// A place in the ring, as an issuing warp walks it: such a warp is one dependent chain,
// in which the division of a step number by the number of stages alone cost 60 ns a
// step.
struct Ring {
    uint32_t s, phase;  // stage; how often the ring has been walked, mod 2
    __device__ __forceinline__ void next(uint32_t stages) {
        if (++s == stages) {
            s = 0;
            phase ^= 1u;
        }
    }
};

// TMA loads of a CTA pair: the data goes to this CTA, the bytes are counted on
// `bar`, an address in the cluster's shared window (the pair's first CTA).
__device__ __forceinline__ void pair_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void pair_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int u,
                                             uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(u), "r"(bar)
        : "memory");
}

__device__ __forceinline__ void pair_load_5d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int u, int v,
                                             uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(u), "r"(v), "r"(bar)
        : "memory");
}

// Four rows of a bf16 matrix (64 columns from x on) into four consecutive 128-byte rows;
// a row outside the matrix reads as zeros.
__device__ __forceinline__ void pair_gather4(uint32_t dst, const CUtensorMap *map, int x, int4 r, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w), "r"(bar)
        : "memory");
}

// 16 bytes global -> shared, zeros where !in (nothing is read then).
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
// A warp's copies of a step are done and visible to the tensor cores: tells the pair.
__device__ __forceinline__ void gathered(uint32_t full_addr, int lane) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive_cluster(full_addr);
}

// Gathering.  The products bring rows by TMA copies of four (pair_gather4).  Such a copy
// takes its lane 85 to 100 cycles to issue and a step has up to 32, so that what bounds
// the ring is how long a step's copies take to leave: with one warp a step they took 1.4
// of the 2.8 us that a stage is on its way (up projection of 16384 tokens, H = 2048: 550
// us with six warps of a step each, 508 with three pairs, 486 with three times four, 707
// with all six on one step; the same rows in dispatch order 465).  cp.async in 16-byte
// pieces took as long as six warps, and half of the rows each way no less.  The weight
// gradients bring theirs by cp.async, a warp a step: their results leave by TMA, which
// the copies of four rows then hold up (dW1 of 16384 tokens: 627 us against 679).
//
// The rings' barriers are waited for by parity, which can tell one phase from the next
// only.  So every warp that waits for a stage is one that the stage's next phase waits
// for: each arrives on every step that it takes part in, whether it had copies to issue
// or not; and no warp is ahead by more than the ring: it waits at each of its steps, and
// its last one was fewer than `stages` steps before.
constexpr int kLoadWarps = 6;  // of the weight gradients, one for each stage of the ring

__device__ __forceinline__ void tma_reduce_add_3d(const CUtensorMap *map, const void *src, int x, int y, int z) {
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::
                     "l"(reinterpret_cast<uint64_t>(map)),
                 "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z)
                 : "memory");
}

// One warp of each CTA of the pair calls these.
__device__ __forceinline__ void pair_tmem_alloc(uint32_t *dst, uint32_t ncols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(ncols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_tmem_dealloc(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}

// D (256 rows over the pair) (+)= A B, issued by one thread of the first CTA.
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Arrive on `bar` of both CTAs when the MMAs issued so far by this thread are done.
__device__ __forceinline__ void pair_commit(uint32_t bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            bar),
        "h"((uint16_t)3)
        : "memory");
}

// Descriptor of an MN-major bf16 operand in the 128-byte swizzled layout: rows of
// 64 MN-contiguous elements along K, 8-row groups 1024 bytes apart, consecutive
// 64-wide MN blocks `mn_stride` bytes apart.
__device__ __forceinline__ uint64_t desc_mn_sw128(uint32_t addr, uint32_t mn_stride) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)((mn_stride >> 4) & 0x3FFFu) << 16) |
           ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// A descriptor moved on by `off` 16-byte units: the address lies in its low word.
__device__ __forceinline__ uint64_t desc_at(uint64_t desc, uint32_t off) {
    return (desc & 0xffffffff00000000ull) | ((uint32_t)desc + off);
}

// kind::f16 instruction descriptor: fp32 D, bf16 A and B, M = 256 over the pair,
// N = n (a multiple of 16).
__host__ __device__ constexpr uint32_t pair_idesc(int n, bool a_mn, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
           ((uint32_t)(n / 8) << 17) | ((uint32_t)(256 / 16) << 24);
}

// i / d for i up to divide_limit(d), by the product with m = ceil(2^32 / d) (0 stands for d
// = 1): exact while i (m d - 2^32) < 2^32.
__host__ __device__ inline uint32_t divide_magic(uint32_t d) { return d == 1 ? 0u : 0xffffffffu / d + 1u; }
inline uint64_t divide_limit(uint32_t d) {
    const uint64_t over = (uint64_t)divide_magic(d) * d - (1ull << 32);  // below d; 0 for a power of two
    return d == 1 || over == 0 ? UINT32_MAX : UINT32_MAX / over;
}
__device__ __forceinline__ int divide_by(int i, uint32_t magic) {
    return magic ? (int)__umulhi((uint32_t)i, magic) : i;
}

// Host: the pair kernels' tensor maps (128-byte swizzle, zero outside the tensor).
// Rows of a bf16 matrix, gathered four at a time, 64 columns each.
bool encode_gather_map(CUtensorMap *map, const void *base, uint64_t rows, uint64_t cols);
// W1 [E][2F][H] as [E][F/16][2][16][H], box 1 x 4 x 2 x 16 x 64: 64 columns of 64
// gate rows and their 64 up rows, 16 of each in turn.
bool encode_gate_up_map(CUtensorMap *map, const void *base, uint64_t E, uint64_t F, uint64_t H);

// A bf16 tensor [planes][rows][cols], cols a multiple of 64, as [planes][cols / 64]
// [rows][64], box 1 x 2 x 64 x 64: 128 columns of 64 rows, MN-major, in one copy (a
// copy costs its thread 60 ns, whatever it carries).
bool encode_mn_pair_map(CUtensorMap *map, const void *base, uint64_t planes, uint64_t rows, uint64_t cols);

}  // namespace dol
