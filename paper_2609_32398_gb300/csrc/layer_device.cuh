// What the kernels of a layer for a few tokens share.
#pragma once

#include "experts_mma.cuh"
#include "layer.cuh"

namespace dol {

__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kBehind>
__device__ __forceinline__ void wait_copies() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kBehind) : "memory");
}

// Two codes of a word (the lower or the upper ones) as fp16.  (By the header's function, which packs
// the halves again, 16 cycles a word and warp; so 6.)
template <int kUpper>
__device__ __forceinline__ unsigned codes_half2(unsigned w) {
    unsigned h;
    if (kUpper) asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, u;\n\t}" : "=r"(h) : "r"(w));
    else asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(h) : "r"(w));
    return h;
}
__device__ __forceinline__ unsigned word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// A word's two bf16 values.
__device__ __forceinline__ f32x2 unpack2(unsigned w) {
    return pair2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

__device__ __forceinline__ unsigned load_acquire(const unsigned *p) {
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Waits, by one thread and with a limit, until *count is n; 1: it is.
__device__ __forceinline__ int wait_count(const unsigned *count, unsigned n, int *status) {
    unsigned long long t0 = 0;
    for (unsigned it = 1; load_acquire(count) < n; ++it) {
        if (it & 255u) continue;
        const unsigned long long t = global_ns();
        if (t0 == 0) t0 = t;
        if (t - t0 > kWaitLimitNs) {
            if (status) atomicOr(status, kDevTimeout);
            return 0;
        }
    }
    return 1;
}

}  // namespace dol
