// What the C entry points of the expert operators share: checks of their arguments and the
// room that a join takes.
#pragma once

#include <climits>

#include "doloss.h"
#include "experts.cuh"

namespace dol {

inline bool off(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }
inline size_t round256(size_t x) { return (x + 255) / 256 * 256; }
inline do_status of(cudaError_t e) { return e == cudaSuccess ? DO_OK : DO_ERR_CUDA; }

// Sizes that every call shares.  Columns are whole pieces of step0 and step1 values.
inline do_status check_sizes(int64_t R, int32_t E, int32_t c0, int32_t c1, int step0, int step1) {
    if (R < 1 || E < 1 || c0 < 1 || c1 < 1) return DO_ERR_INVALID_ARG;
    if (E > 1024 || R > INT32_MAX - 256 || c0 % step0 || c1 % step1 || c0 > (1 << 17) || c1 > (1 << 17))
        return DO_ERR_UNSUPPORTED;
    return DO_OK;
}

// The rows that a join adds are kept in fp32 where they stay in the L2 anyway: the sum
// is then rounded once, and nothing is read from memory twice as wide.  Past that they are
// bf16, half of the bytes that bound the join (0.5 GB each way for 131072 rows of 2048): an
// error of 2.3e-3 of the result's norm instead of 1.7e-3.
inline bool join_wide(int64_t R, int32_t N) { return R * N <= (int64_t)(96 << 20) / 4; }
inline size_t join_bytes(int64_t R, int32_t N) {
    return round256((join_wide(R, N) ? sizeof(float) : sizeof(bf16)) * (size_t)R * (size_t)N);
}

}  // namespace dol
