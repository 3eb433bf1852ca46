// The experts of a handful of routed rows and their join in one kernel: layer_experts.cu for
// a decode step of one or two tokens, where a weight row meets one token and the work is a
// stream of dot products.  Each warp has an equal share, to the pair of gate and up rows, of all
// pairs of all routed rows: a lane loads 16 bytes of each 512 of both rows, 128 KB in flight
// an SM.  For W2 each CTA has a block of out's columns, and its rows (all of them, 172 KB for one
// token of eight experts of 768) are on their way to shared memory right behind the last of W1's, so
// that the memory is not idle while the grid waits for the last activation.  Rows that share an
// expert read its weights again, from the L2.
//
// Order: as in layer_experts.cu, ranges of W1 go by tickets, and nobody waits for one that has
// not been taken by a running CTA.  Sums are fp32, lane by lane in order, then over the
// lanes; sixteen codes of a block of 8-bit weights are summed before most of its power of two is
// applied (dot16).
#include <cuda_fp16.h>

#include "layer.cuh"
#include "layer_device.cuh"
#include "tma.cuh"

namespace dol {
namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32;

// Loads that stay where they are written, and in order.
__device__ __forceinline__ uint4 load_stream(const unsigned char *p, bool in) {
    uint4 v;
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %5, 0;\n\t"
        "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
        "@p ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
        : "l"(p), "r"((int)in));
    return v;
}

// Two fp16 values times the fp16 number c, in fp32: exact.
__device__ __forceinline__ f32x2 halves2(unsigned h, unsigned short c) {
    float lo, hi;
    asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\t"
        "fma.rn.f32.f16 %0, l, %3, %4;\n\tfma.rn.f32.f16 %1, u, %3, %4;\n\t}"
        : "=f"(lo), "=f"(hi)
        : "r"(h), "h"(c), "f"(0.0f));
    return pair2(lo, hi);
}
// kRows weight rows' 16 bytes (8 values, or 16 codes of one block) with the values at x; sums +=.
// Codes of ordinary weights are some 2^12 times the weights: up to 2^-14 of a block's power of two goes
// to each code, on its way from fp16 to fp32, where it costs nothing, and the rest to the sum, so that
// neither a product nor a sum of sixteen leaves fp32's range at either end where the result does not.
// kWide: the values at x are fp32, the lane's 16-byte pieces 512 bytes apart (otherwise bf16, one after
// the other).
template <bool k8, bool kWide, int kRows>
__device__ __forceinline__ void dot16(const uint4 (&w)[kRows], const unsigned char *x, const int (&e)[kRows], float (&sum)[kRows]) {
    f32x2 s[kRows];
    unsigned short first[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        s[i] = pair2(0.0f, 0.0f);
        first[i] = (unsigned short)((k8 ? min(max(e[i] - 112, 1), 15) : 0) << 10);  // an fp16 power of two, 2^-14 to 1
    }
#pragma unroll
    for (int h = 0; h < (k8 ? 2 : 1); ++h) {
        f32x2 x2[4];
        if constexpr (kWide) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(x + 512 * (2 * h + j));
                x2[2 * j] = v.x;
                x2[2 * j + 1] = v.y;
            }
        } else {
            const uint4 v = *reinterpret_cast<const uint4 *>(x + 16 * h);
#pragma unroll
            for (int j = 0; j < 4; ++j) x2[j] = unpack2(word(v, j));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x2 xv = x2[j];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const unsigned c = word(w[i], k8 ? 2 * h + j / 2 : j);
                const f32x2 wv = k8 ? halves2(j & 1 ? codes_half2<1>(c) : codes_half2<0>(c), first[i]) : unpack2(c);
                s[i] = fma2(wv, xv, s[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        float a, b;
        split2(s[i], a, b);
        const int rest = k8 ? max(e[i], min(e[i] + 14, 127)) : 0;
        sum[i] = k8 ? fmaf(a + b, __uint_as_float(rest == 255 ? 0x7fc00000u : (unsigned)rest << 23), sum[i]) : sum[i] + (a + b);
    }
}

// The pairs of gate and up rows [lo, hi) of the list of all R F.
template <bool k8>
struct UpStream {
    static constexpr int kChunk = k8 ? 4 : 8;      // pieces of 512 bytes of both rows in a step
    static constexpr int kSteps = k8 ? 2 : 1;      // on their way together, 64 registers
    const LayerArgs &p;
    const unsigned char *x;  // tokens in shared memory
    const int *ids;          // each routed row's expert, there too
    int x_stride, lane, pieces, chunks, row_bytes, hi;
    // of the loads: pair, chunk and where they are
    int pair, row, f, chunk;
    const unsigned char *w;
    const uint8_t *wx;

    struct Step {
        uint4 w[kChunk][2];
        int e[kChunk][2];
        int row, f, chunk;  // row < 0: none
    };

    __device__ __forceinline__ void locate() {
        const int e = ids[row];
        w = static_cast<const unsigned char *>(p.w1) + ((int64_t)e * 2 * p.F + f) * row_bytes + lane * 16;
        if (k8) wx = p.w1x + ((int64_t)e * 2 * blocks8(p.F) + f / kBlock8) * blocks8(p.H) + lane / 8;
    }
    __device__ __forceinline__ void load(Step &s) {
        s.row = pair < hi ? row : -1;
        s.f = f;
        s.chunk = chunk;
        if (pair >= hi) return;
        const int left = row_bytes - chunk * (kChunk * 512) - lane * 16;
        const unsigned char *up = w + (int64_t)p.F * row_bytes;
#pragma unroll
        for (int j = 0; j < kChunk; ++j) s.w[j][0] = load_stream(w + j * 512, j * 512 < left);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) s.w[j][1] = load_stream(up + j * 512, j * 512 < left);
        if constexpr (k8) {
            const uint8_t *up_x = wx + (int64_t)blocks8(p.F) * blocks8(p.H);
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
                s.e[j][0] = j * 512 < left ? (int)__ldg(wx + 4 * j) : 127;
                s.e[j][1] = j * 512 < left ? (int)__ldg(up_x + 4 * j) : 127;
            }
            wx += kChunk * 4;
        }
        w += kChunk * 512;
        if (++chunk == chunks) {
            chunk = 0;
            ++pair;
            if (++f == p.F) {
                f = 0;
                ++row;
            }
            if (pair < hi) locate();
        }
    }
    __device__ __forceinline__ void sum(const Step &s, float (&d)[2]) {
        if (s.row < 0) return;
        if (s.chunk == 0) d[0] = d[1] = 0.0f;
        const unsigned char *at = x + (s.row / p.k) * x_stride + s.chunk * (kChunk * (k8 ? 1024 : 512)) + lane * (k8 ? 32 : 16);
#pragma unroll
        for (int j = 0; j < kChunk; ++j)
            if (s.chunk * kChunk + j < pieces) dot16<k8, false>(s.w[j], at + j * (k8 ? 1024 : 512), s.e[j], d);
        if (s.chunk == chunks - 1) {
            const float gate = warp_sum(d[0]), up = warp_sum(d[1]);
            // bf16 weights: rounded as for more rows, where the tensor cores take bf16 (2.3e-3 of the result's
            // norm instead of 1.7e-3).  In fp32, one token took 25.1 us against 23.7, and 86.1 against 78.0 with H =
            // 4096, F = 2048; with codes 23.5 against 23.1 and 62.6 against 64.7.
            const float act = gate * sigmoid_f(gate) * up;
            const int64_t to = (int64_t)s.row * p.F + s.f;
            if (lane == 0) {
                if constexpr (k8) static_cast<float *>(p.act)[to] = act;
                else static_cast<bf16 *>(p.act)[to] = __float2bfloat16_rn(act);
            }
        }
    }
    // `then` runs when the last loads have left.
    template <class Then>
    __device__ __forceinline__ void run(int lo, const Then &then) {
        pair = lo;
        chunk = 0;
        row = lo / p.F;
        f = lo - row * p.F;
        if (pair < hi) locate();
        float d[2] = {0.0f, 0.0f};
        Step step[kSteps];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) load(step[i]);
        if (pair >= hi) then();
        while (step[0].row >= 0) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) sum(step[i], d);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) load(step[i]);
            if (pair >= hi) then();
        }
    }
};

// Rows of `pieces` times 16 bytes to shared memory, `stride` bytes apart and zero up to it; piece c
// goes to place(c) of its row.
template <class From, class Place>
__device__ __forceinline__ void bring_rows(unsigned char *to, int rows, int pieces, int stride, const From &from, const Place &place) {
    const int each = stride / 16;
#pragma unroll 4
    for (int i = threadIdx.x; i < rows * each; i += kThreads) {
        const int r = i / each, c = i - r * each;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (c < pieces) v = from(r, c);
        *reinterpret_cast<uint4 *>(to + r * stride + 16 * place(c)) = v;
    }
}

// Shared memory: tokens [T], activations [R], rows of W2 [kWarps][slots], sums [columns][R].
struct FewRoom {
    int x_stride, act_stride, w_stride, slots;
};

template <bool k8>
__global__ void __launch_bounds__(kThreads, 1) layer_few_kernel(const LayerArgs p, const FewRoom room) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, R = p.T * p.k;
    unsigned char *xs = smem, *acts = xs + p.T * room.x_stride;
    unsigned char *rows = acts + R * room.act_stride + warp * room.slots * room.w_stride;
    float *parts = reinterpret_cast<float *>(acts + R * room.act_stride + kWarps * room.slots * room.w_stride);
    __shared__ int s_ticket, s_good, s_ids[kLayerFewRows];
    unsigned *tickets = p.counters, *done = p.counters + 1;
    // the router has waited for what wrote the tokens
    bring_rows(xs, p.T, p.H / 8, room.x_stride, [&](int r, int c) { return __ldcg(reinterpret_cast<const uint4 *>(p.x + (int64_t)r * p.H) + c); },
               [](int c) { return c; });
    pdl_wait();
    if (threadIdx.x == 0) s_ticket = (int)atomicAdd(tickets, 1u);
    if (threadIdx.x < R) s_ids[threadIdx.x] = __ldcg(p.ids + threadIdx.x);
    __syncthreads();
    // out's columns [lo, hi): unit u is column lo + u / R for routed row u % R, a warp has every 16th
    const int lo = (int)((int64_t)p.H * blockIdx.x / p.blocks), hi = (int)((int64_t)p.H * (blockIdx.x + 1) / p.blocks);
    const int units = (int)blockIdx.x < p.blocks ? (hi - lo) * R : 0, row_bytes = p.F * (k8 ? 1 : 2);
    const int next_c = kWarps / R, next_r = kWarps - next_c * R;
    const auto advance = [&](int &c, int &r) {  // from unit u to u + kWarps
        c += next_c;
        r += next_r;
        if (r >= R) {
            r -= R;
            ++c;
        }
    };
    const auto fetch = [&](int first) {
        int c = first / R, r = first - c * R;
#pragma unroll 4
        for (int i = 0; i < room.slots; ++i, advance(c, r)) {
            const int expert = s_ids[r];
            if (first + i * kWarps >= units) break;
            const unsigned char *w = static_cast<const unsigned char *>(p.w2) + ((int64_t)expert * p.H + lo + c) * row_bytes;
#pragma unroll 3
            for (int at = lane * 16; at < room.w_stride; at += 512)
                cp_async16(smem_u32(rows + i * room.w_stride + at), at < row_bytes ? w + at : w, at < row_bytes);
        }
        copies_sent();
    };
    bool fetched = false;
    for (;;) {
        const int ticket = s_ticket;
        if (ticket >= p.ranges) break;
        __syncthreads();
        if (threadIdx.x == 0) s_ticket = (int)atomicAdd(tickets, 1u);  // the next one, taken while this one runs
        const int64_t n = (int64_t)R * p.F, shares = (int64_t)p.ranges * kWarps, me = (int64_t)ticket * kWarps + warp;
        const int bytes = p.H * (k8 ? 1 : 2), pieces = (bytes + 511) / 512;
        constexpr int kChunk = UpStream<k8>::kChunk;
        UpStream<k8> up{p, xs, s_ids, room.x_stride, lane, pieces, (pieces + kChunk - 1) / kChunk, bytes, (int)(n * (me + 1) / shares)};
        up.run((int)(n * me / shares), [&] {
            if (!fetched) fetch(warp);
            fetched = true;
        });
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) atomicAdd(done, 1u);
    }
    if (!fetched) fetch(warp);
    if (threadIdx.x == 0) s_good = wait_count(done, (unsigned)p.ranges, p.status);
    __syncthreads();
    if (!s_good) {
        wait_copies<0>();
        return;
    }
    // with codes, of the 16 values that a lane multiplies with 16 bytes of each 512 of a weight row, so that
    // the lanes' loads follow each other
    const int row_pieces = p.F / (k8 ? 4 : 8);
    bring_rows(acts, R, row_pieces, room.act_stride, [&](int r, int c) { return __ldcg(static_cast<const uint4 *>(p.act) + (int64_t)r * row_pieces + c); },
               [](int c) { return k8 ? (c & -128) + c % 4 * 32 + c / 4 % 32 : c; });
    wait_copies<0>();
    __syncthreads();
    for (int first = warp; first < units; first += room.slots * kWarps) {
        if (first != warp) {
            __syncwarp();
            fetch(first);
            wait_copies<0>();
            __syncwarp();
        }
        int c = first / R, r = first - c * R;
        for (int i = 0; i < room.slots && first + i * kWarps < units; i += 4) {
            // four units at a time (the last one again where there are fewer)
            const unsigned char *w[4], *act[4];
            const uint8_t *ex[4];
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int expert = s_ids[r];
                w[j] = rows + min(i + j, room.slots - 1) * room.w_stride;
                act[j] = acts + r * room.act_stride;
                if (k8) ex[j] = p.w2x + ((int64_t)expert * blocks8(p.H) + min(lo + c, p.H - 1) / kBlock8) * blocks8(p.F) + lane / 8;
                advance(c, r);
            }
            const auto sum_all = [&](const auto &act_of) {
                for (int at = lane * 16; at < room.w_stride; at += 512) {
                    int e[4][1];
#pragma unroll
                    for (int j = 0; j < 4; ++j) e[j][0] = k8 && at < row_bytes ? (int)__ldg(ex[j] + at / 512 * 4) : 127;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint4 row[1] = {*reinterpret_cast<const uint4 *>(w[j] + at)};
                        float sum[1] = {d[j]};
                        dot16<k8, k8>(row, act_of(j) + (k8 ? 4 * at - 48 * lane : at), e[j], sum);
                        d[j] = sum[0];
                    }
                }
            };
            // (where R divides the warps, a warp's units are all of one routed row, whose values are then
            // read once)
            if (kWarps % R == 0) sum_all([&](int) { return act[0]; });
            else sum_all([&](int j) { return act[j]; });
            // over the lanes: first half of them go on with two units, then a quarter with one
            const bool up16 = lane & 16, up8 = lane & 8;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float other = __shfl_xor_sync(kFull, up16 ? d[j] : d[j + 2], 16);
                d[j] = (up16 ? d[j + 2] : d[j]) + other;
            }
            const float other = __shfl_xor_sync(kFull, up8 ? d[0] : d[1], 8);
            float total = (up8 ? d[1] : d[0]) + other;
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) total += __shfl_xor_sync(kFull, total, o);
            const int j = (up16 ? 2 : 0) + (up8 ? 1 : 0), u = first + (i + j) * kWarps;
            if ((lane & 7) == 0 && i + j < room.slots && u < units) parts[u] = total;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (units ? (hi - lo) * p.T : 0); i += kThreads) {
        const int t = i / (hi - lo), c = i - t * (hi - lo);
        float sum = 0.0f;
        for (int q = 0; q < p.k; ++q) sum = fmaf(__ldcg(p.combine + t * p.k + q), parts[c * R + t * p.k + q], sum);
        p.out[(int64_t)t * p.H + lo + c] = __float2bfloat16_rn(sum);
    }
    pdl_trigger();
}

constexpr int kRoom = 232448 - 1024;
FewRoom few_room(const LayerArgs &a, bool eight) {
    // the rows in shared memory have zeros where a last piece of the weights is not full
    const int h = (a.H * (eight ? 1 : 2) + 511) / 512, f = (a.F * (eight ? 1 : 2) + 511) / 512, R = a.T * a.k;
    FewRoom room = {h * (eight ? 1024 : 512), f * (eight ? 2048 : 512), f * 512, 0};
    const int columns = (a.H + a.blocks - 1) / a.blocks;
    const int left = kRoom - a.T * room.x_stride - R * room.act_stride - 4 * R * columns;
    room.slots = left / (kWarps * room.w_stride);
    const int most = (columns * R + kWarps - 1) / kWarps;
    if (room.slots > most) room.slots = most;
    return room;
}

}  // namespace

// Up to four routed rows whose weights would be at most 180 MB in bf16, up to eight of 110 MB, and with
// bf16 weights up to 40 of 80 MB, shared ones counted as often as they are used.  Measured on both sides
// (us in a graph, both kernels of the layer; this against layer_experts.cu).  Eight rows, one token or
// eight, bf16 and codes: H = 2048, F = 768 (75 MB) 23.8 and 28.7, 23.8 and 26.9, all of one expert 17.8 and
// 20.8, 19.8 and 22.5; F = 1024 (101 MB) 31.8 and 31.4, 25.8 and 28.6; F = 1280 (126 MB) 34.0 and 32.3, 31.7
// and 28.3; H = 4096, F = 1536 (302 MB) 68.2 and 60.3, 54.5 and 42.7, of one expert 61.6 and 35.6, 63.2 and 33.2.
// Four: H = 4096, F = 1536 (151 MB) 38.6 and 41.0, 31.8 and 36.1; F = 2048 (201 MB) 49.0 and 47.1, 41.2 and 39.6;
// two with F = 3584 (176 MB) 48.4 and 48.4, 37.0 and 40.2.  More: two tokens of eight experts, H = 2048, F =
// 768 (151 MB), 44.0 and 42.0, 39.6 and 35.3.  R = 35, H
// = 1008, F = 208 (44 MB) 21.1 and 24.2, in 8 bits 23.7 and 22.5; R = 32, H = 1024, F = 256 (50 MB) 23.0
// and 27.6, 30.3 and 26.3, F = 512 (101 MB) 31.3 and 30.9; R = 64, H = 512, F = 256 24.1 and 24.0.
bool layer_few(const LayerArgs &a, bool eight) {
    const int R = a.T * a.k;
    const int64_t bytes = (int64_t)R * 3 * a.F * a.H * 2;
    if (bytes > (R <= 4 ? 180000000 : R <= 8 ? 110000000 : 80000000)) return false;
    return R <= (eight ? 8 : kLayerFewRows) && few_room(a, eight).slots > 0;
}

cudaError_t launch_layer_few(const LayerArgs &a, bool eight, int sms, cudaStream_t s) {
    const FewRoom room = few_room(a, eight);
    const int R = a.T * a.k;
    const size_t smem = (size_t)a.T * room.x_stride + (size_t)R * room.act_stride + (size_t)kWarps * room.slots * room.w_stride +
                        sizeof(float) * R * ((a.H + a.blocks - 1) / a.blocks);
    const cudaError_t e = eight ? ensure_smem_limit<layer_few_kernel<true>>(kRoom) : ensure_smem_limit<layer_few_kernel<false>>(kRoom);
    if (e != cudaSuccess) return e;
    return launch_after(eight ? layer_few_kernel<true> : layer_few_kernel<false>, dim3((unsigned)sms), kThreads, smem, s, a, room);
}

}  // namespace dol
