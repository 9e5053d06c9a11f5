// Device code that the kernels of a prediction share: a (score, label) pair as one key, the largest key of a wavefront.
#pragma once
#include "usl_internal.h"

constexpr int TOPK_SHORT_MERGE = 8 * 256;   // candidates that a merge of 256 lanes holds in registers; more take 512 or 1024
constexpr int TOPK_SHORT_SEGMENT = 8 * 256;  // scores of a workgroup of the pass over them where rows are few
constexpr int TOPK_MAX = 32;                 // largest kk

// The upper word ranks scores (-0 as +0), the lower one equal scores by label (below 2^31, so ~label's top bit says nothing); its last bit says
// that the score is not -0, so that a key holds the score's own bits and no kernel that merges keys waits for the scores themselves.
__device__ __forceinline__ uint64_t score_key(float z, uint32_t label) {
    uint32_t u = __float_as_uint(z);
    const uint32_t minus_zero = u == 0x80000000u;
    if (minus_zero) u = 0u;
    u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return ((uint64_t)u << 32) | (uint64_t)(uint32_t)(~label << 1 | (minus_zero ^ 1u));
}
__device__ __forceinline__ int32_t key_label(uint64_t key) { return (int32_t)~((uint32_t)key >> 1 | 0x80000000u); }
__device__ __forceinline__ float key_score(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32), bits = (u & 0x80000000u) ? u ^ 0x80000000u : ~u;
    return __uint_as_float(bits == 0u && !(key & 1u) ? 0x80000000u : bits);
}

// Largest v of the wavefront, the same register for all lanes: the upper words, then the lower ones of those that have the largest.
// What bounds these kernels is the chain of 2 kk such maxima; lane shifts within the vector unit (rows of 16 lanes, then the last lane
// of a row into the next ones) do not wait for LDS as shuffles do, and a 32-bit maximum takes its shifted operand in the same instruction,
// where 64-bit keys take five (one row of 500k scores, 5 labels: segments 6.7 and 6.2 us, merge 4.0 and 3.8; usl_predict of 4 instances at m = 300k, d = 8k, k = 16 29.4 and 24.3).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_with(uint32_t v) {   // a lane without a source keeps its own
    const uint32_t t = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
    return t > v ? t : v;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max_with<0x111, 0xF>(v);   // row_shr:1, 2, 4, 8: lane 15 of a row has the row's largest
    v = max_with<0x112, 0xF>(v);
    v = max_with<0x114, 0xF>(v);
    v = max_with<0x118, 0xF>(v);
    v = max_with<0x142, 0xA>(v);   // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
    v = max_with<0x143, 0xC>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t plus(uint32_t v) { return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, true); }   // (no source: 0)
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
    v = plus<0x111, 0xF>(v);
    v = plus<0x112, 0xF>(v);
    v = plus<0x114, 0xF>(v);
    v = plus<0x118, 0xF>(v);
    v = plus<0x142, 0xA>(v);
    v = plus<0x143, 0xC>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
    const uint32_t hi = wave_max((uint32_t)(v >> 32)), lo = wave_max((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
    return (uint64_t)hi << 32 | lo;
}

// Largest v of the workgroup, returned to every lane.  red: two sets used in turn, so one barrier is enough.
template <int NT>
struct BlockMax {
    uint64_t (*red)[NT / 64];
    int turn;
    __device__ __forceinline__ uint64_t operator()(uint64_t v) {
        v = wave_max(v);
        uint64_t* set = red[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) set[threadIdx.x >> 6] = v;
        __syncthreads();
        uint64_t r = set[0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) r = set[w] > r ? set[w] : r;
        return r;
    }
};

// The kk largest of the keys that the lanes of WAVES wavefronts hold (0: none), the r-th in lane r of wavefront 0 (0 where there are no more): every wavefront
// its own, without a barrier, then the first one all of theirs.  list: WAVES * kk places.
template <int WAVES, int HELD>
__device__ __forceinline__ uint64_t best_keys(const uint64_t (&held)[HELD], int kk, uint64_t* list) {
    const int lane = threadIdx.x & 63;
    uint64_t prev = ~0ull, found = 0;
    for (int r = 0; r < kk; ++r) {
        uint64_t best = 0;
#pragma unroll
        for (int q = 0; q < HELD; ++q)
            if (held[q] < prev && held[q] > best) best = held[q];
        prev = wave_max(best);
        found = lane == r ? prev : found;
    }
    if (WAVES == 1) return found;
    if (lane < kk) list[(threadIdx.x >> 6) * kk + lane] = found;
    __syncthreads();
    if (threadIdx.x >= 64) return 0;
    uint64_t mine[(WAVES * TOPK_MAX + 63) / 64];
#pragma unroll
    for (int q = 0; q < (WAVES * TOPK_MAX + 63) / 64; ++q) mine[q] = q * 64 + lane < WAVES * kk ? list[q * 64 + lane] : 0ull;
    return best_keys<1>(mine, kk, list);
}
