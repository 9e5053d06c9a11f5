// Device code that the kernels of a prediction share: a (score, label) pair as one key, the largest key of a wavefront.
#pragma once
#include "usl_internal.h"

constexpr int TOPK_SHORT_MERGE = 8 * 256;   // candidates that a merge of 256 lanes holds in registers; more take it 1024
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

template <int NT>
struct TopkSegment {
    uint64_t red[2][NT / 64];
    uint32_t count;
};

// The kk best keys of the EPT scores that each of a workgroup's lanes holds, best first, into dst[kk] (0 where there are no more).  Register e holds
// label seg0 + local_of(e), which grows with e, and counts where is(e, local_of(e)); list: TOPK_MAX * EPT places.
//   1. every lane finds its own best key;
//   2. tau = the kk-th best of the lanes' maxima: at least kk keys of the segment are >= tau, and
//      every key >= tau belongs to one of the kk lanes whose maximum is >= tau, so at most kk*EPT keys pass;
//   3. those keys are collected in LDS and the best kk are peeled off one by one ("largest key below the
//      previous winner": keys are distinct, so nothing has to be removed).
template <int NT, int EPT, typename LABEL, typename IS>
__device__ __forceinline__ void best_of_segment(const float (&v)[EPT], LABEL local_of, IS is, int64_t seg0, int kk, TopkSegment<NT>& shared,
                                                uint64_t* list, uint64_t* dst) {
    BlockMax<NT> block_max = {shared.red, 0};
    // the lane's best score; labels grow with e, so the first of equal scores is the smaller label
    float top = 0.f;
    int top_j = -1;
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
        const int j = local_of(e);
        const bool better = is(e, j) && (top_j < 0 || v[e] > top);
        top = better ? v[e] : top;
        top_j = better ? j : top_j;
    }
    const uint64_t mine = top_j >= 0 ? score_key(top, (uint32_t)(seg0 + top_j)) : 0ull;
    uint64_t tau = ~0ull;
    for (int r = 0; r < kk && tau != 0; ++r) tau = block_max(mine < tau ? mine : 0ull);
    if (threadIdx.x == 0) shared.count = 0;
    __syncthreads();
    // keys are built only for scores that reach tau's score (a cheap float test first)
    const uint32_t tu = (uint32_t)(tau >> 32);
    const float tau_score = tau == 0 ? -INFINITY : __uint_as_float((tu & 0x80000000u) ? (tu & 0x7FFFFFFFu) : ~tu);
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
        const int j = local_of(e);
        if (is(e, j) && v[e] >= tau_score) {
            const uint64_t key = score_key(v[e], (uint32_t)(seg0 + j));
            if (key >= tau) {
                const uint32_t at = atomicAdd(&shared.count, 1u);
                if (at < TOPK_MAX * EPT) list[at] = key;   // (more only where a score is NaN, which no key ranks)
            }
        }
    }
    __syncthreads();
    const uint32_t n = min(shared.count, (uint32_t)(TOPK_MAX * EPT));
    uint64_t prev = ~0ull;
    for (int r = 0; r < kk; ++r) {
        uint64_t best = 0;
        for (uint32_t q = threadIdx.x; q < n; q += NT) {
            const uint64_t key = list[q];
            if (key < prev && key > best) best = key;
        }
        prev = block_max(best);
        if (threadIdx.x == 0) dst[r] = prev;
    }
}
