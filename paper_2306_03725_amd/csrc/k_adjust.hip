// Scores as they are served: penalties for labels that an instance has been shown, a bias per label, a mask of the labels allowed
// (usl_adjustments), written out or ranked straight away.
//
//   c = occurrences of label j in the instance's list;  c > 0:  z <- (z > 0 ? z / repeat : z * repeat) - (presence + frequency * c)
//   z <- z + bias[j];  not allowed: -infinity
//
// A workgroup takes a segment of one instance's scores into registers, all loads in flight at once, and counts the labels of its segment in the instance's
// list: every segment looks at all of it, and no pass has to sort it.  Bound by the stream of the scores where lists are short next to a segment:
// 256 x 500k read and written, with a bias, a mask and lists of up to 500 labels each: 1.04 GB in 206 us, 5.1 TB/s, the rate of a large copy.  Not so lists of thousands, whose
// entries behind the first 1024 are read again by every segment, one after the other: 64 x 500k, lists of up to 1000 labels 57 us written and 51 as the 10 best, of up to 20 000 116 and 172.
#include "k_topk.h"

namespace {

constexpr int AD_NT = 256;
// scores a lane holds: 16, or 8 where that would leave most of the chip without a workgroup.  (32 of them, with 32 KB of counts and 124 registers, leave a
// compute unit three workgroups: 256 x 500k scores written in 241 us, with 16 in 210.)
constexpr int AD_EPT = 16, AD_EPT_FEW = 8;
constexpr int RUN_WORKGROUPS = 4;   // of k_topk_adjusted, to a compute unit: as many as it holds; a run pays for its first threshold (256 x 670k, 10 labels: 162 us, with 8 171, with 16 197)

typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));   // rows and segments begin at any float

struct Adjust {
    const float* bias;
    const uint32_t* allowed;
    int64_t allowed_words;   // from an instance's mask to the next; 0: one mask for all
    const int64_t* off;
    const int32_t* lab;
    float repeat, presence, frequency;
};

// Register e of a lane holds label local_label(e) of the segment: groups of four neighbours.
__device__ __forceinline__ int local_label(int e) { return ((e >> 2) * AD_NT + (int)threadIdx.x) * 4 + (e & 3); }

// Four values from place j of lim, into registers.  full (the same for the workgroup): all of them are there; else those behind the end are the last one again.
// (Not a load under a lane's condition: behind each of those the compiler waits.)
__device__ __forceinline__ void load_four(const float* p, int j, int lim, bool full, float* v) {
    if (full) {
        const f32x4 q = *reinterpret_cast<const f32x4*>(p + j);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = p[min(j + u, lim - 1)];
    }
}

// The labels an instance has been shown: the first of them in registers, for all its segments
struct Shown {
    static constexpr int HELD = 4;
    const int32_t* lab;
    int64_t n;
    int32_t held[HELD];
    __device__ __forceinline__ Shown(const Adjust& a, int instance) : lab(nullptr), n(0) {
        if (!a.off) return;   // (held is not looked at)
        const int64_t p0 = a.off[instance];
        n = a.off[instance + 1] - p0;
        lab = a.lab + p0;
#pragma unroll
        for (int q = 0; q < HELD; ++q) held[q] = -1;
        if (n <= 0) return;
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            const int p = q * AD_NT + (int)threadIdx.x;
            const int32_t label = lab[min((int64_t)p, n - 1)];
            held[q] = p < n ? label : -1;
        }
    }
    __device__ __forceinline__ bool any() const { return n > 0; }   // the same for the whole workgroup
    // counts[j] += occurrences of label seg0 + j
    __device__ __forceinline__ void count(int64_t seg0, int lim, uint32_t* counts) const {
        auto one = [&](int32_t label) {
            const uint32_t j = (uint32_t)label - (uint32_t)seg0;   // (negative and too large ones lie behind every segment)
            if (j < (uint32_t)lim) atomicAdd(&counts[j], 1u);
        };
#pragma unroll
        for (int q = 0; q < HELD; ++q) one(held[q]);
        for (int64_t p = HELD * AD_NT + (int)threadIdx.x; p < n; p += AD_NT) one(lab[p]);   // (each is waited for, and what was asked for before it)
    }
};

// A segment's scores and their labels' bias.  BIAS, MASK: there are any (told at compile time: a register that a branch may or may not load is waited for there).
template <int EPT, bool BIAS, bool MASK>
struct Segment {
    float v[EPT];
    uint32_t mask[EPT / 4];   // the word with a group's four bits, which begin at bit local_label % 32 (a segment begins at a multiple of 32 labels)
    __device__ __forceinline__ void load(const float* row, int64_t seg0, int lim, int instance, const Adjust& a) {
        const bool full = lim == AD_NT * EPT;
#pragma unroll
        for (int e = 0; e < EPT; e += 4) {
            if (MASK) mask[e / 4] = a.allowed[(size_t)instance * a.allowed_words + ((seg0 + min(local_label(e), lim - 1)) >> 5)];
            load_four(row + seg0, local_label(e), lim, full, v + e);
        }
    }
    __device__ __forceinline__ void load_bias(int64_t seg0, int lim, const Adjust& a, float (&bias)[EPT]) const {
#pragma unroll
        for (int e = 0; e < EPT; e += 4)
            if (BIAS) load_four(a.bias + seg0, local_label(e), lim, lim == AD_NT * EPT, bias + e);
    }
    // v becomes the adjusted scores; `hidden` where a label is not allowed or does not exist.  counts: of all lanes' labels, all 0 before and after; between
    // two calls lies a barrier.
    __device__ __forceinline__ void adjust(const Shown& shown, int64_t seg0, int lim, const Adjust& a, const float (&bias)[EPT], uint32_t* counts, float hidden) {
#pragma clang fp contract(off)   // every step is rounded, so that a label is ranked by the bits that are written
        if (shown.any()) {
            shown.count(seg0, lim, counts);
            __syncthreads();
            uint4* four = reinterpret_cast<uint4*>(counts);
#pragma unroll
            for (int e = 0; e < EPT; e += 4) {
                const int at = (e >> 2) * AD_NT + (int)threadIdx.x;
                const uint4 n = four[at];
                if (n.x | n.y | n.z | n.w) {   // few
                    const uint32_t c[4] = {n.x, n.y, n.z, n.w};
                    four[at] = make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float z = v[e + u], less = (z > 0.f ? z / a.repeat : z * a.repeat) - fmaf(a.frequency, (float)c[u], a.presence);
                        v[e + u] = c[u] ? less : z;
                    }
                }
            }
        }
#pragma unroll
        for (int e = 0; e < EPT; e += 4) {
            const int j = local_label(e);
            uint32_t is = MASK ? mask[e / 4] >> (j & 31) : 0xFu;
            if (lim != AD_NT * EPT) is &= (1u << min(max(lim - j, 0), 4)) - 1u;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float z = BIAS ? v[e + u] + bias[e + u] : v[e + u];
                v[e + u] = is >> u & 1u ? z : hidden;
            }
        }
    }
};

template <int EPT>
__device__ __forceinline__ void clear(uint32_t* counts) {
#pragma unroll
    for (int e = 0; e < EPT / 4; ++e) reinterpret_cast<uint4*>(counts)[e * AD_NT + threadIdx.x] = make_uint4(0, 0, 0, 0);
    __syncthreads();
}

// adjusted may be out: a lane reads its scores before it writes them, and no other lane does
template <int EPT, bool BIAS, bool MASK>
__global__ void __launch_bounds__(AD_NT)
k_adjust(const float* out, int64_t m, Adjust a, float* adjusted) {
    __shared__ __align__(16) uint32_t counts[AD_NT * EPT];
    const int64_t seg0 = (int64_t)blockIdx.x * (AD_NT * EPT), row = (int64_t)blockIdx.y * m;
    const int lim = (int)min((int64_t)AD_NT * EPT, m - seg0);
    Segment<EPT, BIAS, MASK> seg;
    float bias[EPT];
    seg.load(out + row, seg0, lim, (int)blockIdx.y, a);
    seg.load_bias(seg0, lim, a, bias);
    const Shown shown(a, (int)blockIdx.y);
    if (shown.any()) clear<EPT>(counts);
    seg.adjust(shown, seg0, lim, a, bias, counts, -INFINITY);
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
        const int j = local_label(e);
        float* to = adjusted + row + seg0 + j;
        if (j + 3 < lim) {
            const f32x4 q = {seg.v[e], seg.v[e + 1], seg.v[e + 2], seg.v[e + 3]};
            *reinterpret_cast<f32x4*>(to) = q;
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j + u < lim) to[u] = seg.v[e + u];
        }
    }
}

// The kk best allowed labels of a run of segments of one instance (number blockIdx.x, + gridDim.x, ...), best first, into
// cand[instance][run][kk] (0: no more).  What is kept is a list of keys (k_topk.h) that holds the kk best of the segments so far, and tau, which the kk-th
// of them is known to reach: a segment whose scores do not reach tau costs one comparison a score.  Of the others the scores go to LDS, and those that
// reach tau are appended; only when the list would overflow are its kk best peeled off, kk maxima over the workgroup, and tau raised to the
// last of them, and if the segment alone is too much for the list, first to the kk-th of the lanes' best (at most kk * EPT labels of the segment reach that).
// A run of one segment takes 2 kk maxima, and so does one of forty where scores come in any order: 256 x 670k, 10 labels: 689 MB in 163 us, 4.2 TB/s.  The next segment's scores are on their way meanwhile.
template <int EPT, bool BIAS, bool MASK>
__global__ void __launch_bounds__(AD_NT, 4)
k_topk_adjusted(const float* __restrict__ out, int64_t m, Adjust a, int kk, int nseg, uint64_t* __restrict__ cand) {
    constexpr int CAP = TOPK_MAX * (EPT + 1), HELD = (CAP + AD_NT - 1) / AD_NT;
    __shared__ __align__(16) uint32_t counts[AD_NT * EPT];
    __shared__ __align__(16) float scores[AD_NT * EPT];
    __shared__ uint64_t list[CAP];
    __shared__ uint64_t red[2][AD_NT / 64];
    __shared__ uint32_t reach[2][AD_NT / 64], length;
    BlockMax<AD_NT> block_max = {red, 0};
    const int tid = (int)threadIdx.x;
    const float* row = out + (int64_t)blockIdx.y * m;
    uint64_t tau = 0;
    float least = -INFINITY;   // tau's score
    uint32_t n = 0;            // entries of the list
    auto raise = [&](uint64_t t) {
        if (t > tau) {
            tau = t;
            least = key_score(t);
        }
    };
    // the kk best of the list, in order
    auto compact = [&]() {
        uint64_t held[HELD];
#pragma unroll
        for (int q = 0; q < HELD; ++q) held[q] = q * AD_NT + tid < (int)n ? list[q * AD_NT + tid] : 0ull;
        __syncthreads();
        uint64_t prev = ~0ull;
        for (int r = 0; r < kk; ++r) {
            uint64_t best = 0;
#pragma unroll
            for (int q = 0; q < HELD; ++q)
                if (held[q] < prev && held[q] > best) best = held[q];
            prev = block_max(best);
            if (tid == 0) list[r] = prev;
        }
        n = min(n, (uint32_t)kk);
        raise(prev);   // (0 while there are fewer than kk)
        if (tid == 0) length = n;
        __syncthreads();
    };
    auto limit = [&](int s) { return (int)min((int64_t)AD_NT * EPT, m - (int64_t)s * (AD_NT * EPT)); };
    Segment<EPT, BIAS, MASK> seg, next;
    int s = (int)blockIdx.x, turn = 0;
    next.load(row, (int64_t)s * (AD_NT * EPT), limit(s), (int)blockIdx.y, a);
    const Shown shown(a, (int)blockIdx.y);
    if (tid == 0) length = 0;
    clear<EPT>(counts);
    for (; s < nseg; s += (int)gridDim.x, turn ^= 1) {
        const int64_t seg0 = (int64_t)s * (AD_NT * EPT);
        float bias[EPT];
        seg = next;
        seg.load_bias(seg0, limit(s), a, bias);   // before the next scores: a wait for the bias would be one for them too
        if (s + (int)gridDim.x < nseg) next.load(row, seg0 + (int64_t)gridDim.x * (AD_NT * EPT), limit(s + (int)gridDim.x), (int)blockIdx.y, a);
        seg.adjust(shown, seg0, limit(s), a, bias, counts, __uint_as_float(0x7FC00000u));   // NaN, which reaches nothing, where a label is not to be given
        uint32_t mine = 0;   // bit e: reaches tau
#pragma unroll
        for (int e = 0; e < EPT; ++e) mine |= seg.v[e] >= least ? 1u << e : 0u;
        const uint32_t wave = wave_sum((uint32_t)__popc(mine));
        if ((tid & 63) == 0) reach[turn][tid >> 6] = wave;
        __syncthreads();
        uint32_t total = 0;
#pragma unroll
        for (int w = 0; w < AD_NT / 64; ++w) total += reach[turn][w];
        if (total == 0) continue;
        if (mine) {   // a lane reads its own scores only
#pragma unroll
            for (int e = 0; e < EPT; e += 4) *reinterpret_cast<float4*>(scores + local_label(e)) = make_float4(seg.v[e], seg.v[e + 1], seg.v[e + 2], seg.v[e + 3]);
        }
        if (n + total > (uint32_t)CAP) {
            if (n) compact();
            float top = 0.f;
            int top_j = -1;   // labels grow with e, so the first of equal scores is the smaller label
            for (uint32_t left = mine; left; left &= left - 1) {
                const int j = local_label(__builtin_ctz(left));
                const float z = scores[j];
                const bool better = z >= least && (top_j < 0 || z > top);
                top = better ? z : top;
                top_j = better ? j : top_j;
            }
            const uint64_t best = top_j >= 0 ? score_key(top, (uint32_t)(seg0 + top_j)) : 0ull;
            uint64_t t = ~0ull;
            for (int r = 0; r < kk && t != 0; ++r) t = block_max(best < t ? best : 0ull);
            raise(t);
        }
        for (uint32_t left = mine; left; left &= left - 1) {
            const int j = local_label(__builtin_ctz(left));
            const uint64_t key = score_key(scores[j], (uint32_t)(seg0 + j));
            if (key >= tau) {
                const uint32_t at = atomicAdd(&length, 1u);
                if (at < (uint32_t)CAP) list[at] = key;
            }
        }
        __syncthreads();
        n = length;
    }
    __syncthreads();
    compact();
    uint64_t* to = cand + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * kk;
    for (int r = tid; r < kk; r += AD_NT) to[r] = list[r];
}

// ... of one segment an instance's run has, where that many workgroups are few: every lane's scores become keys, and no threshold is worth its maxima.
template <int EPT, bool BIAS, bool MASK>
__global__ void __launch_bounds__(AD_NT)
k_topk_adjusted_few(const float* __restrict__ out, int64_t m, Adjust a, int kk, uint64_t* __restrict__ cand) {
    __shared__ __align__(16) uint32_t counts[AD_NT * EPT];
    __shared__ uint64_t list[AD_NT / 64 * TOPK_MAX];
    const int64_t seg0 = (int64_t)blockIdx.x * (AD_NT * EPT);
    const int lim = (int)min((int64_t)AD_NT * EPT, m - seg0);
    Segment<EPT, BIAS, MASK> seg;
    float bias[EPT];
    seg.load(out + (int64_t)blockIdx.y * m, seg0, lim, (int)blockIdx.y, a);
    seg.load_bias(seg0, lim, a, bias);
    const Shown shown(a, (int)blockIdx.y);
    if (shown.any()) clear<EPT>(counts);
    seg.adjust(shown, seg0, lim, a, bias, counts, __uint_as_float(0x7FC00000u));
    uint64_t held[EPT];
#pragma unroll
    for (int e = 0; e < EPT; ++e) held[e] = seg.v[e] == seg.v[e] ? score_key(seg.v[e], (uint32_t)(seg0 + local_label(e))) : 0ull;   // (NaN: not to be given)
    const uint64_t own = best_keys<AD_NT / 64>(held, kk, list);
    if ((int)threadIdx.x < kk) cand[((size_t)blockIdx.y * gridDim.x + blockIdx.x) * kk + threadIdx.x] = own;
}

Adjust of(const usl_ctx* c, const usl_adjustments* a) {
    const int64_t words = (c->m + 31) / 32;
    return Adjust{a->bias, a->allowed, a->allowed_rows == 1 ? 0 : words, a->shown_off, a->shown_lab, a->repeat, a->presence, a->frequency};
}
int segments(const usl_ctx* c, int ept) { return (int)((c->m + AD_NT * ept - 1) / (AD_NT * ept)); }
bool few_segments(const usl_ctx* c, int32_t b) { return (int64_t)segments(c, AD_EPT) * b < c->num_cu; }

}  // namespace

// Best labels: a workgroup for every short segment, or runs of segments under one threshold?  A run pays for its thresholds' maxima and waits out its segments one
// after the other; a segment by itself pays for its lanes' keys, the more the more labels are asked for.  us, by segments and by runs: 20k x 64, 5 labels (640 short
// segments) 10.4 and 15.9; 41k x 173 (3460) 19.3 and 22.5; 46k x 92, 1 label (2116) 10.6 and 15.8; 58k x 49, 10 labels (1421) 18.4 and 20.2; not so 100k x 100, 5 labels
// (4900) 24.3 and 25.1; 58k x 49, 32 labels 43.4 and 37.9; 41k x 600, 5 labels (12 000) 48.4 and 43.4; 747k x 57 79.1 and 50.3.
static bool best_by_segments(const usl_ctx* c, int32_t b, int32_t kk) { return (int64_t)segments(c, AD_EPT_FEW) * b * (kk + 5) <= 35000 / 256 * (int64_t)c->num_cu; }
// Runs of an instance's segments: no more than the chip holds together (one more workgroup takes as long as another round of them: 747k x 57 50.3 us with 17 runs, 104.6 with
// 18), and eight labels asked for are worth a segment of a run (100k x 100, 32 labels: 46.9 us with 5 runs, 55.7 with 10).
static int runs_of(const usl_ctx* c, int nseg, int32_t b, int32_t kk) {
    const int64_t room = (int64_t)c->num_cu * RUN_WORKGROUPS / b, most = kk > 8 ? nseg / (kk / 8) : nseg, runs = room < most ? room : most;
    return runs < 1 ? 1 : (int)runs;
}

size_t usl_adjusted_segments(const usl_ctx* c) {   // b * sets of candidates an instance has, for any b up to max_b
    const size_t by_runs = (size_t)c->num_cu * RUN_WORKGROUPS + c->max_b, by_segments = (size_t)(35000 / 256 * (int64_t)c->num_cu / 6) + 1;
    return by_runs > by_segments ? by_runs : by_segments;
}

// the kernel by what there is to do
#define USL_ADJUST_BY_WHAT(RUN, EPT)                                                          \
    do {                                                                                      \
        if (a->bias) { if (a->allowed) RUN(EPT, true, true); else RUN(EPT, true, false); }    \
        else { if (a->allowed) RUN(EPT, false, true); else RUN(EPT, false, false); }          \
    } while (0)

usl_status usl_launch_adjust(usl_ctx* c, const float* out, const usl_adjustments* a, float* adjusted, int32_t b) {
    const bool few = few_segments(c, b);
    const dim3 grid((unsigned)segments(c, few ? AD_EPT_FEW : AD_EPT), (unsigned)b);
#define USL_ADJUST(EPT, BIAS, MASK) hipLaunchKernelGGL((k_adjust<EPT, BIAS, MASK>), grid, dim3(AD_NT), 0, c->stream, out, c->m, of(c, a), adjusted)
    if (few) USL_ADJUST_BY_WHAT(USL_ADJUST, AD_EPT_FEW);
    else USL_ADJUST_BY_WHAT(USL_ADJUST, AD_EPT);
#undef USL_ADJUST
    return usl_check_launch(c, "adjust_scores");
}

usl_status usl_launch_topk_adjusted(usl_ctx* c, const float* out, const usl_adjustments* a, int32_t b, int32_t kk, int32_t* top_lab, float* top_val) {
    const bool few = best_by_segments(c, b, kk);
    const int nseg = segments(c, few ? AD_EPT_FEW : AD_EPT), runs = few ? nseg : runs_of(c, nseg, b, kk);
    USL_TRY(usl_reserve_topk(c));
    const dim3 grid((unsigned)runs, (unsigned)b);
#define USL_BEST_FEW(EPT, BIAS, MASK) \
    hipLaunchKernelGGL((k_topk_adjusted_few<EPT, BIAS, MASK>), grid, dim3(AD_NT), 0, c->stream, out, c->m, of(c, a), (int)kk, c->topk_cand)
#define USL_BEST(EPT, BIAS, MASK) \
    hipLaunchKernelGGL((k_topk_adjusted<EPT, BIAS, MASK>), grid, dim3(AD_NT), 0, c->stream, out, c->m, of(c, a), (int)kk, nseg, c->topk_cand)
    if (few) USL_ADJUST_BY_WHAT(USL_BEST_FEW, AD_EPT_FEW);
    else USL_ADJUST_BY_WHAT(USL_BEST, AD_EPT);
#undef USL_BEST
#undef USL_BEST_FEW
    return usl_launch_topk_merge(c, runs, b, kk, top_lab, top_val);
}
