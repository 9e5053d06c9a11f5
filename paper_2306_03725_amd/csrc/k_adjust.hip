// Scores as they are served: penalties for labels that an instance has been shown, a bias per label, a mask of the labels allowed
// (usl_adjustments), written out or ranked straight away.
//
//   c = occurrences of label j in the instance's list;  c > 0:  z <- (z > 0 ? z / repeat : z * repeat) - (presence + frequency * c)
//   z <- z + bias[j];  not allowed: -infinity
//
// A workgroup takes a segment of one instance's scores into registers, all loads in flight at once, and while they are on their way counts the labels of
// its segment in the instance's list: the list is short next to the scores, so every segment reads all of it (from the L2), and no pass has to sort it.
#include "k_topk.h"

namespace {

constexpr int AD_NT = 256;
// scores a lane holds: 32 (their counts take 32 KB of LDS), or 8 where that would leave most of the chip without a workgroup
constexpr int AD_EPT = 32, AD_EPT_FEW = 8;

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

// The segment's scores, adjusted; bit e of what is returned: label local_label(e) exists and is allowed.
template <int EPT>
__device__ __forceinline__ uint32_t load_adjusted(const float* __restrict__ row, int64_t seg0, int lim, int instance, const Adjust& a, uint32_t* counts,
                                                  float (&v)[EPT]) {
#pragma clang fp contract(off)   // both kernels round every step, so that a label is ranked by the bits that are written
    const int tid = (int)threadIdx.x;
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
        const int j = local_label(e);
        if (j + 3 < lim) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(row + j);
            v[e] = q.x; v[e + 1] = q.y; v[e + 2] = q.z; v[e + 3] = q.w;
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u) v[e + u] = j + u < lim ? row[j + u] : 0.f;
        }
    }
    uint32_t mask[EPT / 4];   // the four bits of a group; a segment begins at a multiple of 32 labels
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
        const int j = local_label(e);
        mask[e / 4] = !a.allowed || j >= lim ? 0xFu : a.allowed[(size_t)instance * a.allowed_words + ((seg0 + j) >> 5)] >> (j & 31) & 0xFu;
    }
    const int64_t p0 = a.off ? a.off[instance] : 0, p1 = a.off ? a.off[instance + 1] : 0;
    if (p0 < p1) {   // the same for the whole workgroup
        uint4* clear = reinterpret_cast<uint4*>(counts);
#pragma unroll
        for (int e = 0; e < EPT / 4; ++e) clear[e * AD_NT + tid] = make_uint4(0, 0, 0, 0);
        __syncthreads();
        for (int64_t p = p0 + tid; p < p1; p += AD_NT) {
            const int64_t j = (int64_t)a.lab[p] - seg0;
            if (j >= 0 && j < lim) atomicAdd(&counts[j], 1u);
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < EPT; e += 4) {
            const uint4 n = clear[(e >> 2) * AD_NT + tid];
            const uint32_t c[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float z = v[e + u], shown = (z > 0.f ? z / a.repeat : z * a.repeat) - fmaf(a.frequency, (float)c[u], a.presence);
                v[e + u] = c[u] ? shown : z;
            }
        }
    }
    uint32_t is = 0;
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
        const int j = local_label(e);
        float bias[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.bias) {
            if (j + 3 < lim) {
                const f32x4 q = *reinterpret_cast<const f32x4*>(a.bias + seg0 + j);
                bias[0] = q.x; bias[1] = q.y; bias[2] = q.z; bias[3] = q.w;
            } else {
#pragma unroll
                for (int u = 0; u < 4; ++u) bias[u] = j + u < lim ? a.bias[seg0 + j + u] : 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bool ok = mask[e / 4] >> u & 1u;
            v[e + u] = ok ? v[e + u] + bias[u] : -INFINITY;
            if (ok && j + u < lim) is |= 1u << (e + u);
        }
    }
    return is;
}

// adjusted may be out: a lane reads its scores before it writes them, and no other lane does
template <int EPT>
__global__ void __launch_bounds__(AD_NT)
k_adjust(const float* out, int64_t m, Adjust a, float* adjusted) {
    __shared__ __align__(16) uint32_t counts[AD_NT * EPT];
    const int64_t seg0 = (int64_t)blockIdx.x * (AD_NT * EPT);
    const int lim = (int)min((int64_t)AD_NT * EPT, m - seg0);
    const int64_t at = (int64_t)blockIdx.y * m + seg0;
    float v[EPT];
    load_adjusted<EPT>(out + at, seg0, lim, (int)blockIdx.y, a, counts, v);
#pragma unroll
    for (int e = 0; e < EPT; e += 4) {
        const int j = local_label(e);
        float* to = adjusted + at + j;
        if (j + 3 < lim) {
            f32x4 q = {v[e], v[e + 1], v[e + 2], v[e + 3]};
            *reinterpret_cast<f32x4*>(to) = q;
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j + u < lim) to[u] = v[e + u];
        }
    }
}

// The kk best allowed labels of a segment, best first, into cand[instance][segment][kk] (0: no more).
template <int EPT>
__global__ void __launch_bounds__(AD_NT)
k_topk_adjusted(const float* __restrict__ out, int64_t m, Adjust a, int kk, int nseg, uint64_t* __restrict__ cand) {
    __shared__ __align__(16) uint32_t counts[AD_NT * EPT];
    __shared__ uint64_t list[TOPK_MAX * EPT];
    __shared__ TopkSegment<AD_NT> shared;
    const int64_t seg0 = (int64_t)blockIdx.x * (AD_NT * EPT);
    const int lim = (int)min((int64_t)AD_NT * EPT, m - seg0);
    float v[EPT];
    const uint32_t is = load_adjusted<EPT>(out + (int64_t)blockIdx.y * m + seg0, seg0, lim, (int)blockIdx.y, a, counts, v);
    best_of_segment<AD_NT, EPT>(v, [&](int e) -> int { return local_label(e); }, [&](int e, int) -> bool { return is >> e & 1u; }, seg0, kk, shared, list,
                                cand + ((size_t)blockIdx.y * nseg + blockIdx.x) * kk);
}

Adjust of(const usl_ctx* c, const usl_adjustments* a) {
    const int64_t words = (c->m + 31) / 32;
    return Adjust{a->bias, a->allowed, a->allowed_rows == 1 ? 0 : words, a->shown_off, a->shown_lab, a->repeat, a->presence, a->frequency};
}
int segments(const usl_ctx* c, int ept) { return (int)((c->m + AD_NT * ept - 1) / (AD_NT * ept)); }
bool few_segments(const usl_ctx* c, int32_t b) { return (int64_t)segments(c, AD_EPT) * b < c->num_cu; }

}  // namespace

size_t usl_adjusted_segments(const usl_ctx* c) {
    const size_t most = (size_t)segments(c, AD_EPT) * c->max_b, most_few = (size_t)segments(c, AD_EPT_FEW) * (c->num_cu / segments(c, AD_EPT) + 1);
    return most > most_few ? most : most_few;
}

usl_status usl_launch_adjust(usl_ctx* c, const float* out, const usl_adjustments* a, float* adjusted, int32_t b) {
    const bool few = few_segments(c, b);
    const dim3 grid((unsigned)segments(c, few ? AD_EPT_FEW : AD_EPT), (unsigned)b);
    if (few) hipLaunchKernelGGL(k_adjust<AD_EPT_FEW>, grid, dim3(AD_NT), 0, c->stream, out, c->m, of(c, a), adjusted);
    else hipLaunchKernelGGL(k_adjust<AD_EPT>, grid, dim3(AD_NT), 0, c->stream, out, c->m, of(c, a), adjusted);
    return usl_check_launch(c, "adjust_scores");
}

usl_status usl_launch_topk_adjusted(usl_ctx* c, const float* out, const usl_adjustments* a, int32_t b, int32_t kk, int32_t* top_lab, float* top_val) {
    const bool few = few_segments(c, b);
    const int nseg = segments(c, few ? AD_EPT_FEW : AD_EPT);
    USL_TRY(usl_reserve_topk(c));
    const dim3 grid((unsigned)nseg, (unsigned)b);
    if (few) hipLaunchKernelGGL(k_topk_adjusted<AD_EPT_FEW>, grid, dim3(AD_NT), 0, c->stream, out, c->m, of(c, a), (int)kk, nseg, c->topk_cand);
    else hipLaunchKernelGGL(k_topk_adjusted<AD_EPT>, grid, dim3(AD_NT), 0, c->stream, out, c->m, of(c, a), (int)kk, nseg, c->topk_cand);
    return usl_launch_topk_merge(c, nseg, b, kk, top_lab, top_val);
}
