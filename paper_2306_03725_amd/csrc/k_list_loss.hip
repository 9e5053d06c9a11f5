// Losses of a softmax over all labels against short lists: distillation from a teacher's best labels, and a clipped policy objective with a KL term.
//
//   q_j = exp((z_j - top) / T) / S,  S = sum_j exp((z_j - top) / T),  top the row's largest score
//   g_j = scale * (sum of c_e over the entries e of label j - (sum of all c_e) * q_j)
//   distillation:  c_e = -T * p_e,  p the softmax of the teacher's logits / T over the entries;  loss T^2 * sum p_e (log p_e - log q_e)
//   policy (T = 1): c_e = the slope of entry e's loss by its label's log-probability
//
// Three launches: largest score and sum of every segment of a row; a workgroup a row joins them and goes through the row's entries; the gradient, segment by segment.
// An entry counts if its label lies in [0, m), that label's score is above -infinity and (distillation) so is its logit.  Rows without one have no loss and a gradient of zeros, and
// their scores are not looked at.
#include "usl_internal.h"

namespace {

constexpr int LL_NT = 256, LL_EPT = 16, LL_SEG = LL_NT * LL_EPT;

typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));   // rows and segments begin at any float

struct Lists {
    const float* out;
    int64_t m;
    const int64_t* off;
    const int32_t* lab;
    const float *logit;                                // distillation
    const float *old_logp, *ref_logp, *advantage;      // policy
    float low, high, beta;                             // bounds of the ratio, weight of the KL term
    float inv_t;                                       // 1 / T
    double t, scale;
    float* logp;                                       // may be null
    float* loss;
    int nseg, b;
};
struct Part { float top, sum; };
struct Row {
    float top, k;        // g = k * exp((z - top) / T) + the label's entries
    int any;             // entries that count
    int pad;
    double log_sum;      // log S
    double teacher;      // log of the sum of exp(logit / T)
};

// Register e of a lane holds label local_label(e) of the segment: groups of four neighbours.
__device__ __forceinline__ int local_label(int e) { return ((e >> 2) * LL_NT + (int)threadIdx.x) * 4 + (e & 3); }

// A segment's scores, -infinity behind the row's end.  No load under a lane's condition: behind each of those the compiler waits.
__device__ __forceinline__ void load_segment(const float* row, int lim, float (&v)[LL_EPT]) {
    if (lim == LL_SEG) {
#pragma unroll
        for (int e = 0; e < LL_EPT; e += 4) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(row + local_label(e));
            v[e] = q.x; v[e + 1] = q.y; v[e + 2] = q.z; v[e + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < LL_EPT; ++e) v[e] = row[min(local_label(e), lim - 1)];
#pragma unroll
        for (int e = 0; e < LL_EPT; ++e) v[e] = local_label(e) < lim ? v[e] : -INFINITY;
    }
}
__device__ __forceinline__ float shift_of(float top) { return top == -INFINITY ? 0.f : top; }   // (-infinity less itself is NaN)

template <typename T> __device__ __forceinline__ T wave_join(T v, bool largest) {
    for (int o = 32; o > 0; o >>= 1) {
        const T u = __shfl_xor(v, o);
        v = largest ? (u > v ? u : v) : v + u;
    }
    return v;
}
// over the workgroup; red holds LL_NT / 64 values and is free again behind the next barrier
template <typename T> __device__ __forceinline__ T block_join(T v, bool largest, T* red) {
    v = wave_join(v, largest);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    T r = red[0];
#pragma unroll
    for (int w = 1; w < LL_NT / 64; ++w) r = largest ? (red[w] > r ? red[w] : r) : r + red[w];
    return r;
}

template <int N>   // the same for N sums at a time; red holds N * LL_NT / 64 values
__device__ __forceinline__ void block_sums(double (&v)[N], double* red) {
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = wave_join(v[q], false);
    __syncthreads();
#pragma unroll
    for (int q = 0; q < N; ++q)
        if ((threadIdx.x & 63) == 0) red[q * (LL_NT / 64) + (threadIdx.x >> 6)] = v[q];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < N; ++q) {
        v[q] = red[q * (LL_NT / 64)];
#pragma unroll
        for (int w = 1; w < LL_NT / 64; ++w) v[q] += red[q * (LL_NT / 64) + w];
    }
}

__global__ void __launch_bounds__(LL_NT)
k_list_parts(Lists a, Part* __restrict__ parts) {
    __shared__ float red[LL_NT / 64];
    const int i = (int)blockIdx.y;
    if (a.off[i + 1] <= a.off[i]) return;
    const int64_t seg0 = (int64_t)blockIdx.x * LL_SEG;
    float v[LL_EPT];
    load_segment(a.out + (int64_t)i * a.m + seg0, (int)min((int64_t)LL_SEG, a.m - seg0), v);
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < LL_EPT; ++e) top = fmaxf(top, v[e]);   // (fmaxf passes over NaN; the sum does not)
    top = block_join(top, true, red);
    const float from = shift_of(top);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < LL_EPT; ++e) sum += expf((v[e] - from) * a.inv_t);
    sum = block_join(sum, false, red);
    if (threadIdx.x == 0) parts[(size_t)i * a.nseg + blockIdx.x] = Part{top, sum};
}

// An entry's loss and its slope by the log-probability of its label
struct Slope { double loss, c; };
__device__ __forceinline__ Slope policy_of(const Lists& a, int64_t e, double logp) {
    const double adv = (double)a.advantage[e], ratio = exp(logp - (double)a.old_logp[e]);
    const double free = ratio * adv, bound = fmin(fmax(ratio, 1.0 - (double)a.low), 1.0 + (double)a.high) * adv;
    Slope s;
    s.loss = -(free <= bound ? free : bound);
    s.c = free <= bound ? -free : 0.0;
    if (!(free <= bound) && !(bound < free)) s.loss = s.c = free + bound;   // NaN
    if (a.ref_logp) {
        const double gap = (double)a.ref_logp[e] - logp, back = exp(gap);
        s.loss += (double)a.beta * (back - gap - 1.0);
        s.c += (double)a.beta * (1.0 - back);
    }
    return s;
}
// The score of an entry's label; counts: whether the entry does
__device__ __forceinline__ float score_of(const Lists& a, const float* row, int32_t label, bool& counts) {
    const bool inside = (uint32_t)label < (uint32_t)a.m;
    const float z = row[inside ? label : 0];
    counts = inside && !(z == -INFINITY);
    return z;
}
// A lane's first entry, asked for before the row's sum is known; lists are seldom longer than the workgroup
template <bool TEACHER>
struct Entry {
    float z, value;   // value: the teacher's logit
    bool counts;
    __device__ __forceinline__ void load(const Lists& a, const float* row, int64_t e) {
        z = score_of(a, row, a.lab[e], counts);
        if (TEACHER) {
            value = a.logit[e];
            counts = counts && !(value == -INFINITY);
        }
    }
};

template <bool TEACHER>
__global__ void __launch_bounds__(LL_NT)
k_list_rows(Lists a, const Part* __restrict__ parts, Row* __restrict__ rows, double* __restrict__ row_loss) {
    __shared__ double red[3 * LL_NT / 64];
    const int i = (int)blockIdx.x, tid = (int)threadIdx.x;
    const int64_t p0 = a.off[i], n = a.off[i + 1] - p0;
    if (n <= 0) {
        if (tid == 0) {
            rows[i] = Row{};
            row_loss[i] = 0.0;
        }
        return;
    }
    const float* row = a.out + (int64_t)i * a.m;
    parts += (size_t)i * a.nseg;
    const Part held = parts[min(tid, a.nseg - 1)];
    Entry<TEACHER> own;
    own.load(a, row, p0 + min((int64_t)tid, n - 1));
    own.counts = own.counts && tid < n;
    double best = tid < a.nseg ? (double)held.top : -INFINITY;
    for (int s = tid + LL_NT; s < a.nseg; s += LL_NT) best = fmax(best, (double)parts[s].top);
    best = block_join(best, true, red);
    const float top = (float)best, from = shift_of(top);
    auto share = [&](const Part& p) {
        return p.top == -INFINITY && p.sum == 0.f ? 0.0 : (double)p.sum * exp(((double)shift_of(p.top) - (double)from) * (double)a.inv_t);
    };
    double sum = tid < a.nseg ? share(held) : 0.0;
    for (int s = tid + LL_NT; s < a.nseg; s += LL_NT) sum += share(parts[s]);
    double total = 0.0, loss = 0.0, teacher = 0.0, count = 0.0;
    // every entry of this lane's, the first one from registers
    auto each = [&](auto what) {
        if (own.counts) what(own, p0 + tid);
        for (int64_t e = p0 + tid + LL_NT; e < p0 + n; e += LL_NT) {
            Entry<TEACHER> one;
            one.load(a, row, e);
            if (one.counts) what(one, e);
        }
    };
    double log_sum;
    if (TEACHER) {
        double most = -INFINITY;
        each([&](const Entry<TEACHER>& v, int64_t) {
            const double t = (double)v.value * (double)a.inv_t;
            most = t > most ? t : most;
            count += 1.0;
        });
        most = block_join(most, true, red);
        double cross = 0.0, mass = 0.0;
        each([&](const Entry<TEACHER>& v, int64_t) {
            const double t = (double)v.value * (double)a.inv_t, p = exp(t - most);
            mass += p;
            cross += p * ((t - most) - ((double)v.z - (double)from) * (double)a.inv_t);
        });
        double joined[3] = {sum, mass, cross};
        block_sums(joined, red);
        sum = joined[0];
        count = (double)__syncthreads_or(count > 0.0);
        log_sum = log(sum);
        const double log_mass = log(joined[1]);
        teacher = most + log_mass;
        total = -a.t;                                                       // of c_e: the p_e add up to 1
        loss = a.t * a.t * (joined[2] / joined[1] - log_mass + log_sum);
    } else {
        sum = block_join(sum, false, red);
        log_sum = log(sum);
        each([&](const Entry<TEACHER>& v, int64_t e) {
            const Slope s = policy_of(a, e, (double)v.z - (double)from - log_sum);
            count += 1.0;
            loss += s.loss;
            total += s.c;
        });
        if (a.logp)
            for (int64_t e = p0 + tid; e < p0 + n; e += LL_NT) {
                Entry<TEACHER> one = own;
                if (e != p0 + tid) one.load(a, row, e);
                a.logp[e] = one.counts ? (float)((double)one.z - (double)from - log_sum) : -INFINITY;
            }
        double joined[3] = {loss, total, count};
        block_sums(joined, red);
        loss = joined[0];
        total = joined[1];
        count = joined[2];
    }
    if (tid == 0) {
        const bool any = count > 0.0;
        rows[i] = Row{from, any ? (float)(-a.scale * total / sum) : 0.f, any ? 1 : 0, 0, log_sum, teacher};
        row_loss[i] = any ? loss : 0.0;
    }
}

// The rows' losses in a fixed order
__device__ __forceinline__ void add_losses(const Lists& a, const double* row_loss, double* red) {
    double sum = 0.0;
    for (int i = (int)threadIdx.x; i < a.b; i += LL_NT) sum += row_loss[i];
    sum = block_join(sum, false, red);
    if (threadIdx.x == 0) *a.loss = (float)(a.scale * sum);
}
__global__ void __launch_bounds__(LL_NT)
k_list_loss(Lists a, const double* __restrict__ row_loss) {
    __shared__ double red[LL_NT / 64];
    add_losses(a, row_loss, red);
}

// g may be out: a lane writes where it has read, and its segment's entries' scores are read before a barrier, and g is written behind it.
// A label with one entry takes its value from that entry.  Those of several are added up in the list's order, LL_NT entries at a time, by the first entry of the label among
// them: a list of n entries costs n steps, whatever it repeats.  (The first entry of all walking the rest of the list alone: one row of 20000 entries in far pairs, 30938 labels, 37 ms, so 0.67; 64 rows, 500k labels, 177 and 4.0.)
template <bool TEACHER>
__global__ void __launch_bounds__(LL_NT)
k_list_grad(Lists a, const Row* __restrict__ rows, const double* __restrict__ row_loss, float* g) {
    __shared__ __align__(16) uint32_t first[LL_SEG];   // the first entry of a label
    __shared__ __align__(16) uint32_t more[LL_SEG];    // how many it has; then the bits of their sum (in between, with first: of the sum in float64)
    __shared__ uint32_t repeated[LL_SEG / 32];         // labels of several entries
    __shared__ int some;                               // whether there are any
    __shared__ __align__(16) int32_t turn_lab[LL_NT];  // of LL_NT entries: those of such labels, else -1
    __shared__ double turn_c[LL_NT];
    __shared__ double red[LL_NT / 64];
    if (blockIdx.x == 0 && blockIdx.y == 0) add_losses(a, row_loss, red);
    const int i = (int)blockIdx.y, tid = (int)threadIdx.x;
    const int64_t seg0 = (int64_t)blockIdx.x * LL_SEG;
    const int lim = (int)min((int64_t)LL_SEG, a.m - seg0);
    const float* row = a.out + (int64_t)i * a.m;
    float v[LL_EPT];
    const Row r = rows[i];
    if (r.any) {
        load_segment(row + seg0, lim, v);   // (asked for before the row's sums are there, rows without entries would be read too: 256 x 500k 267 us, with them 280)
        const int64_t p0 = a.off[i], n = a.off[i + 1] - p0;
        auto here = [&](int32_t label) { return (uint32_t)label - (uint32_t)seg0 < (uint32_t)lim; };
        auto slope = [&](int64_t e) {   // c_e; 0 if the entry does not count
            Entry<TEACHER> one;
            one.load(a, row, e);
            if (!one.counts) return 0.0;
            if (TEACHER) return -a.t * exp((double)one.value * (double)a.inv_t - r.teacher);
            return policy_of(a, e, (double)one.z - (double)r.top - r.log_sum).c;
        };
        bool mine = false;
        for (int64_t p = tid; p < n; p += LL_NT) mine |= here(a.lab[p0 + p]);
        const bool any = __syncthreads_or(mine);
        if (any) {
#pragma unroll
            for (int e = 0; e < LL_EPT / 4; ++e) {
                reinterpret_cast<uint4*>(first)[e * LL_NT + tid] = make_uint4(~0u, ~0u, ~0u, ~0u);
                reinterpret_cast<uint4*>(more)[e * LL_NT + tid] = make_uint4(0, 0, 0, 0);
            }
            if (tid < LL_SEG / 32) repeated[tid] = 0;
            if (tid == 0) some = 0;
            __syncthreads();
            for (int64_t p = tid; p < n; p += LL_NT) {
                const int32_t label = a.lab[p0 + p];
                if (here(label)) {
                    atomicMin(&first[(uint32_t)label - (uint32_t)seg0], (uint32_t)p);
                    atomicAdd(&more[(uint32_t)label - (uint32_t)seg0], 1u);
                }
            }
            __syncthreads();
            for (int64_t p = tid; p < n; p += LL_NT) {
                const int32_t label = a.lab[p0 + p];
                const uint32_t j = (uint32_t)label - (uint32_t)seg0;
                if (!here(label) || first[j] != (uint32_t)p) continue;
                if (more[j] == 1) more[j] = __float_as_uint((float)(a.scale * slope(p0 + p)));
                else {
                    atomicOr(&repeated[j >> 5], 1u << (j & 31));
                    some = 1;
                }
            }
            __syncthreads();
            if (some) {
                auto is = [&](uint32_t j) { return repeated[j >> 5] >> (j & 31) & 1u; };
                for (uint32_t j = tid; j < LL_SEG; j += LL_NT)
                    if (is(j)) first[j] = more[j] = 0;   // 0.0
                for (int64_t base = 0; base < n; base += LL_NT) {
                    const int32_t label = base + tid < n ? a.lab[p0 + base + tid] : -1;
                    const uint32_t j = (uint32_t)label - (uint32_t)seg0;
                    const bool own = here(label) && is(j);
                    turn_lab[tid] = own ? label : -1;
                    if (own) turn_c[tid] = slope(p0 + base + tid);
                    if (__syncthreads_or(own)) {
                        if (own) {
                            double c = __longlong_as_double((long long)((uint64_t)more[j] << 32 | first[j]));
                            bool lead = true;
#pragma unroll 4
                            for (int t = 0; t < LL_NT; t += 4) {
                                const int4 q = *reinterpret_cast<const int4*>(turn_lab + t);
                                const int same = (q.x == label) | (q.y == label) << 1 | (q.z == label) << 2 | (q.w == label) << 3;
                                if (!same) continue;
                                for (int u = 0; u < 4; ++u)
                                    if (same >> u & 1) {
                                        lead = lead && t + u >= tid;
                                        c += turn_c[t + u];
                                    }
                            }
                            if (lead) {
                                first[j] = (uint32_t)(uint64_t)__double_as_longlong(c);
                                more[j] = (uint32_t)((uint64_t)__double_as_longlong(c) >> 32);
                            }
                        }
                        __syncthreads();
                    }
                }
                for (uint32_t j = tid; j < LL_SEG; j += LL_NT)
                    if (is(j)) more[j] = __float_as_uint((float)(a.scale * __longlong_as_double((long long)((uint64_t)more[j] << 32 | first[j]))));
                __syncthreads();
            }
        }
#pragma unroll
        for (int e = 0; e < LL_EPT; e += 4) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
            if (any) {
                const uint4 q = reinterpret_cast<const uint4*>(more)[(e >> 2) * LL_NT + tid];
                c[0] = __uint_as_float(q.x); c[1] = __uint_as_float(q.y); c[2] = __uint_as_float(q.z); c[3] = __uint_as_float(q.w);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) v[e + u] = fmaf(r.k, expf((v[e + u] - r.top) * a.inv_t), c[u]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < LL_EPT; ++e) v[e] = 0.f;
    }
    float* to = g + (int64_t)i * a.m + seg0;
#pragma unroll
    for (int e = 0; e < LL_EPT; e += 4) {
        const int j = local_label(e);
        if (j + 3 < lim) {
            // g goes past the caches, which hold scores that this launch has yet to read: 256 x 500k 269 -> 241 us (distillation), 280 -> 256 (policy).  (In
            // parts of 64 to 172 MB of rows, all three launches for each: 307 to 257; the last rows first: 269.)
            const f32x4 q = {v[e], v[e + 1], v[e + 2], v[e + 3]};
            __builtin_nontemporal_store(q, reinterpret_cast<f32x4*>(to + j));
        } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j + u < lim) to[j + u] = v[e + u];
        }
    }
}

template <bool TEACHER>
usl_status launch(usl_ctx* c, Lists a, float* g, int32_t b) {
    a.m = c->m;
    a.b = b;
    a.nseg = (int)((c->m + LL_SEG - 1) / LL_SEG);
    // for the largest batch that there can be: one of max_b, or of 320 GB of scores
    int64_t most = ((int64_t)80 << 30) / c->m + 1;
    if (most > c->max_b) most = c->max_b;
    if (most < b) most = b;
    const size_t part_bytes = ((size_t)most * a.nseg * sizeof(Part) + 255) / 256 * 256, row_bytes = ((size_t)most * sizeof(Row) + 255) / 256 * 256;
    USL_TRY(usl_reserve(c, (void**)&c->list_part, &c->list_part_cap, part_bytes + row_bytes + (size_t)most * sizeof(double)));
    Part* parts = (Part*)c->list_part;
    Row* rows = (Row*)(c->list_part + part_bytes);
    double* row_loss = (double*)(c->list_part + part_bytes + row_bytes);
    const dim3 grid((unsigned)a.nseg, (unsigned)b), block(LL_NT);
    const char* what = TEACHER ? "distill_loss_grad" : "policy_loss_grad";
    hipLaunchKernelGGL(k_list_parts, grid, block, 0, c->stream, a, parts);
    USL_TRY(usl_check_launch(c, what));
    hipLaunchKernelGGL(k_list_rows<TEACHER>, dim3((unsigned)b), block, 0, c->stream, a, parts, rows, row_loss);
    USL_TRY(usl_check_launch(c, what));
    if (g) hipLaunchKernelGGL(k_list_grad<TEACHER>, grid, block, 0, c->stream, a, rows, row_loss, g);
    else hipLaunchKernelGGL(k_list_loss, dim3(1), block, 0, c->stream, a, row_loss);
    return usl_check_launch(c, what);
}

}  // namespace

usl_status usl_launch_distill(usl_ctx* c, const float* out, const int64_t* off, const int32_t* lab, const float* logit, float temperature, float scale, float* g,
                              float* loss, int32_t b) {
    Lists a = {};
    a.out = out; a.off = off; a.lab = lab; a.logit = logit; a.loss = loss;
    a.t = (double)temperature;
    a.inv_t = (float)(1.0 / (double)temperature);
    a.scale = (double)scale;
    return launch<true>(c, a, g, b);
}

usl_status usl_launch_policy(usl_ctx* c, const float* out, const int64_t* off, const int32_t* lab, const float* old_logp, const float* ref_logp, const float* advantage,
                             float clip_low, float clip_high, float beta, float scale, float* g, float* logp, float* loss, int32_t b) {
    Lists a = {};
    a.out = out; a.off = off; a.lab = lab; a.old_logp = old_logp; a.ref_logp = ref_logp; a.advantage = advantage; a.logp = logp; a.loss = loss;
    a.low = clip_low; a.high = clip_high; a.beta = beta;
    a.inv_t = 1.f;
    a.t = 1.0;
    a.scale = (double)scale;
    return launch<false>(c, a, g, b);
}
