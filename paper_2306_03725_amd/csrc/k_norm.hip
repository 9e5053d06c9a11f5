// Layer norm of the rows h[b][d] that become the layer's activations x[b][d], and its backward pass:
//   mean = sum_c h / d,  var = sum_c (h - mean)^2 / d,  rstd = (var + eps)^-1/2,  n = (h - mean) rstd,  x = n gamma + beta
//   u = grad_x gamma,  grad_h = rstd (u - mean_c(u) - n mean_c(u n)),  grad_gamma = sum_i grad_x n,  grad_beta = sum_i grad_x
// The deviations are squared around the mean, not the values around zero, so a row far from zero keeps its variance.
#include "usl_internal.h"

namespace {

template <typename TS> __device__ __forceinline__ TS stored(float v);
template <> __device__ __forceinline__ float stored<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t stored<uint16_t>(float v) { return usl_f32_to_bf16(v); }   // the one rounding of a result

// ---- 16 bytes of a row at a time: 4 values of float32, 8 of bfloat16; rows begin at any value --------------------
typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8), aligned(2)));
template <typename TS> constexpr int VEC = 16 / (int)sizeof(TS);
// ... as they lie in memory, in four registers
template <typename TS> struct RawOf;
template <> struct RawOf<float> { typedef f32x4 T; };
template <> struct RawOf<uint16_t> { typedef u16x8 T; };
__device__ __forceinline__ float value(const f32x4& q, int e) { return q[e]; }
__device__ __forceinline__ float value(const u16x8& q, int e) { return usl_bf16_to_f32(q[e]); }

__device__ __forceinline__ void load_vec(const float* p, float (&v)[4]) {
    const f32x4 q = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = q[e];
}
__device__ __forceinline__ void load_vec(const float* p, float (&v)[8]) {
    const f32x4 q = *reinterpret_cast<const f32x4*>(p), r = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = q[e]; v[4 + e] = r[e]; }
}
__device__ __forceinline__ void load_vec(const uint16_t* p, float (&v)[8]) {
    const u16x8 q = *reinterpret_cast<const u16x8*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = usl_bf16_to_f32(q[e]);
}
__device__ __forceinline__ void store_vec(float* p, const float (&v)[4]) {
    const f32x4 q = {v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p) = q;
}
__device__ __forceinline__ void store_vec(float* p, const float (&v)[8]) {
    const f32x4 q = {v[0], v[1], v[2], v[3]}, r = {v[4], v[5], v[6], v[7]};
    *reinterpret_cast<f32x4*>(p) = q;
    *reinterpret_cast<f32x4*>(p + 4) = r;
}
__device__ __forceinline__ void store_vec(uint16_t* p, const float (&v)[8]) {
    u16x8 q;
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = usl_f32_to_bf16(v[e]);
    *reinterpret_cast<u16x8*>(p) = q;
}

// How LANES lanes divide a row of d >= V values: the whole groups of V values are dealt to the lanes in turn, the values behind them (fewer than V) go one
// to a lane.  A lane without a group loads the row's last one instead, and leaves it out of its sums: a load under a lane's condition is waited for by the
// compiler then and there.  (With the last group taken value by value every load and store had V branches, and the kernels spilled.)
template <int LANES, int V>
struct RowShare {
    int lane, whole, rest;   // values in whole groups, values behind them
    __device__ __forceinline__ RowShare(int lane_, int d) : lane(lane_), whole(d / V * V), rest(d % V) {}
    // the lane number taken afresh: what is derived from it is rebuilt with a few instructions instead of living in registers that the row needs
    __device__ __forceinline__ void renew() { asm volatile("" : "+v"(lane)); }
    __device__ __forceinline__ int at(int g) const { return (g * LANES + lane) * V; }
    __device__ __forceinline__ bool has(int g) const { return at(g) < whole; }
    __device__ __forceinline__ bool has_rest() const { return lane < rest; }
    template <typename T>
    __device__ __forceinline__ void load(const T* row, int g, float (&v)[V]) const { load_vec(row + min(at(g), whole - V), v); }
    template <typename RAW, typename T>
    __device__ __forceinline__ RAW load_raw(const T* row, int g) const { return *reinterpret_cast<const RAW*>(row + min(at(g), whole - V)); }
    template <typename T>
    __device__ __forceinline__ float load_rest(const T* row) const { return usl_to_f32(row[min(whole + lane, whole + rest - 1)]); }
};

// ---- sums over lanes --------------------------------------------------------------------------------------------
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ float moved(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xF, true)); }
// over 16 neighbouring lanes, in all of them (lanes that have been added up are alike: a mirror reaches the others as well)
__device__ __forceinline__ float sum16(float v) {
    v += moved<0xB1>(v);    // quads 1 0 3 2
    v += moved<0x4E>(v);    // quads 2 3 0 1
    v += moved<0x141>(v);   // 8 lanes, mirrored
    v += moved<0x140>(v);   // 16
    return v;
}
__device__ __forceinline__ float sum64(float v) {
    v = sum16(v);
    v += moved<0x142, 0xA>(v);   // the last lane of rows 0 and 2 into rows 1 and 3 (0 into the others), of row 1 into rows 2 and 3
    v += moved<0x143, 0xC>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
template <int LANES>
__device__ __forceinline__ float sum_lanes(float v) { return LANES == 16 ? sum16(v) : sum64(v); }

// Sum of v over the workgroup, returned to every lane.  red: one value a wavefront.
template <int NT, typename T>
__device__ __forceinline__ T block_sum(T v, T* red) {
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();   // red is no longer read
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    T s = red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) s += red[w];
    return s;
}

// ---- forward: a row in the registers of LANES lanes, EPL values each (and one of the values behind the groups) --
// Read once, written once; bound by that stream where there are many rows (512 x 32768 bfloat16: 67 MB in 15.1 us, 4.5 TB/s where a large copy
// reaches 5.0), by one launch's latency where there are few (1 x 32768 float32: 5.9 us).  A wavefront takes the mean and the squared deviations of its own values; several wavefronts of a row join theirs
// around the row's mean, behind one barrier:  M2 = sum_w M2_w + n_w (mean_w - mean)^2.
// FULL: there are both a weight and a bias; EARLY: they come with the row, not behind the sums.
template <typename TS, int LANES, int EPL, bool FULL, bool EARLY>
__global__ void __launch_bounds__((LANES < 256 ? 256 : LANES), (LANES == 1024 && EPL <= 32 && !EARLY ? 8 : 1))
k_norm(const TS* h, const float* __restrict__ gamma, const float* __restrict__ beta, float eps, TS* x /* may be h */, float* __restrict__ mean_out,
       float* __restrict__ rstd_out, int b, int d) {
    constexpr int V = VEC<TS>, G = EPL / V, NT = LANES < 256 ? 256 : LANES, WAVES = LANES / 64;
    static_assert(FULL || !EARLY, "nothing to load early");
    int i = (int)blockIdx.x * (NT / LANES) + (int)threadIdx.x / LANES;
    if (LANES >= 64) i = __builtin_amdgcn_readfirstlane(i);
    if (i >= b) return;   // (rows of several wavefronts have a workgroup each)
    RowShare<LANES, V> mine((int)threadIdx.x % LANES, d);
    typename RawOf<TS>::T v[G];
    float wg[EARLY ? G : 1][V], wb[EARLY ? G : 1][V];
    const TS* from = h + (size_t)i * d;
#pragma unroll
    for (int g = 0; g < G; ++g) v[g] = mine.template load_raw<typename RawOf<TS>::T>(from, g);
    float last = mine.load_rest(from);
    if (!mine.has_rest()) last = 0.f;
    if constexpr (EARLY) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            mine.load(gamma, g, wg[g]);
            mine.load(beta, g, wb[g]);
        }
    }
    const float last_w = gamma ? mine.load_rest(gamma) : 1.f, last_b = beta ? mine.load_rest(beta) : 0.f;
    float s = last;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        float t = value(v[g], 0);
#pragma unroll
        for (int e = 1; e < V; ++e) t += value(v[g], e);
        s += mine.has(g) ? t : 0.f;
    }
    int n = d;   // values of this wavefront
    if (LANES > 64) {
        const int wave0 = __builtin_amdgcn_readfirstlane((int)threadIdx.x & ~63);
        n = min(max(mine.rest - wave0, 0), 64);
#pragma unroll
        for (int g = 0; g < G; ++g) n += min(max(mine.whole - (g * LANES + wave0) * V, 0), 64 * V);
    }
    float mean = n ? sum_lanes<LANES>(s) / (float)n : 0.f;
    float m2 = mine.has_rest() ? (last - mean) * (last - mean) : 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) t = fmaf(value(v[g], e) - mean, value(v[g], e) - mean, t);
        m2 += mine.has(g) ? t : 0.f;
    }
    m2 = sum_lanes<LANES>(m2);
    if constexpr (LANES > 64) {
        __shared__ float part[3][WAVES];
        if ((threadIdx.x & 63) == 0) {
            part[0][threadIdx.x >> 6] = mean;
            part[1][threadIdx.x >> 6] = m2;
            part[2][threadIdx.x >> 6] = (float)n;
        }
        __syncthreads();
        const int w = (int)threadIdx.x & 15;   // 16 lanes take a wavefront's each
        const bool is = WAVES == 16 || w < WAVES;
        const float mean_w = part[0][is ? w : 0], m2_w = is ? part[1][w] : 0.f, n_w = is ? part[2][w] : 0.f;
        mean = sum16(mean_w * n_w) / (float)d;
        m2 = sum16(fmaf(n_w * (mean_w - mean), mean_w - mean, m2_w));
    }
    const float rstd = 1.f / sqrtf(m2 / (float)d + eps);
    if (mine.lane == 0) {
        if (mean_out) mean_out[i] = mean;
        if (rstd_out) rstd_out[i] = rstd;
    }
    TS* to = x + (size_t)i * d;
    mine.renew();
#pragma unroll
    for (int g = 0; g < G; ++g) {
        float o[V], w[V], c[V];
        if constexpr (EARLY) {
#pragma unroll
            for (int e = 0; e < V; ++e) { w[e] = wg[g][e]; c[e] = wb[g][e]; }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) { w[e] = 1.f; c[e] = 0.f; }
            if (FULL || gamma) mine.load(gamma, g, w);
            if (FULL || beta) mine.load(beta, g, c);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fmaf((value(v[g], e) - mean) * rstd, w[e], c[e]);
        if (mine.has(g)) store_vec(to + mine.at(g), o);
        if (!EARLY && g % 2) __builtin_amdgcn_sched_barrier(0);   // a few groups' weights at a time
    }
    if (mine.has_rest()) to[mine.whole + mine.lane] = stored<TS>(fmaf((last - mean) * rstd, last_w, last_b));
}

// Rows that registers do not hold: a workgroup a row, which it reads once for every sum and once more to write, a value a lane at a time.  (Sums in 64 bits: a lane may
// have thousands of values.)  512 x 100 003 bfloat16: 148 us, 41 at the rate of a large copy; 64 of float32, a quarter of the chip: 77 and 10.5.
constexpr int ANY_NT = 1024;
template <typename TS>
__global__ void __launch_bounds__(ANY_NT)
k_norm_any(const TS* h, const float* __restrict__ gamma, const float* __restrict__ beta, float eps, TS* x /* may be h */,
           float* __restrict__ mean_out, float* __restrict__ rstd_out, int d) {
    __shared__ double red[ANY_NT / 64];
    const TS* row = h + (size_t)blockIdx.x * d;
    double s = 0.0;
    for (int c = threadIdx.x; c < d; c += ANY_NT) s += usl_load_f32<TS>(row, c);
    const float mean = (float)(block_sum<ANY_NT>(s, red) / d);
    s = 0.0;
    for (int c = threadIdx.x; c < d; c += ANY_NT) {
        const float t = usl_load_f32<TS>(row, c) - mean;
        s += (double)t * t;
    }
    const float rstd = (float)(1.0 / sqrt(block_sum<ANY_NT>(s, red) / d + eps));
    if (threadIdx.x == 0) {
        if (mean_out) mean_out[blockIdx.x] = mean;
        if (rstd_out) rstd_out[blockIdx.x] = rstd;
    }
    for (int c = threadIdx.x; c < d; c += ANY_NT) {
        const float n = (usl_load_f32<TS>(row, c) - mean) * rstd;
        x[(size_t)blockIdx.x * d + c] = stored<TS>(fmaf(n, gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f));
    }
}

// ---- backward, rows of up to 16384: a row in the registers of LANES lanes, EPL values each -----------------------
// A workgroup of 1024 lanes takes 1024 / LANES rows at a time, its share of the batch one after the other, and keeps the sums of grad_x n and grad_x
// of its rows in registers: the inputs are read once.  At the end its row groups' sums are joined through LDS, always in the same order, and left in
// part[workgroup][2][d] (with one workgroup: in the gradients themselves).  Bound by the wait for the rows, which every wavefront has once or a few
// times, and by the launch that adds the parts up: 4099 x 1003 bfloat16, 41 MB: 14.7 us (kernels 12.0 + 3.8 in a trace), 8.3 at the rate of a large copy.
// WEIGHT: there is a gamma.  (The form of 256 lanes, rows of 2049 to 4096, has 11 to 14 of its 128 registers in scratch, the others none: 8192 x 4096 float32 88.6 us, 4096 x 8192 87.4,
// 81.1 at the rate of a large copy.)
constexpr int BWD_NT = 1024;
template <typename TS, int LANES, int EPL, bool WEIGHT>
__global__ void __launch_bounds__(BWD_NT)
k_norm_grad(const float* __restrict__ grad_x, const TS* __restrict__ h, const float* __restrict__ gamma, const float* __restrict__ mean_in,
            const float* __restrict__ rstd_in, float* __restrict__ grad_h, float* __restrict__ to_gamma, float* __restrict__ to_beta, size_t stride, int b, int d) {
    constexpr int V = VEC<TS>, G = EPL / V, ROWS = BWD_NT / LANES, WAVES = LANES / 64;
    extern __shared__ __align__(16) float lds[];   // [row groups, or up to 4 those but the first][2][EPL + 1][LANES]
    __shared__ float part[2][2][BWD_NT / 64];
    RowShare<LANES, V> mine((int)threadIdx.x % LANES, d);
    int group = (int)threadIdx.x / LANES;
    if (LANES >= 64) group = __builtin_amdgcn_readfirstlane(group);
    float sg[G][V] = {}, sb[G][V] = {}, last_sg = 0.f, last_sb = 0.f;
    int turn = 0;
    for (int i0 = (int)blockIdx.x * ROWS; i0 < b; i0 += (int)gridDim.x * ROWS, turn ^= 1) {
        const int i = i0 + group;
        const bool in = i < b;
        mine.renew();
        const size_t at = (size_t)(in ? i : 0) * d;   // (a row group without a row takes row 0, and adds nothing)
        float gx[G][V], n[G][V], su = 0.f, sn = 0.f;
        const float mean = mean_in[in ? i : 0], rstd = rstd_in[in ? i : 0];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            mine.load(grad_x + at, g, gx[g]);
            mine.load(h + at, g, n[g]);
        }
        float last_g = mine.load_rest(grad_x + at), last_n = mine.load_rest(h + at);
        if (!in || !mine.has_rest()) last_g = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float w[V], t = 0.f, q = 0.f;
            if (WEIGHT) mine.load(gamma, g, w);   // (from the L1: kept across the rows they would cost the registers that the sums need)
            if (G > 2 && g % 2) __builtin_amdgcn_sched_barrier(0);   // two groups' at a time
            if (!in) {
#pragma unroll
                for (int e = 0; e < V; ++e) gx[g][e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {   // (a lane without the group: its sums of columns go nowhere)
                n[g][e] = (n[g][e] - mean) * rstd;
                sg[g][e] = fmaf(gx[g][e], n[g][e], sg[g][e]);
                sb[g][e] += gx[g][e];
                if (WEIGHT) gx[g][e] *= w[e];   // u
                t += gx[g][e];
                q = fmaf(gx[g][e], n[g][e], q);
            }
            su += mine.has(g) ? t : 0.f;
            sn += mine.has(g) ? q : 0.f;
        }
        last_n = (last_n - mean) * rstd;
        last_sg = fmaf(last_g, last_n, last_sg);
        last_sb += last_g;
        if (WEIGHT) last_g *= mine.load_rest(gamma);
        if (!mine.has_rest()) last_g = last_n = 0.f;
        su = sum_lanes<LANES>(su + last_g);
        sn = sum_lanes<LANES>(fmaf(last_g, last_n, sn));
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) {
                part[turn][0][threadIdx.x >> 6] = su;
                part[turn][1][threadIdx.x >> 6] = sn;
            }
            __syncthreads();   // (two sets in turn: a set is written again behind the next barrier, which all reach behind their reads)
            const int q = (int)threadIdx.x & 15;   // 16 lanes take a wavefront's each
            const bool is = WAVES == 16 || q < WAVES;
            su = sum16(is ? part[turn][0][group * WAVES + (is ? q : 0)] : 0.f);
            sn = sum16(is ? part[turn][1][group * WAVES + (is ? q : 0)] : 0.f);
        }
        const float mu = su / (float)d, mn = sn / (float)d;
        mine.renew();
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float o[V];
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = rstd * (gx[g][e] - mu - n[g][e] * mn);
            if (in && mine.has(g)) store_vec(grad_h + at + mine.at(g), o);
        }
        if (in && mine.has_rest()) grad_h[at + mine.whole + mine.lane] = rstd * (last_g - mu - last_n * mn);
    }
    if (!to_gamma && !to_beta) return;
    if constexpr (ROWS <= 4) {   // long rows: the first group joins the others' sums to its own
        constexpr int E = EPL + 1, ENTRIES = 2 * E * LANES;   // [2][value of a lane, the rest][lane]
        if (ROWS > 1 && group > 0) {
            float* own = lds + (group - 1) * ENTRIES + mine.lane;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    own[(g * V + e) * LANES] = sg[g][e];
                    own[(E + g * V + e) * LANES] = sb[g][e];
                }
            own[EPL * LANES] = last_sg;
            own[(E + EPL) * LANES] = last_sb;
        }
        if (ROWS > 1) __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int r = 0; r < ROWS - 1; ++r) {
            const float* other = lds + r * ENTRIES + mine.lane;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    sg[g][e] += other[(g * V + e) * LANES];
                    sb[g][e] += other[(E + g * V + e) * LANES];
                }
            last_sg += other[EPL * LANES];
            last_sb += other[(E + EPL) * LANES];
        }
        float* rows[2] = {to_gamma ? to_gamma + blockIdx.x * stride : nullptr, to_beta ? to_beta + blockIdx.x * stride : nullptr};
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (!rows[which]) continue;
#pragma unroll
            for (int g = 0; g < G; ++g)
                if (mine.has(g)) store_vec(rows[which] + mine.at(g), which ? sb[g] : sg[g]);
            if (mine.has_rest()) rows[which][mine.whole + mine.lane] = which ? last_sb : last_sg;
        }
    } else {   // every row group leaves its sums, and every lane joins those of a few columns
        constexpr int E = EPL + 1, ENTRIES = 2 * E * LANES;   // [2][value of a lane, the rest][lane]
        float* own = lds + group * ENTRIES + mine.lane;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                own[(g * V + e) * LANES] = sg[g][e];
                own[(E + g * V + e) * LANES] = sb[g][e];
            }
        own[EPL * LANES] = last_sg;
        own[(E + EPL) * LANES] = last_sb;
        __syncthreads();
        for (int at = (int)threadIdx.x; at < ENTRIES; at += BWD_NT) {
            float s = lds[at];
#pragma unroll
            for (int r = 1; r < ROWS; ++r) s += lds[r * ENTRIES + at];
            const int lane = at % LANES, q = at / LANES % E;
            float* to = at < E * LANES ? to_gamma : to_beta;
            const int c = q == EPL ? mine.whole + lane : (q / V * LANES + lane) * V + q % V;
            if (to && (q == EPL ? lane < mine.rest : c < mine.whole)) to[blockIdx.x * stride + c] = s;
        }
    }
}

// ---- backward, wide rows: the rows' sums first, then tiles of columns and rows -----------------------------------
// The inputs are read twice, the second time mostly from the cache behind the L2s, and that is what bounds it: 256 x 32768 float32: 34.0 us (in a trace sums
// 13.5, 67 MB, tiles 18.4, 101 MB, parts 4.3); one pass would be 20.3 at the rate of a large copy.  (A row of this width and its sums of columns do not fit the registers
// of a compute unit beside each other, and sums left by every row are as many bytes as the inputs.)
// sums[i][split][2]: sums of u and u n over a share of row i's columns.  grid (splits, rows)
constexpr int SUMS_NT = 512;
template <typename TS, bool WEIGHT>
__global__ void __launch_bounds__(SUMS_NT)
k_norm_grad_sums(const float* __restrict__ grad_x, const TS* __restrict__ h, const float* __restrict__ gamma, const float* __restrict__ mean_in,
                 const float* __restrict__ rstd_in, float* __restrict__ sums, int d, int cols) {
    constexpr int V = VEC<TS>, AHEAD = 16 / V;
    __shared__ double red[SUMS_NT / 64];
    const float* gx_row = grad_x + (size_t)blockIdx.y * d;
    const float mean = mean_in[blockIdx.y], rstd = rstd_in[blockIdx.y];
    const TS* h_row = h + (size_t)blockIdx.y * d;
    const int c0 = (int)blockIdx.x * cols, whole = d / V * V, end = min(whole, c0 + cols);
    double su = 0.0, sn = 0.0;
    for (int c = c0 + (int)threadIdx.x * V; c < end; c += SUMS_NT * V * AHEAD) {
        float gx[AHEAD][V], v[AHEAD][V], w[AHEAD][V], t = 0.f, q = 0.f;
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int ca = min(c + a * SUMS_NT * V, end - V);   // (behind the end: the last group once more, and nothing is made of it)
            load_vec(gx_row + ca, gx[a]);
            load_vec(h_row + ca, v[a]);
            if (WEIGHT) load_vec(gamma + ca, w[a]);
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            float ta = 0.f, qa = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float u = WEIGHT ? gx[a][e] * w[a][e] : gx[a][e];
                ta += u;
                qa = fmaf(u, (v[a][e] - mean) * rstd, qa);
            }
            t += c + a * SUMS_NT * V < end ? ta : 0.f;
            q += c + a * SUMS_NT * V < end ? qa : 0.f;
        }
        su += t;
        sn += q;
    }
    if (blockIdx.x == 0 && (int)threadIdx.x < d - whole) {   // the values behind the whole groups
        const int c = whole + (int)threadIdx.x;
        const float u = gamma ? gx_row[c] * gamma[c] : gx_row[c];
        su += u;
        sn += (double)u * ((usl_to_f32(h_row[c]) - mean) * rstd);
    }
    const double all = block_sum<SUMS_NT>(su, red), alln = block_sum<SUMS_NT>(sn, red);
    if (threadIdx.x == 0) {
        float* to = sums + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2;
        to[0] = (float)all;
        to[1] = (float)alln;
    }
}

// grad_h of a tile, and the tile's sums of grad_x n and grad_x over its rows into part[blockIdx.y][2][d] (with one part: the gradients themselves).  A lane has 4 columns.  grid (columns, rows)
constexpr int TILE_NT = 256, TILE_COLS = TILE_NT * 4, TILE_AT_ONCE = 8, TILE_ROWS = 2048 /* their statistics take 32 KB of LDS */;
__device__ __forceinline__ void load_four(const float* p, float (&v)[4]) { load_vec(p, v); }
typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void load_four(const uint16_t* p, float (&v)[4]) {
    const u16x4 q = *reinterpret_cast<const u16x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = usl_bf16_to_f32(q[e]);
}
template <typename TS>
__global__ void __launch_bounds__(TILE_NT)
k_norm_grad_tile(const float* __restrict__ grad_x, const TS* __restrict__ h, const float* __restrict__ gamma, const float* __restrict__ mean_in,
                 const float* __restrict__ rstd_in, const float* __restrict__ sums, int splits, float* __restrict__ grad_h, float* __restrict__ to_gamma, float* __restrict__ to_beta,
                 size_t stride, int b, int d, int rows) {
    extern __shared__ __align__(16) float of_row[];   // [rows][4]: mean, rstd, mean of u, mean of u n
    const int i0 = (int)blockIdx.y * rows, n = min(rows, b - i0), lane = threadIdx.x & 63;
    const int start = (int)blockIdx.x * TILE_COLS + (int)threadIdx.x * 4, c = min(start, max(d - 4, 0));   // (the last lane takes the last four: a neighbour's again)
    const bool full = d >= 4;
    float gx[2][TILE_AT_ONCE][4], v[2][TILE_AT_ONCE][4], w[4] = {1.f, 1.f, 1.f, 1.f}, sg[4] = {}, sb[4] = {};
    // (loads without conditions, which the compiler would wait for: what is not there is another row's or column's)
    auto load = [&](int r0, float (&g)[TILE_AT_ONCE][4], float (&x)[TILE_AT_ONCE][4]) {
#pragma unroll
        for (int a = 0; a < TILE_AT_ONCE; ++a) {
            const size_t at = (size_t)(i0 + min(r0 + a, n - 1)) * d;
            if (full) {
                load_four(grad_x + at + c, g[a]);
                load_four(h + at + c, x[a]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    g[a][e] = grad_x[at + min(c + e, d - 1)];
                    x[a][e] = usl_to_f32(h[at + min(c + e, d - 1)]);
                }
            }
        }
    };
    load(0, gx[0], v[0]);
    if (gamma) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = gamma[min(c + e, d - 1)];
    }
    for (int r = (int)(threadIdx.x >> 6); r < n; r += TILE_NT / 64) {
        float su = 0.f, sn = 0.f;
        for (int s = lane; s < splits; s += 64) {
            const float* from = sums + ((size_t)(i0 + r) * splits + s) * 2;
            su += from[0];
            sn += from[1];
        }
        su = sum64(su);
        sn = sum64(sn);
        if (lane == 0) {
            of_row[r * 4] = mean_in[i0 + r];
            of_row[r * 4 + 1] = rstd_in[i0 + r];
            of_row[r * 4 + 2] = su / (float)d;
            of_row[r * 4 + 3] = sn / (float)d;
        }
    }
    __syncthreads();
    if (start >= d) return;
    auto put = [&](float* to, const float (&o)[4]) {
        if (full) store_vec(to + c, o);
        else
            for (int e = 0; e < 4; ++e)
                if (c + e < d) to[c + e] = o[e];
    };
    auto work = [&](int r0, const float (&g)[TILE_AT_ONCE][4], const float (&x)[TILE_AT_ONCE][4]) {
#pragma unroll
        for (int a = 0; a < TILE_AT_ONCE; ++a) {
            if (r0 + a >= n) break;
            const float4 k = *reinterpret_cast<const float4*>(of_row + (r0 + a) * 4);
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = g[a][e] * w[e], m = (x[a][e] - k.x) * k.y;
                o[e] = k.y * (u - k.z - m * k.w);
                sg[e] = fmaf(g[a][e], m, sg[e]);
                sb[e] += g[a][e];
            }
            put(grad_h + (size_t)(i0 + r0 + a) * d, o);
        }
    };
    // the next rows are asked for before these are written: the wait for a load is one for every store before it too
    for (int r0 = 0; r0 < n; r0 += 2 * TILE_AT_ONCE) {
        load(r0 + TILE_AT_ONCE, gx[1], v[1]);
        work(r0, gx[0], v[0]);
        load(r0 + 2 * TILE_AT_ONCE, gx[0], v[0]);
        work(r0 + TILE_AT_ONCE, gx[1], v[1]);
    }
    if (to_gamma) put(to_gamma + blockIdx.y * stride, sg);
    if (to_beta) put(to_beta + blockIdx.y * stride, sb);
}

// The parts' sums, added up in a fixed order: a lane takes COLS columns of one of the two sums and every GROUPS-th part, the groups join through LDS.
template <int COLS, int GROUPS>
__global__ void __launch_bounds__(64 * GROUPS)
k_norm_sum_parts(const float* __restrict__ part, int parts, int d, float* __restrict__ grad_gamma, float* __restrict__ grad_beta) {
    constexpr int AT_ONCE = 8;
    __shared__ float red[GROUPS][64 * COLS];
    const int lane = threadIdx.x & 63, group = threadIdx.x >> 6, c = ((int)blockIdx.x * 64 + lane) * COLS;
    float* to = blockIdx.y ? grad_beta : grad_gamma;
    if (!to) return;
    float s[COLS] = {};
    const float* from = part + (size_t)blockIdx.y * d;
    const int first = min(c, d - COLS);   // (the last lanes take the last columns: the same sums as another lane's)
    for (int p0 = group; p0 < parts; p0 += AT_ONCE * GROUPS) {
        float v[AT_ONCE][COLS];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const float* at = from + (size_t)min(p0 + u * GROUPS, parts - 1) * 2 * d + first;
            if constexpr (COLS == 4) load_vec(at, v[u]);
            else v[u][0] = *at;
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
            for (int e = 0; e < COLS; ++e) s[e] += p0 + u * GROUPS < parts ? v[u][e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < COLS; ++e) red[group][lane * COLS + e] = s[e];
    __syncthreads();
    for (int q = threadIdx.x; q < 64 * COLS; q += 64 * GROUPS) {
        float t = red[0][q];
#pragma unroll
        for (int g = 1; g < GROUPS; ++g) t += red[g][q];
        to[min((int)blockIdx.x * 64 * COLS + q / COLS * COLS, d - COLS) + q % COLS] = t;
    }
}

}  // namespace

struct NormArgs {
    const void* h;
    const float *gamma, *beta;
    float eps;
    void* x;
    float *mean, *rstd;
    int32_t b;
};
template <typename TS, int LANES, int EPL, bool FULL, bool EARLY>
static void launch_norm(usl_ctx* c, const NormArgs& a) {
    constexpr int NT = LANES < 256 ? 256 : LANES, ROWS = NT / LANES;
    hipLaunchKernelGGL((k_norm<TS, LANES, EPL, FULL, EARLY>), dim3((unsigned)((a.b + ROWS - 1) / ROWS)), dim3(NT), 0, c->stream, (const TS*)a.h, a.gamma, a.beta, a.eps,
                       (TS*)a.x, a.mean, a.rstd, a.b, c->d);
}
// Weight and bias come with the row where registers are left for them: always for 16 values a lane, never for 64; for 32 where there is at most one row to a compute
// unit, whose wait for them nothing else covers (1 x 32768 float32 6.5 us, early 6.0; 512 x 32768 bfloat16, two rows to a compute unit: 14.9, early, one, 17.7).
template <typename TS, int LANES, int EPL>
static void launch_norm(usl_ctx* c, const NormArgs& a) {
    if (!a.gamma || !a.beta) return launch_norm<TS, LANES, EPL, false, false>(c, a);
    if constexpr (EPL <= 16) launch_norm<TS, LANES, EPL, true, true>(c, a);
    else if constexpr (EPL > 32) launch_norm<TS, LANES, EPL, true, false>(c, a);
    else if (a.b <= c->num_cu) launch_norm<TS, LANES, EPL, true, true>(c, a);
    else launch_norm<TS, LANES, EPL, true, false>(c, a);
}
// Lanes of a row by its length: 16 where four rows fit a wavefront, then a wavefront, then as many as keep 16 values each; the longest rows of a
// workgroup have 32 or 64 values a lane.
template <typename TS>
static usl_status norm(usl_ctx* c, const NormArgs& a) {
    const int d = c->d;
    if (d < VEC<TS> || d > 65536)
        hipLaunchKernelGGL(k_norm_any<TS>, dim3((unsigned)a.b), dim3(ANY_NT), 0, c->stream, (const TS*)a.h, a.gamma, a.beta, a.eps, (TS*)a.x, a.mean, a.rstd, d);
    else if (d <= 128) launch_norm<TS, 16, 8>(c, a);
    else if (d <= 256) launch_norm<TS, 16, 16>(c, a);
    else if (d <= 512) launch_norm<TS, 64, 8>(c, a);
    else if (d <= 1024) launch_norm<TS, 64, 16>(c, a);
    else if (d <= 2048) launch_norm<TS, 64, 32>(c, a);
    else if (d <= 4096) launch_norm<TS, 256, 16>(c, a);
    else if (d <= 8192) launch_norm<TS, 512, 16>(c, a);
    else if (d <= 16384) launch_norm<TS, 1024, 16>(c, a);
    else if (d <= 32768) launch_norm<TS, 1024, 32>(c, a);
    else launch_norm<TS, 1024, 64>(c, a);
    return usl_check_launch(c, "layer_norm");
}

usl_status usl_launch_norm(usl_ctx* c, const void* h, const float* gamma, const float* beta, float eps, void* x, float* mean, float* rstd, int32_t b) {
    const NormArgs a = {h, gamma, beta, eps, x, mean, rstd, b};
    return c->storage == USL_F32 ? norm<float>(c, a) : norm<uint16_t>(c, a);
}

// How the backward pass is cut up.
struct NormShape {
    bool registers;   // rows in registers, one pass
    int lanes, parts; // lanes of a row; sets of sums over rows
    int rows, splits; // two passes: rows of a tile, shares of a row
};
static NormShape norm_shape(const usl_ctx* c, int b) {
    NormShape s = {};
    const int d = c->d, es = c->storage == USL_F32 ? 4 : 2;
    s.lanes = d <= 128 ? 16 : d <= 1024 ? 64 : d <= 2048 ? 128 : d <= 4096 ? 256 : d <= 8192 ? 512 : 1024;
    const int at_once = BWD_NT / s.lanes, all = (b + at_once - 1) / at_once;
    s.parts = all < c->num_cu ? all : c->num_cu;
    // The sums that a workgroup leaves are written and read once: 16 bytes a column and workgroup, against 4 + es bytes a value for reading the inputs again.
    // Below half a million values neither counts, and one pass is a launch less (10 x 4840 bfloat16: 16.4 us and 10.8).
    s.registers = d <= 16384 && d * es >= 16 && ((int64_t)s.parts * 16 <= (int64_t)b * (4 + es) || (int64_t)b * d <= 1 << 19);
    if (s.registers) return s;
    const int tiles = (d + TILE_COLS - 1) / TILE_COLS, want = (c->num_cu * 2 + tiles - 1) / tiles;
    s.rows = (b + want - 1) / want;
    s.rows = s.rows < 8 ? 8 : s.rows > TILE_ROWS ? TILE_ROWS : s.rows;
    s.parts = (b + s.rows - 1) / s.rows;
    const int most = (d + 4095) / 4096;
    s.splits = (c->num_cu * 2 + b - 1) / b;
    if (s.splits > most) s.splits = most;
    return s;
}

template <typename TS>
static usl_status norm_grad(usl_ctx* c, const float* grad_x, const void* h, const float* gamma, const float* mean, const float* rstd, float* grad_h,
                            float* grad_gamma, float* grad_beta, int32_t b) {
    const NormShape s = norm_shape(c, b);
    const int d = c->d;
    const bool sums = grad_gamma || grad_beta;
    // scratch for any batch up to max_b: at most parts_most sets of sums, and max_b + 2 num_cu pairs of a row's sums
    const int tiles = (d + TILE_COLS - 1) / TILE_COLS, want = (c->num_cu * 2 + tiles - 1) / tiles;
    const int by_tiles = want > (c->max_b + TILE_ROWS - 1) / TILE_ROWS ? want : (c->max_b + TILE_ROWS - 1) / TILE_ROWS;
    const int parts_most = d <= 16384 && by_tiles < c->num_cu ? c->num_cu : by_tiles;
    const size_t held = (size_t)(parts_most < c->max_b ? parts_most : c->max_b) * 2 * d;
    if (!s.registers || (sums && s.parts > 1))
        USL_TRY(usl_reserve(c, (void**)&c->norm_part, &c->norm_part_cap, (held + 2 * ((size_t)c->max_b + 2 * c->num_cu)) * 4));
    const bool direct = s.parts == 1;
    float* to_gamma = !sums ? nullptr : direct ? grad_gamma : c->norm_part;
    float* to_beta = !sums ? nullptr : direct ? grad_beta : c->norm_part + d;
    if (s.registers) {
#define USL_NORM_GRAD(LANES, EPL) do { if (gamma) USL_NORM_GRAD_W(LANES, EPL, true); else USL_NORM_GRAD_W(LANES, EPL, false); } while (0)
#define USL_NORM_GRAD_W(LANES, EPL, WEIGHT)                                                                                                                      \
    do {                                                                                                                                               \
        constexpr size_t lds = (size_t)(LANES >= 256 ? BWD_NT - LANES : BWD_NT) * 2 * (EPL + 1) * 4;                                                                      \
        if (lds >= 65536)                                                                                                                              \
            USL_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void*>(k_norm_grad<TS, LANES, EPL, WEIGHT>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)); \
        hipLaunchKernelGGL((k_norm_grad<TS, LANES, EPL, WEIGHT>), dim3((unsigned)s.parts), dim3(BWD_NT), lds, c->stream, grad_x, (const TS*)h, gamma, mean,     \
                           rstd, grad_h, to_gamma, to_beta, (size_t)2 * d, b, d);                                                                      \
    } while (0)
        if (d <= 128) USL_NORM_GRAD(16, 8);
        else if (d <= 512) USL_NORM_GRAD(64, 8);
        else if (d <= 1024) USL_NORM_GRAD(64, 16);
        else if (d <= 2048) USL_NORM_GRAD(128, 16);
        else if (d <= 4096) USL_NORM_GRAD(256, 16);
        else if (d <= 8192) USL_NORM_GRAD(512, 16);
        else USL_NORM_GRAD(1024, 16);
#undef USL_NORM_GRAD_W
#undef USL_NORM_GRAD
        USL_TRY(usl_check_launch(c, "layer_norm_backward"));
        if (!sums || direct) return USL_OK;
    } else {
        float* row_sums = c->norm_part + held;
        const int cols = ((d + s.splits - 1) / s.splits + 15) / 16 * 16;
        const dim3 grid((unsigned)s.splits, (unsigned)b);
        if (gamma) hipLaunchKernelGGL((k_norm_grad_sums<TS, true>), grid, dim3(SUMS_NT), 0, c->stream, grad_x, (const TS*)h, gamma, mean, rstd, row_sums, d, cols);
        else hipLaunchKernelGGL((k_norm_grad_sums<TS, false>), grid, dim3(SUMS_NT), 0, c->stream, grad_x, (const TS*)h, gamma, mean, rstd, row_sums, d, cols);
        hipLaunchKernelGGL(k_norm_grad_tile<TS>, dim3((unsigned)tiles, (unsigned)s.parts), dim3(TILE_NT), (size_t)s.rows * 16, c->stream, grad_x, (const TS*)h, gamma,
                           mean, rstd, row_sums, s.splits, grad_h, to_gamma, to_beta, (size_t)2 * d, b, d, s.rows);
        USL_TRY(usl_check_launch(c, "layer_norm_backward"));
        if (!sums || direct) return USL_OK;
    }
    // few sets of long sums, or many of short ones
    if (s.parts <= 32 && d >= 4)
        hipLaunchKernelGGL((k_norm_sum_parts<4, 4>), dim3((unsigned)((d + 255) / 256), 2), dim3(256), 0, c->stream, c->norm_part, s.parts, d, grad_gamma, grad_beta);
    else
        hipLaunchKernelGGL((k_norm_sum_parts<1, 16>), dim3((unsigned)((d + 63) / 64), 2), dim3(1024), 0, c->stream, c->norm_part, s.parts, d, grad_gamma, grad_beta);
    return usl_check_launch(c, "layer_norm_backward");
}

usl_status usl_launch_norm_grad(usl_ctx* c, const float* grad_x, const void* h, const float* gamma, const float* mean, const float* rstd, float* grad_h,
                                float* grad_gamma, float* grad_beta, int32_t b) {
    return c->storage == USL_F32 ? norm_grad<float>(c, grad_x, h, gamma, mean, rstd, grad_h, grad_gamma, grad_beta, b)
                                 : norm_grad<uint16_t>(c, grad_x, h, gamma, mean, rstd, grad_h, grad_gamma, grad_beta, b);
}
