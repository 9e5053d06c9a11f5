// The gated block's backward pass: from grad_x, e, the matrices and the projections that the forward pass kept,
//
//   G_gate = grad_x * up * act'(gate),  G_up = grad_x * act(gate)
//   grad_e = G_gate V_gate + G_up V_up,  grad_V_gate = G_gate^T e,  grad_V_up = G_up^T e
//
// The instances go through in chunks; for each, a first launch writes G = [G_gate | G_up] and a copy of e whose rows are padded with zeros, then two products
// (k_dense.h).  With bfloat16 storage G, a product of float32 numbers, is the exact sum of three bfloat16 ones (8 + 8 + 8 bits, cut off, not rounded), and each
// product is three on the matrix cores that share their other operand: gradients are float32 numbers, and G rounded to bfloat16 would leave them 1e-3 off, two parts 2e-6.
#include "k_dense.h"

using namespace dense;

namespace {

constexpr int PAD = 128;   // columns of G and of e's copy are padded to it
constexpr int PREP_NT = 256;

template <typename T> constexpr int PARTS = sizeof(T) == 2 ? 3 : 1;

struct Grad {
    const float* grad_x;
    const void *e, *V[2], *gate, *up;
    float *grad_e, *grad_V[2];
    char *G, *E;               // chunk: [parts][rows][2 * dp], [rows][wp]
    float* sums;               // [splits][rows][w]
    int d, w, dp, wp, b;       // b: instances of this chunk
    int rows;                  // padded instances of the chunk
    int first;                 // not 0: grad_V is overwritten, else added to
    int splits, steps_each;    // of grad_e's sums over d
};

template <typename T> __device__ __forceinline__ void split(float v, T (&part)[PARTS<T>]);
template <> __device__ __forceinline__ void split<float>(float v, float (&part)[1]) { part[0] = v; }
template <> __device__ __forceinline__ void split<bf16>(float v, bf16 (&part)[3]) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7F800000u) == 0x7F800000u) {   // an infinity or NaN has no rest
        part[0] = bf16{usl_f32_to_bf16(v)};
        part[1] = part[2] = bf16{0};
        return;
    }
    const float rest = v - __uint_as_float(u & 0xFFFF0000u);
    const uint32_t r = __float_as_uint(rest);
    const float last = rest - __uint_as_float(r & 0xFFFF0000u);
    part[0] = bf16{(uint16_t)(u >> 16)};
    part[1] = bf16{(uint16_t)(r >> 16)};
    part[2] = bf16{(uint16_t)(__float_as_uint(last) >> 16)};
}

// G and e's copy.  Grid: (columns of G / PREP_NT + columns of e / PREP_NT, rows)
template <typename T, int ACT>
__global__ void __launch_bounds__(PREP_NT)
k_gated_slopes(Grad a) {
    const int i = (int)blockIdx.y, blocks = (a.dp + PREP_NT - 1) / PREP_NT;
    if ((int)blockIdx.x >= blocks) {
        const int c = ((int)blockIdx.x - blocks) * PREP_NT + (int)threadIdx.x;
        if (c < a.wp) ((T*)a.E)[(size_t)i * a.wp + c] = i < a.b && c < a.w ? ((const T*)a.e)[(size_t)i * a.w + c] : narrow<T>(0.f);
        return;
    }
    const int c = (int)blockIdx.x * PREP_NT + (int)threadIdx.x;
    if (c >= a.dp) return;
    float by_gate = 0.f, by_up = 0.f;
    if (i < a.b && c < a.d) {
        const size_t at = (size_t)i * a.d + c;
        float value, slope;
        act_and_slope<ACT>(widen(((const T*)a.gate)[at]), value, slope);
        const float g = a.grad_x[at];
        by_gate = g * widen(((const T*)a.up)[at]) * slope;
        by_up = g * value;
    }
    T part[PARTS<T>];
    T* to = (T*)a.G + (size_t)i * 2 * a.dp + c;
    const size_t next = (size_t)a.rows * 2 * a.dp;
    split<T>(by_gate, part);
#pragma unroll
    for (int q = 0; q < PARTS<T>; ++q) to[q * next] = part[q];
    split<T>(by_up, part);
#pragma unroll
    for (int q = 0; q < PARTS<T>; ++q) to[q * next + a.dp] = part[q];
}

// grad_V: [w] along m, [2][d] along n, the instances along K.  Tiles of 128 x 128, four wavefronts.
template <typename T>
__global__ void __launch_bounds__(256)
k_gated_grad_v(Grad a) {
    constexpr int P = PARTS<T>, F = 4;
    using S = StageKO<T, 128, 4>;
    constexpr int STEP = (1 + P) * S::BYTES;
    __shared__ __align__(1024) char lds[2 * STEP];
    const int m0 = (int)blockIdx.x * 128, n0 = (int)blockIdx.y * 128, wave = (int)threadIdx.x >> 6, wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    const size_t pitch_e = (size_t)a.wp * sizeof(T), pitch_g = (size_t)2 * a.dp * sizeof(T), next = a.rows * pitch_g;
    const char *E = a.E + (size_t)m0 * sizeof(T), *G = a.G + (size_t)n0 * sizeof(T);
    f32x4 acc[F][F];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int h = 0; h < F; ++h) acc[f][h] = f32x4{0, 0, 0, 0};
    const int steps = a.rows / S::DEPTH;
    auto ask = [&](int s) {
        const uint32_t to = lds_at(lds + (s & 1) * STEP);
        S::direct(to, E + (size_t)s * S::DEPTH * pitch_e, S::DEPTH, pitch_e, S::ROW);
#pragma unroll
        for (int q = 0; q < P; ++q) S::direct(to + (1 + q) * S::BYTES, G + q * next + (size_t)s * S::DEPTH * pitch_g, S::DEPTH, pitch_g, S::ROW);
    };
    ask(0);
    for (int s = 0; s < steps; ++s) {
        landed();
        __syncthreads();
        if (s + 1 < steps) ask(s + 1);
        const char* from = lds + (s & 1) * STEP;
        i32x4 x[F];
#pragma unroll
        for (int f = 0; f < F; ++f) x[f] = S::frag(from, wm + f * 16);
#pragma unroll
        for (int q = P - 1; q >= 0; --q)   // the small parts first
#pragma unroll
            for (int h = 0; h < F; ++h) {
                const i32x4 y = S::frag(from + (1 + q) * S::BYTES, wn + h * 16);
#pragma unroll
                for (int f = 0; f < F; ++f) acc[f][h] = Core<T>::mul(x[f], y, acc[f][h]);
            }
    }
    const int l = (int)threadIdx.x & 63;
    const bool aligned = a.w % 4 == 0 && ((uintptr_t)a.grad_V[0] | (uintptr_t)a.grad_V[1]) % 16 == 0;
#pragma unroll
    for (int h = 0; h < F; ++h) {
        const int n = n0 + wn + h * 16 + (l & 15), which = n >= a.dp, row = n - which * a.dp;
        float* to = a.grad_V[which];
        if (row >= a.d || !to) continue;
        to += (size_t)row * a.w;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int m = m0 + wm + f * 16 + (l >> 4) * 4;
            f32x4 v = acc[f][h];
            if (aligned && m + 3 < a.w) {
                f32x4* p = reinterpret_cast<f32x4*>(to + m);
                if (!a.first) v += *p;
                *p = v;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (m + j < a.w) to[m + j] = a.first ? v[j] : to[m + j] + v[j];
            }
        }
    }
}

// Sums of grad_e over a piece of [2][d]: [w] along m, the instances along n.  DIRECT: V's rows and bases are multiples of 16 bytes.
template <typename T, bool DIRECT>
__global__ void __launch_bounds__(256)
k_gated_grad_e(Grad a) {
    constexpr int P = PARTS<T>, F = 4;
    using SV = StageKO<T, 128, 4>;
    using SG = StageKC<128, 64, 1, 4>;
    constexpr int STEP = SV::BYTES + P * SG::BYTES;
    __shared__ __align__(1024) char lds[2 * STEP];
    const int m0 = (int)blockIdx.x * 128, n0 = (int)blockIdx.y * 128, wave = (int)threadIdx.x >> 6, wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
    const size_t pitch_v = (size_t)a.w * sizeof(T), pitch_g = (size_t)2 * a.dp * sizeof(T), next = a.rows * pitch_g;
    const int rows = a.rows - n0;   // (of the tile's 128; those behind the last instance hold zeros)
    f32x4 acc[F][F];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int h = 0; h < F; ++h) acc[f][h] = f32x4{0, 0, 0, 0};
    const int first = (int)blockIdx.z * a.steps_each, last = min(first + a.steps_each, 2 * a.dp / SV::DEPTH);
    i32x4 held[SV::LOADS];
    auto ask = [&](int s) {
        char* to = lds + (s & 1) * STEP;
        const int k = s * SV::DEPTH, which = k >= a.dp, row = k - which * a.dp;   // rows behind V's end meet zeros of G, and are not read
        const char* V = (const char*)a.V[which] + (size_t)min(row, a.d - 1) * pitch_v + (size_t)m0 * sizeof(T);
        if constexpr (DIRECT) SV::direct(lds_at(to), V, a.d - row, pitch_v, (a.w - m0) * (int)sizeof(T));
        else SV::fetch(held, V, a.d - row, pitch_v, (a.w - m0) * (int)sizeof(T));
#pragma unroll
        for (int q = 0; q < P; ++q)
            SG::direct(lds_at(to + SV::BYTES + q * SG::BYTES), a.G + q * next + (size_t)n0 * pitch_g + (size_t)k * sizeof(T), rows, (uint32_t)pitch_g, 64);
    };
    auto place = [&](int s) {
        if constexpr (!DIRECT) SV::put(lds + (s & 1) * STEP, held);
    };
    if (first < last) {
        ask(first);
        place(first);
    }
    for (int s = first; s < last; ++s) {
        landed();
        __syncthreads();
        if (s + 1 < last) ask(s + 1);
        const char* from = lds + (s & 1) * STEP;
        i32x4 x[F];
#pragma unroll
        for (int f = 0; f < F; ++f) x[f] = SV::frag(from, wm + f * 16);
#pragma unroll
        for (int q = P - 1; q >= 0; --q)
#pragma unroll
            for (int h = 0; h < F; ++h) {
                const i32x4 y = SG::frag(from + SV::BYTES + q * SG::BYTES, wn, h, 0);
#pragma unroll
                for (int f = 0; f < F; ++f) acc[f][h] = Core<T>::mul(x[f], y, acc[f][h]);
            }
        if (s + 1 < last) place(s + 1);
    }
    const int l = (int)threadIdx.x & 63;
    float* sums = a.sums + (size_t)blockIdx.z * a.b * a.w;
#pragma unroll
    for (int h = 0; h < F; ++h) {
        const int i = n0 + wn + h * 16 + (l & 15);
        if (i >= a.b) continue;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int m = m0 + wm + f * 16 + (l >> 4) * 4;
            float* to = sums + (size_t)i * a.w + m;
            if (a.w % 4 == 0 && m + 3 < a.w) *reinterpret_cast<f32x4*>(to) = acc[f][h];
            else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (m + j < a.w) to[j] = acc[f][h][j];
            }
        }
    }
}

// grad_e: the pieces' sums, in a fixed order
__global__ void __launch_bounds__(256)
k_gated_join(const float* __restrict__ sums, float* __restrict__ grad_e, size_t n, int splits) {
    for (size_t v = (size_t)blockIdx.x * 256 + threadIdx.x; v < n; v += (size_t)gridDim.x * 256) {
        float s = sums[v];
        for (int q = 1; q < splits; ++q) s += sums[(size_t)q * n + v];
        grad_e[v] = s;
    }
}

constexpr size_t SCRATCH = (size_t)1 << 30;   // what the chunk of instances is cut to, if 256 of them take less

template <typename T>
usl_status run(usl_ctx* c, Grad a, int32_t act, int32_t b) {
    constexpr int ES = (int)sizeof(T), DEPTH = 64 / ES;
    const char* what = "gated_block_backward";
    a.dp = (a.d + PAD - 1) / PAD * PAD;
    a.wp = (a.w + PAD - 1) / PAD * PAD;
    const size_t row = ((size_t)PARTS<T> * 2 * a.dp + a.wp) * ES;
    auto padded = [](size_t n) { return (n + 31) / 32 * 32; };   // a step of K, and more than a wavefront's rows
    size_t most = padded((size_t)c->max_b);
    if (most * row > SCRATCH) most = padded(SCRATCH / row < 256 ? 256 : SCRATCH / row);
    if (most > padded((size_t)c->max_b)) most = padded((size_t)c->max_b);
    if (most > 32768) most = 32768;   // a row is a grid dimension
    const int tiles_w = a.wp / 128, k_steps = 2 * a.dp / DEPTH;
    auto splits_of = [&](int rows) {   // two workgroups to a compute unit; at least eight steps each
        const int tiles = tiles_w * ((rows + 127) / 128), want = (2 * c->num_cu + tiles - 1) / tiles, room = (k_steps + 7) / 8;
        return want < room ? want : room;
    };
    size_t sums_most = 0;
    for (size_t r = 32; r <= most; r += 32) {   // (not always the largest batch's)
        const size_t s = (size_t)splits_of((int)r) * r * a.w;
        if (s > sums_most) sums_most = s;
    }
    USL_TRY(usl_reserve(c, (void**)&c->gated_scratch, &c->gated_scratch_cap, most * row + sums_most * 4));
    a.G = c->gated_scratch;
    const char *e = (const char*)a.e, *gate = (const char*)a.gate, *up = (const char*)a.up;
    const float* grad_x = a.grad_x;
    float* grad_e = a.grad_e;
    for (int32_t i0 = 0; i0 < b; i0 += (int32_t)most) {
        a.b = (int)(b - i0 < (int32_t)most ? b - i0 : (int32_t)most);
        a.rows = (int)padded((size_t)a.b);
        a.first = i0 == 0;
        a.E = a.G + (size_t)a.rows * PARTS<T> * 2 * a.dp * ES;
        a.sums = (float*)(a.G + (size_t)a.rows * row);
        a.e = e + (size_t)i0 * a.w * ES;
        a.gate = gate + (size_t)i0 * a.d * ES;
        a.up = up + (size_t)i0 * a.d * ES;
        a.grad_x = grad_x + (size_t)i0 * a.d;
        const dim3 slopes((unsigned)((a.dp + PREP_NT - 1) / PREP_NT + (a.wp + PREP_NT - 1) / PREP_NT), (unsigned)a.rows);
        if (act == USL_SILU) hipLaunchKernelGGL((k_gated_slopes<T, 0>), slopes, dim3(PREP_NT), 0, c->stream, a);
        else hipLaunchKernelGGL((k_gated_slopes<T, 1>), slopes, dim3(PREP_NT), 0, c->stream, a);
        USL_TRY(usl_check_launch(c, what));
        if (a.grad_V[0] || a.grad_V[1]) {
            hipLaunchKernelGGL(k_gated_grad_v<T>, dim3((unsigned)tiles_w, (unsigned)(2 * a.dp / 128)), dim3(256), 0, c->stream, a);
            USL_TRY(usl_check_launch(c, what));
        }
        if (!grad_e) continue;
        a.splits = splits_of(a.rows);
        a.steps_each = (k_steps + a.splits - 1) / a.splits;
        a.splits = (k_steps + a.steps_each - 1) / a.steps_each;
        const dim3 grid((unsigned)tiles_w, (unsigned)((a.rows + 127) / 128), (unsigned)a.splits);
        const bool direct = (a.w * ES | (uintptr_t)a.V[0] | (uintptr_t)a.V[1]) % 16 == 0;
        if (direct) hipLaunchKernelGGL((k_gated_grad_e<T, true>), grid, dim3(256), 0, c->stream, a);
        else hipLaunchKernelGGL((k_gated_grad_e<T, false>), grid, dim3(256), 0, c->stream, a);
        USL_TRY(usl_check_launch(c, what));
        const size_t n = (size_t)a.b * a.w;
        const unsigned blocks = (unsigned)((n + 255) / 256 < 4096 ? (n + 255) / 256 : 4096);
        hipLaunchKernelGGL(k_gated_join, dim3(blocks), dim3(256), 0, c->stream, a.sums, grad_e + (size_t)i0 * a.w, n, a.splits);
        USL_TRY(usl_check_launch(c, what));
    }
    return USL_OK;
}

}  // namespace

usl_status usl_launch_gated_backward(usl_ctx* c, const float* grad_x, const void* e, const void* V_gate, const void* V_up, const void* gate, const void* up, int32_t w,
                                     int32_t act, float* grad_e, float* grad_V_gate, float* grad_V_up, int32_t b) {
    Grad a = {};
    a.grad_x = grad_x; a.e = e; a.V[0] = V_gate; a.V[1] = V_up; a.gate = gate; a.up = up;
    a.grad_e = grad_e; a.grad_V[0] = grad_V_gate; a.grad_V[1] = grad_V_up;
    a.d = c->d; a.w = w;
    return c->storage == USL_F32 ? run<float>(c, a, act, b) : run<bf16>(c, a, act, b);
}
