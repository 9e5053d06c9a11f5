// The gated block's backward pass: from grad_x, e, the matrices and the projections that the forward pass kept,
//
//   G_gate = grad_x * up * act'(gate),  G_up = grad_x * act(gate)
//   grad_e = G_gate V_gate + G_up V_up,  grad_V_gate = G_gate^T e,  grad_V_up = G_up^T e
//
// The instances go through in chunks; for each, a first launch writes G = [G_gate | G_up] and a copy of e whose rows are padded with zeros, then two products
// (k_dense.h).  G lies in blocks of 128 columns, the instances one behind the other: with whole rows, a power of two apart, a tile's 32 or 128 rows met in
// one channel of the caches.  With bfloat16 storage G, a product of float32 numbers, is the exact sum of three bfloat16 ones (8 + 8 + 8 bits, cut off, not rounded), and each
// product is three on the matrix cores that share their other operand: gradients are float32 numbers, and G rounded to bfloat16 would leave them 1e-3 off, two parts 2e-6.
#include "k_dense.h"

using namespace dense;

namespace {

constexpr int PREP_NT = 256;

template <typename T> constexpr int PARTS = sizeof(T) == 2 ? 3 : 1;

struct Grad {
    const float* grad_x;
    const void *e, *V[2], *gate, *up;
    float *grad_e, *grad_V[2];
    char *G, *E;               // chunk: [parts][2 * dp / 128][rows][128], [rows][wp]
    float* sums;               // [splits][rows][w]
    int d, w, dp, wp, b;       // b: instances of this chunk
    int rows;                  // padded instances of the chunk
    int first;                 // not 0: grad_V is overwritten, else added to
    int tiles_m, tiles_n;      // of a product
    int splits, steps_each;    // of grad_e's sums over d
};

// Eight neighbours from any address as float32
typedef uint32_t AnyWords __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void load_eight(const float* p, float (&v)[8]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const AnyWords q = reinterpret_cast<const AnyWords*>(p)[u];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[u * 4 + j] = __uint_as_float(q[j]);
    }
}
__device__ __forceinline__ void load_eight(const bf16* p, float (&v)[8]) {
    const AnyWords q = *reinterpret_cast<const AnyWords*>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(j & 1 ? q[j / 2] & 0xFFFF0000u : q[j / 2] << 16);
}
// v as the sum of PARTS<T> numbers, each eight to its place: to, to + next, ...
__device__ __forceinline__ void store_parts(float* to, size_t, const float (&v)[8]) {
    reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store_parts(bf16* to, size_t next, const float (&v)[8]) {
    uint32_t rest[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) rest[j] = __float_as_uint(v[j]);
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        uint32_t cut[8];   // the upper half of a word
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cut[j] = rest[j] & 0xFFFF0000u;
            const bool odd = (rest[j] & 0x7F800000u) == 0x7F800000u;   // an infinity or NaN has no rest, and a NaN stays one
            const uint32_t left = __float_as_uint(__uint_as_float(rest[j]) - __uint_as_float(cut[j]));
            if (q == 0) cut[j] |= odd && (rest[j] & 0x7FFFFFu) ? 0x400000u : 0u;
            rest[j] = odd ? 0u : left;
        }
        uint4 w;
        w.x = cut[0] >> 16 | cut[1]; w.y = cut[2] >> 16 | cut[3]; w.z = cut[4] >> 16 | cut[5]; w.w = cut[6] >> 16 | cut[7];
        *reinterpret_cast<uint4*>(to + q * next) = w;
    }
}

// G and e's copy, eight columns a lane.  Grid: (groups of 8 columns of G and of e / PREP_NT, rows).  Bound by its bytes.
template <typename T, int ACT>
__global__ void __launch_bounds__(PREP_NT)
k_gated_slopes(Grad a) {
    const int i = (int)blockIdx.y, groups = a.dp / 8;
    int c = ((int)blockIdx.x * PREP_NT + (int)threadIdx.x);
    if (c >= groups) {
        c = (c - groups) * 8;
        if (c >= a.wp) return;
        const T* e = (const T*)a.e + (size_t)i * a.w + c;
        T* to = (T*)a.E + (size_t)i * a.wp + c;
        if (i < a.b && c + 8 <= a.w) {
#pragma unroll
            for (int u = 0; u < (int)sizeof(T) / 2; ++u) reinterpret_cast<uint4*>(to)[u] = __builtin_bit_cast(uint4, reinterpret_cast<const AnyWords*>(e)[u]);
        } else {
            for (int j = 0; j < 8; ++j) to[j] = i < a.b && c + j < a.w ? e[j] : narrow<T>(0.f);
        }
        return;
    }
    c *= 8;
    float gate[8], up[8], g[8];
    const size_t at = (size_t)i * a.d + c;
    if (i < a.b && c + 8 <= a.d) {
        load_eight((const T*)a.gate + at, gate);
        load_eight((const T*)a.up + at, up);
        load_eight(a.grad_x + at, g);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool is = i < a.b && c + j < a.d;
            gate[j] = is ? widen(((const T*)a.gate)[at + j]) : 0.f;
            up[j] = is ? widen(((const T*)a.up)[at + j]) : 0.f;
            g[j] = is ? a.grad_x[at + j] : 0.f;
        }
    }
    float by_up[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float value, slope;
        act_and_slope<ACT>(gate[j], value, slope);
        gate[j] = g[j] * up[j] * slope;
        by_up[j] = g[j] * value;
    }
    T* to = (T*)a.G + ((size_t)(c >> 7) * a.rows + i) * 128 + (c & 127);
    const size_t next = (size_t)a.rows * 2 * a.dp;
    store_parts(to, next, gate);
    store_parts(to + (size_t)a.dp * a.rows, next, by_up);
}

// One of `inner` tiles of one of `outer` pieces.  Workgroups go to the chiplets in turn; each of those takes a run of tiles, so that those of a piece, which share
// what they read, meet in its cache.  false: one too many
__device__ __forceinline__ bool tile_of(int inner, int outer, int& in, int& out) {
    const int each = (inner * outer + 7) / 8, at = ((int)blockIdx.x & 7) * each + ((int)blockIdx.x >> 3);
    in = at % inner;
    out = at / inner;
    return out < outer;
}
unsigned tiles_grid(int inner, int outer) { return (unsigned)((inner * outer + 7) / 8 * 8); }

// grad_V: [w] along m, [2][d] along n, the instances along K.  Tiles of MT x NT, a wavefront F x F fragments of it.  The parts of G meet the same fragments of e, so
// what has to come from the caches for a product on the matrix cores falls with MT.
template <typename T, int MT, int NT, int F, int STAGES>
__global__ void __launch_bounds__(MT * NT / (4 * F * F), 2)
k_gated_grad_v(Grad a) {
    constexpr int P = PARTS<T>, WM = F * 16, WAVES = MT / WM * (NT / WM);
    using SE = StageKO<T, MT, WAVES>;
    using SG = StageKO<T, NT, WAVES>;
    constexpr int STEP = SE::BYTES + P * SG::BYTES, LOADS = SE::LOADS + P * SG::LOADS;
    extern __shared__ __align__(1024) char lds[];
    int tm, tn;
    if (!tile_of(a.tiles_m, 2 * a.dp / NT, tm, tn)) return;
    const int m0 = tm * MT, n0 = tn * NT, wave = (int)threadIdx.x >> 6, wm = wave / (NT / WM) * WM, wn = wave % (NT / WM) * WM;
    const size_t pitch_e = (size_t)a.wp * sizeof(T), pitch_g = 128 * sizeof(T), next_part = (size_t)a.rows * 2 * a.dp * sizeof(T);
    const char *E = a.E + (size_t)m0 * sizeof(T), *G = a.G + (size_t)(n0 >> 7) * a.rows * pitch_g + (size_t)(n0 & 127) * sizeof(T);
    f32x4 acc[F][F];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int h = 0; h < F; ++h) acc[f][h] = f32x4{0, 0, 0, 0};
    const int steps = a.rows / SE::DEPTH;
    int lane_e[F], lane_g[F];
#pragma unroll
    for (int f = 0; f < F; ++f) {
        lane_e[f] = SE::lane(wm + f * 16);
        lane_g[f] = SG::lane(wn + f * 16);
    }
    auto place = [&](int s) { return lds + s % STAGES * STEP; };
    constexpr int GROUPS = P > 1 ? P : 2, Y = P * F / GROUPS;   // a part, or half of the only one; the small parts first
    walk<F, GROUPS, Y, STAGES>(
        steps, [&](int s) { arrived<STAGES, LOADS>(s, steps); },
        [&](int s) {
            if (s >= steps) return;
            const uint32_t to = lds_at(place(s));
            SE::direct(to, E + (size_t)s * SE::DEPTH * pitch_e, SE::DEPTH, pitch_e, SE::ROW);
#pragma unroll
            for (int q = 0; q < P; ++q) SG::direct(to + SE::BYTES + q * SG::BYTES, G + q * next_part + (size_t)s * SE::DEPTH * pitch_g, SE::DEPTH, pitch_g, SG::ROW);
        },
        [&](int s, i32x4 (&x)[F]) {
#pragma unroll
            for (int f = 0; f < F; ++f) x[f] = SE::frag(place(s), lane_e[f]);
        },
        [&](int s, int g, i32x4 (&y)[Y]) {
#pragma unroll
            for (int h = 0; h < Y; ++h) y[h] = SG::frag(place(s) + SE::BYTES + (P - 1 - (g * Y + h) / F) * SG::BYTES, lane_g[(g * Y + h) % F]);
        },
        [&](int g, const i32x4 (&x)[F], const i32x4 (&y)[Y]) {
#pragma unroll
            for (int h = 0; h < Y; ++h)
#pragma unroll
                for (int f = 0; f < F; ++f) acc[f][(g * Y + h) % F] = Core<T>::mul(x[f], y[h], acc[f][(g * Y + h) % F]);
        });
    const int l = (int)threadIdx.x & 63;
#pragma unroll
    for (int h = 0; h < F; ++h) {
        const int n = n0 + wn + h * 16 + (l & 15), which = n >= a.dp, row = n - which * a.dp;
        float* to = a.grad_V[which];
        if (row >= a.d || !to) continue;
        to += (size_t)row * a.w;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int m = m0 + wm + f * 16 + (l >> 4) * 4;
            if (m >= a.w) continue;
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = a.first ? acc[f][h][j] : acc[f][h][j] + to[min(m + j, a.w - 1)];
            put_many(to + m, v, a.w - m);
        }
    }
}

// Sums of grad_e over a piece of [2][d]: [w] along m, the instances along n.  Tiles of MT x NT, a wavefront 64 x 16 * FN of it.  V comes straight into
// LDS, with rows and bases that are multiples of 4 bytes all but the steps at its end (20 x 2014 -> 36853 float32 376 us, so 344); else through registers, asked for two steps ahead and put into LDS one step ahead.
template <typename T, int MT, int NT, int FN, int STAGES, int HOW>
__global__ void __launch_bounds__(MT * NT / (16 * FN), 2)
k_gated_grad_e(Grad a) {
    constexpr int P = PARTS<T>, F = 4, WAVES = MT / 64 * (NT / (FN * 16));
    using SV = StageKO<T, MT, WAVES>;
    using SG = StageKC<NT, 64, 1, WAVES>;
    constexpr int STEP = SV::BYTES + P * SG::BYTES, LOADS = (HOW != REGISTERS ? SV::LOADS : 0) + P * SG::LOADS;
    static_assert(HOW != REGISTERS || STAGES == 3, "two steps ahead");
    extern __shared__ __align__(1024) char lds[];
    int tile, piece;
    if (!tile_of(a.tiles_m * a.tiles_n, a.splits, tile, piece)) return;
    const int m0 = tile % a.tiles_m * MT, n0 = tile / a.tiles_m * NT, wave = (int)threadIdx.x >> 6, wm = wave % (MT / 64) * 64, wn = wave / (MT / 64) * (FN * 16);
    const size_t pitch_v = (size_t)a.w * sizeof(T), pitch_g = 128 * sizeof(T), next_part = (size_t)a.rows * 2 * a.dp * sizeof(T);
    const int rows = a.rows - n0;   // (those behind the last instance hold zeros)
    f32x4 acc[F][FN];
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int h = 0; h < FN; ++h) acc[f][h] = f32x4{0, 0, 0, 0};
    const int first = piece * a.steps_each, steps = min(a.steps_each, 2 * a.dp / SV::DEPTH - first);
    int lane_v[F];
#pragma unroll
    for (int f = 0; f < F; ++f) lane_v[f] = SV::lane(wm + f * 16);
    const int lane_g = SG::lane(wn);
    auto place = [&](int s) { return lds + s % STAGES * STEP; };
    auto ask_g = [&](int s) {
        if (s >= steps) return;
        const int k = (first + s) * SV::DEPTH;
#pragma unroll
        for (int q = 0; q < P; ++q)
            SG::direct(lds_at(place(s) + SV::BYTES + q * SG::BYTES), a.G + q * next_part + ((size_t)(k >> 7) * a.rows + n0) * pitch_g + (size_t)(k & 127) * sizeof(T), rows,
                       (uint32_t)pitch_g, 64);
    };
    struct Held { i32x4 v[SV::LOADS]; };
    auto ask_v = [&](int s, Held* h) {
        if (s >= steps) return;
        const int k = (first + s) * SV::DEPTH, which = k >= a.dp, row = k - which * a.dp;   // rows behind V's end meet zeros of G, and are not read
        const char* V = (const char*)a.V[which] + (size_t)min(row, a.d - 1) * pitch_v + (size_t)m0 * sizeof(T);
        if (HOW == WORDS && a.d - row <= SV::DEPTH) {
            Held last;
            landed<0>();   // (arrived() counts on as many loads of every step behind its own: here they are fewer, and what lies before is there)
            SV::fetch(last.v, V, a.d - row, pitch_v, (a.w - m0) * (int)sizeof(T), m0 * (int)sizeof(T));
            SV::put(place(s), last.v);
        } else if (HOW != REGISTERS) SV::direct(lds_at(place(s)), V, a.d - row, pitch_v, (a.w - m0) * (int)sizeof(T));
        else SV::fetch(h->v, V, a.d - row, pitch_v, (a.w - m0) * (int)sizeof(T), m0 * (int)sizeof(T));
    };
    constexpr int GROUPS = P > 1 ? P : 2, Y = P * FN / GROUPS;
    auto first_of = [&](int s, i32x4 (&x)[F]) {
#pragma unroll
        for (int f = 0; f < F; ++f) x[f] = SV::frag(place(s), lane_v[f]);
    };
    auto group_of = [&](int s, int g, i32x4 (&y)[Y]) {
#pragma unroll
        for (int h = 0; h < Y; ++h) y[h] = SG::frag(place(s) + SV::BYTES + (P - 1 - (g * Y + h) / FN) * SG::BYTES, lane_g, (g * Y + h) % FN);
    };
    auto multiply = [&](int g, const i32x4 (&x)[F], const i32x4 (&y)[Y]) {
#pragma unroll
        for (int h = 0; h < Y; ++h)
#pragma unroll
            for (int f = 0; f < F; ++f) acc[f][(g * Y + h) % FN] = Core<T>::mul(x[f], y[h], acc[f][(g * Y + h) % FN]);
    };
    if constexpr (HOW != REGISTERS) {
        walk<F, GROUPS, Y, STAGES>(
            steps, [&](int s) { arrived<STAGES, LOADS>(s, steps); },
            [&](int s) {
                ask_v(s, nullptr);
                ask_g(s);
            },
            first_of, group_of, multiply);
    } else {
        Held one, two;
        auto turn = [&](int s, Held& after, Held& behind) {   // after: V of step s + 1; behind: to hold that of step s + 2
            if (s + 2 <= steps) landed<LOADS>();   // (G of step s + 1 may be on its way; loads into registers behind it only make the wait longer)
            else landed<0>();
            __syncthreads();
            ask_g(s + 2);
            ask_v(s + 2, &behind);
            i32x4 x[F], y[Y];
            first_of(s, x);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                group_of(s, g, y);
                multiply(g, x, y);
            }
            if (s + 1 < steps) SV::put(place(s + 1), after.v);
        };
        ask_g(0);
        ask_g(1);
        ask_v(0, &two);
        ask_v(1, &one);
        SV::put(lds, two.v);
        for (int s = 0; s < steps; s += 2) {
            turn(s, one, two);
            if (s + 1 < steps) turn(s + 1, two, one);
        }
    }
    const int l = (int)threadIdx.x & 63;
    float* sums = a.sums + (size_t)piece * a.b * a.w;
#pragma unroll
    for (int h = 0; h < FN; ++h) {
        const int i = n0 + wn + h * 16 + (l & 15);
        if (i >= a.b) continue;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int m = m0 + wm + f * 16 + (l >> 4) * 4;
            if (m >= a.w) continue;
            const float v[4] = {acc[f][h][0], acc[f][h][1], acc[f][h][2], acc[f][h][3]};
            put_many(sums + (size_t)i * a.w + m, v, a.w - m);
        }
    }
}

// grad_e: the pieces' sums, in a fixed order: each of four wavefronts every fourth piece, then theirs
__global__ void __launch_bounds__(256)
k_gated_join(const float* __restrict__ sums, float* __restrict__ grad_e, size_t n, int splits) {
    __shared__ float part[4][64];
    const int l = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const size_t v = (size_t)blockIdx.x * 64 + l, at = v < n ? v : n - 1;
    float s = 0.f;
#pragma unroll 8
    for (int q = wave; q < splits; q += 4) s += sums[(size_t)q * n + at];
    part[wave][l] = s;
    __syncthreads();
    if (wave == 0 && v < n) grad_e[v] = part[0][l] + part[1][l] + part[2][l] + part[3][l];
}

constexpr size_t SCRATCH = (size_t)1 << 30, CHUNK = 256;   // bytes that a chunk of instances is cut to, if CHUNK of them take less

template <typename F>
usl_status lds_for(usl_ctx* c, F* kernel, int bytes) {
    if (bytes > 64 * 1024) USL_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return USL_OK;
}

template <typename T, int MT, int NT, int F, int STAGES>
usl_status grad_v(usl_ctx* c, Grad a) {
    constexpr int BYTES = STAGES * (MT + PARTS<T> * NT) * 64;
    USL_TRY(lds_for(c, k_gated_grad_v<T, MT, NT, F, STAGES>, BYTES));
    a.tiles_m = (a.w + MT - 1) / MT;
    hipLaunchKernelGGL((k_gated_grad_v<T, MT, NT, F, STAGES>), dim3(tiles_grid(a.tiles_m, 2 * a.dp / NT)), dim3(MT * NT / (4 * F * F)), BYTES, c->stream, a);
    return usl_check_launch(c, "gated_block_backward");
}

template <typename T, int MT, int NT, int FN, int STAGES, int HOW>
usl_status grad_e_tiles(usl_ctx* c, const Grad& a) {
    constexpr int BYTES = STAGES * (MT + PARTS<T> * NT) * 64;
    USL_TRY(lds_for(c, k_gated_grad_e<T, MT, NT, FN, STAGES, HOW>, BYTES));
    hipLaunchKernelGGL((k_gated_grad_e<T, MT, NT, FN, STAGES, HOW>), dim3(tiles_grid(a.tiles_m * a.tiles_n, a.splits)), dim3(MT * NT / (16 * FN)), BYTES, c->stream, a);
    return usl_check_launch(c, "gated_block_backward");
}

template <typename T, int MT, int NT, int FN>
usl_status grad_e(usl_ctx* c, const Grad& a, int how) {
    if (how == DIRECT) return grad_e_tiles<T, MT, NT, FN, 4, DIRECT>(c, a);
    if constexpr (sizeof(T) == 2 || MT == 128)   // (rows of float32 are rows of words, but for those below 16 bytes)
        if (how == REGISTERS) return grad_e_tiles<T, MT, NT, FN, 3, REGISTERS>(c, a);
    return grad_e_tiles<T, MT, NT, FN, 4, WORDS>(c, a);
}

// Tiles of grad_e.  Instances 32 or 64 at a time where there are no more, and 64 where V comes straight into LDS and they leave out an eighth of what 128 at a time
// would multiply; 256 columns of w where every compute unit then has at least 16 steps to go, else 128, which share the work among twice the workgroups and leave
// half the sums.  (Backward of 300 x 200 -> 1000 float32, 25 us, 7 more with 256 columns; of 1 x 130 -> 45688 float32 with 32 instances at a time 117 us, with 64 at a time 127;
// with 64 and 128 at a time: 155 x 256 -> 55424 float32 221 and 244, bfloat16 140 and 145, 300 x 384 -> 16384 float32 193 and 204, 512 x 768 -> 16384 482 and 457,
// 150 x 301 -> 30001 bfloat16, V through registers, 171 and 129.)
struct Tiles { int m, n; };
Tiles tiles_of(const usl_ctx* c, int w, int rows, int k_steps, bool direct) {
    const int by_64 = (rows + 63) / 64, by_128 = (rows + 127) / 128;
    const int n = rows <= 32 ? 32 : rows <= 64 || (direct && by_64 * 8 <= by_128 * 14) ? 64 : 128;
    const bool wide = w > 128 && (int64_t)((w + 255) / 256) * ((rows + n - 1) / n) * (k_steps / 16) >= c->num_cu;
    return wide ? Tiles{256, n} : Tiles{128, 128};
}

// Tiles of grad_V, 64 x 64 or 256 x 128 of the values of grad_V.  The tall ones take half of what the small ones do from the caches for a product on the matrix
// cores.  With float32 storage, whose products take four instructions each, that is never the bound and the small tiles share the work better.  With bfloat16 a compute unit does a
// value of a small tile at 0.55 of the rate, and the choice is by what falls to the unit that has the most.  (Whole backward passes, small tiles and tall ones:
// float32 512 x 768 -> 8192 242 and 278 us, 64 x 256 -> 131072 226 and 244, 300 x 200 -> 1000 25 and 60; bfloat16 512 x 768 -> 32768 440 and 373,
// 512 x 1024 -> 4096 88 and 81, 680 x 256 -> 17920 156 and 157, 256 x 512 -> 4096 35 and 38, 779 x 1302 -> 357 39 and 59.)
template <typename T>
bool tall_v(const usl_ctx* c, int w, int dp) {
    if (sizeof(T) == 4 || w <= 128) return false;
    auto most = [&](int m, int n) { return ((int64_t)((w + m - 1) / m) * (2 * dp / n) + c->num_cu - 1) / c->num_cu * m * n; };
    return most(256, 128) * 0.55 <= most(64, 64);
}

template <typename T>
usl_status run(usl_ctx* c, Grad a, int32_t act, int32_t b) {
    constexpr int ES = (int)sizeof(T), DEPTH = 64 / ES;
    const char* what = "gated_block_backward";
    a.dp = (a.d + 127) / 128 * 128;
    a.wp = a.w <= 128 ? 128 : (a.w + 255) / 256 * 256;
    // What an instance of a chunk takes: its rows of G and of e's copy; with grad_e's sums, if they are one piece
    auto taken = [&](int w, int wp) { return ((size_t)PARTS<T> * 2 * a.dp + wp) * ES + (size_t)w * 4; };
    auto padded = [](size_t n) { return (n + 31) / 32 * 32; };   // a step of K, and more than a wavefront's rows
    const size_t row = taken(0, a.wp), each = taken(a.w, a.wp), all = padded((size_t)(c->max_b < 32768 ? c->max_b : 32768));   // a row is a grid dimension
    auto smaller = [](size_t p, size_t q) { return p < q ? p : q; };
    auto larger = [](size_t p, size_t q) { return p > q ? p : q; };
    const size_t most = smaller(all, larger(SCRATCH / each / 32 * 32, CHUNK));
    // Several pieces of grad_e's sums: no more tiles than compute units, of 128 x 256 at most
    const size_t pieces = (size_t)c->num_cu * 128 * 256 * 4;
    // Never less for a larger w, though the chunk is shorter: only a w larger than any before makes a call allocate
    auto need = [&](size_t of) { return pieces + smaller(all * of, larger(SCRATCH, CHUNK * of)); };
    const int k_steps = 2 * a.dp / DEPTH;
    const uintptr_t rows_at = a.w * ES | (uintptr_t)a.V[0] | (uintptr_t)a.V[1];
    const int how = rows_at % 16 == 0 ? DIRECT : rows_at % 4 == 0 && a.w * ES >= 16 ? WORDS : REGISTERS;   // (16 bytes from a row on end in the next one at the latest)
    auto cut = [&](Grad& g, int rows) {   // a workgroup to a compute unit; at least four steps each
        const Tiles t = tiles_of(c, g.w, rows, k_steps, how != REGISTERS);
        g.tiles_m = (g.w + t.m - 1) / t.m;
        g.tiles_n = (rows + t.n - 1) / t.n;
        const int tiles = g.tiles_m * g.tiles_n, want = c->num_cu / tiles, room = (k_steps + 3) / 4;   // (one more than there is room for takes another round)
        g.splits = want < 1 ? 1 : want < room ? want : room;
        g.steps_each = (k_steps + g.splits - 1) / g.splits;
        g.splits = (k_steps + g.steps_each - 1) / g.steps_each;
        return t;
    };
    USL_TRY(usl_reserve_kept(c, (void**)&c->gated_scratch, &c->gated_scratch_cap, need(each), need(taken(65536, 65536))));
    a.G = c->gated_scratch;
    const char *e = (const char*)a.e, *gate = (const char*)a.gate, *up = (const char*)a.up;
    const float* grad_x = a.grad_x;
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
        const dim3 slopes((unsigned)(((a.dp + a.wp) / 8 + PREP_NT - 1) / PREP_NT), (unsigned)a.rows);
        if (act == USL_SILU) hipLaunchKernelGGL((k_gated_slopes<T, 0>), slopes, dim3(PREP_NT), 0, c->stream, a);
        else hipLaunchKernelGGL((k_gated_slopes<T, 1>), slopes, dim3(PREP_NT), 0, c->stream, a);
        USL_TRY(usl_check_launch(c, what));
        if (a.grad_V[0] || a.grad_V[1]) {
            const bool tall = tall_v<T>(c, a.w, a.dp);
            if constexpr (ES == 2)
                if (tall) USL_TRY((grad_v<T, 256, 128, 4, 4>(c, a)));
            if (!tall) USL_TRY((grad_v<T, 64, 64, 2, 4>(c, a)));
        }
        if (!a.grad_e) continue;
        const Tiles t = cut(a, a.rows);
        if (t.m == 128) USL_TRY((grad_e<T, 128, 128, 4>(c, a, how)));
        else if (t.n == 32) USL_TRY((grad_e<T, 256, 32, 2>(c, a, how)));
        else if (t.n == 64) USL_TRY((grad_e<T, 256, 64, 4>(c, a, how)));
        else USL_TRY((grad_e<T, 256, 128, 4>(c, a, how)));
        const size_t n = (size_t)a.b * a.w;
        hipLaunchKernelGGL(k_gated_join, dim3((unsigned)((n + 63) / 64)), dim3(256), 0, c->stream, a.sums, a.grad_e + (size_t)i0 * a.w, n, a.splits);
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
