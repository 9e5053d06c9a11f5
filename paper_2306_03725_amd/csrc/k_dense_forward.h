// Kernels of one or two projections of the rows of e, with what follows them in the epilogue (k_gated.hip, k_int8.hip).
#pragma once
#include <math.h>

#include "k_dense.h"

namespace dense {

struct Forward {
    const void* V[2];          // [d][w]: gate and up, or one matrix
    const void* e;             // [b][w]
    const float* V_scale[2];   // 8-bit integers: [d]
    const float* e_scale;      // [b]
    void *x, *gate, *up;       // [b][d]; gate, up may be null
    int d, b, row_bytes;       // of a row of V and e
    int tiles_d, tiles_b;
    int whole;                 // results' rows consist of whole 64-byte pieces of memory
};

// What 8-bit integers' sums are multiplied by: a lane's N neighbours of each matrix
template <typename T, int MATS, int N>
struct Scales {
    float v[MATS][N];
    __device__ __forceinline__ void load(const Forward& a, int d0) {
        if (sizeof(T) == 1)
#pragma unroll
            for (int q = 0; q < MATS; ++q)
#pragma unroll
                for (int j = 0; j < N; ++j) v[q][j] = a.V_scale[q][min(d0 + j, a.d - 1)];
    }
};
// gate and up go past the caches, which have V and e to keep: 512 x 768 -> 32768 bfloat16 74 us, so 67 (x too: 68); the results from 8-bit integers too: 1024 x 512 ->
// 65536 67 and 59, 500 x 750 -> 32768 gated 60 and 58.  Where rows of the results end inside 64 bytes of memory, two tiles write them, and past the caches that is two
// writes of a part; through the caches, with the two tiles on one chiplet, it is one: 942 x 128 -> 65033 bfloat16 250 us, on one chiplet 218, and through the caches 156;
// 512 x 768 -> 32760 96, 83, 76.  From 8 bits past them all the same: 942 x 512 -> 65033 gated 125, through them 148 (on two chiplets 142 and 149).
// 16 instances' values of WD neighbouring activations, a lane N of one instance's, to rows of memory: through LDS, so that a store takes whole lines of it.
// (16 rows of 64 bytes to a store, the other half of every line by the next one: 512 x 768 -> 32768 bfloat16, three outputs, 85 us, and with more between the
// two 98; in whole lines 73.)  `mine`: the wavefront's own LDS.
template <typename TO, int WD, bool PAST_CACHES, int N>
__device__ __forceinline__ void put_tile(char* mine, TO* to, const float (&v)[N], int i0, int b, int d0, int d, bool past) {
    constexpr int ROW = WD * (int)sizeof(TO), PITCH = ROW + 16, EACH = 16 / (int)sizeof(TO), GROUPS = ROW / 16;
    static_assert(N * 4 == WD, "four lanes share a row");
    const int l = (int)threadIdx.x & 63;
    if constexpr (N < EACH) {   // 8 bytes a lane: not worth the way
        const int i = i0 + (l & 15), c = d0 + (l >> 4) * N;
        if (i < b && c < d) put_many(to + (size_t)i * d + c, v, d - c);
    } else {
        TO r[N];
#pragma unroll
        for (int j = 0; j < N; ++j) r[j] = narrow<TO>(v[j]);
        uint4 q[N / EACH > 0 ? N / EACH : 1];
        __builtin_memcpy(q, r, sizeof(r));
#pragma unroll
        for (int u = 0; u < N / EACH; ++u) *reinterpret_cast<uint4*>(mine + (l & 15) * PITCH + (l >> 4) * (ROW / 4) + u * 16) = q[u];
#pragma unroll
        for (int t = 0; t < 16 * GROUPS / 64; ++t) {
            const int at = t * 64 + l, row = at / GROUPS, c = d0 + at % GROUPS * EACH, i = i0 + row;
            const uint4 w = *reinterpret_cast<const uint4*>(mine + row * PITCH + at % GROUPS * 16);
            if (i >= b || c >= d) continue;
            TO* p = to + (size_t)i * d + c;
            if (d - c >= EACH) {
                typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
                if (PAST_CACHES && past) {   // (the two lines around it keep the compiler from making one store of the two)
                    asm volatile("; past the caches" ::: "memory");
                    __builtin_nontemporal_store(__builtin_bit_cast(Words, w), reinterpret_cast<Words*>(p));
                    asm volatile("; past the caches" ::: "memory");
                } else *reinterpret_cast<Words*>(p) = __builtin_bit_cast(Words, w);
            } else {
                TO one[EACH];
                __builtin_memcpy(one, &w, 16);
#pragma unroll
                for (int j = 0; j < EACH - 1; ++j)
                    if (j < d - c) p[j] = one[j];
            }
        }
    }
}

// How rows come into LDS.  DIRECT: they and their bases are multiples of 16 bytes; STAGES steps of K then have room in LDS, one being multiplied and the others on their
// way.  WORDS: of 4; the same for whole steps, and what is left of a row through registers behind them.  Else everything through registers, asked for two steps ahead.
// us, in words and through registers, and with a row of a few numbers more, directly: 60 x 1830 -> 7059 bfloat16 17.1, 34.2, 16.2; 47 x 1990 -> 11048 float32 79, 111, 78;
// 910 x 940 -> 1147 from 8 bits 12.8, 16.0, 12.1; 773 x 542 -> 4324 bfloat16 32.2, 33.5, 25.0.
// A tile of BD activations of BB instances.
template <typename T, typename TO, int MATS, int ACT, int BD, int BB, int WAVES_D, int WAVES_B, int STAGES, int HOW>
__global__ void __launch_bounds__(64 * WAVES_D * WAVES_B, 2)   // (two wavefronts to a SIMD: sums and fragments in 256 registers)
k_dense_forward(Forward a) {
    constexpr int WAVES = WAVES_D * WAVES_B, KB = 64, FD = BD / WAVES_D / 16, FB = BB / WAVES_B / 16;
    static_assert(HOW != REGISTERS || STAGES == 2, "two sets of registers");
    using Acc = typename Core<T>::Acc;
    // V's rows, gate's before up's; a lane's neighbours of all fragments are neighbours.  TOGETHER: the rows of one matrix are too few for all wavefronts.
    constexpr bool TOGETHER = BD < 16 * WAVES;
    using SV = StageKC<MATS * BD, KB, FD, WAVES>;
    using SQ = StageKC<TOGETHER ? MATS * BD : BD, KB, FD, WAVES>;
    using SE = StageKC<BB, KB, 1, WAVES>;
    constexpr int STEP = SV::BYTES + SE::BYTES, LOADS = (TOGETHER ? 1 : MATS) * SQ::LOADS + SE::LOADS;
    extern __shared__ __align__(1024) char lds[];
    // Workgroups go to the chiplets in turn: the tiles of one piece of V, which share its rows, go to one of them, one after the other; so do those of its neighbours where
    // a piece of memory holds results of two tiles, to be one write of the chiplet's cache.
    const int turn = (int)blockIdx.x >> 3, xcd = (int)blockIdx.x & 7, tb = turn % a.tiles_b, nth = turn / a.tiles_b;
    const int td = a.whole ? nth * 8 + xcd : (int)((int64_t)xcd * a.tiles_d >> 3) + nth;
    if (td >= (a.whole ? a.tiles_d : (int)((int64_t)(xcd + 1) * a.tiles_d >> 3))) return;
    const int d0 = td * BD, b0 = tb * BB, wave = (int)threadIdx.x >> 6, wd = wave % WAVES_D * (BD / WAVES_D), wb = wave / WAVES_D * (BB / WAVES_B);
    const int rows_d = min(a.d - d0, BD), rows_b = min(a.b - b0, BB);
    const uint32_t pitch = (uint32_t)a.row_bytes;
    const char *V[2], *e = (const char*)a.e + (size_t)b0 * pitch;
#pragma unroll
    for (int q = 0; q < 2; ++q) V[q] = (const char*)a.V[MATS == 1 ? 0 : q] + (size_t)d0 * pitch;
    Acc acc[MATS][FD][FB];
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int f = 0; f < FD; ++f)
#pragma unroll
            for (int h = 0; h < FB; ++h) acc[q][f][h] = Acc{0, 0, 0, 0};
    const int steps = HOW == WORDS ? a.row_bytes / KB : (a.row_bytes + KB - 1) / KB;
    const int lane_v = SV::lane(wd), lane_e = SE::lane(wb);
    struct Held { i32x4 v[TOGETHER ? 1 : MATS][SQ::LOADS], e[SE::LOADS]; };
    auto ask = [&](Held& h, int s) {
        const int at = s * KB, left = a.row_bytes - at;
        if (left <= 0) return;
        const char* const from[2] = {V[0] + at, V[1] + at};
        if constexpr (TOGETHER) SQ::fetch_two(h.v[0], from, BD, rows_d, pitch, left, at);
        else
#pragma unroll
            for (int q = 0; q < MATS; ++q) SQ::fetch(h.v[q], from[q], rows_d, pitch, left, at);
        SE::fetch(h.e, e + at, rows_b, pitch, left, at);
    };
    auto put = [&](const Held& h, char* to) {
#pragma unroll
        for (int q = 0; q < (TOGETHER ? 1 : MATS); ++q) SQ::put(to + q * SQ::BYTES, h.v[q]);
        SE::put(to + SV::BYTES, h.e);
    };
    auto multiply = [&](const char* from) {
        i32x4 eb[FB];
#pragma unroll
        for (int f = 0; f < FB; ++f) eb[f] = SE::frag(from + SV::BYTES, lane_e, f);
#pragma unroll
        for (int q = 0; q < MATS; ++q)
#pragma unroll
            for (int f = 0; f < FD; ++f) {
                const i32x4 v = SV::frag(from + q * (BD * KB), lane_v, f);
#pragma unroll
                for (int g = 0; g < FB; ++g) acc[q][f][g] = Core<T>::mul(v, eb[g], acc[q][f][g]);
            }
    };
    if constexpr (HOW != REGISTERS) {
        constexpr int GROUPS = 2, Y = MATS * FD / GROUPS;   // a matrix, or half of one's fragments
        auto place = [&](int s) { return lds + s % STAGES * STEP; };
        walk<FB, GROUPS, Y, STAGES>(
            steps, [&](int s) { arrived<STAGES, LOADS>(s, steps); },
            [&](int s) {
                if (s >= steps) return;
                const int at = s * KB, left = a.row_bytes - at;
                const uint32_t to = lds_at(place(s));
                const char* const from[2] = {V[0] + at, V[1] + at};
                if constexpr (TOGETHER) SV::direct_two(to, from, BD, rows_d, pitch, left);
                else
#pragma unroll
                    for (int q = 0; q < MATS; ++q) SQ::direct(to + q * SQ::BYTES, from[q], rows_d, pitch, left);
                SE::direct(to + SV::BYTES, e + at, rows_b, pitch, left);
            },
            [&](int s, i32x4 (&x)[FB]) {
#pragma unroll
                for (int f = 0; f < FB; ++f) x[f] = SE::frag(place(s) + SV::BYTES, lane_e, f);
            },
            [&](int s, int g, i32x4 (&y)[Y]) {
#pragma unroll
                for (int f = 0; f < Y; ++f) y[f] = SV::frag(place(s) + (g * Y + f) / FD * (BD * KB), lane_v, (g * Y + f) % FD);
            },
            [&](int g, const i32x4 (&x)[FB], const i32x4 (&y)[Y]) {
#pragma unroll
                for (int f = 0; f < Y; ++f)
#pragma unroll
                    for (int h = 0; h < FB; ++h) {
                        Acc& to = acc[(g * Y + f) / FD][(g * Y + f) % FD][h];
                        to = Core<T>::mul(y[f], x[h], to);
                    }
            });
        if (HOW == WORDS && steps * KB < a.row_bytes) {
            Held rest;
            ask(rest, steps);
            __syncthreads();   // the last whole step has been read
            put(rest, lds);
            __syncthreads();
            multiply(lds);
        }
    } else {
        Held one, two;   // steps s + 1 and s + 2
        auto place = [&](const Held& h, int s) {
            if (s < steps) put(h, lds + (s & 1) * STEP);
        };
        ask(two, 0);
        ask(one, 1);
        place(two, 0);
        for (int s = 0; s < steps; s += 2) {
            __syncthreads();
            ask(two, s + 2);
            multiply(lds);
            place(one, s + 1);
            __syncthreads();
            if (s + 1 >= steps) break;
            ask(one, s + 3);
            multiply(lds + STEP);
            place(two, s + 2);
        }
    }
    constexpr int N = 4 * FD, WD = BD / WAVES_D;
    static_assert(WAVES * 16 * (WD * (int)sizeof(TO) + 16) <= STAGES * STEP, "room for the outputs");
    const int l = (int)threadIdx.x & 63, i0 = b0 + wb, c0 = d0 + wd;
    char* mine = lds + wave * 16 * (WD * (int)sizeof(TO) + 16);
    Scales<T, MATS, N> scales;
    scales.load(a, c0 + (l >> 4) * N);
    const bool past = sizeof(T) == 1 || a.whole;
    __syncthreads();   // the last step has been read
#pragma unroll
    for (int g = 0; g < FB; ++g) {
        const float e_scale = sizeof(T) == 1 ? a.e_scale[min(i0 + g * 16 + (l & 15), a.b - 1)] : 1.f;
        float v[MATS][N];
#pragma unroll
        for (int q = 0; q < MATS; ++q)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                v[q][j] = (float)acc[q][j / 4][g][j % 4];
                if (sizeof(T) == 1) v[q][j] *= e_scale * scales.v[q][j];
            }
        if (MATS == 1) {
            put_tile<TO, WD, true>(mine, (TO*)a.x, v[0], i0 + g * 16, a.b, c0, a.d, past);
            continue;
        }
        float x[N];
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = act_of<ACT, sizeof(TO) == 2>(v[0][j]) * v[MATS - 1][j];
        put_tile<TO, WD, sizeof(T) == 1>(mine, (TO*)a.x, x, i0 + g * 16, a.b, c0, a.d, past);
        if (a.gate) put_tile<TO, WD, true>(mine, (TO*)a.gate, v[0], i0 + g * 16, a.b, c0, a.d, past);
        if (a.up) put_tile<TO, WD, true>(mine, (TO*)a.up, v[MATS - 1], i0 + g * 16, a.b, c0, a.d, past);
    }
}

// Few results: the matrices go from memory into fragments, 16 rows and 16 instances to a workgroup whose wavefronts share K and join their sums through LDS.  Bound by the rows' way from memory, 64 bytes of each to a load: 7 x 562 -> 37570 float32, 169 MB, 53 us.
template <typename T, typename TO, int MATS, int ACT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
k_dense_few(Forward a) {
    using Acc = typename Core<T>::Acc;
    __shared__ Acc sums[WAVES][MATS][64];
    const int l = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, d0 = (int)blockIdx.x * 16, i = (int)blockIdx.y * 16 + (l & 15);
    const size_t row_v = (size_t)min(d0 + (l & 15), a.d - 1) * a.row_bytes, row_e = (size_t)min(i, a.b - 1) * a.row_bytes;
    const char* e = (const char*)a.e + row_e + (l >> 4) * 16;
    const char* V[MATS];
#pragma unroll
    for (int q = 0; q < MATS; ++q) V[q] = (const char*)a.V[q] + row_v + (l >> 4) * 16;
    Acc acc[MATS];
#pragma unroll
    for (int q = 0; q < MATS; ++q) acc[q] = Acc{0, 0, 0, 0};
    const int whole = a.row_bytes / 64, steps = (a.row_bytes + 63) / 64, each = (steps + WAVES - 1) / WAVES;
    const int first = wave * each, last = min(first + each, whole);
#pragma unroll 8
    for (int s = first; s < last; ++s) {
        const i32x4 y = *reinterpret_cast<const i32x4_any*>(e + (size_t)s * 64);
#pragma unroll
        for (int q = 0; q < MATS; ++q) acc[q] = Core<T>::mul(*reinterpret_cast<const i32x4_any*>(V[q] + (size_t)s * 64), y, acc[q]);
    }
    if (whole < steps && first <= whole && whole < first + each) {   // the end of the rows
        const int before = whole * 64 + (l >> 4) * 16, left = a.row_bytes - before;
        const i32x4 y = sixteen(e + (size_t)whole * 64, left, before);
#pragma unroll
        for (int q = 0; q < MATS; ++q) acc[q] = Core<T>::mul(sixteen(V[q] + (size_t)whole * 64, left, before), y, acc[q]);
    }
#pragma unroll
    for (int q = 0; q < MATS; ++q) sums[wave][q][l] = acc[q];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int v = 1; v < WAVES; ++v) acc[q] += sums[v][q][l];
    const int at = d0 + (l >> 4) * 4;
    if (i < a.b && at < a.d) {
        Scales<T, MATS, 4> scales;
        scales.load(a, at);
        const float e_scale = sizeof(T) == 1 ? a.e_scale[i] : 1.f;
        float v[MATS][4];
#pragma unroll
        for (int q = 0; q < MATS; ++q)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[q][j] = (float)acc[q][j];
                if (sizeof(T) == 1) v[q][j] *= e_scale * scales.v[q][j];
            }
        const size_t to = (size_t)i * a.d + at;
        if (MATS == 1) {
            put_many((TO*)a.x + to, v[0], a.d - at);
            return;
        }
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = act_of<ACT, sizeof(TO) == 2>(v[0][j]) * v[MATS - 1][j];
        put_many((TO*)a.x + to, x, a.d - at);
        if (a.gate) put_many((TO*)a.gate + to, v[0], a.d - at);
        if (a.up) put_many((TO*)a.up + to, v[MATS - 1], a.d - at);
    }
}

template <typename T, typename TO, int MATS, int ACT, int BD, int BB, int WAVES_D, int WAVES_B, int STAGES, int HOW>
usl_status launch_tiles(usl_ctx* c, Forward a, const char* what) {
    constexpr int BYTES = STAGES * (MATS * BD + BB) * 64;
    const auto kernel = k_dense_forward<T, TO, MATS, ACT, BD, BB, WAVES_D, WAVES_B, STAGES, HOW>;
    a.tiles_d = (a.d + BD - 1) / BD;
    a.tiles_b = (a.b + BB - 1) / BB;
    const dim3 grid((unsigned)((a.tiles_d + 7) / 8 * 8 * a.tiles_b)), block(64 * WAVES_D * WAVES_B);
    if (BYTES > 64 * 1024) USL_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, BYTES));
    hipLaunchKernelGGL(kernel, grid, block, BYTES, c->stream, a);
    return usl_check_launch(c, what);
}

template <typename T, typename TO, int MATS, int ACT, int BD, int BB, int STAGES>
usl_status launch_any(usl_ctx* c, const Forward& a, const char* what, int how) {
    if (how == DIRECT) return launch_tiles<T, TO, MATS, ACT, BD, BB, 2, 2, STAGES, DIRECT>(c, a, what);
    if constexpr (sizeof(T) < 4)   // (float32 numbers lie at multiples of 4 bytes)
        if (how == REGISTERS) return launch_tiles<T, TO, MATS, ACT, BD, BB, 2, 2, 2, REGISTERS>(c, a, what);
    return launch_tiles<T, TO, MATS, ACT, BD, BB, 2, 2, STAGES, WORDS>(c, a, what);
}

// Which tiles?  A compute unit's time is that of the tiles that fall to it, whole ones of them, each as long as its area over its rate: large ones read fragments less often
// (in float32 the matrix cores are so slow that it does not matter), small ones leave less undone at the edges and fall to the compute units more evenly.  Rates from
// 512 x 768 -> 32768 (bfloat16 128 x 256 67 us, 128 x 128 83, 64 x 64 114, 32 x 64 160).  us, gated, w = 768, bfloat16 if not said otherwise, by what the rule takes and by others:
//   256 x -> 32768  128 x 256 37, 128 x 128 46        256 x -> 16384  128 x 128 20, 128 x 256 25, 64 x 64 25
//   128 x -> 32768  128 x 128 29.5, 64 x 64 37        64 x -> 32768   64 x 64 25, 128 x 128 27
//   512 x -> 4096   64 x 64 14, 128 x 128 18          100 x 1000 -> 3000  32 x 64 9.8, 64 x 64 12.1
//   float32: 169 x 256 -> 16512  64 x 64 40, 128 x 128 72;  1000 x 500 -> 20000  348 and 406;  512 x 768 -> 32768  128 x 256 398, 64 x 64 406
//   from 8 bits, rows of at most 768: 942 x 128 -> 65536  128 x 128 74, 128 x 256 87;  942 x 512 -> 65536  117 and 125;  942 x 768 -> 65536  161 and 164;  942 x 2048 -> 65536  322 and 308
// At most 16 instances: tiles of 64 x 16 where there is one for every compute unit: 1 x -> 32768 19.2, rows straight into fragments 21.6; 8 x -> 16384 9.8 and 11.6; 8 x -> 8192
// 7.2 and 7.1; 8 x -> 32768 float32 42.5 and 51.4; 1 x 512 -> 65536 from 8 bits 10.0 and 10.5.
// Rows straight into fragments otherwise, and for up to two fragments to a compute unit (four in float32), whose wavefronts then share K: 48 x 1792 -> 64 6.9, 32 x 64 14.1;
// 100 x 1000 -> 1000 8.9 and 9.7; not 200 x 512 -> 1024 (832 fragments) 7.6 and 6.3.  float32: 64 x 880 -> 2471 15.4 and 24.5, 200 x 512 -> 1024 12.9 and 15.2; not
// 333 x 512 -> 1024 (1344) 18.6 and 15.4.
template <typename T, typename TO, int MATS, int ACT>
usl_status launch_forward(usl_ctx* c, Forward a, const char* what) {
    constexpr int FEW = MATS == 1 ? 128 : 64, MANY = MATS == 1 ? 256 : 128;
    constexpr bool SLOW = sizeof(T) == 4;
    const uintptr_t rows = a.row_bytes | (uintptr_t)a.V[0] | (uintptr_t)a.V[MATS - 1] | (uintptr_t)a.e;
    const int how = rows % 16 == 0 ? DIRECT : rows % 4 == 0 ? WORDS : REGISTERS;
    a.whole = ((size_t)a.d * sizeof(TO) | (uintptr_t)a.x | (uintptr_t)a.gate | (uintptr_t)a.up) % 64 == 0;
    auto tiles = [&](int d, int b) { return (int64_t)((a.d + d - 1) / d) * ((a.b + b - 1) / b); };
    if (how == DIRECT && a.b <= 16 && tiles(FEW, 16) >= c->num_cu) return launch_tiles<T, TO, MATS, ACT, FEW, 16, 4, 1, 5, DIRECT>(c, a, what);
    if (a.b <= 16 || tiles(16, 16) <= (SLOW ? 4 : 2) * c->num_cu) {
        hipLaunchKernelGGL((k_dense_few<T, TO, MATS, ACT, 4>), dim3((unsigned)((a.d + 15) / 16), (unsigned)((a.b + 15) / 16)), dim3(256), 0, c->stream, a);
        return usl_check_launch(c, what);
    }
    const bool short_ones = sizeof(T) == 1 && MATS == 2 && a.row_bytes <= 768;
    auto cost = [&](int d, int b, double rate) { return (double)((tiles(d, b) + c->num_cu - 1) / c->num_cu) * d * b / rate; };
    const double by_many = how != REGISTERS ? cost(MANY, 256, 1.0) : INFINITY, by_128 = cost(128, 128, SLOW ? 1.0 : short_ones ? 1.05 : 0.8), by_64 = cost(64, 64, SLOW ? 0.97 : 0.59),
                 by_32 = MATS == 2 ? cost(32, 64, SLOW ? 0.9 : 0.42) : INFINITY;
    if (by_many <= by_128 && by_many <= by_64 && by_many <= by_32)
        return how == DIRECT ? launch_tiles<T, TO, MATS, ACT, MANY, 256, 2, 4, 4, DIRECT>(c, a, what) : launch_tiles<T, TO, MATS, ACT, MANY, 256, 2, 4, 4, WORDS>(c, a, what);
    if (by_128 <= by_64 && by_128 <= by_32) return launch_any<T, TO, MATS, ACT, 128, 128, 3>(c, a, what, how);
    if constexpr (MATS == 2)
        if (by_32 < by_64) return launch_any<T, TO, MATS, ACT, 32, 64, 4>(c, a, what, how);
    return launch_any<T, TO, MATS, ACT, 64, 64, 4>(c, a, what, how);
}

}  // namespace dense
