// Kernels of one or two projections of the rows of e, with what follows them in the epilogue (k_gated.hip, k_int8.hip).
#pragma once
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
};

// Four neighbours of an instance's output from their sums
template <typename T, typename TO, int MATS, int ACT>
__device__ __forceinline__ void finish(const Forward& a, const typename Core<T>::Acc (&acc)[MATS], int i, int d0, bool aligned) {
    float v[MATS][4];
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[q][j] = (float)acc[q][j];
            if (sizeof(T) == 1) v[q][j] *= a.e_scale[i] * a.V_scale[q][min(d0 + j, a.d - 1)];
        }
    const size_t at = (size_t)i * a.d + d0;
    auto put = [&](void* to, const float (&f)[4]) {
        TO r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = narrow<TO>(f[j]);
        TO* p = (TO*)to + at;
        if (aligned && d0 + 3 < a.d) {
            struct alignas(4 * sizeof(TO)) Four { TO v[4]; };
            *reinterpret_cast<Four*>(p) = *reinterpret_cast<const Four*>(__builtin_assume_aligned(r, 4));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (d0 + j < a.d) p[j] = r[j];
        }
    };
    if (MATS == 1) {
        put(a.x, v[0]);
        return;
    }
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = act_of<ACT>(v[0][j]) * v[MATS - 1][j];
    put(a.x, x);
    if (a.gate) put(a.gate, v[0]);
    if (a.up) put(a.up, v[MATS - 1]);
}

// A tile of BD activations of BB instances.  DIRECT: rows and bases are multiples of 16 bytes.
template <typename T, typename TO, int MATS, int ACT, int BD, int BB, int WAVES_D, int WAVES_B, bool DIRECT>
__global__ void __launch_bounds__(64 * WAVES_D * WAVES_B)
k_dense_forward(Forward a) {
    constexpr int WAVES = WAVES_D * WAVES_B, KB = 128, FD = BD / WAVES_D / 16, FB = BB / WAVES_B / 16;
    using Acc = typename Core<T>::Acc;
    using SV = StageKC<BD, KB, FD, WAVES>;
    using SE = StageKC<BB, KB, 1, WAVES>;
    constexpr int STEP = MATS * SV::BYTES + SE::BYTES;
    extern __shared__ __align__(1024) char lds[];   // two steps
    // Workgroups go to the chiplets in turn: the tiles of one piece of V, which share its rows, go to one of them, one after the other.
    const int turn = (int)blockIdx.x >> 3, td = turn / a.tiles_b * 8 + ((int)blockIdx.x & 7), tb = turn % a.tiles_b;
    if (td >= a.tiles_d) return;
    const int d0 = td * BD, b0 = tb * BB, wave = (int)threadIdx.x >> 6, wd = wave % WAVES_D * (BD / WAVES_D), wb = wave / WAVES_D * (BB / WAVES_B);
    const int rows_d = min(a.d - d0, BD), rows_b = min(a.b - b0, BB);
    const uint32_t pitch = (uint32_t)a.row_bytes;
    const char* V[MATS];
#pragma unroll
    for (int q = 0; q < MATS; ++q) V[q] = (const char*)a.V[q] + (size_t)d0 * pitch;
    const char* e = (const char*)a.e + (size_t)b0 * pitch;
    Acc acc[MATS][FD][FB];
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int f = 0; f < FD; ++f)
#pragma unroll
            for (int h = 0; h < FB; ++h) acc[q][f][h] = Acc{0, 0, 0, 0};
    const int steps = (a.row_bytes + KB - 1) / KB;
    i32x4 held_v[DIRECT ? 1 : MATS][SV::LOADS], held_e[SE::LOADS];
    auto ask = [&](int s) {
        const int at = s * KB, left = a.row_bytes - at;
        char* to = lds + (s & 1) * STEP;
#pragma unroll
        for (int q = 0; q < MATS; ++q) {
            if constexpr (DIRECT) SV::direct(lds_at(to + q * SV::BYTES), V[q] + at, rows_d, pitch, left);
            else SV::template fetch<T>(held_v[q], V[q] + at, rows_d, pitch, left);
        }
        if constexpr (DIRECT) SE::direct(lds_at(to + MATS * SV::BYTES), e + at, rows_b, pitch, left);
        else SE::template fetch<T>(held_e, e + at, rows_b, pitch, left);
    };
    auto place = [&](int s) {
        if constexpr (!DIRECT) {
            char* to = lds + (s & 1) * STEP;
#pragma unroll
            for (int q = 0; q < MATS; ++q) SV::put(to + q * SV::BYTES, held_v[q]);
            SE::put(to + MATS * SV::BYTES, held_e);
        }
    };
    ask(0);
    place(0);
    for (int s = 0; s < steps; ++s) {
        if (DIRECT) landed();
        __syncthreads();   // step s is there, and nobody reads the one before it any more
        if (s + 1 < steps) ask(s + 1);
        const char* from = lds + (s & 1) * STEP;
#pragma unroll
        for (int h = 0; h < KB / 64; ++h) {
            i32x4 eb[FB];
#pragma unroll
            for (int f = 0; f < FB; ++f) eb[f] = SE::frag(from + MATS * SV::BYTES, wb, f, h);
#pragma unroll
            for (int q = 0; q < MATS; ++q)
#pragma unroll
                for (int f = 0; f < FD; ++f) {
                    const i32x4 v = SV::frag(from + q * SV::BYTES, wd, f, h);
#pragma unroll
                    for (int g = 0; g < FB; ++g) acc[q][f][g] = Core<T>::mul(v, eb[g], acc[q][f][g]);
                }
        }
        if (s + 1 < steps) place(s + 1);
    }
    const int l = (int)threadIdx.x & 63;
    const bool aligned = a.d % 4 == 0 && ((uintptr_t)a.x | (uintptr_t)a.gate | (uintptr_t)a.up) % (4 * sizeof(TO)) == 0;
#pragma unroll
    for (int g = 0; g < FB; ++g) {
        const int i = b0 + wb + g * 16 + (l & 15);
        if (i < a.b)
#pragma unroll
            for (int f = 0; f < FD; ++f) {
                const int at = d0 + wd + frag_row<FD>(f, (l >> 4) * 4);
                Acc one[MATS];
#pragma unroll
                for (int q = 0; q < MATS; ++q) one[q] = acc[q][f][g];
                if (at < a.d) finish<T, TO, MATS, ACT>(a, one, i, at, aligned);
            }
    }
}

// At most 16 instances: the matrices go from memory into fragments, 16 rows to a workgroup whose wavefronts share K and join their sums through LDS.
template <typename T, typename TO, int MATS, int ACT, int WAVES>
__global__ void __launch_bounds__(64 * WAVES)
k_dense_few(Forward a) {
    using Acc = typename Core<T>::Acc;
    __shared__ Acc sums[WAVES][MATS][64];
    const int l = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, d0 = (int)blockIdx.x * 16;
    const size_t row_v = (size_t)min(d0 + (l & 15), a.d - 1) * a.row_bytes, row_e = (size_t)min(l & 15, a.b - 1) * a.row_bytes;
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
        const int left = a.row_bytes - whole * 64 - (l >> 4) * 16;
        const i32x4 y = sixteen<T>(e + (size_t)whole * 64, left);
#pragma unroll
        for (int q = 0; q < MATS; ++q) acc[q] = Core<T>::mul(sixteen<T>(V[q] + (size_t)whole * 64, left), y, acc[q]);
    }
#pragma unroll
    for (int q = 0; q < MATS; ++q) sums[wave][q][l] = acc[q];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int q = 0; q < MATS; ++q)
#pragma unroll
        for (int v = 1; v < WAVES; ++v) acc[q] += sums[v][q][l];
    const bool aligned = a.d % 4 == 0 && ((uintptr_t)a.x | (uintptr_t)a.gate | (uintptr_t)a.up) % (4 * sizeof(TO)) == 0;
    const int at = d0 + (l >> 4) * 4;
    if ((l & 15) < a.b && at < a.d) finish<T, TO, MATS, ACT>(a, acc, l & 15, at, aligned);
}

template <typename T, typename TO, int MATS, int ACT, int BD, int BB, int WAVES_D, int WAVES_B>
usl_status launch_tiles(usl_ctx* c, Forward a, const char* what) {
    constexpr int BYTES = 2 * (MATS * BD + BB) * 128;
    a.tiles_d = (a.d + BD - 1) / BD;
    a.tiles_b = (a.b + BB - 1) / BB;
    const dim3 grid((unsigned)((a.tiles_d + 7) / 8 * 8 * a.tiles_b)), block(64 * WAVES_D * WAVES_B);
    const bool direct = (a.row_bytes | (uintptr_t)a.V[0] | (uintptr_t)a.V[MATS - 1] | (uintptr_t)a.e) % 16 == 0;
    const auto kernel = direct ? k_dense_forward<T, TO, MATS, ACT, BD, BB, WAVES_D, WAVES_B, true> : k_dense_forward<T, TO, MATS, ACT, BD, BB, WAVES_D, WAVES_B, false>;
    if (BYTES > 64 * 1024) USL_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, BYTES));
    hipLaunchKernelGGL(kernel, grid, block, BYTES, c->stream, a);
    return usl_check_launch(c, what);
}

template <typename T, typename TO, int MATS, int ACT>
usl_status launch_forward(usl_ctx* c, const Forward& a, const char* what) {
    if (a.b <= 16) {
        hipLaunchKernelGGL((k_dense_few<T, TO, MATS, ACT, 4>), dim3((unsigned)((a.d + 15) / 16)), dim3(256), 0, c->stream, a);
        return usl_check_launch(c, what);
    }
    if ((int64_t)((a.d + 127) / 128) * ((a.b + 127) / 128) >= c->num_cu) return launch_tiles<T, TO, MATS, ACT, 128, 128, 2, 2>(c, a, what);
    return launch_tiles<T, TO, MATS, ACT, 64, 64, 2, 2>(c, a, what);
}

}  // namespace dense
