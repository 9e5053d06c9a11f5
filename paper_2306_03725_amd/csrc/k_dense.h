// Device code of the dense products around the layer: out[n][m] = sum over kk of A[m][kk] * B[n][kk] on the matrix cores, both operands staged through
// LDS.  m is the axis along which the output is contiguous: a lane of a 16 x 16 tile holds four neighbours in m of one n.
//
// K is walked in steps.  An operand's tile of a step is either KC (its rows are m or n, with the step's values of K side by side) or KO (its rows are
// values of K, as its memory has them: the transpose is made by the reads, ds_read_b64_tr_b16 for 16-bit numbers).  A fragment is 16 bytes a lane in both
// cases: lane l has row l % 16 and the bytes of group l / 16 of 64 bytes of K.
//
// Tiles go from memory to LDS without registers between (buffer_load_dwordx4 ... lds: a wavefront's 64 x 16 bytes land one behind the other), so
// which 16 bytes a lane asks for decides what lies where: groups of 16 bytes of a row are permuted by a key of the row, by which the lanes whose reads meet
// (k_lanes.h) touch every bank once.  Rows behind the end are the last row again (their results are dropped), groups behind the end of K are asked for out of
// the buffer's range and arrive as zeros.
#pragma once
#include "usl_internal.h"

namespace dense {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(1)));   // 16 bytes from any address

struct bf16 { uint16_t bits; };

// A step of 64 bytes of K on the matrix cores
template <typename T> struct Core;
template <> struct Core<bf16> {
    using Acc = f32x4;
    static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Core<float> {   // the j-th of four products takes value j of every lane: K in another order, the same for both operands
    using Acc = f32x4;
    static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
        return c;
    }
};
template <> struct Core<int8_t> {
    using Acc = i32x4;
    static __device__ __forceinline__ Acc mul(i32x4 a, i32x4 b, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }
};

__device__ __forceinline__ uint32_t lds_at(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }

// What a lane asks a buffer for when it wants zeros: behind the end that the buffer below claims
constexpr uint32_t NOWHERE = 0x80000000u;

// A buffer from p on: every offset that is used lies inside the caller's memory or is NOWHERE.
__device__ __forceinline__ i32x4 buffer_at(const void* p) {
    const uint64_t a = (uint64_t)p;
    i32x4 r;
    r.x = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    r.y = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xFFFF);
    r.z = 0x7FFFFFF0;
    r.w = 0x00020000;
    return r;
}
// 16 bytes a lane from buffer + off to LDS, at `to` + 16 * lane.  M0 is written without the compiler's knowledge: the kernels here have no other use of it.
__device__ __forceinline__ void to_lds(uint32_t to, const i32x4& buffer, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane((int)to)), "v"(off), "s"(buffer) : "memory");
}
template <int LATER>   // what this wavefront asked for is there, but for the LATER loads behind it; behind a barrier, what all did
__device__ __forceinline__ void landed() {
    static_assert(LATER < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LATER) : "memory");
}

// The `bytes` bytes from p on, zeros behind them; may be 0 or less.  before: bytes of the same row that lie before p.  Any address.
__device__ __forceinline__ i32x4 sixteen(const char* p, int bytes, int before) {
    if (bytes >= 16) return *reinterpret_cast<const i32x4_any*>(p);
    unsigned __int128 r = 0;
    if (bytes > 0 && before + bytes >= 16) {   // the last 16 bytes of the row, without those before p
        r = __builtin_bit_cast(unsigned __int128, *reinterpret_cast<const i32x4_any*>(p - (16 - bytes))) >> 8 * (16 - bytes);
    } else {
#pragma unroll 1
        for (int j = 0; j < bytes; ++j) r |= (unsigned __int128)(uint8_t)p[j] << 8 * j;
    }
    return __builtin_bit_cast(i32x4, r);
}

// How rows come into LDS: through registers, from any address; or straight, from multiples of 16 bytes, or of 4 but for what ends inside 16
enum { REGISTERS, DIRECT, WORDS };

// ---- KC: ROWS rows of KB (128 or 64) bytes of K
// The row of a tile that fragment f's row i is.  SPREAD fragments side by side: a lane's four neighbours of each of them are 4 * SPREAD neighbours.
template <int SPREAD>
__device__ __forceinline__ int frag_row(int f, int i) {
    return SPREAD == 1 ? f * 16 + i : (f / SPREAD) * (16 * SPREAD) + (i >> 2) * (4 * SPREAD) + (f % SPREAD) * 4 + (i & 3);
}
// Which group of 16 bytes of a row lies at place p of it (and the other way round).  The 16 lanes that meet read rows i = 0-3 and 12-15 of a fragment at one
// group, rows 4-11 at the next one (k_lanes.h).  128 bytes: two rows cover the banks, 8 rows' keys have to differ.  64: four rows.
template <int KB, int SPREAD>
__device__ __forceinline__ int place_of(int row, int p) {
    const int q = SPREAD == 1 ? row >> 2 : row / (4 * SPREAD);   // i >> 2 of the fragment's row
    if (KB == 128) return p ^ ((row & 3) | (q & 1) << 2);
    return p ^ ((q >> 1 & 1) | ((q ^ q >> 1) & 1) << 1);
}
template <int ROWS, int KB, int SPREAD, int WAVES>
struct StageKC {
    // rows of a wavefront's load; where there are fewer loads than wavefronts, some ask for the same rows, so that all have asked for as many
    static constexpr int AT_ONCE = 1024 / KB, LOADS = ROWS < AT_ONCE * WAVES ? 1 : ROWS / AT_ONCE / WAVES;
    static_assert(ROWS % AT_ONCE == 0 && (ROWS < AT_ONCE * WAVES ? AT_ONCE * WAVES % ROWS == 0 : LOADS * AT_ONCE * WAVES == ROWS), "rows are dealt evenly");
    static constexpr int BYTES = ROWS * KB;
    static __device__ __forceinline__ int first_of(int t) { return (t * WAVES + (int)(threadIdx.x >> 6)) * AT_ONCE % ROWS; }
    static __device__ __forceinline__ int row_of(int t) { return first_of(t) + (int)(threadIdx.x & 63) / (KB / 16); }
    static __device__ __forceinline__ int group_of(int t) { return place_of<KB, SPREAD>(row_of(t), (int)(threadIdx.x & 63) % (KB / 16)); }
    // from: row 0 of the tile at this step's first byte; rows: how many there are; left: bytes of K from here to the end, a multiple of 16 or KB and more; from's address a multiple of 4
    static __device__ __forceinline__ void direct(uint32_t lds, const char* from, int rows, uint32_t pitch, int left) {
        const i32x4 buffer = buffer_at(from);
#pragma unroll
        for (int t = 0; t < LOADS; ++t) {
            const int g = group_of(t) * 16;
            const uint32_t off = (uint32_t)min(row_of(t), rows - 1) * pitch + (uint32_t)g;
            to_lds(lds + (uint32_t)(first_of(t) * KB), buffer, g < left ? off : NOWHERE);
        }
    }
    // the same of two matrices whose rows follow one another, `each` (a multiple of a load's rows) of them at a time
    static __device__ __forceinline__ void direct_two(uint32_t lds, const char* const (&from)[2], int each, int rows, uint32_t pitch, int left) {
#pragma unroll
        for (int t = 0; t < LOADS; ++t) {
            const int first = first_of(t), which = __builtin_amdgcn_readfirstlane(first >= each), g = group_of(t) * 16;
            const i32x4 buffer = buffer_at(from[which]);
            const uint32_t off = (uint32_t)min(row_of(t) - which * each, rows - 1) * pitch + (uint32_t)g;
            to_lds(lds + (uint32_t)(first * KB), buffer, g < left ? off : NOWHERE);
        }
    }
    // the same through registers, for rows at any address: fetch, then (behind the step before) put
    // (before: bytes of K before the step)
    static __device__ __forceinline__ void fetch(i32x4 (&held)[LOADS], const char* from, int rows, uint32_t pitch, int left, int before) {
        if (left >= KB) {
#pragma unroll
            for (int t = 0; t < LOADS; ++t) held[t] = *reinterpret_cast<const i32x4_any*>(from + (size_t)min(row_of(t), rows - 1) * pitch + group_of(t) * 16);
        } else {
#pragma unroll
            for (int t = 0; t < LOADS; ++t) {
                const int g = group_of(t) * 16;
                held[t] = sixteen(from + (size_t)min(row_of(t), rows - 1) * pitch + g, left - g, before + g);
            }
        }
    }
    static __device__ __forceinline__ void fetch_two(i32x4 (&held)[LOADS], const char* const (&from)[2], int each, int rows, uint32_t pitch, int left, int before) {
#pragma unroll
        for (int t = 0; t < LOADS; ++t) {
            const int which = first_of(t) >= each, g = group_of(t) * 16;
            const char* p = from[which] + (size_t)min(row_of(t) - which * each, rows - 1) * pitch + g;
            held[t] = left >= KB ? *reinterpret_cast<const i32x4_any*>(p) : sixteen(p, left - g, before + g);
        }
    }
    static __device__ __forceinline__ void put(char* lds, const i32x4 (&held)[LOADS]) {
#pragma unroll
        for (int t = 0; t < LOADS; ++t) *reinterpret_cast<i32x4*>(lds + first_of(t) * KB + (int)(threadIdx.x & 63) * 16) = held[t];
    }
    // Where this lane's 16 bytes of fragment 0 lie, row0 being the wavefront's first row of the tile (a multiple of 16 * SPREAD), and how far on those of
    // fragment f: the key of a row is that of its fragment's row.  KB = 64.
    static __device__ __forceinline__ int lane(int row0) {
        static_assert(KB == 64, "a fragment is a step");
        const int l = (int)threadIdx.x & 63, row = row0 + frag_row<SPREAD>(0, l & 15);
        int at = row * KB + place_of<KB, SPREAD>(row, l >> 4) * 16;
        asm volatile("" : "+v"(at));   // (one register, not one for every place that it is added to)
        return at;
    }
    static constexpr int on(int f) { return SPREAD == 1 ? f * 16 * KB : (f / SPREAD * 16 * SPREAD + f % SPREAD * 4) * KB; }
    static __device__ __forceinline__ i32x4 frag(const char* lds, int lane, int f) { return *reinterpret_cast<const i32x4*>(lds + lane + on(f)); }
};

// ---- KO: rows of COLS values, a row for each value of K in a step of 64 bytes of K
template <typename T, int COLS, int WAVES>
struct StageKO {
    static constexpr int DEPTH = 64 / (int)sizeof(T), ROW = COLS * (int)sizeof(T), GROUPS = ROW / 16, AT_ONCE = 64 / GROUPS, LOADS = DEPTH / AT_ONCE / WAVES;
    static_assert(GROUPS <= 64 && LOADS * AT_ONCE * WAVES == DEPTH, "rows are dealt evenly");
    static constexpr int BYTES = DEPTH * ROW;
    // 16-bit: 32 lanes read 32 bytes of the rows k = 0-3 and 8-11 (then 4-7 and 12-15, ...): blocks of 32 bytes are permuted by a key that differs between those.
    // 32-bit: 64 lanes read 64 bytes of the rows j, 4 + j, 8 + j, 12 + j: blocks of 64 bytes by k / 4.
    static __device__ __forceinline__ int group_at(int k, int p) {
        if (sizeof(T) == 2) return p ^ (((k & 3) | (k >> 3 & 1) << 2) << 1 & (GROUPS - 1));
        return p ^ ((k >> 2 & 3) << 2 & (GROUPS - 1));
    }
    static __device__ __forceinline__ int row_of(int t) { return (t * WAVES + (int)(threadIdx.x >> 6)) * AT_ONCE + (int)(threadIdx.x & 63) / GROUPS; }
    static __device__ __forceinline__ int group_of(int t) { return group_at(row_of(t), (int)(threadIdx.x & 63) % GROUPS); }
    // from: the tile's first column in the step's first row; depth: rows of K from here to the end; width: bytes from the first column to the end of a row
    static __device__ __forceinline__ void direct(uint32_t lds, const char* from, int depth, size_t pitch, int width) {
        const i32x4 buffer = buffer_at(from);
#pragma unroll
        for (int t = 0; t < LOADS; ++t) {
            const int g = group_of(t) * 16, k = row_of(t);
            to_lds(lds + (uint32_t)((t * WAVES + (int)(threadIdx.x >> 6)) * 1024), buffer, k < depth && g < width ? (uint32_t)k * (uint32_t)pitch + (uint32_t)g : NOWHERE);
        }
    }
    // The same through registers.  Columns behind a row's end come out as the next row's numbers, as long as there is a next row, and as zeros in the matrix's last step
    // (a column has its own results; cut off in every step: 20 x 2014 -> 36853 backward, float32, 654 us, so 376).  before: bytes of a row before the first column
    static __device__ __forceinline__ void fetch(i32x4 (&held)[LOADS], const char* from, int depth, size_t pitch, int width, int before) {
        if (depth > DEPTH && pitch >= 16) {
#pragma unroll
            for (int t = 0; t < LOADS; ++t) {
                const int g = group_of(t) * 16;
                held[t] = *reinterpret_cast<const i32x4_any*>(from + (size_t)row_of(t) * pitch + (g < width ? g : 0));
            }
        } else {
#pragma unroll
            for (int t = 0; t < LOADS; ++t) {
                const int g = group_of(t) * 16, k = row_of(t);
                held[t] = sixteen(from + (size_t)k * pitch + g, k < depth ? width - g : 0, before + g);
            }
        }
    }
    static __device__ __forceinline__ void put(char* lds, const i32x4 (&held)[LOADS]) {
#pragma unroll
        for (int t = 0; t < LOADS; ++t) *reinterpret_cast<i32x4*>(lds + (t * WAVES + (int)(threadIdx.x >> 6)) * 1024 + (int)(threadIdx.x & 63) * 16) = held[t];
    }
    // Where this lane reads for the fragment of the 16 columns from col (a multiple of 16) on.  16-bit: 16 lanes give the addresses of 4 x 16 numbers, four
    // lanes a row, and receive a column each; the other four of a lane's eight values of K lie four rows on, under the same key.  32-bit: the lane's first value of K;
    // the others lie in the rows behind it, under the same key.
    static __device__ __forceinline__ int lane(int col) {
        const int l = (int)threadIdx.x & 63, g = l >> 4;
        int at;
        if (sizeof(T) == 2) {
            const int k = 8 * g + ((l & 15) >> 2), c = col * 2 + (l & 3) * 8;
            at = k * ROW + group_at(k, c >> 4) * 16 + (c & 8);
        } else {
            const int k = 4 * g, c = (col + (l & 15)) * 4;
            at = k * ROW + group_at(k, c >> 4) * 16 + (c & 15);
        }
        asm volatile("" : "+v"(at));
        return at;
    }
    static __device__ __forceinline__ i32x4 frag(const char* lds, int lane) {
        if (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) i16x4 lds4;
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + lane));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + lane + 4 * ROW));
            return __builtin_bit_cast(i32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        i32x4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = *reinterpret_cast<const int*>(lds + lane + j * ROW);
        return r;
    }
};

// ---- the walk along K
// Fragments of a step are read in a first set of X, which every product of the step uses, and GROUPS of Y.  A group is read while the one before it is being
// multiplied, and the next step's first ones during the last group's products: a wavefront that has read the last group says so by the barrier, behind which the
// next step is there for all, and this step's place is free for step s + STAGES.
//   arrive(s): this wavefront's part of step s has landed; ask(s): step s is asked for, if there is one; first(s, x), group(s, g, y): fragments; multiply(g, x, y)
template <int X, int GROUPS, int Y, int STAGES, typename Arrive, typename Ask, typename First, typename Group, typename Multiply>
__device__ __forceinline__ void walk(int steps, Arrive arrive, Ask ask, First first, Group group, Multiply multiply) {
    static_assert(GROUPS > 1, "a group is read while another is multiplied");
    i32x4 xa[X], xb[X], ya[Y], yb[Y];
    auto step = [&](int s, i32x4 (&x)[X], i32x4 (&xn)[X], i32x4 (&y)[Y], i32x4 (&yn)[Y]) {   // y holds the first group
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            i32x4 (&now)[Y] = g & 1 ? yn : y, (&then)[Y] = g & 1 ? y : yn;
            if (g + 1 < GROUPS) group(s, g + 1, then);
            else {   // (behind the last step too: what is read there is in LDS, and is not used; a branch would cost registers)
                arrive(s + 1);
                __syncthreads();
                first(s + 1, xn);
                group(s + 1, 0, then);
                ask(s + STAGES);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(g, x, now);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int s = 0; s < STAGES; ++s) ask(s);
    arrive(0);
    __syncthreads();
    first(0, xa);
    group(0, 0, ya);
    // the next step's first group is in y if the groups are even, else in yn
    int s = 0;
    for (; s + 2 <= steps; s += 2) {
        step(s, xa, xb, ya, yb);
        if (GROUPS % 2) step(s + 1, xb, xa, yb, ya);
        else step(s + 1, xb, xa, ya, yb);
    }
    if (s < steps) step(s, xa, xb, ya, yb);
}
// ... of which a wavefront asks for LOADS pieces a step: waits for step s, where all that may be are behind it
template <int STAGES, int LOADS>
__device__ __forceinline__ void arrived(int s, int steps) {
    if (s == 0 && steps >= STAGES) landed<(STAGES - 1) * LOADS>();
    else if (s > 0 && s + STAGES - 1 <= steps) landed<(STAGES - 2) * LOADS>();   // (step s + STAGES - 1 is asked for behind the barrier)
    else landed<0>();
}

// ---- the block's activations
// Off by 16 roundings of float32 relative to their value at most, far into the tails (measured over a million gates: SiLU 4.8, GELU 7.2, the slopes less); below
// 2^-118 they may be 0.  SHORT, for results that bfloat16 cuts to 2^-8: by 2^-15 (SiLU: 88 roundings of the exponent; GELU: 2 * 87 of them, and 4.7e-6 of the polynomial).
// us, with the short forms and with the others: 512 x 768 -> 32768 bfloat16 SiLU 69 and 71, GELU 72 and 77; 942 x 128 -> 65536 from 8 bits 60 and 70, 75 and 84.  With float32 results the
// others take 399 and 405 there where the short ones take 397 and 400, in the backward pass as long as those.

// 2^((c + c_rest) (v + v_rest)), the rests what c and v would be with more bits: |c v| roundings of the product are caught by fma and put right behind the exponential.
__device__ __forceinline__ float power_of(float v, float v_rest, float c, float c_rest) {
    const float y = v * c, rest = fmaf(v_rest, c, fmaf(v, c_rest, fmaf(v, c, -y))), p = __builtin_amdgcn_exp2f(y);
    return fmaf(p, rest * 0.69314718f, p);
}
// 1 / (1 + exp(-a)), and what it leaves of 1.  (Behind 200 there is nothing but 0 and 1; a NaN comes back by the factor a.)
__device__ __forceinline__ float sigmoid_of(float a, float& left) {
    const float p = power_of(fminf(fabsf(a), 200.f), 0.f, -1.44269504f, -1.925963e-8f), r = __builtin_amdgcn_rcpf(1.f + p);
    left = a < 0.f ? r : p * r;
    return a < 0.f ? p * r : r;
}
// Phi(a), the normal distribution's function, and its density.  Phi(-v) = exp(-v^2 / 2) t P(t), t = 1 / (1 + c v), P the polynomial whose largest relative error over
// 0 <= v <= 14 is least, fitted in 64 bits by Lawson's weights: degree 8, c = 0.35, 3.2e-8; SHORT degree 5, c = 0.31, 4.7e-6.
template <bool SHORT>
__device__ __forceinline__ float phi_of(float a, float& density) {
    const float v = fminf(fabsf(a), 20.f), s = v * v, t = __builtin_amdgcn_rcpf(fmaf(SHORT ? 0.31f : 0.35f, v, 1.f));
    float e, p;
    if (SHORT) {
        e = __builtin_amdgcn_exp2f(s * -0.72134752f);
        p = fmaf(-0.0739290938f, t, 0.180450201f);
        p = fmaf(p, t, 0.0157448575f);
        p = fmaf(p, t, 0.133429706f);
        p = fmaf(p, t, 0.120441295f);
        p = fmaf(p, t, 0.123860702f);
    } else {
        e = power_of(s, fmaf(v, v, -s), -0.72134752f, -9.629815e-9f);
        p = fmaf(-0.029145895f, t, 0.143971547f);
        p = fmaf(p, t, -0.255713969f);
        p = fmaf(p, t, 0.159173876f);
        p = fmaf(p, t, -0.0231096633f);
        p = fmaf(p, t, 0.10550794f);
        p = fmaf(p, t, 0.119832881f);
        p = fmaf(p, t, 0.139861867f);
        p = fmaf(p, t, 0.139621407f);
    }
    const float tail = e * t * p;
    density = 0.39894228f * e;
    return a < 0.f ? tail : 1.f - tail;
}
template <int ACT, bool SHORT>   // 0: a / (1 + exp(-a)); 1: a * Phi(a), the normal distribution's function
__device__ __forceinline__ float act_of(float a) {
    if (ACT == 0 && SHORT) return a * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -1.44269504f));
    float other;
    return a * (ACT == 0 ? sigmoid_of(a, other) : phi_of<SHORT>(a, other));
}
template <int ACT>
__device__ __forceinline__ void act_and_slope(float a, float& value, float& slope) {
    if (ACT == 0) {
        float left;
        const float p = sigmoid_of(a, left);
        value = a * p;
        slope = fmaf(value, left, p);
    } else {
        float density;
        const float phi = phi_of<false>(a, density);
        value = a * phi;
        slope = fmaf(a, density, phi);
    }
}

template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 narrow<bf16>(float v) { return __builtin_bit_cast(bf16, (__bf16)v); }   // nearest, ties to even
// N neighbours (a multiple of 4) to memory at any address; `there` of them exist (1 at least)
template <typename T, int N>
__device__ __forceinline__ void put_many(T* to, const float (&v)[N], int there) {
    constexpr int BYTES = N * (int)sizeof(T), WIDE = BYTES % 16 == 0 ? 4 : 2;   // words of a store
    typedef uint32_t Words __attribute__((ext_vector_type(WIDE), aligned(2)));
    T r[N];
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = narrow<T>(v[j]);
    if (there >= N) {
        Words q[BYTES / 4 / WIDE];
        __builtin_memcpy(q, r, BYTES);
#pragma unroll
        for (int u = 0; u < BYTES / 4 / WIDE; ++u) reinterpret_cast<Words*>(to)[u] = q[u];
    } else {
#pragma unroll
        for (int j = 0; j < N - 1; ++j)
            if (j < there) to[j] = r[j];
    }
}
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16 v) { return usl_bf16_to_f32(v.bits); }

}  // namespace dense
