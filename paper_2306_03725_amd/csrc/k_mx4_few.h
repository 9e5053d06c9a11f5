// Scores of one group of instances (b <= Q) from values in 4 bits (k_mx4.h): idx and codes stream, nothing is reused.
//
// A lane takes four neighbouring slots of a label (16 bytes of idx, half a word of codes, which it shares with its neighbour), gathers their activations from
// the row in LDS, and the LPL lanes of a label add up their sums; after LPL rounds every lane has a label's.  A round of the whole grid is a run of
// consecutive labels, 64 / LPL to a wavefront.  A round's first label is the same for the wavefront, so addresses are scalar bases and 32-bit offsets that never
// change; what would lie behind the last label begins earlier (labels that two wavefronts share get the same bits twice).
// Bound by the stream of idx and codes: m = 670k, k = 64, b = 1, bfloat16: 197 MB in 39.6 us, 5.0 TB/s, the rate of a large copy (31 us where they are still in the
// cache behind the L2s; with runs of 64 labels to a wavefront 41, and 33).
// The scale is the conversion's operand, so that every weight is what usl_dequantize_mx4 makes of it and the sums have usl_forward's range (sums of codes, scaled at the
// end, do not).  It comes with its piece; where that is six loads already (APART), a label's scale is loaded a turn ahead by the lane that ends with its sum, and
// handed to the others by a permutation (m = 500k, d = 32k, k = 30, b = 1, bfloat16: 19.4 us, with a load a piece 21.1; k = 32, with it, 13.6).
#pragma once
#include "k_products_common.h"

namespace usl_products {

enum Mx4Slots { MX4_ALL_SLOTS, MX4_FOURS, MX4_ANY_SLOTS };   // k = 4 LPL; k a multiple of 4; any k

// AHEAD: rounds in flight, a divisor of LPL
template <int LPL, typename TS, int Q, Mx4Slots SLOTS, int AHEAD>
__global__ void __launch_bounds__(1024)
k_mx4_few(const char* __restrict__ xi, const int32_t* __restrict__ idx, const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
          float* __restrict__ out, int64_t m, int k_, int b, int row_bytes) {
    typedef typename Unit<TS, Q>::T U;
    constexpr int R = 64 / LPL;              // labels of a round
    constexpr bool APART = SLOTS == MX4_ANY_SLOTS && LPL <= 8;
    extern __shared__ __align__(16) unsigned char lds_raw[];
    const uint32_t lds0 = lds_base(lds_raw);
    const int k = SLOTS == MX4_ALL_SLOTS ? 4 * LPL : k_, words = mx4_words(k), blocks = mx4_blocks(k);
    const int nw = (int)blockDim.x >> 6;
    stage_async(xi, lds0, row_bytes, (int)threadIdx.x, (int)blockDim.x);
    const int lane = threadIdx.x & 63, sub = lane & (LPL - 1), t = sub * 4;
    // what a slot that does not exist reads: a unit of zeros behind the row
    const uint32_t nowhere = (uint32_t)row_bytes / (uint32_t)sizeof(U);
    if (threadIdx.x < 4) reinterpret_cast<uint32_t*>(lds_raw)[(uint32_t)row_bytes / 4 + threadIdx.x] = 0u;
    const uint32_t col_at = (uint32_t)((lane / LPL) * k + (t < k ? t : 0)) * 4u;
    const uint32_t word_at = (uint32_t)((lane / LPL) * words + min(t >> 3, words - 1)) * 4u;
    const uint32_t scale_at = (uint32_t)((lane / LPL) * blocks + min(t / MX4_BLOCK, blocks - 1));
    uint32_t any_at[4];
    if (SLOTS == MX4_ANY_SLOTS) {
#pragma unroll
        for (int q = 0; q < 4; ++q) any_at[q] = (uint32_t)((lane / LPL) * k + min(t + q, k - 1)) * 4u;
    }
    struct Piece { uint32_t c[4], w, s; };
    auto fetch = [&](int64_t j, Piece& p) {   // j: first label of a round
        const char* cols = reinterpret_cast<const char*>(idx + j * k);
        if constexpr (SLOTS == MX4_ANY_SLOTS) {
#pragma unroll
            for (int q = 0; q < 4; ++q) p.c[q] = *reinterpret_cast<const uint32_t*>(cols + any_at[q]);
        } else {
            const uint4 c = *reinterpret_cast<const uint4*>(cols + col_at);
            p.c[0] = c.x; p.c[1] = c.y; p.c[2] = c.z; p.c[3] = c.w;
        }
        p.w = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(codes + j * words) + word_at);
        if (!APART) p.s = (scales + j * blocks)[scale_at];
    };
    auto dot4 = [&](const Piece& p, float scale, float (&acc)[Q]) {
        U v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = lds_read<U>(lds0 + (SLOTS != MX4_ALL_SLOTS && t + q >= k ? nowhere : p.c[q]) * (uint32_t)sizeof(U));
        const uint32_t half = p.w >> (16 * (sub & 1));
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
            if constexpr (sizeof(TS) == 4) {
                const f32x2 w = q ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(half, scale, 1) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(half, scale, 0);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if constexpr (Q == 1) acc[0] = fmaf(w[u], v[q + u], acc[0]);
                    else {
#pragma unroll
                        for (int i = 0; i < Q; ++i) acc[i] = fmaf(w[u], v[q + u][i], acc[i]);
                    }
                }
            } else {
                const uint32_t w = __builtin_bit_cast(uint32_t, q ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(half, scale, 1)
                                                                 : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(half, scale, 0));
                if constexpr (Q == 1) acc[0] = dot2((uint32_t)v[q] | ((uint32_t)v[q + 1] << 16), w, acc[0]);
                else if constexpr (Q == 2) {
                    acc[0] = dot2(join_lo(v[q], v[q + 1]), w, acc[0]);
                    acc[1] = dot2(join_hi(v[q], v[q + 1]), w, acc[1]);
                } else {
                    acc[0] = dot2(join_lo(v[q].x, v[q + 1].x), w, acc[0]);
                    acc[1] = dot2(join_hi(v[q].x, v[q + 1].x), w, acc[1]);
                    acc[2] = dot2(join_lo(v[q].y, v[q + 1].y), w, acc[2]);
                    acc[3] = dot2(join_hi(v[q].y, v[q + 1].y), w, acc[3]);
                }
            }
        }
    };
    const int64_t waves = (int64_t)gridDim.x * nw, wave = (int64_t)blockIdx.x * nw + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int rounds = (int)((m + waves * R - 1) / (waves * R));
    auto first_of = [&](int round) { return min((round * waves + wave) * R, m - R); };
    auto mine_of = [&](int r0) { return min(((r0 + sub) * waves + wave) * R, m - R) + lane / LPL; };   // the label whose sum this lane ends with, of rounds r0 ... r0 + LPL - 1
    uint32_t next = 127u;
    if (APART) next = scales[mine_of(0)];
    Piece p[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) fetch(first_of(a), p[a]);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int r0 = 0; r0 < rounds; r0 += LPL) {
        const float held = mx4_scale(next);
        if (APART) next = scales[mine_of(r0 + LPL)];
        float sum[Q] = {};
#pragma unroll 1
        for (int r1 = 0; r1 < LPL && r0 + r1 < rounds; r1 += AHEAD) {
#pragma unroll
            for (int a = 0; a < AHEAD; ++a) {
                float acc[Q] = {};
                dot4(p[a], APART ? __int_as_float(__builtin_amdgcn_ds_bpermute(((lane & ~(LPL - 1)) + r1 + a) * 4, __float_as_int(held))) : mx4_scale(p[a].s), acc);
                fetch(first_of(r0 + r1 + a + AHEAD), p[a]);   // (behind the last round: the last labels again, and nothing is made of them)
#pragma unroll
                for (int i = 0; i < Q; ++i) {   // (lanes that have been added up are alike: a mirror reaches the others as well)
                    if (LPL > 1) acc[i] += moved<0xB1>(acc[i]);    // quads 1 0 3 2
                    if (LPL > 2) acc[i] += moved<0x4E>(acc[i]);    // quads 2 3 0 1
                    if (LPL > 4) acc[i] += moved<0x141>(acc[i]);   // 8 lanes, mirrored
                    if (LPL > 8) acc[i] += moved<0x140>(acc[i]);   // 16
                }
#pragma unroll
                for (int i = 0; i < Q; ++i) sum[i] = sub == r1 + a ? acc[i] : sum[i];
            }
        }
        if (r0 + sub < rounds) {
            const int64_t mine = mine_of(r0);
#pragma unroll
            for (int i = 0; i < Q; ++i)
                if (i < b) out[(size_t)i * m + mine] = sum[i];
        }
    }
}

}  // namespace usl_products
