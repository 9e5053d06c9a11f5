// The layer's values as microscaled 4-bit numbers (k_mx4.h): to them, back, and the scores of a layer that holds them.
#include "k_mx4.h"

namespace {

// Scale byte of a block whose largest magnitude has these bits: 2^(floor(log2 amax) - 2), so that the largest code's magnitudes, 4 to 6, meet it; at
// least 2^-127.  An infinity or a NaN anywhere makes all of the block's values NaN, as one product with it would.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax) {
    if (amax >= 0x7F800000u) return 255u;
    const int e = (int)(amax >> 23) - 2;   // (denormal numbers have exponent field 0, and end at the least scale like all below 2^-124)
    return e < 0 ? 0u : (uint32_t)e;
}

// A lane takes four neighbouring slots of a label; the lanes of a block of 32 slots are neighbours, 8 of them (1, 2 or 4 where a label has 16 slots or
// fewer), so their largest magnitude is found by lane permutations, and two lanes make a word.  ITEMS such pieces of a lane are on their way together.
// Bound by the stream of the values.
constexpr int ITEMS = 2;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));        // a row of k values begins at any of them
typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));

int lanes_of_label(int k) { return k <= 4 ? 1 : k <= 8 ? 2 : k <= 16 ? 4 : mx4_blocks(k) * 8; }

// Piece `item` of this lane: label (m: none) and first slot
struct Pieces {
    int64_t j0, m;
    uint32_t rest, per;   // the workgroup's first piece is number `rest` of label j0; pieces of a label
    __device__ __forceinline__ Pieces(int64_t m_, int per_) : m(m_), per((uint32_t)per_) {
        const int64_t first = (int64_t)blockIdx.x * (256 * ITEMS);
        j0 = first / per_;
        rest = (uint32_t)(first - j0 * per_);
    }
    __device__ __forceinline__ int64_t label(int item, int* slot) const {
        const uint32_t at = rest + (uint32_t)item * 256 + threadIdx.x;
        const uint32_t q = (per & (per - 1)) == 0 ? at >> __builtin_ctz(per) : at / per;
        *slot = (int)(at - q * per) * 4;
        return min(j0 + q, m);
    }
};

template <int CTRL>
__device__ __forceinline__ uint32_t max_of_pair(uint32_t v) {
    const uint32_t t = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
    return t > v ? t : v;
}

// G: lanes of a block; FOURS: k is a multiple of 4.  Loads have no conditions, which the compiler would wait for: a lane whose piece does not exist loads
// another one, and makes nothing of it.
template <typename TS, int G, bool FOURS>
__global__ void __launch_bounds__(256)
k_mx4_quantize(const TS* __restrict__ W, uint32_t* __restrict__ codes, uint8_t* __restrict__ scales, int64_t m, int k, int per) {
    const Pieces pieces(m, per);
    float v[ITEMS][4];
    int64_t label[ITEMS];
    int slot[ITEMS];
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        label[u] = pieces.label(u, &slot[u]);
        const TS* row = W + (size_t)min(label[u], m - 1) * k;
        if constexpr (FOURS && sizeof(TS) == 4) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(row + min(slot[u], k - 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = q[e];
        } else if constexpr (FOURS) {
            const u16x4 q = *reinterpret_cast<const u16x4*>(row + min(slot[u], k - 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = usl_bf16_to_f32(q[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = usl_to_f32(row[min(slot[u] + e, k - 1)]);
        }
    }
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (slot[u] + (FOURS ? 0 : e) >= k) v[u][e] = 0.f;
    }
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        uint32_t amax = 0;   // bits of magnitudes: their order is the numbers', infinities and NaN above
#pragma unroll
        for (int q = 0; q < 4; ++q) amax = max(amax, __float_as_uint(v[u][q]) & 0x7FFFFFFFu);
        if (G > 1) amax = max_of_pair<0xB1>(amax);    // quads 1 0 3 2
        if (G > 2) amax = max_of_pair<0x4E>(amax);    // quads 2 3 0 1
        if (G > 4) amax = max_of_pair<0x141>(amax);   // 8 lanes, mirrored
        const uint32_t byte = mx4_scale_byte(amax);
        const float inv = __uint_as_float((254u - byte) << 23);   // 2^(127 - byte): the products are exact, or far below the least code
        uint32_t half = 0;                                        // (the conversion rounds to nearest even and ends at 6)
        half = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(half, v[u][0] * inv, v[u][1] * inv, 1.f, 0);
        half = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(half, v[u][2] * inv, v[u][3] * inv, 1.f, 1);
        half = byte == 255u ? 0u : half & 0xFFFFu;
        const uint32_t upper = G > 1 ? (uint32_t)__builtin_amdgcn_update_dpp(0, (int)half, 0xB1, 0xF, 0xF, true) : 0u;
        const int t = slot[u];
        if (label[u] >= m) continue;
        if ((t & 7) == 0 && t < k) codes[label[u] * mx4_words(k) + (t >> 3)] = half | upper << 16;
        if ((t & 31) == 0) scales[label[u] * mx4_blocks(k) + t / MX4_BLOCK] = (uint8_t)byte;
    }
}

template <typename TS>
__global__ void __launch_bounds__(256)
k_mx4_dequantize(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, TS* __restrict__ W, int64_t m, int k, int per) {
    const Pieces pieces(m, per);
    uint32_t word[ITEMS], byte[ITEMS];
    int64_t label[ITEMS];
    int slot[ITEMS];
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        label[u] = pieces.label(u, &slot[u]);
        const int64_t j = min(label[u], m - 1);
        word[u] = codes[j * mx4_words(k) + min(slot[u] >> 3, mx4_words(k) - 1)];
        byte[u] = scales[j * mx4_blocks(k) + min(slot[u] / MX4_BLOCK, mx4_blocks(k) - 1)];
    }
#pragma unroll
    for (int u = 0; u < ITEMS; ++u) {
        const int t = slot[u];
        const uint32_t half = word[u] >> (4 * (t & 4));
        const float scale = mx4_scale(byte[u]);
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(half, 1.f, 0), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(half, 1.f, 1);
        const float v[4] = {lo.x * scale, lo.y * scale, hi.x * scale, hi.y * scale};
        if (label[u] >= m) continue;
        TS* to = W + (size_t)label[u] * k + t;
        if (t + 4 <= k) {
            if constexpr (sizeof(TS) == 4) {
                const f32x4 q = {v[0], v[1], v[2], v[3]};
                *reinterpret_cast<f32x4*>(to) = q;
            } else {   // exact: a 4-bit number has fewer bits, and the scale is a power of two
                const u16x4 q = {usl_f32_to_bf16(v[0]), usl_f32_to_bf16(v[1]), usl_f32_to_bf16(v[2]), usl_f32_to_bf16(v[3])};
                *reinterpret_cast<u16x4*>(to) = q;
            }
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (t + q < k) {
                    if constexpr (sizeof(TS) == 4) to[q] = v[q];
                    else to[q] = usl_f32_to_bf16(v[q]);
                }
        }
    }
}

// out[i][j] = sum over the label's slots of value * x[i][idx[j][t]].  Any k, any d (wider than the columns that fit 16 bits, or more than 64 slots): a
// lane a label, activations from memory, AT_ONCE instances for each look at a label's slots.  Bound by the gathers, and by slots read k apart once for every AT_ONCE instances: 100k labels,
// k = 96, d = 32k, b = 64 3.2 ms (usl_forward, which stages rows there, 6.1), b = 1 155 us (98); k = 32, d = 100k, b = 16 0.49 ms (2.1).
constexpr int AT_ONCE = 8;
template <typename TS>
__global__ void __launch_bounds__(256)
k_mx4_forward_any(const TS* __restrict__ x, const int32_t* __restrict__ idx, const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                  float* __restrict__ out, int64_t m, int d, int k, int b) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= m) return;
    const int i0 = (int)blockIdx.y * AT_ONCE;
    float sum[AT_ONCE] = {};
    for (int t = 0; t < k; ++t) {
        const float w = mx4_value(codes, scales, j, t, k);
        const size_t col = (size_t)idx[j * k + t];
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) sum[q] = fmaf(w, usl_load_f32<TS>(x, (size_t)min(i0 + q, b - 1) * d + col), sum[q]);
    }
#pragma unroll
    for (int q = 0; q < AT_ONCE; ++q)
        if (i0 + q < b) out[(size_t)(i0 + q) * m + j] = sum[q];
}

}  // namespace

// m = 500k, k = 32, float32, both calls one after the other: 137 MB in 30.2 us, 4.5 TB/s, where a large copy reaches 5.0.  (A lane a block of 32, its slots
// one after the other, took 544.)
usl_status usl_launch_mx4_quantize(usl_ctx* c, const void* W, uint32_t* codes, uint8_t* scales) {
    const int per = lanes_of_label(c->k);
    const unsigned n = (unsigned)((c->m * per + 256 * ITEMS - 1) / (256 * ITEMS));
#define USL_QUANTIZE_F(TS, G, FOURS) hipLaunchKernelGGL((k_mx4_quantize<TS, G, FOURS>), dim3(n), dim3(256), 0, c->stream, (const TS*)W, codes, scales, c->m, c->k, per)
#define USL_QUANTIZE(TS, G) do { if (c->k % 4 == 0) USL_QUANTIZE_F(TS, G, true); else USL_QUANTIZE_F(TS, G, false); } while (0)
#define USL_QUANTIZE_G(TS)                       \
    do {                                         \
        if (per == 1) USL_QUANTIZE(TS, 1);       \
        else if (per == 2) USL_QUANTIZE(TS, 2);  \
        else if (per == 4) USL_QUANTIZE(TS, 4);  \
        else USL_QUANTIZE(TS, 8);                \
    } while (0)
    if (c->storage == USL_F32) USL_QUANTIZE_G(float);
    else USL_QUANTIZE_G(uint16_t);
#undef USL_QUANTIZE_G
#undef USL_QUANTIZE
#undef USL_QUANTIZE_F
    return usl_check_launch(c, "quantize_mx4");
}

usl_status usl_launch_mx4_dequantize(usl_ctx* c, const uint32_t* codes, const uint8_t* scales, void* W) {
    const int per = lanes_of_label(c->k);
    const unsigned n = (unsigned)((c->m * per + 256 * ITEMS - 1) / (256 * ITEMS));
    if (c->storage == USL_F32) hipLaunchKernelGGL(k_mx4_dequantize<float>, dim3(n), dim3(256), 0, c->stream, codes, scales, (float*)W, c->m, c->k, per);
    else hipLaunchKernelGGL(k_mx4_dequantize<uint16_t>, dim3(n), dim3(256), 0, c->stream, codes, scales, (uint16_t*)W, c->m, c->k, per);
    return usl_check_launch(c, "dequantize_mx4");
}

usl_status usl_launch_forward_mx4_any(usl_ctx* c, const void* x, const int32_t* idx, const uint32_t* codes, const uint8_t* scales, float* out, int32_t b) {
    const dim3 grid((unsigned)((c->m + 255) / 256), (unsigned)((b + AT_ONCE - 1) / AT_ONCE));
    if (c->storage == USL_F32)
        hipLaunchKernelGGL(k_mx4_forward_any<float>, grid, dim3(256), 0, c->stream, (const float*)x, idx, codes, scales, out, c->m, c->d, c->k, b);
    else
        hipLaunchKernelGGL(k_mx4_forward_any<uint16_t>, grid, dim3(256), 0, c->stream, (const uint16_t*)x, idx, codes, scales, out, c->m, c->d, c->k, b);
    return usl_check_launch(c, "forward_mx4");
}
