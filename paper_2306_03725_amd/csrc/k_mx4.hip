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
// Nearest code of v, a half between two magnitudes to the one with the even mantissa, beyond 6 to 6.
__device__ __forceinline__ uint32_t mx4_nearest(float v) {
    const float a = fabsf(v);
    const uint32_t em = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
    return em | (__float_as_uint(v) >> 28 & 8u);
}

// a lane a block
template <typename TS>
__global__ void __launch_bounds__(256)
k_mx4_quantize(const TS* __restrict__ W, uint32_t* __restrict__ codes, uint8_t* __restrict__ scales, int64_t m, int k) {
    const int nb = mx4_blocks(k), nw = mx4_words(k);
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= m * nb) return;
    const int64_t j = at / nb;
    const int blk = (int)(at - j * nb), t0 = blk * MX4_BLOCK, t1 = min(k, t0 + MX4_BLOCK);
    uint32_t amax = 0;
    for (int t = t0; t < t1; ++t) amax = max(amax, __float_as_uint(usl_load_f32<TS>(W, (size_t)j * k + t)) & 0x7FFFFFFFu);
    const uint32_t byte = mx4_scale_byte(amax);
    scales[at] = (uint8_t)byte;
    const float inv = byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23);   // 2^(127 - byte), exact
    for (int t = t0; t < t1; t += 8) {
        uint32_t word = 0;
        for (int q = 0; q < 8 && t + q < t1; ++q) word |= (byte == 255u ? 0u : mx4_nearest(usl_load_f32<TS>(W, (size_t)j * k + t + q) * inv)) << (4 * q);
        codes[j * nw + t / 8] = word;
    }
}

// a lane a word
template <typename TS>
__global__ void __launch_bounds__(256)
k_mx4_dequantize(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales, TS* __restrict__ W, int64_t m, int k) {
    const int nb = mx4_blocks(k), nw = mx4_words(k);
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= m * nw) return;
    const int64_t j = at / nw;
    const int t0 = (int)(at - j * nw) * 8;
    const uint32_t word = codes[at];
    const float scale = mx4_scale(scales[j * nb + t0 / MX4_BLOCK]);
    for (int q = 0; q < 8 && t0 + q < k; ++q) {
        const float v = mx4_code(word >> (4 * q)) * scale;
        if constexpr (sizeof(TS) == 4) W[j * k + t0 + q] = v;
        else W[j * k + t0 + q] = usl_f32_to_bf16(v);   // exact: a 4-bit number has fewer bits, and the scale is a power of two
    }
}

// out[i][j] = sum over the label's blocks of scale * sum over its slots of code * x[i][idx[j][t]].  Any k, any d: a lane a label, activations from memory.
template <typename TS>
__global__ void __launch_bounds__(256)
k_mx4_forward_any(const TS* __restrict__ x, const int32_t* __restrict__ idx, const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                  float* __restrict__ out, int64_t m, int d, int k, int b, int inst) {
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= m) return;
    const int nb = mx4_blocks(k), nw = mx4_words(k), i0 = blockIdx.y * inst, i1 = min(b, i0 + inst);
    for (int i = i0; i < i1; ++i) {
        const TS* row = x + (size_t)i * d;
        float sum = 0.f;
        for (int blk = 0; blk < nb; ++blk) {
            const int t0 = blk * MX4_BLOCK, t1 = min(k, t0 + MX4_BLOCK);
            float acc = 0.f;
            for (int t = t0; t < t1; ++t)
                acc = fmaf(mx4_code(codes[j * nw + t / 8] >> (4 * (t % 8))), usl_load_f32<TS>(row, (size_t)idx[j * k + t]), acc);
            sum = fmaf(mx4_scale(scales[j * nb + blk]), acc, sum);
        }
        out[(size_t)i * m + j] = sum;
    }
}

unsigned blocks_of(int64_t lanes) { return (unsigned)((lanes + 255) / 256); }

}  // namespace

usl_status usl_launch_mx4_quantize(usl_ctx* c, const void* W, uint32_t* codes, uint8_t* scales) {
    const unsigned n = blocks_of(c->m * mx4_blocks(c->k));
    if (c->storage == USL_F32) hipLaunchKernelGGL(k_mx4_quantize<float>, dim3(n), dim3(256), 0, c->stream, (const float*)W, codes, scales, c->m, c->k);
    else hipLaunchKernelGGL(k_mx4_quantize<uint16_t>, dim3(n), dim3(256), 0, c->stream, (const uint16_t*)W, codes, scales, c->m, c->k);
    return usl_check_launch(c, "quantize_mx4");
}

usl_status usl_launch_mx4_dequantize(usl_ctx* c, const uint32_t* codes, const uint8_t* scales, void* W) {
    const unsigned n = blocks_of(c->m * mx4_words(c->k));
    if (c->storage == USL_F32) hipLaunchKernelGGL(k_mx4_dequantize<float>, dim3(n), dim3(256), 0, c->stream, codes, scales, (float*)W, c->m, c->k);
    else hipLaunchKernelGGL(k_mx4_dequantize<uint16_t>, dim3(n), dim3(256), 0, c->stream, codes, scales, (uint16_t*)W, c->m, c->k);
    return usl_check_launch(c, "dequantize_mx4");
}

usl_status usl_launch_forward_mx4(usl_ctx* c, const void* x, const int32_t* idx, const uint32_t* codes, const uint8_t* scales, float* out, int32_t b) {
    const int64_t nblk = (c->m + 255) / 256;
    int parts = (int)((c->num_cu * 8 + nblk - 1) / nblk);
    if (parts > b) parts = b;
    const int inst = (b + parts - 1) / parts;
    const dim3 grid((unsigned)nblk, (unsigned)((b + inst - 1) / inst));
    if (c->storage == USL_F32)
        hipLaunchKernelGGL(k_mx4_forward_any<float>, grid, dim3(256), 0, c->stream, (const float*)x, idx, codes, scales, out, c->m, c->d, c->k, b, inst);
    else
        hipLaunchKernelGGL(k_mx4_forward_any<uint16_t>, grid, dim3(256), 0, c->stream, (const uint16_t*)x, idx, codes, scales, out, c->m, c->d, c->k, b, inst);
    return usl_check_launch(c, "forward_mx4");
}
