// Products in 8-bit integers with a scale for each row of both operands: quantisation, one projection, the gated block (k_dense_forward.h).
// Sums are exact in 32 bits: 127 * 127 * 65536 < 2^31.
#include "k_dense_forward.h"

using namespace dense;

namespace {

constexpr int Q_NT = 256;
constexpr int64_t Q_ROWS = 1 << 22;   // of a launch: it takes less than 2^32 work items

// A row to a workgroup: the largest magnitude, then the codes.  scale = max(largest / 127, 2^-126); code = value / scale to the nearest, halves to even.
// A row with an infinity or NaN has NaN as its scale, and codes 0.
template <typename TS>
__global__ void __launch_bounds__(Q_NT)
k_quantize_i8(const TS* __restrict__ rows, int w, int8_t* __restrict__ codes, float* __restrict__ scales) {
    __shared__ uint32_t most[Q_NT / 64];
    const size_t row = blockIdx.x;
    rows += row * (size_t)w;
    codes += row * (size_t)w;
    uint32_t top = 0;   // magnitudes in the order of their bits, NaN and infinity on top
    for (int c = (int)threadIdx.x; c < w; c += Q_NT) top = max(top, __float_as_uint(widen(rows[c])) & 0x7FFFFFFFu);
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q_NT / 64; ++q) top = max(top, most[q]);
    const bool finite = top < 0x7F800000u;
    const float scale = finite ? fmaxf(__fdiv_rn(__uint_as_float(top), 127.f), 0x1p-126f) : __uint_as_float(0x7FC00000u);
    for (int c = (int)threadIdx.x; c < w; c += Q_NT) {
        const float q = finite ? rintf(__fdiv_rn(widen(rows[c]), scale)) : 0.f;
        codes[c] = (int8_t)fminf(fmaxf(q, -127.f), 127.f);
    }
    if (threadIdx.x == 0) scales[row] = scale;
}

template <typename TO>
usl_status product(usl_ctx* c, const Forward& a, int mats, int act, const char* what) {
    if (mats == 1) return launch_forward<int8_t, TO, 1, 0>(c, a, what);
    return act == USL_SILU ? launch_forward<int8_t, TO, 2, 0>(c, a, what) : launch_forward<int8_t, TO, 2, 1>(c, a, what);
}

}  // namespace

usl_status usl_launch_quantize_i8(usl_ctx* c, const void* rows, int64_t n, int32_t w, int8_t* codes, float* scales) {
    const size_t wide = c->storage == USL_F32 ? 4 : 2;
    for (int64_t at = 0; at < n; at += Q_ROWS) {
        const void* from = (const char*)rows + (size_t)at * (size_t)w * wide;
        int8_t* to = codes + (size_t)at * (size_t)w;
        const dim3 grid((unsigned)(n - at < Q_ROWS ? n - at : Q_ROWS)), block(Q_NT);
        if (c->storage == USL_F32) hipLaunchKernelGGL(k_quantize_i8<float>, grid, block, 0, c->stream, (const float*)from, (int)w, to, scales + at);
        else hipLaunchKernelGGL(k_quantize_i8<bf16>, grid, block, 0, c->stream, (const bf16*)from, (int)w, to, scales + at);
        USL_TRY(usl_check_launch(c, "quantize_i8"));
    }
    return USL_OK;
}

usl_status usl_launch_dense_i8(usl_ctx* c, const int8_t* e, const float* e_scales, const int8_t* V0, const float* s0, const int8_t* V1, const float* s1, int32_t w,
                               int32_t act, void* x, int32_t b) {
    Forward a = {};
    a.V[0] = V0; a.V[1] = V1; a.e = e;
    a.V_scale[0] = s0; a.V_scale[1] = s1; a.e_scale = e_scales;
    a.x = x;
    a.d = c->d; a.b = b; a.row_bytes = w;
    const int mats = V1 ? 2 : 1;
    const char* what = V1 ? "gated_block_i8" : "project_i8";
    return c->storage == USL_F32 ? product<float>(c, a, mats, act, what) : product<bf16>(c, a, mats, act, what);
}
