// Layer norm of the rows h[b][d] that become the layer's activations x[b][d], and its backward pass:
//   mean = sum_c h / d,  var = sum_c (h - mean)^2 / d,  rstd = (var + eps)^-1/2,  n = (h - mean) rstd,  x = n gamma + beta
//   u = grad_x gamma,  grad_h = rstd (u - mean_c(u) - n mean_c(u n)),  grad_gamma = sum_i grad_x n,  grad_beta = sum_i grad_x
// The deviations are squared around the mean, not the values around zero, so a row far from zero keeps its variance.
#include "usl_internal.h"

namespace {

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

template <typename TS> __device__ __forceinline__ TS stored(float v);
template <> __device__ __forceinline__ float stored<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t stored<uint16_t>(float v) { return usl_f32_to_bf16(v); }   // the one rounding of a result

// ---- any d: a workgroup a row, which it reads once for every sum and once more to write -------------------------
// (Sums in 64 bits: a lane may have thousands of values.)

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

template <typename TS>
__global__ void __launch_bounds__(ANY_NT)
k_norm_grad_any(const float* __restrict__ grad_x, const TS* __restrict__ h, const float* __restrict__ gamma, const float* __restrict__ mean_in,
                const float* __restrict__ rstd_in, float* __restrict__ grad_h, int d) {
    __shared__ double red[ANY_NT / 64];
    const size_t at = (size_t)blockIdx.x * d;
    const float mean = mean_in[blockIdx.x], rstd = rstd_in[blockIdx.x];
    double su = 0.0, sn = 0.0;
    for (int c = threadIdx.x; c < d; c += ANY_NT) {
        const float u = grad_x[at + c] * (gamma ? gamma[c] : 1.f), n = (usl_load_f32<TS>(h, at + c) - mean) * rstd;
        su += u;
        sn += (double)u * n;
    }
    const float mu = (float)(block_sum<ANY_NT>(su, red) / d), mn = (float)(block_sum<ANY_NT>(sn, red) / d);
    for (int c = threadIdx.x; c < d; c += ANY_NT) {
        const float u = grad_x[at + c] * (gamma ? gamma[c] : 1.f), n = (usl_load_f32<TS>(h, at + c) - mean) * rstd;
        grad_h[at + c] = rstd * (u - mu - n * mn);
    }
}

// ---- the sums over the rows ------------------------------------------------------------------------------------
// part[p][0][c] and part[p][1][c]: sums of grad_x n and of grad_x over the rows [p * rows, p * rows + rows).  A lane a column.
template <typename TS>
__global__ void __launch_bounds__(256)
k_norm_columns(const float* __restrict__ grad_x, const TS* __restrict__ h, const float* __restrict__ mean, const float* __restrict__ rstd,
               float* __restrict__ part, int b, int d, int rows) {
    const int c = blockIdx.x * 256 + threadIdx.x, i0 = blockIdx.y * rows, i1 = min(b, i0 + rows);
    if (c >= d) return;
    float sg = 0.f, sb = 0.f;
    for (int i = i0; i < i1; ++i) {
        const float g = grad_x[(size_t)i * d + c];
        sg = fmaf(g, (usl_load_f32<TS>(h, (size_t)i * d + c) - mean[i]) * rstd[i], sg);
        sb += g;
    }
    part[((size_t)blockIdx.y * 2) * d + c] = sg;
    part[((size_t)blockIdx.y * 2 + 1) * d + c] = sb;
}

// ... added up in a fixed order.  grid (columns, 2)
__global__ void __launch_bounds__(256)
k_norm_sum_parts(const float* __restrict__ part, int parts, int d, float* __restrict__ grad_gamma, float* __restrict__ grad_beta) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    float* to = blockIdx.y ? grad_beta : grad_gamma;
    if (c >= d || !to) return;
    float s = 0.f;
    for (int p = 0; p < parts; ++p) s += part[((size_t)p * 2 + blockIdx.y) * d + c];
    to[c] = s;
}

}  // namespace

template <typename TS>
static usl_status norm(usl_ctx* c, const void* h, const float* gamma, const float* beta, float eps, void* x, float* mean, float* rstd, int32_t b) {
    hipLaunchKernelGGL(k_norm_any<TS>, dim3((unsigned)b), dim3(ANY_NT), 0, c->stream, (const TS*)h, gamma, beta, eps, (TS*)x, mean, rstd, c->d);
    return usl_check_launch(c, "layer_norm");
}

usl_status usl_launch_norm(usl_ctx* c, const void* h, const float* gamma, const float* beta, float eps, void* x, float* mean, float* rstd, int32_t b) {
    return c->storage == USL_F32 ? norm<float>(c, h, gamma, beta, eps, x, mean, rstd, b) : norm<uint16_t>(c, h, gamma, beta, eps, x, mean, rstd, b);
}

// Parts that the rows of a batch are summed in: enough for four workgroups to a compute unit, at least 8 rows each.
static int norm_rows_of_part(const usl_ctx* c, int b) {
    const int tiles = (c->d + 255) / 256, want = (c->num_cu * 4 + tiles - 1) / tiles;
    int rows = (b + want - 1) / want;
    return rows < 8 ? 8 : rows;
}

template <typename TS>
static usl_status norm_grad(usl_ctx* c, const float* grad_x, const void* h, const float* gamma, const float* mean, const float* rstd, float* grad_h,
                            float* grad_gamma, float* grad_beta, int32_t b) {
    if (grad_gamma || grad_beta) {
        const int rows = norm_rows_of_part(c, b), parts = (b + rows - 1) / rows;
        const int most = (c->max_b + 7) / 8 < c->num_cu * 4 ? (c->max_b + 7) / 8 : c->num_cu * 4;   // of any batch: no later call grows it
        USL_TRY(usl_reserve(c, (void**)&c->norm_part, &c->norm_part_cap, (size_t)(most > parts ? most : parts) * 2 * c->d * 4));
        const unsigned tiles = (unsigned)((c->d + 255) / 256);
        hipLaunchKernelGGL(k_norm_columns<TS>, dim3(tiles, (unsigned)parts), dim3(256), 0, c->stream, grad_x, (const TS*)h, mean, rstd, c->norm_part, b, c->d, rows);
        hipLaunchKernelGGL(k_norm_sum_parts, dim3(tiles, 2), dim3(256), 0, c->stream, c->norm_part, parts, c->d, grad_gamma, grad_beta);
    }
    hipLaunchKernelGGL(k_norm_grad_any<TS>, dim3((unsigned)b), dim3(ANY_NT), 0, c->stream, grad_x, (const TS*)h, gamma, mean, rstd, grad_h, c->d);
    return usl_check_launch(c, "layer_norm_backward");
}

usl_status usl_launch_norm_grad(usl_ctx* c, const float* grad_x, const void* h, const float* gamma, const float* mean, const float* rstd, float* grad_h,
                                float* grad_gamma, float* grad_beta, int32_t b) {
    return c->storage == USL_F32 ? norm_grad<float>(c, grad_x, h, gamma, mean, rstd, grad_h, grad_gamma, grad_beta, b)
                                 : norm_grad<uint16_t>(c, grad_x, h, gamma, mean, rstd, grad_h, grad_gamma, grad_beta, b);
}
