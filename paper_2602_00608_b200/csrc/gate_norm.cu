// Gated residual add and modulated norm in one pass over a token's channels: x and h are read once, x_out and y written once.
// A token's r stays in registers between its statistics and its use; the variance is that of the centred values (two
// reductions), so a large common offset does not cancel.
#include "block_ops.h"

namespace vd {
namespace {

constexpr int THREADS = 512, PER = 32;                       // channels: up to THREADS * PER

__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
    for (int x = 16; x; x >>= 1) v += __shfl_xor_sync(0xffffffffu, v, x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
    for (int i = 0; i < THREADS / 32; ++i) s += red[i];
    return s;
}

// z -> (z - mean) / sqrt(var + eps) or z / sqrt(mean z^2 + eps)
__device__ __forceinline__ void unit(float (&z)[PER], int C, int norm, float eps, float* red) {
    if (norm == VD_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) if ((int)threadIdx.x + i * THREADS < C) s += z[i];
        const float mean = block_sum(s, red) / (float)C;
#pragma unroll
        for (int i = 0; i < PER; ++i) z[i] -= mean;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) if ((int)threadIdx.x + i * THREADS < C) q = fmaf(z[i], z[i], q);
    const float rstd = 1.f / sqrtf(block_sum(q, red) / (float)C + eps);
#pragma unroll
    for (int i = 0; i < PER; ++i) z[i] *= rstd;
}

__global__ void __launch_bounds__(THREADS) gate_norm_kernel(const GateNormArgs a) {
    __shared__ float red[THREADS / 32];
    const vd_gate_norm_desc& d = a.d;
    const int b = (int)(blockIdx.x / d.tokens), t = (int)(blockIdx.x % d.tokens), C = d.channels, group = t / d.mod_tokens;
    const int64_t x0 = b * d.x_batch + t * d.x_token, h0 = b * d.h_batch + t * d.h_token, xo0 = b * d.xo_batch + t * d.xo_token,
                  y0 = b * d.y_batch + t * d.y_token, g0 = b * d.gate_batch + group * d.gate_group,
                  sc0 = b * d.scale_batch + group * d.scale_group, sh0 = b * d.shift_batch + group * d.shift_group;
    float r[PER];
    if (a.h) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * THREADS;
            r[i] = c < C ? load_as_f32(a.h, d.h_dtype, h0 + c) : 0.f;
        }
        if (d.post_norm) unit(r, C, d.norm, d.eps, red);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int c = threadIdx.x + i * THREADS;
        if (c >= C) continue;
        const float x = load_as_f32(a.x, d.x_dtype, x0 + c);
        if (a.h) {
            float u = r[i];
            if (a.post_weight) u *= a.post_weight[c];
            if (a.gate) u *= load_as_f32(a.gate, d.mod_dtype, g0 + c);
            r[i] = fmaf(d.residual_scale, u, x);
        } else {
            r[i] = x;
        }
    }
    if (a.x_out) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = threadIdx.x + i * THREADS;
            if (c < C) store_from_f32(a.x_out, d.x_dtype, xo0 + c, r[i]);
        }
    }
    if (!a.y) return;
    unit(r, C, d.norm, d.eps, red);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int c = threadIdx.x + i * THREADS;
        if (c >= C) continue;
        float y = r[i];
        if (a.weight) y *= a.weight[c];
        if (a.bias) y += a.bias[c];
        if (a.scale) y *= 1.f + load_as_f32(a.scale, d.mod_dtype, sc0 + c);
        if (a.shift) y += load_as_f32(a.shift, d.mod_dtype, sh0 + c);
        store_from_f32(a.y, d.y_dtype, y0 + c, y);
    }
}

}  // namespace

cudaError_t launch_gate_norm(const GateNormArgs& a, cudaStream_t s) {
    gate_norm_kernel<<<(unsigned)(a.d.batch * a.d.tokens), THREADS, 0, s>>>(a);
    return cudaGetLastError();
}

}  // namespace vd
