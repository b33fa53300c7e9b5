// Gated residual add and modulated norm in one pass over a token's channels: x and h are read once, x_out and y written once.
// A token's r stays in registers between its statistics and its use; the variance is that of the centred values (two
// reductions), so a large common offset does not cancel.
// Bound by HBM: 12 bytes per channel with an fp32 stream and bf16 blocks.  TPR threads share a token, NV vectors of V channels each; all
// of a token's loads are under way before the first sum.  x, h and the outputs pass L1 by; the rows of gate, scale and shift and
// the weights, which the tokens of a frame share, are read through it.  21600 tokens of 1920: 498 MB in 86.7 us, 5.75 TB/s of the 6.6 that a copy
// reaches; what is left are a block's two sums, during which it loads nothing (a persistent block that loads the next token meanwhile has
// fewer blocks beside it: 122 us instead of 96).
#include "block_ops.h"

namespace vd {
namespace {

constexpr int MAX_CHANNELS = 16384;

template <typename T, int V> struct Raw;                     // V channels as they lie in memory
template <> struct Raw<float, 8> { float4 a, b; };
template <> struct Raw<__nv_bfloat16, 8> { uint4 a; };
template <> struct Raw<float, 2> { float2 a; };
template <> struct Raw<__nv_bfloat16, 2> { uint32_t a; };
template <> struct Raw<float, 1> { float a; };
template <> struct Raw<__nv_bfloat16, 1> { unsigned short a; };

__device__ __forceinline__ void get_stream(Raw<float, 8>& r, const float* p) { r.a = __ldcs((const float4*)p); r.b = __ldcs((const float4*)p + 1); }
__device__ __forceinline__ void get_stream(Raw<__nv_bfloat16, 8>& r, const __nv_bfloat16* p) { r.a = __ldcs((const uint4*)p); }
__device__ __forceinline__ void get_stream(Raw<float, 2>& r, const float* p) { r.a = __ldcs((const float2*)p); }
__device__ __forceinline__ void get_stream(Raw<__nv_bfloat16, 2>& r, const __nv_bfloat16* p) { r.a = __ldcs((const uint32_t*)p); }
__device__ __forceinline__ void get_stream(Raw<float, 1>& r, const float* p) { r.a = __ldcs(p); }
__device__ __forceinline__ void get_stream(Raw<__nv_bfloat16, 1>& r, const __nv_bfloat16* p) { r.a = __ldcs((const unsigned short*)p); }
__device__ __forceinline__ void get(Raw<float, 8>& r, const float* p) { r.a = *(const float4*)p; r.b = *((const float4*)p + 1); }
__device__ __forceinline__ void get(Raw<__nv_bfloat16, 8>& r, const __nv_bfloat16* p) { r.a = *(const uint4*)p; }
__device__ __forceinline__ void get(Raw<float, 2>& r, const float* p) { r.a = *(const float2*)p; }
__device__ __forceinline__ void get(Raw<__nv_bfloat16, 2>& r, const __nv_bfloat16* p) { r.a = *(const uint32_t*)p; }
__device__ __forceinline__ void get(Raw<float, 1>& r, const float* p) { r.a = *p; }
__device__ __forceinline__ void get(Raw<__nv_bfloat16, 1>& r, const __nv_bfloat16* p) { r.a = *(const unsigned short*)p; }

__device__ __forceinline__ void up(const Raw<float, 8>& r, float (&f)[8]) {
    f[0] = r.a.x; f[1] = r.a.y; f[2] = r.a.z; f[3] = r.a.w; f[4] = r.b.x; f[5] = r.b.y; f[6] = r.b.z; f[7] = r.b.w;
}
__device__ __forceinline__ void up(const Raw<__nv_bfloat16, 8>& r, float (&f)[8]) {
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void up(const Raw<float, 2>& r, float (&f)[2]) { f[0] = r.a.x; f[1] = r.a.y; }
__device__ __forceinline__ void up(const Raw<__nv_bfloat16, 2>& r, float (&f)[2]) { f[0] = __uint_as_float(r.a << 16); f[1] = __uint_as_float(r.a & 0xffff0000u); }
__device__ __forceinline__ void up(const Raw<float, 1>& r, float (&f)[1]) { f[0] = r.a; }
__device__ __forceinline__ void up(const Raw<__nv_bfloat16, 1>& r, float (&f)[1]) { f[0] = __uint_as_float((uint32_t)r.a << 16); }

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&t);
}
__device__ __forceinline__ void put(float* p, const float (&f)[8]) {
    *(float4*)p = make_float4(f[0], f[1], f[2], f[3]);
    *((float4*)p + 1) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void put(__nv_bfloat16* p, const float (&f)[8]) {
    *(uint4*)p = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}
__device__ __forceinline__ void put(float* p, const float (&f)[2]) { *(float2*)p = make_float2(f[0], f[1]); }
__device__ __forceinline__ void put(__nv_bfloat16* p, const float (&f)[2]) { *(uint32_t*)p = pack2(f[0], f[1]); }
__device__ __forceinline__ void put(float* p, const float (&f)[1]) { *p = f[0]; }
__device__ __forceinline__ void put(__nv_bfloat16* p, const float (&f)[1]) { *p = __float2bfloat16_rn(f[0]); }

// the sum over the TPR threads of a token; `red`: one of two areas in turn, so that one barrier per sum is enough
template <int TPR>
__device__ __forceinline__ float token_sum(float v, float (*red)[TPR / 32], int& turn) {
#pragma unroll
    for (int x = 16; x; x >>= 1) v += __shfl_xor_sync(0xffffffffu, v, x);
    if (TPR == 32) return v;
    float* area = red[turn];
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) area[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 32; ++i) s += area[i];
    return s;
}

template <int V, int TPR, int NV>
__device__ __forceinline__ void unit(float (&z)[NV][V], int C, int lane, int norm, float eps, float (*red)[TPR / 32], int& turn) {
    const float n = (float)C;                                // (divided by, not multiplied with its reciprocal: a token of one value has that mean)
    if (norm == VD_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) s += z[i][e];        // (zeros beyond the last channel)
        const float mean = token_sum<TPR>(s, red, turn) / n;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) z[i][e] = (lane + i * TPR) * V < C ? z[i][e] - mean : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) q = fmaf(z[i][e], z[i][e], q);
    const float rstd = rsqrtf(token_sum<TPR>(q, red, turn) / n + eps);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) z[i][e] *= rstd;
}

// XT: the residual stream; HT: h, y, gate, scale and shift.  (Nine blocks of 128 threads to an SM where a thread has vectors of 8: 21600 tokens
// of 1920 as the compiler likes it 90 us, eight blocks; nine 86.7; ten 90.)
template <typename XT, typename HT, int V, int TPR, int NV>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, V == 8 && TPR == 128 ? 9 : 0) gate_norm_kernel(const GateNormArgs a) {
    constexpr int TOKENS = TPR < 128 ? 128 / TPR : 1;        // of a block; a token of several warps has the block to itself
    static_assert(TPR == 32 || TPR >= 128, "");
    __shared__ float red[2][TPR / 32];
    const vd_gate_norm_desc& d = a.d;
    const uint32_t token = blockIdx.x * TOKENS + (TOKENS > 1 ? threadIdx.x / TPR : 0), all = (uint32_t)d.batch * (uint32_t)d.tokens;    // (below 2^31)
    if (token >= all) return;                                // (whole warps)
    const int lane = TOKENS > 1 ? threadIdx.x % TPR : threadIdx.x;
    const int b = (int)(token / (uint32_t)d.tokens), t = (int)(token - (uint32_t)b * (uint32_t)d.tokens), C = d.channels,
              group = (int)((uint32_t)t / (uint32_t)d.mod_tokens);
    const XT* x = (const XT*)a.x + b * d.x_batch + t * d.x_token;
    const HT* h = (const HT*)a.h + b * d.h_batch + t * d.h_token;
    int turn = 0;
    float r[NV][V];
    Raw<XT, V> rx[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((lane + i * TPR) * V < C) get_stream(rx[i], x + (lane + i * TPR) * V);
    if (a.h) {
        Raw<HT, V> rh[NV], rg[NV];
        const HT* gate = (const HT*)a.gate + b * d.gate_batch + group * d.gate_group;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((lane + i * TPR) * V < C) get_stream(rh[i], h + (lane + i * TPR) * V);
        if (a.gate)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if ((lane + i * TPR) * V < C) get(rg[i], gate + (lane + i * TPR) * V);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((lane + i * TPR) * V < C) up(rh[i], r[i]);
            else
#pragma unroll
                for (int e = 0; e < V; ++e) r[i][e] = 0.f;
        }
        if (d.post_norm) {
            unit<V, TPR, NV>(r, C, lane, d.norm, d.eps, red, turn);
            if (a.post_weight)
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if ((lane + i * TPR) * V < C) {
                        Raw<float, V> w;
                        float f[V];
                        get(w, a.post_weight + (lane + i * TPR) * V);
                        up(w, f);
#pragma unroll
                        for (int e = 0; e < V; ++e) r[i][e] *= f[e];
                    }
        }
        if (a.gate)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if ((lane + i * TPR) * V < C) {
                    float f[V];
                    up(rg[i], f);
#pragma unroll
                    for (int e = 0; e < V; ++e) r[i][e] *= f[e];
                }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((lane + i * TPR) * V < C) {
                float f[V];
                up(rx[i], f);
#pragma unroll
                for (int e = 0; e < V; ++e) r[i][e] = fmaf(d.residual_scale, r[i][e], f[e]);
            }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((lane + i * TPR) * V < C) up(rx[i], r[i]);
            else
#pragma unroll
                for (int e = 0; e < V; ++e) r[i][e] = 0.f;
        }
    }
    if (a.x_out) {
        XT* xo = (XT*)a.x_out + b * d.xo_batch + t * d.xo_token;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((lane + i * TPR) * V < C) put(xo + (lane + i * TPR) * V, r[i]);
    }
    if (!a.y) return;
    // the modulation's loads are under way during the sums
    Raw<HT, V> rs[NV], rt[NV];
    const HT* scale = (const HT*)a.scale + b * d.scale_batch + group * d.scale_group;
    const HT* shift = (const HT*)a.shift + b * d.shift_batch + group * d.shift_group;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((lane + i * TPR) * V < C) {
            if (a.scale) get(rs[i], scale + (lane + i * TPR) * V);
            if (a.shift) get(rt[i], shift + (lane + i * TPR) * V);
        }
    unit<V, TPR, NV>(r, C, lane, d.norm, d.eps, red, turn);
    HT* y = (HT*)a.y + b * d.y_batch + t * d.y_token;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((lane + i * TPR) * V < C) {
            float f[V];
            Raw<float, V> w;
            if (a.weight) {
                get(w, a.weight + (lane + i * TPR) * V);
                up(w, f);
#pragma unroll
                for (int e = 0; e < V; ++e) r[i][e] *= f[e];
            }
            if (a.bias) {
                get(w, a.bias + (lane + i * TPR) * V);
                up(w, f);
#pragma unroll
                for (int e = 0; e < V; ++e) r[i][e] += f[e];
            }
            if (a.scale) {
                up(rs[i], f);
#pragma unroll
                for (int e = 0; e < V; ++e) r[i][e] = fmaf(r[i][e], f[e], r[i][e]);
            }
            if (a.shift) {
                up(rt[i], f);
#pragma unroll
                for (int e = 0; e < V; ++e) r[i][e] += f[e];
            }
            put(y + (lane + i * TPR) * V, r[i]);
        }
}

// h, y and the modulation in types of their own: one channel at a time, types looked at per access, 32 slots of 512 threads whatever the width
// (fp32 modulation of bf16 blocks, fp32 stream: 21600 x 1920 1410 us, with a bf16 modulation 87; 2700 x 16384 1082 and 140)
constexpr int MIXED_THREADS = 512, MIXED_PER = MAX_CHANNELS / MIXED_THREADS;
__global__ void __launch_bounds__(MIXED_THREADS) gate_norm_mixed_kernel(const GateNormArgs a) {
    __shared__ float red[2][MIXED_THREADS / 32];
    const vd_gate_norm_desc& d = a.d;
    const int b = (int)(blockIdx.x / d.tokens), t = (int)(blockIdx.x % d.tokens), C = d.channels, group = t / d.mod_tokens, tid = threadIdx.x;
    const int64_t x0 = b * d.x_batch + t * d.x_token, h0 = b * d.h_batch + t * d.h_token, xo0 = b * d.xo_batch + t * d.xo_token,
                  y0 = b * d.y_batch + t * d.y_token, g0 = b * d.gate_batch + group * d.gate_group,
                  sc0 = b * d.scale_batch + group * d.scale_group, sh0 = b * d.shift_batch + group * d.shift_group;
    int turn = 0;
    float r[MIXED_PER][1];
#pragma unroll
    for (int i = 0; i < MIXED_PER; ++i) r[i][0] = a.h && tid + i * MIXED_THREADS < C ? load_as_f32(a.h, d.h_dtype, h0 + tid + i * MIXED_THREADS) : 0.f;
    if (d.post_norm) unit<1, MIXED_THREADS, MIXED_PER>(r, C, tid, d.norm, d.eps, red, turn);
#pragma unroll
    for (int i = 0; i < MIXED_PER; ++i) {
        const int c = tid + i * MIXED_THREADS;
        if (c >= C) continue;
        float u = r[i][0];
        if (a.post_weight) u *= a.post_weight[c];
        if (a.gate) u *= load_as_f32(a.gate, d.mod_dtype, g0 + c);
        const float x = load_as_f32(a.x, d.x_dtype, x0 + c);
        r[i][0] = a.h ? fmaf(d.residual_scale, u, x) : x;
        if (a.x_out) store_from_f32(a.x_out, d.x_dtype, xo0 + c, r[i][0]);
    }
    if (!a.y) return;
    unit<1, MIXED_THREADS, MIXED_PER>(r, C, tid, d.norm, d.eps, red, turn);
#pragma unroll
    for (int i = 0; i < MIXED_PER; ++i) {
        const int c = tid + i * MIXED_THREADS;
        if (c >= C) continue;
        float y = r[i][0];
        if (a.weight) y *= a.weight[c];
        if (a.bias) y += a.bias[c];
        if (a.scale) y = fmaf(y, load_as_f32(a.scale, d.mod_dtype, sc0 + c), y);
        if (a.shift) y += load_as_f32(a.shift, d.mod_dtype, sh0 + c);
        store_from_f32(a.y, d.y_dtype, y0 + c, y);
    }
}

template <typename XT, typename HT, int V, int TPR, int NV> cudaError_t launch(const GateNormArgs& a, cudaStream_t s) {
    constexpr int threads = TPR < 128 ? 128 : TPR;
    const int64_t tokens = (int64_t)a.d.batch * a.d.tokens, per = threads / TPR;
    gate_norm_kernel<XT, HT, V, TPR, NV><<<(unsigned)((tokens + per - 1) / per), threads, 0, s>>>(a);
    return cudaGetLastError();
}

template <typename XT, typename HT> cudaError_t launch_typed(const GateNormArgs& a, cudaStream_t s) {
    const vd_gate_norm_desc& d = a.d;
    const int C = d.channels;
    // 16-byte accesses everywhere?
    const int xs = sizeof(XT), hs = sizeof(HT);
    uint64_t at = (uintptr_t)a.x | (uintptr_t)a.h | (uintptr_t)a.gate | (uintptr_t)a.x_out | (uintptr_t)a.weight | (uintptr_t)a.bias |
                  (uintptr_t)a.post_weight | (uintptr_t)a.scale | (uintptr_t)a.shift | (uintptr_t)a.y;
    at |= (uint64_t)((d.x_batch | d.x_token | (a.x_out ? d.xo_batch | d.xo_token : 0)) * xs);
    at |= (uint64_t)((a.h ? d.h_batch | d.h_token : 0) * hs) | (uint64_t)((a.y ? d.y_batch | d.y_token : 0) * hs);
    at |= (uint64_t)((a.gate ? d.gate_batch | d.gate_group : 0) * hs) | (uint64_t)((a.scale ? d.scale_batch | d.scale_group : 0) * hs) |
          (uint64_t)((a.shift ? d.shift_batch | d.shift_group : 0) * hs);
    if (C % 8 == 0 && at % 16 == 0) {
        const int vecs = C / 8;
        if (vecs <= 32) return launch<XT, HT, 8, 32, 1>(a, s);
        if (vecs <= 64) return launch<XT, HT, 8, 32, 2>(a, s);
        if (vecs <= 128) return launch<XT, HT, 8, 128, 1>(a, s);
        if (vecs <= 256) return launch<XT, HT, 8, 128, 2>(a, s);
        if (vecs <= 512) return launch<XT, HT, 8, 256, 2>(a, s);
        if (vecs <= 1024) return launch<XT, HT, 8, 512, 2>(a, s);
        return launch<XT, HT, 8, 512, 4>(a, s);
    }
    const uint64_t even = d.x_batch | d.x_token | (a.x_out ? d.xo_batch | d.xo_token : 0) | (a.h ? d.h_batch | d.h_token : 0) |
                          (a.y ? d.y_batch | d.y_token : 0) | (a.gate ? d.gate_batch | d.gate_group : 0) |
                          (a.scale ? d.scale_batch | d.scale_group : 0) | (a.shift ? d.shift_batch | d.shift_group : 0);
    const uint64_t x_at = (uintptr_t)a.x | (uintptr_t)a.x_out, f_at = (uintptr_t)a.weight | (uintptr_t)a.bias | (uintptr_t)a.post_weight,
                   h_at = (uintptr_t)a.h | (uintptr_t)a.y | (uintptr_t)a.gate | (uintptr_t)a.scale | (uintptr_t)a.shift;
    if (C % 2 == 0 && even % 2 == 0 && x_at % (2 * xs) == 0 && h_at % (2 * hs) == 0 && f_at % 8 == 0) {
        // (920 tokens of 4436, bf16, norms on both sides: one channel at a time 49 us, two 21.)  The fewest threads and then the fewest slots that hold a
        // token, against the next step, us, 6.4 million values, norms on both sides, fp32 (bf16): 254 channels 24.8 / 49.6 (24.0 / 52.2), 1022 26.5 / 32.9
        // (24.7 / 32.4), 2046 26.8 / 41.2 (25.6 / 41.2), 4098 30.2 / 44.6 (28.0 / 44.6), 5118 30.5 / 39.9 (28.3 / 39.2), 8190 37.1 / 42.3 (35.2 / 42.4)
        const int n = C / 2;
        if (n <= 128) return launch<XT, HT, 2, 32, 4>(a, s);
        if (n <= 512) return launch<XT, HT, 2, 128, 4>(a, s);
        if (n <= 1024) return launch<XT, HT, 2, 256, 4>(a, s);
        if (n <= 2560) return launch<XT, HT, 2, 512, 5>(a, s);
        if (n <= 4096) return launch<XT, HT, 2, 512, 8>(a, s);
        return launch<XT, HT, 2, 512, MAX_CHANNELS / 1024>(a, s);
    }
    // One channel at a time: the issue slots bound it (600 instructions for a warp's five channels), so few threads with many channels each, the
    // barriers, divisions and addresses being each warp's; but slots that find no channel cost too.  3039 tokens of 1111, fp32, norms on both
    // sides: 256 threads of eight 23.3 us, of five 18.6, 128 of nine 16.9; of 2401: 512 of five 51, 256 of ten 39; of 3501: 512 of seven 60, 256 of 14 62.
    // Each step against the next at the widest token that it takes, us, 6.4 million values, norms on both sides, fp32 (bf16): 127 channels 30.5 / 82.2
    // (29.9 / 86.3), 511 29.4 / 33.0 (29.8 / 33.0), 767 26.9 / 28.9 (27.5 / 30.8), 897 28.0 / 28.9 (29.4 / 30.2), 1151 26.4 / 27.1 (28.6 / 29.0), 1279
    // 26.8 / 28.6 (28.7 / 31.4), 1535 26.8 / 32.9 (31.3 / 32.9), 2047 28.9 / 29.8 (30.3 / 33.1), 2559 28.8 / 39.2 (32.3 / 40.5), 3583 33.1 / 36.8
    // (35.9 / 40.0), 5119 32.1 / 49.3 (36.1 / 54.0), 8191 43.2 / 53.4 (49.4 / 61.7).
    if (C <= 128) return launch<XT, HT, 1, 32, 4>(a, s);
    if (C <= 512) return launch<XT, HT, 1, 128, 4>(a, s);
    if (C <= 768) return launch<XT, HT, 1, 128, 6>(a, s);
    if (C <= 1024) return launch<XT, HT, 1, 128, 8>(a, s);
    if (C <= 1152) return launch<XT, HT, 1, 128, 9>(a, s);
    if (C <= 1280) return launch<XT, HT, 1, 128, 10>(a, s);
    if (C <= 1536) return launch<XT, HT, 1, 128, 12>(a, s);
    if (C <= 2048) return launch<XT, HT, 1, 256, 8>(a, s);
    if (C <= 2560) return launch<XT, HT, 1, 256, 10>(a, s);
    if (C <= 3584) return launch<XT, HT, 1, 512, 7>(a, s);
    if (C <= 5120) return launch<XT, HT, 1, 512, 10>(a, s);
    if (C <= 8192) return launch<XT, HT, 1, 512, 16>(a, s);
    return launch<XT, HT, 1, 512, MAX_CHANNELS / 512>(a, s);
}

}  // namespace

cudaError_t launch_gate_norm(const GateNormArgs& a, cudaStream_t s) {
    const vd_gate_norm_desc& d = a.d;
    const bool mods = a.gate || a.scale || a.shift;
    // the type of h, y and the modulation, as far as they are there
    const int t = a.h ? d.h_dtype : a.y ? d.y_dtype : d.x_dtype;
    if ((a.y && d.y_dtype != t) || (mods && d.mod_dtype != t)) {
        gate_norm_mixed_kernel<<<(unsigned)(d.batch * d.tokens), MIXED_THREADS, 0, s>>>(a);
        return cudaGetLastError();
    }
    if (d.x_dtype == VD_BF16) return t == VD_BF16 ? launch_typed<__nv_bfloat16, __nv_bfloat16>(a, s) : launch_typed<__nv_bfloat16, float>(a, s);
    return t == VD_BF16 ? launch_typed<float, __nv_bfloat16>(a, s) : launch_typed<float, float>(a, s);
}

}  // namespace vd
