// Attention to states of another length, the kernel without restrictions: any head size up to 256, any strides and alignment.
// A warp takes one row (batch item, token, head) and walks the keys one by one, running maximum and sum as in
//   m' = max(m, s),  l' = l 2^(m - m') + 2^(s - m'),  o' = o 2^(m - m') + 2^(s - m') v.
// Lane i holds channels i, i + 32, ... of q and o.  Scores are in units of log 2.  The others are checked against it: nothing is shared with them.
#include "block_ops.h"

namespace vd {
namespace {

constexpr int WARPS = 4, MAX_PER_LANE = 8;

template <typename T> __device__ __forceinline__ float up(T v) { return (float)v; }
template <> __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__global__ void __launch_bounds__(WARPS * 32) xattn_plain_kernel(const XAttnArgs a, float scale_log2) {
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5), rows = (int64_t)a.B * a.Tq * a.H;
    if (row >= rows) return;
    const int h = (int)(row % a.H), b = (int)(row / a.H / a.Tq), t = (int)(row / a.H % a.Tq), kvh = h / (a.H / a.Hkv);
    const T* q = (const T*)a.q + b * a.sq.batch + t * a.sq.token + h * a.sq.head;
    const T* k = (const T*)a.k + b * a.sk.batch + kvh * a.sk.head;
    const T* v = (const T*)a.v + b * a.sv.batch + kvh * a.sv.head;
    T* o = (T*)a.o + b * a.so.batch + t * a.so.token + h * a.so.head;
    const int len = a.kv_lens ? min(max(a.kv_lens[b], 0), a.Tk) : a.Tk;
    float qr[MAX_PER_LANE], acc[MAX_PER_LANE];
#pragma unroll
    for (int i = 0; i < MAX_PER_LANE; ++i) {
        qr[i] = lane + 32 * i < a.D ? up(q[lane + 32 * i]) : 0.f;
        acc[i] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    for (int u = 0; u < len; ++u) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < MAX_PER_LANE; ++i)
            if (lane + 32 * i < a.D) s = fmaf(qr[i], up(k[u * a.sk.token + lane + 32 * i]), s);
#pragma unroll
        for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
        s *= scale_log2;
        const float m2 = fmaxf(m, s), ref = m2 == -INFINITY ? 0.f : m2;     // (a score that is NaN makes the row NaN below)
        const float keep = exp2f(m - ref), p = exp2f(s - ref);
        l = fmaf(l, keep, p);
#pragma unroll
        for (int i = 0; i < MAX_PER_LANE; ++i)
            if (lane + 32 * i < a.D) acc[i] = fmaf(acc[i], keep, p * up(v[u * a.sv.token + lane + 32 * i]));
        m = m2;
    }
    const float inv = len ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < MAX_PER_LANE; ++i)
        if (lane + 32 * i < a.D) o[lane + 32 * i] = (T)(acc[i] * inv);
}

}  // namespace

cudaError_t launch_xattn_plain(const XAttnArgs& a, cudaStream_t s) {
    const int64_t rows = (int64_t)a.B * a.Tq * a.H;
    const dim3 grid((unsigned)((rows + WARPS - 1) / WARPS)), block(WARPS * 32);
    const float scale_log2 = a.scale * 1.4426950408889634f;
    if (a.dtype == VD_BF16) xattn_plain_kernel<__nv_bfloat16><<<grid, block, 0, s>>>(a, scale_log2);
    else xattn_plain_kernel<float><<<grid, block, 0, s>>>(a, scale_log2);
    return cudaGetLastError();
}

}  // namespace vd
