// Rotary positions: one read and one write of the tensor.  angle = position * turns per position, in 64 bits: at position 10^6 an
// fp32 product would leave 0.06 of a turn in doubt; the whole turns go before sin and cos are taken in fp32.
// Bound by HBM.  A token's (cos, sin) are made once, in shared memory, and used by all its heads; a thread owns the same channels of
// several heads, 16 bytes each, whose loads are under way while the table is made.  21600 tokens, 60 heads of 64, bf16: 53.6 us, 6.2 TB/s of the
// 6.6 that a copy reaches.
#include "block_ops.h"

namespace vd {
namespace {

__device__ __forceinline__ float2 turn_of(const RotaryArgs& a, int b, int t, int pair) {
    int axis = 0;
    while (axis < a.axes - 1 && pair >= a.axis_end[axis]) ++axis;
    const int64_t pos = a.pos ? (int64_t)a.pos[b * a.pos_batch + t * a.pos_token + axis] : a.first + t;
    const double turns = (double)pos * a.freqs[pair];
    float sn, cs;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
    return make_float2(cs * a.amplitude, sn * a.amplitude);
}

constexpr int MAX_THREADS = 256, HEADS = 4;                  // HEADS: of a thread, loaded ahead

__device__ __forceinline__ void turn_pair(float& u, float& v, float2 cs) {
    const float x = u;
    u = fmaf(x, cs.x, -v * cs.y);
    v = fmaf(x, cs.y, v * cs.x);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&t);
}
// 16 bytes as V = 8 bf16 or 4 fp32 values
__device__ __forceinline__ void up(const uint4& r, float (&f)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void up(const uint4& r, float (&f)[4]) {
    f[0] = __uint_as_float(r.x); f[1] = __uint_as_float(r.y); f[2] = __uint_as_float(r.z); f[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ uint4 down(const float (&f)[8]) { return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])); }
__device__ __forceinline__ uint4 down(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// blockDim: (units of a head, heads, tokens).  A unit is 16 bytes (HALF: of either half of the turned channels), or 16 copied bytes.
template <typename T, bool HALF>
__global__ void __launch_bounds__(MAX_THREADS) rotary_vec_kernel(const RotaryArgs a) {
    constexpr int V = 16 / sizeof(T);
    extern __shared__ float2 table[];                        // [tokens][pairs]
    const int pairs = a.R / 2, turning = HALF ? pairs / V : a.R / V, unit = threadIdx.x;
    const uint32_t token = blockIdx.x * blockDim.z + threadIdx.z, tokens = (uint32_t)a.B * (uint32_t)a.T;      // (below 2^31)
    const bool here = token < tokens, turns = unit < turning;
    const int b = here ? (int)(token / (uint32_t)a.T) : 0, t = here ? (int)(token % (uint32_t)a.T) : 0;
    const int c = turns ? unit * V : a.R + (unit - turning) * V;
    const T* x = (const T*)a.x + b * a.sx.batch + t * a.sx.token + c;
    T* y = (T*)a.y + b * a.sy.batch + t * a.sy.token + c;
    float2 cs[HALF ? V : V / 2];
    for (int h0 = threadIdx.y; h0 < a.H; h0 += HEADS * (int)blockDim.y) {
        uint4 r0[HEADS], r1[HEADS];
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            const int h = h0 + i * (int)blockDim.y;
            if (here && h < a.H) {
                r0[i] = *(const uint4*)(x + h * a.sx.head);
                if (HALF && turns) r1[i] = *(const uint4*)(x + h * a.sx.head + pairs);
            }
        }
        if (h0 == (int)threadIdx.y) {                        // (every thread has a head: blockDim.y <= H)
            const int n = (int)(blockDim.x * blockDim.y * blockDim.z);
            for (int i = ((int)threadIdx.z * blockDim.y + threadIdx.y) * blockDim.x + threadIdx.x; i < (int)blockDim.z * pairs; i += n) {
                const int z = blockDim.z == 1 ? 0 : i / pairs;
                const uint32_t tk = blockIdx.x * blockDim.z + (uint32_t)z;
                if (tk < tokens) table[i] = turn_of(a, (int)(tk / (uint32_t)a.T), (int)(tk % (uint32_t)a.T), i - z * pairs);
            }
            __syncthreads();
            if (turns)
#pragma unroll
                for (int e = 0; e < (HALF ? V : V / 2); ++e) cs[e] = table[threadIdx.z * pairs + (HALF ? unit * V : unit * V / 2) + e];
        }
#pragma unroll
        for (int i = 0; i < HEADS; ++i) {
            const int h = h0 + i * (int)blockDim.y;
            if (!here || h >= a.H) continue;
            if (turns) {
                float f[V];
                up(r0[i], f);
                if (HALF) {
                    float g[V];
                    up(r1[i], g);
#pragma unroll
                    for (int e = 0; e < V; ++e) turn_pair(f[e], g[e], cs[HALF ? e : 0]);
                    *(uint4*)(y + h * a.sy.head + pairs) = down(g);
                } else {
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) turn_pair(f[2 * e], f[2 * e + 1], cs[e]);
                }
                r0[i] = down(f);
            }
            *(uint4*)(y + h * a.sy.head) = r0[i];
        }
    }
}

// any size and alignment: a block per token; thread-strided over (head, pair or copied channel).  (21600 tokens x 60 heads, bf16: of 40 in halves
// 142 us, of 64 with 20 channels turned 304, of 64 at odd elements 211; in 16-byte pieces 64 takes 52.)
__global__ void __launch_bounds__(MAX_THREADS) rotary_kernel(const RotaryArgs a) {
    extern __shared__ float2 table[];                        // of the token's pairs
    const int b = (int)(blockIdx.x / (uint32_t)a.T), t = (int)(blockIdx.x % (uint32_t)a.T), pairs = a.R / 2, work = pairs + a.D - a.R;
    for (int i = threadIdx.x; i < pairs; i += blockDim.x) table[i] = turn_of(a, b, t, i);
    __syncthreads();
    for (int64_t i = threadIdx.x; i < (int64_t)a.H * work; i += blockDim.x) {
        const int h = (int)(i / work), w = (int)(i % work);
        const int64_t x0 = b * a.sx.batch + t * a.sx.token + h * a.sx.head, y0 = b * a.sy.batch + t * a.sy.token + h * a.sy.head;
        if (w < pairs) {
            const int c0 = a.interleaved ? 2 * w : w, c1 = a.interleaved ? 2 * w + 1 : w + pairs;
            float u = load_as_f32(a.x, a.dtype, x0 + c0), v = load_as_f32(a.x, a.dtype, x0 + c1);
            turn_pair(u, v, table[w]);
            store_from_f32(a.y, a.dtype, y0 + c0, u);
            store_from_f32(a.y, a.dtype, y0 + c1, v);
        } else {
            const int c = a.R + w - pairs;
            store_from_f32(a.y, a.dtype, y0 + c, load_as_f32(a.x, a.dtype, x0 + c));
        }
    }
}

template <typename T> cudaError_t launch_vec(const RotaryArgs& a, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int units = (a.interleaved ? a.R / V : a.R / 2 / V) + (a.D - a.R) / V;
    const int64_t tokens = (int64_t)a.B * a.T;
    // A thread takes HEADS heads where there are tokens enough, and small tokens share a block of 128 threads: many small blocks, each with
    // its loads under way, hide one another's tables (us: 21600 x 60 heads of 64 two heads a thread 82, four 56, eight 55; 8192 x 40 of 128
    // 50, 31, 33; three axes, interleaved, and one, halves).
    const int each = tokens >= 8 * 148 ? HEADS : 1;
    int heads = (a.H + each - 1) / each;
    if (heads > MAX_THREADS / units) heads = MAX_THREADS / units;
    int per = 128 / (units * heads);
    while (per > 1 && (tokens + per - 1) / per < 4 * 148) --per;
    if (per > 16) per = 16;
    if (per < 1) per = 1;
    const dim3 grid((unsigned)((tokens + per - 1) / per)), block(units, heads, per);
    const size_t smem = (size_t)per * (a.R / 2) * sizeof(float2);
    if (a.interleaved) rotary_vec_kernel<T, false><<<grid, block, smem, s>>>(a);
    else rotary_vec_kernel<T, true><<<grid, block, smem, s>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t s) {
    const int size = a.dtype == VD_BF16 ? 2 : 4, V = 16 / size;
    const uint64_t at = (uintptr_t)a.x | (uintptr_t)a.y |
                        (uint64_t)((a.sx.batch | a.sx.token | a.sx.head | a.sy.batch | a.sy.token | a.sy.head) * size);
    // 16 bytes at a time where every unit starts on such a boundary
    if (at % 16 == 0 && a.D % V == 0 && a.R % (a.interleaved ? V : 2 * V) == 0)
        return a.dtype == VD_BF16 ? launch_vec<__nv_bfloat16>(a, s) : launch_vec<float>(a, s);
    rotary_kernel<<<(unsigned)((int64_t)a.B * a.T), MAX_THREADS, a.R / 2 * sizeof(float2), s>>>(a);
    return cudaGetLastError();
}

}  // namespace vd
