// Rotary positions: one read and one write of the tensor.  angle = position * turns per position, in 64 bits: at position 10^6
// an fp32 product would leave 2^-24 * 10^6 = 0.06 of a turn's last digits; the whole turns go before sin and cos are taken in fp32.
#include "block_ops.h"

namespace vd {
namespace {

__device__ __forceinline__ void sincos_of(const RotaryArgs& a, int b, int t, int pair, float* sn, float* cs) {
    int axis = 0;
    while (axis < a.axes - 1 && pair >= a.axis_end[axis]) ++axis;
    const int64_t pos = a.pos ? (int64_t)a.pos[b * a.pos_batch + t * a.pos_token + axis] : a.first + t;
    const double turns = (double)pos * a.freqs[pair];
    sincospif(2.f * (float)(turns - rint(turns)), sn, cs);
    *sn *= a.amplitude;
    *cs *= a.amplitude;
}

// a block per token; thread-strided over (head, pair or copied channel)
__global__ void __launch_bounds__(256) rotary_kernel(const RotaryArgs a) {
    extern __shared__ float2 turn[];                         // (cos, sin) of the token's pairs
    const int b = (int)(blockIdx.x / a.T), t = (int)(blockIdx.x % a.T), pairs = a.R / 2, work = pairs + a.D - a.R;
    for (int i = threadIdx.x; i < pairs; i += blockDim.x) sincos_of(a, b, t, i, &turn[i].y, &turn[i].x);
    __syncthreads();
    for (int64_t i = threadIdx.x; i < (int64_t)a.H * work; i += blockDim.x) {
        const int h = (int)(i / work), w = (int)(i % work);
        const int64_t x0 = b * a.sx.batch + t * a.sx.token + h * a.sx.head, y0 = b * a.sy.batch + t * a.sy.token + h * a.sy.head;
        if (w < pairs) {
            const int c0 = a.interleaved ? 2 * w : w, c1 = a.interleaved ? 2 * w + 1 : w + pairs;
            const float u = load_as_f32(a.x, a.dtype, x0 + c0), v = load_as_f32(a.x, a.dtype, x0 + c1);
            const float2 cs = turn[w];
            store_from_f32(a.y, a.dtype, y0 + c0, fmaf(u, cs.x, -v * cs.y));
            store_from_f32(a.y, a.dtype, y0 + c1, fmaf(u, cs.y, v * cs.x));
        } else {
            const int c = a.R + w - pairs;
            store_from_f32(a.y, a.dtype, y0 + c, load_as_f32(a.x, a.dtype, x0 + c));
        }
    }
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t s) {
    rotary_kernel<<<(unsigned)(a.B * a.T), 256, a.R / 2 * sizeof(float2), s>>>(a);
    return cudaGetLastError();
}

}  // namespace vd
