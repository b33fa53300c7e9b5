// Internal declarations of the transformer-block operators (vd_block.h).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "vd_block.h"
#include "vd_internal.h"

namespace vd {

struct Strides { int64_t batch, token, head; };

struct XAttnArgs {
    const void* q; const void* k; const void* v; void* o;
    const int32_t* kv_lens;     // [B] or null
    int dtype, B, Tq, Tk, H, Hkv, D;
    Strides sq, sk, sv, so;
    float scale;
};
cudaError_t launch_xattn_plain(const XAttnArgs& a, cudaStream_t s);
bool xattn_rows_supported(const XAttnArgs& a);
cudaError_t launch_xattn_rows(const XAttnArgs& a, cudaStream_t s);
cudaError_t launch_xattn_f32(const XAttnArgs& a, cudaStream_t s);
bool xattn_tc_supported(const XAttnArgs& a);
cudaError_t launch_xattn_tc(const XAttnArgs& a, cudaStream_t s);
struct XAttnDivision { int splits; uint32_t items, whole, grid; };       // the first `whole` items are a CTA's each, the others a cluster's of `splits` CTAs
cudaError_t xattn_tc_division(const XAttnArgs& a, XAttnDivision* d);
void xattn_tc_meeting_limit(long long cycles);

struct RotaryArgs {
    const void* x; void* y;
    const int32_t* pos;         // or null
    const double* freqs;
    int dtype, B, T, H, D, R, interleaved, axes;
    int axis_end[VD_ROTARY_MAX_AXES];       // first pair behind the axis
    float amplitude;
    Strides sx, sy;
    int64_t pos_batch, pos_token, first;
};
cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t s);

struct GateNormArgs {
    vd_gate_norm_desc d;
    const void* x; const void* h; const float* post_weight; const void* gate; void* x_out;
    const float* weight; const float* bias; const void* scale; const void* shift; void* y;
};
cudaError_t launch_gate_norm(const GateNormArgs& a, cudaStream_t s);

#ifdef __CUDACC__
__device__ __forceinline__ float load_as_f32(const void* p, int dtype, int64_t i) {
    return dtype == VD_BF16 ? __bfloat162float(((const __nv_bfloat16*)p)[i]) : ((const float*)p)[i];
}
__device__ __forceinline__ void store_from_f32(void* p, int dtype, int64_t i, float v) {
    if (dtype == VD_BF16) ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v);
    else ((float*)p)[i] = v;
}
#endif

}  // namespace vd
