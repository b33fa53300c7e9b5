// Tensor maps of bf16 attention operands: 64 channels (128 bytes, swizzled) wide boxes, zeros beyond the tensor.
#pragma once
#include "block_ops.h"
#include "tc_common.cuh"

namespace vd {

inline bool encode_map(CUtensorMap* tm, const void* base, int rank, const uint64_t* dims, const uint64_t* strides_bytes, const uint32_t* box) {
    tc::EncodeTiledFn enc = tc::encode_fn();
    if (!enc) return false;
    cuuint64_t d[5], st[4];
    cuuint32_t bx[5], es[5];
    for (int i = 0; i < rank; ++i) { d[i] = dims[i]; bx[i] = box[i]; es[i] = 1; }
    for (int i = 0; i + 1 < rank; ++i) st[i] = strides_bytes[i];
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d, st, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// bytes between the elements of a dimension; one that is never stepped along gets any valid stride
inline bool stride_ok(int64_t stride, int64_t n, uint64_t* bytes) {
    if (n <= 1) { *bytes = 256; return true; }
    *bytes = (uint64_t)stride * 2;
    return stride > 0 && stride % 8 == 0 && stride < (1ll << 38);
}
// k or v as [D, keys, heads, batch], in boxes of `keys` keys x 64 channels; where a stride is 0 the coordinate stays 0
inline bool encode_kv(CUtensorMap* tm, const XAttnArgs& a, const void* p, const Strides& s, int keys, int* use_head, int* use_batch) {
    *use_head = s.head != 0;
    *use_batch = s.batch != 0;
    const uint64_t dims[4] = {(uint64_t)a.D, (uint64_t)a.Tk, s.head ? (uint64_t)a.Hkv : 1, s.batch ? (uint64_t)a.B : 1};
    uint64_t st[3];
    const uint32_t box[4] = {64, (uint32_t)keys, 1, 1};
    return stride_ok(s.token, dims[1], &st[0]) && stride_ok(s.head, dims[2], &st[1]) && stride_ok(s.batch, dims[3], &st[2]) && encode_map(tm, p, 4, dims, st, box);
}
// strides, sizes and addresses that the maps of k and v can hold
inline bool kv_maps_supported(const XAttnArgs& a, int most_channels) {
    uint64_t unused;
    return a.dtype == VD_BF16 && a.D % 8 == 0 && a.D <= most_channels && a.Tk >= 1 && (((uintptr_t)a.k | (uintptr_t)a.v) & 15) == 0 &&
           stride_ok(a.sk.token, a.Tk, &unused) && stride_ok(a.sv.token, a.Tk, &unused) &&
           (a.sk.head == 0 || stride_ok(a.sk.head, a.Hkv, &unused)) && (a.sv.head == 0 || stride_ok(a.sv.head, a.Hkv, &unused)) &&
           (a.sk.batch == 0 || stride_ok(a.sk.batch, a.B, &unused)) && (a.sv.batch == 0 || stride_ok(a.sv.batch, a.B, &unused));
}

}  // namespace vd
