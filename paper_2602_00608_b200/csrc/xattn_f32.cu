// Attention to states of another length in single precision, on the FP32 pipes (no operand or sum in fewer bits; the tensor core
// drops what falls off a running sum, and one of several hundred keys shows it), and of what the tensor core's kernel does not take:
// heads of any width up to 256, any alignment and stride (2000 x 3000, 8 heads of 100, bf16: 626 us; a warp per row, xattn_plain.cu, 7608).
// A CTA of 128 threads takes 16 RT rows of a key head (a row: a token and one of the heads that share it) and walks blocks of 8 KJ keys;
// two CTAs share an SM (one with heads beyond 128 channels), so that one computes
// while the other exchanges.  What bounds it is the way from shared memory to the registers, 128 bytes a clock for all warps, broadcast or
// not: an fma.rn.f32x2 of a thread may take two of a thread's bytes.  So a thread holds as much as its registers allow:
//   scores   RT rows x KJ keys, pairs along the channels, so that both operands are pairs as they lie in memory.  Its keys are 8 apart and
//            a key's row is an odd multiple of 16 bytes long: no bank conflicts
//   output   the same RT rows x DM / 8 channels, pairs of channels; P goes through shared memory among the 8 threads of a row, its 16-byte
//            pieces exchanged by key, without a barrier
// 2 x 1350 x up to 777, 12 heads of 80 on 4: 197 us, 36 TFLOP/s of the pipes' 74, shared memory 61 % busy, FMA pipes 57 %.
// (Three CTAs an SM, other unrolling of the two loops: no gain.)
// k, v and q come by cp.async, k and v one step ahead of their use.  Where there are few rows a cluster divides the keys (xattn_meet.cuh).
#include "block_ops.h"
#include "xattn_meet.cuh"

namespace vd {
namespace {

using namespace tc;
using namespace xa;

constexpr int THREADS = 128;

template <int DM_> struct Cfg {                              // DM: channels that are held, a multiple of 16
    static constexpr int DM = DM_, RT = DM > 80 ? 4 : 8, KJ = DM > 128 ? 4 : DM > 80 ? 8 : 6, ROWS = 16 * RT, KEYS = 8 * KJ;
    static constexpr int NC = DM / 8, QUADS = NC / 4, REST = NC % 4;     // channels of a thread's output: QUADS times four, 32 apart, and two more
    // Q [ROWS][DM], K [KEYS][DM + 4], V [KEYS][DM], P [KEYS][ROWS]
    static constexpr int Q_AT = 0, K_AT = ROWS * DM, V_AT = K_AT + KEYS * (DM + 4), P_AT = V_AT + KEYS * DM, END = P_AT + KEYS * ROWS;
    static constexpr int SMEM = END * 4;
    static_assert((DM + 4) % 8 == 4 && (REST == 0 || REST == 2), "an odd multiple of 16 bytes; whole pairs");
    static_assert((DM > 128 ? 1 : 2) * (SMEM + 1024) <= 228 * 1024, "two CTAs share an SM");
    static_assert(ROWS * (DM + 2) <= END, "the meeting's memory lies over the others");
};

template <typename T> __device__ __forceinline__ float one(T v) { return (float)v; }
template <> __device__ __forceinline__ float one(__nv_bfloat16 v) { return __bfloat162float(v); }

// WHOLE: fp32 in whole, aligned pieces of 16 bytes.  Otherwise either type, converted on its way in, so that what is in shared memory and all
// that follows is the same: one value at a time, or bf16 in pieces of four where they are whole (2000 x 3000, 8 heads of 256 3.1 -> 1.8 ms).
template <typename T, int DM, bool WHOLE>
__global__ void __launch_bounds__(THREADS, DM > 128 ? 1 : 2) xattn_f32_kernel(const RowParams p) {
    using C = Cfg<DM>;
    constexpr int RT = C::RT, KJ = C::KJ, ROWS = C::ROWS, KEYS = C::KEYS, KS = DM + 4, NC = C::NC;
    extern __shared__ __align__(16) float smem[];
    float *s_q = smem + C::Q_AT, *s_k = smem + C::K_AT, *s_v = smem + C::V_AT, *s_p = smem + C::P_AT;
    const XAttnArgs& a = p.a;
    const int tid = threadIdx.x, cx = tid & 7, ry = tid >> 3;                // rows RT ry, keys cx, channels 4 cx
    const int split = p.splits > 1 ? (int)cluster_ctarank() : 0;
    const Work w = work_of<ROWS>(p);
    const int tiles = (w.len + KEYS - 1) / KEYS, mine = tiles > split ? (tiles - split + p.splits - 1) / p.splits : 0;
    const T* k = (const T*)a.k + w.b * a.sk.batch + w.kvh * a.sk.head + cx * 4;      // loads: eight threads per key or row
    const T* v = (const T*)a.v + w.b * a.sv.batch + w.kvh * a.sv.head + cx * 4;
    constexpr int CHUNKS = (DM / 4 + 7) / 8;                 // of a thread's part of a key
    auto chunk_held = [&](int c) { return DM % 32 == 0 || c + 1 < CHUNKS || cx + 8 * c < DM / 4; };
    // zeros where there are no channels or keys (0 * NaN is NaN)
    const bool pieces = (((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v) & 7) == 0 && a.D % 4 == 0 &&
                        ((a.sq.batch | a.sq.token | a.sq.head | a.sk.batch | a.sk.token | a.sk.head | a.sv.batch | a.sv.token | a.sv.head) & 3) == 0;
    auto bring = [&](float* dst, const T* src, int c, bool here) {            // four channels from cx * 4 + c * 32
        const int left = here ? a.D - (cx * 4 + c * 32) : 0;
        if constexpr (WHOLE) {
            cp_async16(smem_u32(dst + c * 32), left > 0 ? src + c * 32 : (const T*)a.q, left > 0 ? 16u : 0u);
        } else {
            float f[4] = {};
            if (sizeof(T) == 2 && pieces) {
                const uint2 x = left > 0 ? *(const uint2*)(src + c * 32) : make_uint2(0u, 0u);
                f[0] = __uint_as_float(x.x << 16); f[1] = __uint_as_float(x.x & 0xffff0000u);
                f[2] = __uint_as_float(x.y << 16); f[3] = __uint_as_float(x.y & 0xffff0000u);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < left) f[e] = one(src[c * 32 + e]);
            }
            *(float4*)(dst + c * 32) = make_float4(f[0], f[1], f[2], f[3]);
        }
    };
    auto load = [&](float* dst, int stride, const T* src, int64_t token, int key0) {
        float* at = dst + ry * stride + cx * 4;
        const T* row = src + (key0 + ry) * token;
#pragma unroll
        for (int r = 0; r < KEYS; r += 16, row += 16 * token) {
            const bool here = key0 + r + ry < w.len;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
                if (chunk_held(c)) bring(at + r * stride, row, c, here);
        }
    };
    for (int r = ry; r < ROWS; r += 16) {
        const bool here = r < w.rows;
        const T* row = (const T*)a.q + w.at(p, a.sq, here ? r : 0) + cx * 4;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if (chunk_held(c)) bring(s_q + r * DM + cx * 4, row, c, here);
    }
    if (mine) load(s_k, KS, k, a.sk.token, split * KEYS);
    cp_async_commit();
    if (mine) load(s_v, DM, v, a.sv.token, split * KEYS);
    cp_async_commit();

    unsigned long long o[RT][NC / 2];
    float m_ref[RT], l[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        m_ref[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int u = 0; u < NC / 2; ++u) o[i][u] = 0ull;
    }
    for (int t = 0; t < mine; ++t) {
        const int key0 = (split + t * p.splits) * KEYS, next = key0 + p.splits * KEYS;
        asm volatile("cp.async.wait_group 1;" ::: "memory"); // K (and Q) of this block
        __syncthreads();
        float s[RT][KJ];
        {
            unsigned long long acc[RT][KJ];
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < KJ; ++j) acc[i][j] = 0ull;
            const float* qp = s_q + ry * RT * DM;
            const float* kp = s_k + cx * KS;
#pragma unroll 2
            for (int d = 0; d < a.D; d += 4) {
                ulonglong2 kk[KJ];
#pragma unroll
                for (int j = 0; j < KJ; ++j) kk[j] = *(const ulonglong2*)(kp + j * 8 * KS + d);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const ulonglong2 q = *(const ulonglong2*)(qp + i * DM + d);
#pragma unroll
                    for (int j = 0; j < KJ; ++j) acc[i][j] = fmaf2(q.y, kk[j].y, fmaf2(q.x, kk[j].x, acc[i][j]));
                }
            }
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < KJ; ++j) s[i][j] = sum2(acc[i][j]) * p.scale_log2;
        }
        __syncthreads();                                     // K has been read
        if (t + 1 < mine) load(s_k, KS, k, a.sk.token, next);
        cp_async_commit();
        if (key0 + KEYS > w.len)
#pragma unroll
            for (int j = 0; j < KJ; ++j)
                if (key0 + cx + 8 * j >= w.len)
#pragma unroll
                    for (int i = 0; i < RT; ++i) s[i][j] = -INFINITY;
        bool grow = false;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float top = s[i][0];
#pragma unroll
            for (int j = 1; j < KJ; ++j) top = fmaxf(top, s[i][j]);
            grow = grow || top > m_ref[i] + RESCALE_THRESHOLD;
        }
        if (__any_sync(0xffffffffu, grow)) {                 // (a row's 8 threads sit side by side)
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float top = m_ref[i];
#pragma unroll
                for (int j = 0; j < KJ; ++j) top = fmaxf(top, s[i][j]);
#pragma unroll
                for (int x = 1; x < 8; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                const float f = top == -INFINITY ? 1.f : ex2(m_ref[i] - top);
                m_ref[i] = top;
                l[i] *= f;
#pragma unroll
                for (int u = 0; u < NC / 2; ++u) o[i][u] = fmaf2(o[i][u], pack2(f, f), 0ull);
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const float ref = m_ref[i] == -INFINITY ? 0.f : m_ref[i];
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                s[i][j] = ex2(s[i][j] - ref);
                l[i] += s[i][j];
            }
        }
#pragma unroll
        for (int j = 0; j < KJ; ++j) {                       // pieces of four rows, exchanged by key
            float* row = s_p + (cx + 8 * j) * ROWS;
#pragma unroll
            for (int h = 0; h < RT / 4; ++h)
                *(float4*)(row + (((ry * (RT / 4) + h) ^ cx) << 2)) = make_float4(s[4 * h][j], s[4 * h + 1][j], s[4 * h + 2][j], s[4 * h + 3][j]);
        }
        asm volatile("cp.async.wait_group 1;" ::: "memory"); // V of this block
        __syncthreads();
#pragma unroll 8
        for (int key = 0; key < KEYS; ++key) {
            const float* row = s_p + key * ROWS;
            float pr[RT];
#pragma unroll
            for (int h = 0; h < RT / 4; ++h) {
                const float4 x = *(const float4*)(row + (((ry * (RT / 4) + h) ^ (key & 7)) << 2));
                pr[4 * h] = x.x; pr[4 * h + 1] = x.y; pr[4 * h + 2] = x.z; pr[4 * h + 3] = x.w;
            }
            unsigned long long vv[NC / 2];
            const float* at = s_v + key * DM;
#pragma unroll
            for (int q = 0; q < C::QUADS; ++q) {
                const ulonglong2 x = *(const ulonglong2*)(at + q * 32 + cx * 4);
                vv[2 * q] = x.x; vv[2 * q + 1] = x.y;
            }
            if (C::REST) vv[NC / 2 - 1] = *(const unsigned long long*)(at + C::QUADS * 32 + cx * 2);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const unsigned long long x = pack2(pr[i], pr[i]);
#pragma unroll
                for (int u = 0; u < NC / 2; ++u) o[i][u] = fmaf2(x, vv[u], o[i][u]);
            }
        }
        __syncthreads();                                     // V has been read (and P, by its threads)
        if (t + 1 < mine) load(s_v, DM, v, a.sv.token, next);
        cp_async_commit();
    }
    cp_async_wait_all();
    float2* om = (float2*)(smem + ROWS * DM);
    if (p.splits > 1) __syncthreads();                       // the meeting's memory lies over the stages
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
        for (int x = 1; x < 8; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
        const int r = ry * RT + i;
        const bool here = r < w.rows;
        if (p.splits > 1 && cx == 0) om[r] = make_float2(m_ref[i], l[i]);
        T* out = here ? (T*)a.o + w.at(p, a.so, r) : nullptr;
        const float f = w.len ? 1.f / l[i] : 0.f;
#pragma unroll
        for (int u = 0; u < NC; u += 2) {
            const int d = u < C::QUADS * 4 ? (u / 4) * 32 + cx * 4 + u % 4 : C::QUADS * 32 + cx * 2;
            float lo, hi;
            unpack2(o[i][u / 2], lo, hi);
            if (p.splits > 1) {
                smem[r * DM + d] = lo;
                smem[r * DM + d + 1] = hi;
            } else if (here) {
                if (d < a.D) out[d] = (T)(lo * f);
                if (d + 1 < a.D) out[d + 1] = (T)(hi * f);
            }
        }
    }
    if (p.splits > 1) {
        __syncthreads();
        meet_cluster<T, DM, THREADS>(p, smem, om, w, split, tid);
    }
}

template <typename T, int DM, bool WHOLE> cudaError_t launch(const XAttnArgs& a, cudaStream_t s) {
    constexpr int smem = Cfg<DM>::SMEM;
    const RowParams p = plan_rows<xattn_f32_kernel<T, DM, WHOLE>>(a, THREADS, Cfg<DM>::ROWS, smem, Cfg<DM>::KEYS);
    return cc::launch_clusters<xattn_f32_kernel<T, DM, WHOLE>>({(int64_t)p.groups * a.Hkv * a.B * p.splits, THREADS, smem, smem, p.splits}, s, p);
}
template <typename T> cudaError_t launch_any(const XAttnArgs& a, cudaStream_t s) {
    if (a.D <= 64) return launch<T, 64, false>(a, s);
    if (a.D <= 128) return launch<T, 128, false>(a, s);
    return launch<T, 256, false>(a, s);
}

}  // namespace

cudaError_t launch_xattn_f32(const XAttnArgs& a, cudaStream_t s) {
    const uint64_t at = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v;
    const int64_t st = a.sq.batch | a.sq.token | a.sq.head | a.sk.batch | a.sk.token | a.sk.head | a.sv.batch | a.sv.token | a.sv.head;
    if (a.dtype == VD_BF16) return launch_any<__nv_bfloat16>(a, s);
    if (a.D % 4 != 0 || at % 16 != 0 || st % 4 != 0) return launch_any<float>(a, s);
    if (a.D <= 32) return launch<float, 32, true>(a, s);
    if (a.D <= 48) return launch<float, 48, true>(a, s);
    if (a.D <= 64) return launch<float, 64, true>(a, s);
    if (a.D <= 80) return launch<float, 80, true>(a, s);
    if (a.D <= 96) return launch<float, 96, true>(a, s);
    if (a.D <= 128) return launch<float, 128, true>(a, s);
    return launch<float, 256, true>(a, s);
}

}  // namespace vd
