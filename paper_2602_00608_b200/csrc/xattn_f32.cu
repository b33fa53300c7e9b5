// Attention to states of another length in single precision, on the FP32 pipes (no operand or sum in fewer bits; the tensor core
// drops what falls off a running sum, and one of several hundred keys shows it).  A CTA of 128 threads takes 64 rows of a key head
// (a row: a token and one of the heads that share it) and walks blocks of 16 NJ keys; two CTAs share an SM, so that one computes
// while the other exchanges.  A thread holds 8 rows x NJ keys of the scores, as pairs along the channels, so that both operands are
// pairs as they lie in memory (fma.rn.f32x2), and 8 rows x NC channels of the output, as pairs of rows.  The keys of a thread are 16
// apart and a key's row in shared memory is an odd multiple of 16 bytes: no bank conflicts.  P goes through shared memory, its
// 16-byte pieces exchanged by key.  k, v and q come by cp.async, k and v one step ahead of their use.
// Where there are few rows a cluster divides the keys (xattn_meet.cuh).
#include "block_ops.h"
#include "xattn_meet.cuh"

namespace vd {
namespace {

using namespace tc;
using namespace xa;

constexpr int ROWS = 64, THREADS = 128;

template <int NC> struct Cfg {                               // NC: output channels of a thread
    static constexpr int DM = NC * 16, NJ = NC > 6 ? 3 : 4, KEYS = NJ * 16;
    static constexpr int VEC = NC % 4 == 0 ? 4 : NC % 2 == 0 ? 2 : 1;
    // Q [64][DM], K [KEYS][DM + 4], V [KEYS][DM], P [KEYS][64]
    static constexpr int Q_AT = 0, K_AT = ROWS * DM, V_AT = K_AT + KEYS * (DM + 4), P_AT = V_AT + KEYS * DM, END = P_AT + KEYS * ROWS;
    static constexpr int SMEM = END * 4;
    static_assert((DM + 4) % 8 == 4, "an odd multiple of 16 bytes");
    static_assert(2 * (SMEM + 1024) <= 228 * 1024, "two CTAs share an SM");
    static_assert(ROWS * (DM + 2) <= END, "the meeting's memory lies over the others");
};

template <int NC>
__global__ void __launch_bounds__(THREADS, 2) xattn_f32_kernel(const RowParams p) {
    using C = Cfg<NC>;
    constexpr int DM = C::DM, NJ = C::NJ, KEYS = C::KEYS, KS = DM + 4;
    extern __shared__ __align__(16) float smem[];
    float *s_q = smem + C::Q_AT, *s_k = smem + C::K_AT, *s_v = smem + C::V_AT, *s_p = smem + C::P_AT;
    const XAttnArgs& a = p.a;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int split = p.splits > 1 ? (int)cluster_ctarank() : 0;
    const Work w = work_of<ROWS>(p);
    const int tiles = (w.len + KEYS - 1) / KEYS, mine = tiles > split ? (tiles - split + p.splits - 1) / p.splits : 0;
    const int chunks = a.D / 4, lc = tid & 7, lr = tid >> 3; // loads: eight threads per key or row
    const float* k = (const float*)a.k + w.b * a.sk.batch + w.kvh * a.sk.head;
    const float* v = (const float*)a.v + w.b * a.sv.batch + w.kvh * a.sv.head;
    // zeros where there are no channels, rows or keys (0 * NaN is NaN)
    auto load = [&](float* dst, int stride, const float* src, int64_t token, int key0) {
#pragma unroll
        for (int r = 0; r < KEYS; r += 16) {
            const int key = key0 + r + lr;
            const bool here = key < w.len;
            const float* row = src + (here ? key : 0) * token;
            for (int c = lc; c < DM / 4; c += 8) {
                const bool in = here && c < chunks;
                cp_async16(smem_u32(dst + (r + lr) * stride + c * 4), in ? row + c * 4 : src, in ? 16u : 0u);
            }
        }
    };
    for (int r = lr; r < ROWS; r += 16) {
        const bool here = r < w.rows;
        const float* row = (const float*)a.q + w.at(p, a.sq, here ? r : 0);
        for (int c = lc; c < DM / 4; c += 8) {
            const bool in = here && c < chunks;
            cp_async16(smem_u32(s_q + r * DM + c * 4), in ? row + c * 4 : (const float*)a.q, in ? 16u : 0u);
        }
    }
    if (mine) load(s_k, KS, k, a.sk.token, split * KEYS);
    cp_async_commit();
    if (mine) load(s_v, DM, v, a.sv.token, split * KEYS);
    cp_async_commit();

    unsigned long long o[4][NC];                             // rows 8 ty + 2i, + 1
    float m_ref[8], l[8];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < NC; ++u) o[i][u] = 0ull;
#pragma unroll
    for (int i = 0; i < 8; ++i) { m_ref[i] = -INFINITY; l[i] = 0.f; }

    for (int t = 0; t < mine; ++t) {
        const int key0 = (split + t * p.splits) * KEYS, next = key0 + p.splits * KEYS;
        asm volatile("cp.async.wait_group 1;" ::: "memory"); // K (and Q) of this block
        __syncthreads();
        float s[8][NJ];
        {
            unsigned long long acc[8][NJ];
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc[i][j] = 0ull;
            const float* qp = s_q + ty * 8 * DM;
            const float* kp = s_k + tx * KS;
#pragma unroll 2
            for (int d = 0; d < a.D; d += 4) {
                ulonglong2 kk[NJ];
#pragma unroll
                for (int j = 0; j < NJ; ++j) kk[j] = *(const ulonglong2*)(kp + j * 16 * KS + d);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const ulonglong2 q = *(const ulonglong2*)(qp + i * DM + d);
#pragma unroll
                    for (int j = 0; j < NJ; ++j) acc[i][j] = fmaf2(q.y, kk[j].y, fmaf2(q.x, kk[j].x, acc[i][j]));
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) s[i][j] = sum2(acc[i][j]) * p.scale_log2;
        }
        __syncthreads();                                     // K has been read
        if (t + 1 < mine) load(s_k, KS, k, a.sk.token, next);
        cp_async_commit();
        bool grow = false;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const bool here = key0 + tx + 16 * j < w.len;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!here) s[i][j] = -INFINITY;
                grow = grow || s[i][j] > m_ref[i] + RESCALE_THRESHOLD;
            }
        }
        if (__any_sync(0xffffffffu, grow)) {                 // (a row's 16 threads sit in one half of a warp)
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float top = m_ref[i];
#pragma unroll
                for (int j = 0; j < NJ; ++j) top = fmaxf(top, s[i][j]);
#pragma unroll
                for (int x = 1; x < 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                f[i] = top == -INFINITY ? 1.f : ex2(m_ref[i] - top);
                m_ref[i] = top;
                l[i] *= f[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int u = 0; u < NC; ++u) o[i][u] = fmaf2(o[i][u], pack2(f[2 * i], f[2 * i + 1]), 0ull);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float ref = m_ref[i] == -INFINITY ? 0.f : m_ref[i];
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                s[i][j] = ex2(s[i][j] - ref);
                l[i] += s[i][j];
            }
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) {                       // pieces of four rows, exchanged by key
            float* row = s_p + (tx + 16 * j) * ROWS;
            *(float4*)(row + (((ty * 2) ^ tx) << 2)) = make_float4(s[0][j], s[1][j], s[2][j], s[3][j]);
            *(float4*)(row + (((ty * 2 + 1) ^ tx) << 2)) = make_float4(s[4][j], s[5][j], s[6][j], s[7][j]);
        }
        asm volatile("cp.async.wait_group 1;" ::: "memory"); // V of this block
        __syncthreads();
#pragma unroll 4
        for (int key = 0; key < KEYS; ++key) {
            const float* row = s_p + key * ROWS;
            const ulonglong2 p0 = *(const ulonglong2*)(row + (((ty * 2) ^ (key & 15)) << 2)), p1 = *(const ulonglong2*)(row + (((ty * 2 + 1) ^ (key & 15)) << 2));
            float vv[NC];
#pragma unroll
            for (int u = 0; u < NC; u += C::VEC) {
                const float* at = s_v + key * DM + (u / C::VEC) * 16 * C::VEC + tx * C::VEC;
                if constexpr (C::VEC == 4) { const float4 x = *(const float4*)at; vv[u] = x.x; vv[u + 1] = x.y; vv[u + 2] = x.z; vv[u + 3] = x.w; }
                else if constexpr (C::VEC == 2) { const float2 x = *(const float2*)at; vv[u] = x.x; vv[u + 1] = x.y; }
                else vv[u] = *at;
            }
#pragma unroll
            for (int u = 0; u < NC; ++u) {
                const unsigned long long x = pack2(vv[u], vv[u]);
                o[0][u] = fmaf2(p0.x, x, o[0][u]);
                o[1][u] = fmaf2(p0.y, x, o[1][u]);
                o[2][u] = fmaf2(p1.x, x, o[2][u]);
                o[3][u] = fmaf2(p1.y, x, o[3][u]);
            }
        }
        __syncthreads();                                     // V and P have been read
        if (t + 1 < mine) load(s_v, DM, v, a.sv.token, next);
        cp_async_commit();
    }
    cp_async_wait_all();
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
    float2* om = (float2*)(smem + ROWS * DM);
    if (p.splits > 1) __syncthreads();                       // the meeting's memory lies over the stages
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = ty * 8 + i;
        if (p.splits > 1) {
            if (tx == 0) om[r] = make_float2(m_ref[i], l[i]);
#pragma unroll
            for (int u = 0; u < NC; ++u) {
                float lo, hi;
                unpack2(o[i >> 1][u], lo, hi);
                smem[r * DM + (u / C::VEC) * 16 * C::VEC + tx * C::VEC + u % C::VEC] = i & 1 ? hi : lo;
            }
        } else if (r < w.rows) {
            float* out = (float*)a.o + w.at(p, a.so, r);
            const float inv = w.len ? 1.f / l[i] : 0.f;
#pragma unroll
            for (int u = 0; u < NC; ++u) {
                const int d = (u / C::VEC) * 16 * C::VEC + tx * C::VEC + u % C::VEC;
                float lo, hi;
                unpack2(o[i >> 1][u], lo, hi);
                if (d < a.D) out[d] = (i & 1 ? hi : lo) * inv;
            }
        }
    }
    if (p.splits > 1) {
        __syncthreads();
        meet_cluster<float, DM, THREADS>(p, smem, om, w, split, tid);
    }
}

template <int NC> cudaError_t launch(const XAttnArgs& a, cudaStream_t s) {
    const RowParams p = plan_rows<xattn_f32_kernel<NC>>(a, THREADS, ROWS, Cfg<NC>::SMEM, Cfg<NC>::KEYS);
    return cc::launch_clusters<xattn_f32_kernel<NC>>({(int64_t)p.groups * a.Hkv * a.B * p.splits, THREADS, Cfg<NC>::SMEM, Cfg<NC>::SMEM, p.splits}, s, p);
}

}  // namespace

bool xattn_f32_supported(const XAttnArgs& a) {
    const uint64_t at = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v;
    const int64_t st = a.sq.batch | a.sq.token | a.sq.head | a.sk.batch | a.sk.token | a.sk.head | a.sv.batch | a.sv.token | a.sv.head;
    return a.dtype == VD_F32 && a.D % 4 == 0 && a.D <= 128 && at % 16 == 0 && st % 4 == 0;
}

cudaError_t launch_xattn_f32(const XAttnArgs& a, cudaStream_t s) {
    const int nc = (a.D + 15) / 16;
    if (nc <= 2) return launch<2>(a, s);
    if (nc <= 3) return launch<3>(a, s);
    if (nc <= 4) return launch<4>(a, s);
    if (nc <= 5) return launch<5>(a, s);
    if (nc <= 6) return launch<6>(a, s);
    return launch<8>(a, s);
}

}  // namespace vd
