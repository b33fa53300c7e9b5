// Attention to states of another length for few rows per key head (a new token or a few, with the heads that share it): bound by the
// bytes of k and v, which each CTA streams straight into registers.
// LPK lanes hold a key's channels, 16 bytes each (twice that for fp32 heads beyond 128), a warp 32 / LPK keys a load, U loads of k and
// of v under way.  The U x R partial scores of a lane are added over the LPK lanes by halving (N - 1 shuffles for N sums
// instead of N log2 LPK), which leaves each lane with one whole score, whose exponential it takes and hands back to the others.
// The running maximum is a warp's, moved only when a score exceeds it by 2^8 (every lane's sums share it, so they add without
// weights).  With more rows the arithmetic is what bounds this, and bf16 takes matrix instructions instead (below).  Warps meet in shared memory; where there are few heads, a cluster of up to eight CTAs divides the keys and meets in
// distributed shared memory.  Fixed orders throughout: the same bits each time.
#include <algorithm>

#include "block_ops.h"
#include "conv_cluster.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace vd {
namespace {

using namespace tc;

constexpr int WARPS = 8, MAX_SPLITS = 8;
constexpr float RESCALE_THRESHOLD = 8.0f;

struct RowParams {
    XAttnArgs a;
    int g, groups;               // groups: of R rows, of a (batch item, key head)
    int splits;
    float scale_log2;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint4 ldg_stream(const void* p) {
    uint4 r;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}
// 16 bytes as pairs of floats
template <typename T> struct Vec;
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void up(const uint4& r, unsigned long long (&f)[4]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
};
template <> struct Vec<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void up(const uint4& r, unsigned long long (&f)[2]) {
        f[0] = pack2(__uint_as_float(r.x), __uint_as_float(r.y));
        f[1] = pack2(__uint_as_float(r.z), __uint_as_float(r.w));
    }
};
__device__ __forceinline__ void unpack2(unsigned long long v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }

// v[i] summed over the L lanes of a group; lane x of it is left with sum x / (L / N) in v[0]
template <int N, int L> __device__ __forceinline__ float sum_scatter(float (&v)[N], int lane) {
    static_assert(N <= L, "");
    int cnt = N;
#pragma unroll
    for (int w = L / 2; w >= 1; w >>= 1) {
        if (cnt > 1) {
            cnt >>= 1;
            const bool upper = (lane & w) != 0;
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                if (i >= cnt) break;
                const float send = upper ? v[i] : v[i + cnt], keep = upper ? v[i + cnt] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, w);
            }
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], w);
        }
    }
    return v[0];
}

// a CTA's row group, and what its rows are
struct Work {
    int b, kvh, row0, rows, len;
    __device__ __forceinline__ int64_t at(const RowParams& p, const Strides& s, int r) const {
        const int row = row0 + r, t = row / p.g, h = kvh * p.g + row - t * p.g;
        return b * s.batch + t * s.token + h * s.head;
    }
};
template <int R> __device__ __forceinline__ Work work_of(const RowParams& p) {
    Work w;
    const int64_t item = blockIdx.x / p.splits;
    w.row0 = (int)(item % p.groups) * R;
    w.kvh = (int)(item / p.groups % p.a.Hkv);
    w.b = (int)(item / p.groups / p.a.Hkv);
    w.rows = min(R, p.a.Tq * p.g - w.row0);
    w.len = p.a.kv_lens ? min(max(p.a.kv_lens[w.b], 0), p.a.Tk) : p.a.Tk;
    return w;
}
// shared memory: the warps' accumulators, the CTA's, and (maximum, sum) of either; `rows` rows of DM channels each
template <int DM> struct Shared {
    float* base;
    int rows;
    __device__ __forceinline__ Shared(float* b, int r) : base(b), rows(r) {}
    __device__ __forceinline__ float* acc(int warp, int r) const { return base + (warp * rows + r) * DM; }
    __device__ __forceinline__ float* out(int r) const { return acc(WARPS, r); }
    __device__ __forceinline__ float2* ml(int warp, int r) const { return (float2*)acc(WARPS + 1, 0) + warp * rows + r; }
    __device__ __forceinline__ float2* om(int r) const { return ml(WARPS, r); }
};
constexpr int shared_bytes(int rows, int dm) { return (WARPS + 1) * rows * (dm + 2) * 4; }

// The warps' shares are in shared memory: added up and written, or left there for the cluster, whose CTAs each finish a part.
template <typename T, int DM> __device__ __forceinline__ void meet(const RowParams& p, const Shared<DM>& sh, const Work& w, int split, int tid) {
    const XAttnArgs& a = p.a;
    __syncthreads();
    for (int i = tid; i < w.rows * DM; i += WARPS * 32) {
        const int r = i / DM, d = i % DM;
        float2 ml[WARPS];
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
            ml[k] = *sh.ml(k, r);
            m = fmaxf(m, ml[k].x);
        }
        const float ref = m == -INFINITY ? 0.f : m;
        float o = 0.f, sum = 0.f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
            const float f = ex2(ml[k].x - ref);
            o = fmaf(f, sh.acc(k, r)[d], o);
            sum = fmaf(f, ml[k].y, sum);
        }
        if (p.splits == 1) {
            if (d < a.D) ((T*)a.o)[w.at(p, a.so, r) + d] = (T)(w.len ? o / sum : 0.f);
        } else {
            sh.out(r)[d] = o;
            if (d == 0) *sh.om(r) = make_float2(m, sum);
        }
    }
    if (p.splits == 1) return;
    cluster_sync_all();                                      // every CTA's share is in its shared memory
    for (int i = split * (WARPS * 32) + tid; i < w.rows * DM; i += p.splits * WARPS * 32) {
        const int r = i / DM, d = i % DM;
        if (d >= a.D) continue;
        float m[MAX_SPLITS], sum[MAX_SPLITS], o[MAX_SPLITS], top = -INFINITY;
#pragma unroll
        for (int c = 0; c < MAX_SPLITS; ++c)
            if (c < p.splits) {
                const uint32_t om = map_to_cta(smem_u32(sh.om(r)), (uint32_t)c), at = map_to_cta(smem_u32(sh.out(r) + d), (uint32_t)c);
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m[c]), "=f"(sum[c]) : "r"(om) : "memory");
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o[c]) : "r"(at) : "memory");
                top = fmaxf(top, m[c]);
            }
        const float ref = top == -INFINITY ? 0.f : top;
        float total = 0.f, out = 0.f;
#pragma unroll
        for (int c = 0; c < MAX_SPLITS; ++c)
            if (c < p.splits) {
                const float f = ex2(m[c] - ref);
                total = fmaf(f, sum[c], total);
                out = fmaf(f, o[c], out);
            }
        ((T*)a.o)[w.at(p, a.so, r) + d] = (T)(w.len ? out / total : 0.f);
    }
    cluster_sync_all();                                      // nobody leaves while others read its memory
}

template <typename T, int R, int U, int LPK, int NVL>
__global__ void __launch_bounds__(WARPS * 32, 2) xattn_rows_kernel(const RowParams p) {
    constexpr int E = Vec<T>::E, P = E / 2, N = R * U, KPL = 32 / LPK, KPI = KPL * U, SPAN = LPK * E;     // KPI: keys of a warp's round
    constexpr int DUP = LPK / N, DM = SPAN * NVL;            // DUP: lanes that hold the same score; DM: channels that are held
    static_assert(N <= LPK, "");
    extern __shared__ float smem[];
    const Shared<DM> sh(smem, R);
    const XAttnArgs& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, x = lane % LPK, kg = lane / LPK;
    const int split = p.splits > 1 ? (int)cluster_ctarank() : 0;
    const Work w = work_of<R>(p);
    const int b = w.b, kvh = w.kvh, len = w.len;
    unsigned long long q[NVL][R][P], acc[NVL][R][P];
    bool live[NVL];
#pragma unroll
    for (int n = 0; n < NVL; ++n) {
        live[n] = n * SPAN + x * E < a.D;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (live[n]) v = *(const uint4*)((const T*)a.q + w.at(p, a.sq, min(r, w.rows - 1)) + n * SPAN + x * E);
            Vec<T>::up(v, q[n][r]);
#pragma unroll
            for (int i = 0; i < P; ++i) acc[n][r][i] = 0ull;
        }
    }
    const T* k = (const T*)a.k + b * a.sk.batch + kvh * a.sk.head + x * E;
    const T* v = (const T*)a.v + b * a.sv.batch + kvh * a.sv.head + x * E;
    const int mine = x / DUP, my_row = mine / U, my_u = mine % U;        // the score this lane is left with
    float m_ref = -INFINITY, l = 0.f;                        // of my_row
    for (int64_t base = (int64_t)(split * WARPS + warp) * KPI; base < len; base += (int64_t)p.splits * WARPS * KPI) {
        uint4 kr[U][NVL], vr[U][NVL];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t key = base + u * KPL + kg;
#pragma unroll
            for (int n = 0; n < NVL; ++n) {
                kr[u][n] = make_uint4(0, 0, 0, 0);
                if (key < len && live[n]) kr[u][n] = ldg_stream(k + key * a.sk.token + n * SPAN);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t key = base + u * KPL + kg;
#pragma unroll
            for (int n = 0; n < NVL; ++n) {
                vr[u][n] = make_uint4(0, 0, 0, 0);
                if (key < len && live[n]) vr[u][n] = ldg_stream(v + key * a.sv.token + n * SPAN);
            }
        }
        float s[N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            unsigned long long part[R] = {};
#pragma unroll
            for (int n = 0; n < NVL; ++n) {
                unsigned long long f[P];
                Vec<T>::up(kr[u][n], f);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < P; ++i) part[r] = fmaf2(q[n][r][i], f[i], part[r]);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) s[r * U + u] = sum2(part[r]);
        }
        float sc = sum_scatter<N, LPK>(s, lane) * p.scale_log2;
        if (base + my_u * KPL + kg >= len) sc = -INFINITY;
        if (__any_sync(0xffffffffu, sc > m_ref + RESCALE_THRESHOLD)) {
            float mx = fmaxf(sc, m_ref);
#pragma unroll
            for (int d = LPK; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
#pragma unroll
            for (int d = DUP; d < DUP * U; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            const float factor = mx == -INFINITY ? 1.f : ex2(m_ref - mx);
            m_ref = mx;
            l *= factor;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f = __shfl_sync(0xffffffffu, factor, (lane & ~(LPK - 1)) | (r * U * DUP));
#pragma unroll
                for (int n = 0; n < NVL; ++n)
#pragma unroll
                    for (int i = 0; i < P; ++i) acc[n][r][i] = fmaf2(acc[n][r][i], pack2(f, f), 0ull);
            }
        }
        const float e = ex2(sc - (m_ref == -INFINITY ? 0.f : m_ref));    // (NaN scores and infinite ones make it NaN)
        l += e;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            unsigned long long pr[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float f = __shfl_sync(0xffffffffu, e, (lane & ~(LPK - 1)) | ((r * U + u) * DUP));
                pr[r] = pack2(f, f);
            }
#pragma unroll
            for (int n = 0; n < NVL; ++n) {
                unsigned long long f[P];
                Vec<T>::up(vr[u][n], f);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < P; ++i) acc[n][r][i] = fmaf2(pr[r], f[i], acc[n][r][i]);
            }
        }
    }
    // ---- a warp's keys: lanes of other keys, then the warps of the CTA, then the CTAs of the cluster
#pragma unroll
    for (int d = LPK; d < 32; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
#pragma unroll
    for (int d = DUP; d < DUP * U; d <<= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    if (kg == 0 && my_u == 0 && x % DUP == 0) *sh.ml(warp, my_row) = make_float2(m_ref, l);
#pragma unroll
    for (int n = 0; n < NVL; ++n)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float f0, f1;
                unpack2(acc[n][r][i], f0, f1);
#pragma unroll
                for (int d = LPK; d < 32; d <<= 1) {
                    f0 += __shfl_xor_sync(0xffffffffu, f0, d);
                    f1 += __shfl_xor_sync(0xffffffffu, f1, d);
                }
                if (kg == 0) *(float2*)(sh.acc(warp, r) + n * SPAN + x * E + 2 * i) = make_float2(f0, f1);
            }
    meet<T, DM>(p, sh, w, split, tid);
}

// bf16, up to 16 rows: scores and products on the matrix instructions (mma m16n8k16; with this few rows the bytes bound the call, and
// operands go from memory to registers as they are).  Rows are the products' narrow side, eight at a time.  A lane
// (g, c) = (lane / 4, lane % 4):
//   S^T = K Q^T    holds 16-byte chunks c, c + 4, ... of keys g and g + 8: a chunk's first two words are its share of one product, the
//                  others of the next, and Q's chunks are taken alike, so the channels' order does not matter
//   O^T = V^T P^T  P^T is S^T as the products left it, turned by movmatrix; holds chunks g (+ 8) of keys 2c, 2c + 1, 2c + 8, 2c + 9: product i
//                  takes channels 2i and 2i + 1 of every chunk, pairs of keys put together by byte permutes
// The next round's k loads go out once k is in the scores, those of v once v is in the output.
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// DC: 64-channel groups; KB: blocks of 16 keys of a warp's round; NR: groups of eight rows
template <int DC, int KB, int NR>
__global__ void __launch_bounds__(WARPS * 32) xattn_rows_mma_kernel(const RowParams p) {
    constexpr int R = NR * 8, DM = DC * 64, QC = DC * 2;     // QC: Q and K chunks of a lane
    extern __shared__ float smem[];
    const Shared<DM> sh(smem, R);
    const XAttnArgs& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    const int split = p.splits > 1 ? (int)cluster_ctarank() : 0;
    const Work w = work_of<R>(p);
    const int chunks = a.D / 8;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    uint4 q[NR][QC];                                         // row 8 n + g
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int j = 0; j < QC; ++j)
            q[n][j] = c + 4 * j < chunks && n * 8 + g < w.rows ? *(const uint4*)((const __nv_bfloat16*)a.q + w.at(p, a.sq, n * 8 + g) + (c + 4 * j) * 8) : zero;
    const __nv_bfloat16* k = (const __nv_bfloat16*)a.k + w.b * a.sk.batch + w.kvh * a.sk.head + c * 8;
    const __nv_bfloat16* v = (const __nv_bfloat16*)a.v + w.b * a.sv.batch + w.kvh * a.sv.head + g * 8;
    float o[DC][4][NR][4] = {};
    float m[NR][2], l[NR][2];                                // of rows 8 n + 2c, + 1
#pragma unroll
    for (int n = 0; n < NR; ++n) { m[n][0] = m[n][1] = -INFINITY; l[n][0] = l[n][1] = 0.f; }
    uint4 kr[KB][2][QC], vr[KB][4][DC];
    auto load_k = [&](int base) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int key = base + kb * 16 + h * 8 + g;
                const __nv_bfloat16* at = k + key * a.sk.token;
#pragma unroll
                for (int j = 0; j < QC; ++j) {
                    kr[kb][h][j] = zero;
                    if (key < w.len && c + 4 * j < chunks) kr[kb][h][j] = ldg_stream(at + j * 32);
                }
            }
    };
    auto load_v = [&](int base) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = base + kb * 16 + 2 * c + (i & 1) + (i >> 1) * 8;
                const __nv_bfloat16* at = v + key * a.sv.token;
#pragma unroll
                for (int dc = 0; dc < DC; ++dc) {
                    vr[kb][i][dc] = zero;
                    if (key < w.len && dc * 8 + g < chunks) vr[kb][i][dc] = ldg_stream(at + dc * 64);
                }
            }
    };
    const int step = p.splits * WARPS * (KB * 16);
    int base = (split * WARPS + warp) * (KB * 16);           // (below 2^31: a round reaches at most 2^15 keys further than the last key)
    if (base < w.len) { load_k(base); load_v(base); }
    for (; base < w.len; base += step) {
        float s[KB][NR][4];                                  // keys g (first two) and g + 8 of rows 8 n + 2c, + 1
        bool grow = false;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                float d0[4] = {0.f, 0.f, 0.f, 0.f}, d1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < QC; ++j) {
                    const uint4 x = kr[kb][0][j], y = kr[kb][1][j];
                    mma_16816(d0, x.x, y.x, x.y, y.y, q[n][j].x, q[n][j].y);
                    mma_16816(d1, x.z, y.z, x.w, y.w, q[n][j].z, q[n][j].w);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[kb][n][e] = base + kb * 16 + (e >> 1) * 8 + g < w.len ? (d0[e] + d1[e]) * p.scale_log2 : -INFINITY;
                    grow = grow || s[kb][n][e] > m[n][e & 1] + RESCALE_THRESHOLD;
                }
            }
        }
        const bool more = base + step < w.len;
        if (more) load_k(base + step);
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float top = m[n][e];
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) top = fmaxf(top, fmaxf(s[kb][n][e], s[kb][n][e + 2]));
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    const float f = top == -INFINITY ? 1.f : ex2(m[n][e] - top);
                    m[n][e] = top;
                    l[n][e] *= f;
#pragma unroll
                    for (int dc = 0; dc < DC; ++dc)
#pragma unroll
                        for (int i = 0; i < 4; ++i) { o[dc][i][n][e] *= f; o[dc][i][n][e + 2] *= f; }
                }
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            uint32_t b0[NR], b1[NR];
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const float r0 = m[n][0] == -INFINITY ? 0.f : m[n][0], r1 = m[n][1] == -INFINITY ? 0.f : m[n][1];
                const float e0 = ex2(s[kb][n][0] - r0), e1 = ex2(s[kb][n][1] - r1), e2 = ex2(s[kb][n][2] - r0), e3 = ex2(s[kb][n][3] - r1);
                l[n][0] += e0 + e2;
                l[n][1] += e1 + e3;
                b0[n] = transpose_8x8(pack_bf16(e0, e1));
                b1[n] = transpose_8x8(pack_bf16(e2, e3));
            }
#pragma unroll
            for (int dc = 0; dc < DC; ++dc) {
                const uint4 x0 = vr[kb][0][dc], x1 = vr[kb][1][dc], x2 = vr[kb][2][dc], x3 = vr[kb][3][dc];
                const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w}, w2[4] = {x2.x, x2.y, x2.z, x2.w}, w3[4] = {x3.x, x3.y, x3.z, x3.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a0 = __byte_perm(w0[i], w1[i], 0x5410), a1 = __byte_perm(w0[i], w1[i], 0x7632),
                                   a2 = __byte_perm(w2[i], w3[i], 0x5410), a3 = __byte_perm(w2[i], w3[i], 0x7632);
#pragma unroll
                    for (int n = 0; n < NR; ++n) mma_16816(o[dc][i][n], a0, a1, a2, a3, b0[n], b1[n]);
                }
            }
        }
        if (more) load_v(base + step);
    }
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
            if (g == 0) *sh.ml(warp, n * 8 + 2 * c + e) = make_float2(m[n][e], l[n][e]);
#pragma unroll
            for (int dc = 0; dc < DC; ++dc)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *(float2*)(sh.acc(warp, n * 8 + 2 * c + e) + (dc * 8 + g) * 8 + 2 * i) = make_float2(o[dc][i][n][e], o[dc][i][n][e + 2]);
        }
    meet<__nv_bfloat16, DM>(p, sh, w, split, tid);
}

// KERNEL for groups of `rows` rows, `round` keys of a CTA at a time
template <auto KERNEL> cudaError_t launch_split(const XAttnArgs& a, int rows, int dm, int round, cudaStream_t s) {
    RowParams p{a, a.H / a.Hkv, 0, 1, a.scale * 1.4426950408889634f};
    p.groups = (int)(((int64_t)a.Tq * p.g + rows - 1) / rows);
    const int64_t items = (int64_t)p.groups * a.Hkv * a.B;
    const int smem = shared_bytes(rows, dm);
    // two CTAs per SM; a split has at least one round of keys for each of its warps
    while (p.splits < MAX_SPLITS && items * p.splits < 148 && a.Tk > p.splits * round && cc::clusters_fit<KERNEL>(WARPS * 32, smem, 2 * p.splits)) p.splits *= 2;
    return cc::launch_clusters<KERNEL>({items * p.splits, WARPS * 32, smem, smem, p.splits}, s, p);
}
template <typename T, int R, int U, int LPK, int NVL> cudaError_t launch(const XAttnArgs& a, cudaStream_t s) {
    return launch_split<xattn_rows_kernel<T, R, U, LPK, NVL>>(a, R, LPK * Vec<T>::E * NVL, 32 / LPK * U * WARPS, s);
}
template <int DC, int KB> cudaError_t launch_mma(const XAttnArgs& a, int64_t rows, cudaStream_t s) {
    return rows <= 8 ? launch_split<xattn_rows_mma_kernel<DC, KB, 1>>(a, 8, DC * 64, KB * 16 * WARPS, s)
                     : launch_split<xattn_rows_mma_kernel<DC, KB, 2>>(a, 16, DC * 64, KB * 16 * WARPS, s);
}

template <typename T, int R> cudaError_t launch_rows(const XAttnArgs& a, cudaStream_t s) {
    const int chunks = a.D / Vec<T>::E;
    if (chunks <= 8) return launch<T, R, 8 / R, 8, 1>(a, s);
    if (chunks <= 16) return launch<T, R, R == 1 ? 8 : 4, 16, 1>(a, s);
    if (chunks <= 32) return launch<T, R, R == 1 ? 8 : 4, 32, 1>(a, s);
    if constexpr (sizeof(T) == 4) return launch<T, R, R == 4 ? 2 : 4, 32, 2>(a, s);
    return cudaErrorInvalidValue;
}

}  // namespace

bool xattn_rows_supported(const XAttnArgs& a) {
    const int e = a.dtype == VD_BF16 ? 8 : 4;
    const uint64_t at = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v;
    const int64_t st = a.sq.batch | a.sq.token | a.sq.head | a.sk.batch | a.sk.token | a.sk.head | a.sv.batch | a.sv.token | a.sv.head;
    return a.D % e == 0 && at % 16 == 0 && st % e == 0;
}

cudaError_t launch_xattn_rows(const XAttnArgs& a, cudaStream_t s) {
    const int64_t rows = (int64_t)a.Tq * (a.H / a.Hkv);
    if (a.dtype == VD_BF16) {
        if (rows == 1 || a.D > 128) return rows == 1 ? launch_rows<__nv_bfloat16, 1>(a, s) : rows == 2 ? launch_rows<__nv_bfloat16, 2>(a, s) : launch_rows<__nv_bfloat16, 4>(a, s);
        return a.D <= 64 ? launch_mma<1, 2>(a, rows, s) : launch_mma<2, 1>(a, rows, s);
    }
    return rows == 1 ? launch_rows<float, 1>(a, s) : rows == 2 ? launch_rows<float, 2>(a, s) : launch_rows<float, 4>(a, s);
}

}  // namespace vd
