// Attention to states of another length for few rows per key head (a new token or a few, with the heads that share it): bound by the
// bytes of k and v, which each CTA streams straight into registers.
// LPK lanes hold a key's channels, 16 bytes each (twice that for fp32 heads beyond 128), a warp 32 / LPK keys a load, U loads of k and
// of v under way.  The U x R partial scores of a lane are added over the LPK lanes by halving (N - 1 shuffles for N sums
// instead of N log2 LPK), which leaves each lane with one whole score, whose exponential it takes and hands back to the others.
// The running maximum is a warp's, moved only when a score exceeds it by 2^8 (every lane's sums share it, so they add without
// weights).  With more rows the arithmetic is what bounds this, and bf16 takes matrix instructions instead (below).  Warps meet in shared memory;
// where there are few heads, a cluster of up to eight CTAs divides the keys and meets in distributed shared memory.  Fixed orders throughout:
// the same bits each time.  4 sequences of up to 16384 keys, 8 key heads of 128 with 4 rows each: 218 MB in 41 us, 5.3 TB/s with the launch and
// the meeting, DRAM 70 % busy.  Eight warps a CTA (us, 4 / 8 / 16 warps: 8 x 16 heads, 512 keys of 64 8.5 / 6.5 / 8.5; 256 x 2000 of 128
// 45.0 / 43.3 / 58.3; fp32, 512 x 1000 of 64 42.9 / 43.4 / 47.5, 32 x 4096 of 80 26.5 / 20.1 / 24.9).
#include "block_ops.h"
#include "xattn_maps.h"
#include "xattn_meet.cuh"

namespace vd {
namespace {

using namespace tc;
using namespace xa;

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

// The warps' shares are in shared memory: added up and written, or left there for the cluster, whose CTAs each finish a part.
template <typename T, int DM, int WARPS> __device__ __forceinline__ void meet(const RowParams& p, const Shared<DM, WARPS>& sh, const Work& w, int split, int tid) {
    const XAttnArgs& a = p.a;
    __syncthreads();
    for (int i = tid; i < w.rows * DM && tid < WARPS * 32; i += WARPS * 32) {
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
    if (p.splits > 1) meet_cluster<T, DM, WARPS * 32>(p, sh.out(0), sh.om(0), w, split, tid);
}

template <typename T, int R, int U, int LPK, int NVL, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, 2) xattn_rows_kernel(const RowParams p) {
    constexpr int E = Vec<T>::E, P = E / 2, N = R * U, KPL = 32 / LPK, KPI = KPL * U, SPAN = LPK * E;     // KPI: keys of a warp's round
    constexpr int DUP = LPK / N, DM = SPAN * NVL;            // DUP: lanes that hold the same score; DM: channels that are held
    static_assert(N <= LPK, "");
    extern __shared__ float smem[];
    const Shared<DM, WARPS> sh(smem, R);
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
    meet<T, DM, WARPS>(p, sh, w, split, tid);
}

// bf16, up to 16 rows: scores and products on the matrix instructions (mma m16n8k16: with this few rows the bytes bound the call, not
// the products), k and v through a ring of shared-memory stages that one thread keeps filled by bulk tensor loads: up to 192 KB
// of an SM under way.  Rows are the products' narrow side, eight at a time:
//   S^T = K Q^T      K by ldmatrix as it lies in the stage, Q in registers
//   O^T = V^T P^T    V by transposing ldmatrix, P^T is S^T as the products left it, turned by movmatrix
// A warp takes 16 keys of every stage and keeps a maximum, a sum and an output of its own.
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <int DP> struct StreamCfg {                         // (heads beyond 128 channels: half the keys a stage, so that three still fit)
    static constexpr int WARPS = DP == 256 ? 4 : 8, KEYS = WARPS * 16, THREADS = (WARPS + 1) * 32;
    static constexpr int STAGES = DP == 64 ? 6 : 3, TILE = KEYS * DP * 2, SMEM = STAGES * 2 * TILE + 128 + 1024;
    static_assert(SMEM <= 232448 && shared_bytes(WARPS, 16, DP) <= STAGES * 2 * TILE, "shared memory of one CTA; the meeting's lies over the stages");
};
struct StreamBars { uint64_t full[6], empty[6]; uint32_t abort_flag; };
static_assert(sizeof(StreamBars) <= 128, "");
struct StreamParams {
    RowParams p;
    int kb, vb, kh, vh;          // 0: the batch (head) coordinate of k or v stays 0
};
// NR: groups of eight rows
template <int DP, int NR>
__global__ void __launch_bounds__(StreamCfg<DP>::THREADS, 1)
xattn_stream_kernel(const StreamParams sp, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
    using C = StreamCfg<DP>;
    constexpr int R = NR * 8, KS = DP / 16, WARPS = C::WARPS, KEYS = C::KEYS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* stages = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    StreamBars* bars = (StreamBars*)(stages + C::STAGES * 2 * C::TILE);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const RowParams& p = sp.p;
    const XAttnArgs& a = p.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    if (tid == 0) {
        for (int i = 0; i < C::STAGES; ++i) { mbar_init(smem_u32(&bars->full[i]), 1); mbar_init(smem_u32(&bars->empty[i]), WARPS); }
        bars->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async_smem();
    }
    __syncthreads();
    const int split = p.splits > 1 ? (int)cluster_ctarank() : 0;
    const Work w = work_of<R>(p);
    const int tiles = (w.len + KEYS - 1) / KEYS, mine = tiles > split ? (tiles - split + p.splits - 1) / p.splits : 0;
    const Shared<DP, WARPS> sh((float*)stages, R);
    float o[KS][NR][4] = {};                                 // channels 16 i + g, + 8 of rows 8 n + 2c, + 1
    float m[NR][2], l[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) { m[n][0] = m[n][1] = -INFINITY; l[n][0] = l[n][1] = 0.f; }
    if (warp == WARPS) {
        if (lane == 0) {
            bool ok = true;
            int i = 0;
            for (; i < mine && ok; ++i) {
                const int st = i % C::STAGES, tile = split + i * p.splits;
                ok = mbar_wait(smem_u32(&bars->empty[st]), ((i / C::STAGES) & 1) ^ 1, abort_flag);
                if (!ok) break;
                const uint32_t full = smem_u32(&bars->full[st]), dst = smem_u32(stages + st * 2 * C::TILE);
                mbar_arrive_expect_tx(full, 2 * C::TILE);
                for (int x = 0; x < DP / 64; ++x) {
                    tma_load_4d(dst + x * (KEYS * 128), &tm_k, x * 64, tile * KEYS, w.kvh * sp.kh, w.b * sp.kb, full);
                    tma_load_4d(dst + C::TILE + x * (KEYS * 128), &tm_v, x * 64, tile * KEYS, w.kvh * sp.vh, w.b * sp.vb, full);
                }
            }
            if (!ok || *abort_flag) cc::land_loads(bars->full, C::STAGES, i);     // (else the others wait for all of them)
        }
        __syncwarp();
    } else {
        uint32_t q[KS][NR][2];                               // row 8 n + g, channels 16 k + 2c, + 1 and + 8, + 9
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int ch = k * 16 + h * 8 + 2 * c;
                    q[k][n][h] = ch < a.D && n * 8 + g < w.rows ? *(const uint32_t*)((const __nv_bfloat16*)a.q + w.at(p, a.sq, n * 8 + g) + ch) : 0u;
                }
        // addresses within a tile: lane's row of the four 8x8 matrices; 16-byte chunk x of row r lies at x ^ (r & 7)
        const int k_row = warp * 16 + (lane & 7) + ((lane >> 3) & 1) * 8, v_row = warp * 16 + (lane & 7) + (lane >> 4) * 8;
        const uint32_t k_at = (uint32_t)(k_row * 128), v_at = (uint32_t)(v_row * 128), k_hi = (uint32_t)(lane >> 4), v_hi = (uint32_t)((lane >> 3) & 1), sw = (uint32_t)(lane & 7);
        bool ok = true;
        for (int i = 0; i < mine; ++i) {
            const int st = i % C::STAGES, left = w.len - (split + i * p.splits) * KEYS - warp * 16;       // keys of this warp's 16 that count
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->full[st]), (i / C::STAGES) & 1, abort_flag)) && ok;
            if (left > 0) {
                const uint32_t kt = smem_u32(stages + st * 2 * C::TILE) + k_at, vt = smem_u32(stages + st * 2 * C::TILE + C::TILE) + v_at;
                if (left < 16) {                             // 0 * NaN is NaN: values that do not count become zeros (the last stage: never filled again)
                    for (int x = lane; x < (16 - left) * 8; x += 32)
#pragma unroll
                        for (int y = 0; y < DP / 64; ++y)
                            *(uint4*)(stages + st * 2 * C::TILE + C::TILE + y * (KEYS * 128) + (warp * 16 + left) * 128 + x * 16) = make_uint4(0, 0, 0, 0);
                    __syncwarp();
                }
                float s[NR][4], s1[NR][4];                   // keys g (first two) and g + 8 of rows 8 n + 2c, + 1
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][e] = s1[n][e] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t f[4];
                    ldsm4(f, kt + (uint32_t)((k >> 2) * (KEYS * 128)) + (((uint32_t)((k & 3) * 2) + k_hi) ^ sw) * 16u);
#pragma unroll
                    for (int n = 0; n < NR; ++n) mma_16816(k & 1 ? s1[n] : s[n], f, q[k][n][0], q[k][n][1]);
                }
                bool grow = false;
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[n][e] = (e >> 1) * 8 + g < left ? (s[n][e] + s1[n][e]) * p.scale_log2 : -INFINITY;
                        grow = grow || s[n][e] > m[n][e & 1] + RESCALE_THRESHOLD;
                    }
                if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                    for (int n = 0; n < NR; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = fmaxf(m[n][e], fmaxf(s[n][e], s[n][e + 2]));
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                            const float f = top == -INFINITY ? 1.f : ex2(m[n][e] - top);
                            m[n][e] = top;
                            l[n][e] *= f;
#pragma unroll
                            for (int k = 0; k < KS; ++k) { o[k][n][e] *= f; o[k][n][e + 2] *= f; }
                        }
                }
                uint32_t b0[NR], b1[NR];
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const float r0 = m[n][0] == -INFINITY ? 0.f : m[n][0], r1 = m[n][1] == -INFINITY ? 0.f : m[n][1];
                    const float e0 = ex2(s[n][0] - r0), e1 = ex2(s[n][1] - r1), e2 = ex2(s[n][2] - r0), e3 = ex2(s[n][3] - r1);
                    l[n][0] += e0 + e2;
                    l[n][1] += e1 + e3;
                    b0[n] = transpose_8x8(pack_bf16(e0, e1));
                    b1[n] = transpose_8x8(pack_bf16(e2, e3));
                }
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t f[4];
                    ldsm4_t(f, vt + (uint32_t)((k >> 2) * (KEYS * 128)) + (((uint32_t)((k & 3) * 2) + v_hi) ^ sw) * 16u);
#pragma unroll
                    for (int n = 0; n < NR; ++n) mma_16816(o[k][n], f, b0[n], b1[n]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars->empty[st]));
        }
        if (!ok) l[0][0] = l[0][1] = l[NR - 1][0] = l[NR - 1][1] = __int_as_float(0x7fffffff);
    }
    __syncthreads();                                         // every load has landed and been used: the stages become the meeting's memory
    if (warp < WARPS) {
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
                if (g == 0) *sh.ml(warp, n * 8 + 2 * c + e) = make_float2(m[n][e], l[n][e]);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    sh.acc(warp, n * 8 + 2 * c + e)[k * 16 + g] = o[k][n][e];
                    sh.acc(warp, n * 8 + 2 * c + e)[k * 16 + g + 8] = o[k][n][e + 2];
                }
            }
    }
    meet<__nv_bfloat16, DP, WARPS>(p, sh, w, split, tid);
}

template <typename T, int R, int U, int LPK, int NVL> cudaError_t launch(const XAttnArgs& a, cudaStream_t s) {
    constexpr int W = 8, smem = shared_bytes(W, R, LPK * Vec<T>::E * NVL);
    const RowParams p = plan_rows<xattn_rows_kernel<T, R, U, LPK, NVL, W>>(a, W * 32, R, smem, 32 / LPK * U * W);
    return cc::launch_clusters<xattn_rows_kernel<T, R, U, LPK, NVL, W>>({(int64_t)p.groups * a.Hkv * a.B * p.splits, W * 32, smem, smem, p.splits}, s, p);
}
template <int DP, int NR> cudaError_t launch_stream(const XAttnArgs& a, cudaStream_t s) {
    using C = StreamCfg<DP>;
    CUtensorMap tk, tv;
    StreamParams sp;
    if (!encode_kv(&tk, a, a.k, a.sk, C::KEYS, &sp.kh, &sp.kb) || !encode_kv(&tv, a, a.v, a.sv, C::KEYS, &sp.vh, &sp.vb)) return cudaErrorInvalidValue;
    sp.p = plan_rows<xattn_stream_kernel<DP, NR>>(a, C::THREADS, NR * 8, C::SMEM, C::KEYS);
    return cc::launch_clusters<xattn_stream_kernel<DP, NR>>({(int64_t)sp.p.groups * a.Hkv * a.B * sp.p.splits, C::THREADS, C::SMEM, C::SMEM, sp.p.splits}, s, sp, tk, tv);
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
        // One row: few heads with long contexts want the ring's bytes in flight, many heads have them anyway and short contexts end
        // sooner without it (us, lanes / ring: 16 heads x 16000 keys of 64 23.5 / 16.6, 4 x 8000 of 128, 4 rows 33.7 / 12.5; 256 x 2000 43.1 / 45.4,
        // 32 x 100 4.8 / 6.5).  Two to four rows: 256 x 2000, two rows 48.0 / 45.8, 32 x 16384, four rows 103 / 47.
        // Heads of 256: 32 x 16384, one row 82 / 86, four 150 / 87, sixteen of 8000 keys 259 / 58.  Short contexts: 32 x 1000 of 128,
        // two rows 8.5 / 10.5, x 2000 11.1 / 10.9; 256 x 50, four rows 8.6 / 14.5, x 200 17.1 / 14.6.
        const bool ring = rows > 4 || a.Tk > (rows > 2 ? 128 : 1024);
        if ((rows > 1 ? ring : ring && a.D <= 128 && (int64_t)a.B * a.Hkv < 148) && kv_maps_supported(a, 256)) {
            if (a.D <= 64) return rows <= 8 ? launch_stream<64, 1>(a, s) : launch_stream<64, 2>(a, s);
            if (a.D <= 128) return rows <= 8 ? launch_stream<128, 1>(a, s) : launch_stream<128, 2>(a, s);
            return rows <= 8 ? launch_stream<256, 1>(a, s) : launch_stream<256, 2>(a, s);
        }
        return rows == 1 ? launch_rows<__nv_bfloat16, 1>(a, s) : rows == 2 ? launch_rows<__nv_bfloat16, 2>(a, s) : launch_rows<__nv_bfloat16, 4>(a, s);
    }
    return rows == 1 ? launch_rows<float, 1>(a, s) : rows == 2 ? launch_rows<float, 2>(a, s) : launch_rows<float, 4>(a, s);
}

}  // namespace vd
