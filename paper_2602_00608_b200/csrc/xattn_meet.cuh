// What the attention kernels for few rows and for single precision share: rows of a key head taken in groups, the division of the keys
// among the CTAs of a cluster, and how these add their shares up.
#pragma once
#include <mutex>

#include "block_ops.h"
#include "conv_cluster.cuh"
#include "tc_common.cuh"
#include "tc_pair.cuh"

namespace vd {
namespace xa {

using namespace tc;

constexpr int MAX_SPLITS = 8;
constexpr float RESCALE_THRESHOLD = 8.0f;                    // log2 units: sums may grow by 2^8 before their reference moves

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
__device__ __forceinline__ void unpack2(unsigned long long v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }

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
template <int DM, int WARPS> struct Shared {
    float* base;
    int rows;
    __device__ __forceinline__ Shared(float* b, int r) : base(b), rows(r) {}
    __device__ __forceinline__ float* acc(int warp, int r) const { return base + (warp * rows + r) * DM; }
    __device__ __forceinline__ float* out(int r) const { return acc(WARPS, r); }
    __device__ __forceinline__ float2* ml(int warp, int r) const { return (float2*)acc(WARPS + 1, 0) + warp * rows + r; }
    __device__ __forceinline__ float2* om(int r) const { return ml(WARPS, r); }
};
constexpr int shared_bytes(int warps, int rows, int dm) { return (warps + 1) * rows * (dm + 2) * 4; }

// CTAs of a cluster, each with its rows' unnormalised outputs [rows][DM] and (maximum, sum) in shared memory: added up in a fixed
// order and written, every CTA a part.
template <typename T, int DM, int THREADS>
__device__ __forceinline__ void meet_cluster(const RowParams& p, const float* out_rows, const float2* om, const Work& w, int split, int tid) {
    const XAttnArgs& a = p.a;
    cluster_sync_all();                                      // every CTA's share is in its shared memory
    for (int i = split * THREADS + tid; i < w.rows * DM && tid < THREADS; i += p.splits * THREADS) {
        const int r = i / DM, d = i % DM;
        if (d >= a.D) continue;
        float m[MAX_SPLITS], sum[MAX_SPLITS], o[MAX_SPLITS], top = -INFINITY;
#pragma unroll
        for (int c = 0; c < MAX_SPLITS; ++c)
            if (c < p.splits) {
                const uint32_t at_om = map_to_cta(smem_u32(om + r), (uint32_t)c), at = map_to_cta(smem_u32(out_rows + r * DM + d), (uint32_t)c);
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m[c]), "=f"(sum[c]) : "r"(at_om) : "memory");
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

// clusters of `splits` CTAs of KERNEL that the current device holds at once (0: none), asked once per device
template <auto KERNEL> int clusters_held(int threads, int smem, int splits) {
    static std::mutex mu;
    static int known[cc::kMaxDevices][MAX_SPLITS] = {};      // 0: not asked, else the answer + 1
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= cc::kMaxDevices || cc::set_smem_limit<KERNEL>(smem) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    std::lock_guard<std::mutex> lock(mu);
    int& k = known[dev][splits - 1];
    if (k == 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)splits);
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = (size_t)smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)splits; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, (const void*)KERNEL, &cfg) != cudaSuccess) { cudaGetLastError(); n = 0; }
        k = n + 1;
    }
    return k - 1;
}

// CTAs that share the keys of a group: the fewest waves of clusters x (rounds of a CTA + what a CTA costs besides, in rounds)
template <auto KERNEL> RowParams plan_rows(const XAttnArgs& a, int threads, int rows, int smem, int round) {
    RowParams p{a, a.H / a.Hkv, 0, 1, a.scale * 1.4426950408889634f};
    p.groups = (int)(((int64_t)a.Tq * p.g + rows - 1) / rows);
    const int64_t items = (int64_t)p.groups * a.Hkv * a.B;
    double best = 0.0;
    for (int n = 1; n <= MAX_SPLITS && (n == 1 || (n - 1) * round < a.Tk); ++n) {
        const int held = clusters_held<KERNEL>(threads, smem, n);
        if (held < 1) continue;
        const double cost = (double)((items + held - 1) / held) * ((a.Tk + n * round - 1) / (n * round) + (n == 1 ? 2.0 : 3.0));
        if (best == 0.0 || cost < best) { best = cost; p.splits = n; }
    }
    return p;
}
}  // namespace xa
}  // namespace vd
