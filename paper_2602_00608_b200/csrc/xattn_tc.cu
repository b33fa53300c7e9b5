// Attention to states of another length on tcgen05/TMEM (bf16, heads of up to 256 channels):
//   o[b,t,h] = sum_{u < len[b]} softmax_u(scale q[b,t,h].k[b,u,h/g]) v[b,u,h/g]
// An item is up to 256 rows of one key head: two tiles of 128 rows (a row is a token and one of the g heads that share the key head,
// packed by the tensor map), each with a warpgroup of its own, one thread per row, so that a row's maximum and sum need no other
// thread.  The two tiles take every block of 128 keys from shared memory together, and while one is in its softmax the tensor core
// works for the other:
//   S = Q K^T      K as it lies in memory, K-major
//   softmax        running maximum with lazy rescaling of the output accumulator (by powers of two, exactly); P in bf16 back to tensor memory,
//                  a half at a time, so that the second half's exponentials overlap the first half's product
//   O += P V       P from tensor memory, V as it lies in memory (MN-major): nothing is transposed
// Heads beyond 128 channels: an item is one tile, whose products (2048 clocks) the softmax of half a tile at a time still overlaps: 9472 x 8192, 8
// heads of 256 520 us, 1220 TFLOP/s (in tiles on the FP32 pipes 2000 x 3000 takes 1843 us, here 62); their keys are not divided.
// CTAs are persistent, one per SM (contexts of one tile: two); the next item's Q, K and scores are under way during an item's last rows.
// Rounded to bf16 are P (a half step, up to 2^-8 of a value, as the operand type asks) and the output; S, O, maxima and sums are fp32.
// What bounds it.  A tile of 128 rows x 128 keys with heads of 128 takes the tensor core 1024 clocks (4096 multiply-adds each) and the special
// function units as many (16 exponentials each): 9472 x 8192, 16 heads 477 us in a burst, 1330 TFLOP/s of the 1625 that a large matrix
// product reaches, tensor pipe 62 % busy (4096 keys); run for long, the board's power holds back both (5400 x 14400 1060 TFLOP/s of 1397).
// Heads of 64 halve the products and leave the exponentials: 8 x 1350 x 1350, 30 heads 187 us, special function units 63 % busy, the rest the
// chain of scores, maximum, exponentials and product, which two tiles overlap and tensor memory has no room for a third.
// Keys behind a row's length: scores are replaced before the maximum, P is zero there, and the up to 15 rows of V that the last
// product still reads are zeroed in shared memory, since 0 * NaN is NaN.
// Every wait is bounded (see tc_common.cuh; where CTAs wait for one another the bound grows with the keys); rows of an item whose wait gave
// up are NaN.
#include <math.h>

#include <algorithm>
#include <atomic>

#include "block_ops.h"
#include "conv_cluster.cuh"
#include "tc_common.cuh"
#include "xattn_maps.h"
#include "xattn_meet.cuh"

namespace vd {
namespace {

using namespace tc;

constexpr int ROWS = 128, KEYS = 128, CHUNK = 64;            // of a tile; channels of a 128-byte row
constexpr int HALF = KEYS / 2;                               // keys of P that go to the tensor core at a time
constexpr int SOFTMAX_WARPS = 8, LOAD_WARP = 8, MMA_WARP = 9, NUM_THREADS = 352;     // MMA_WARP + s issues for tile s
constexpr int MAX_LENS = 128;                                // lengths that are kept in shared memory
constexpr int MAX_SPLITS = xa::MAX_SPLITS;
// What a meeting costs, in tiles, by the loops and with all loads under way (18000 clocks; a tile is 2000 to 3000).  Dividing: 2 x 300 x 3000, 8 heads of
// 128 49 -> 33 us; 5400 x 14400, 16 heads (352 items on 148 SMs: 2 rounds and a rest instead of 3) 596 -> 523; 9472 x 8192, 16 heads of 64 469 -> 453.
constexpr double MEET_REST = 8.0, MEET_ALL = 5.0;
constexpr float RESCALE_THRESHOLD = 8.0f;                    // log2 units: accumulators may grow by 2^8

template <int DP, bool SHORT = false> struct Cfg {
    static constexpr int CHUNKS = DP / CHUNK;
    static constexpr int TILE_BYTES = ROWS * DP * 2;         // of Q (a tile), K or V
    static constexpr int TILES = DP == 256 ? 1 : 2;          // of an item: tensor memory has no room for two O of 256 channels
    static constexpr int STAGES = SHORT || DP == 256 ? 2 : DP == 128 ? 3 : 6, Q_BUFS = SHORT || DP > 64 ? 1 : 2;
    static constexpr bool O_OVER_Q = DP == 256;              // shared memory has none for O on its way out: it takes Q's place
    // Tensor memory has room for a P of its own beside the scores where O takes 64 columns: the next scores then do not wait for the
    // products of P.  Columns of tile s: S at 128 s, O at O_COL + O_STEP s, P at P_COL + P_STEP s.  SHORT: the second half of S is O's.
    static constexpr bool APART = DP == 64;
    static constexpr uint32_t TMEM = SHORT ? 256 : 512, P_COL = APART && !SHORT ? 384 : 0, P_STEP = APART && !SHORT ? 64 : 128;
    static constexpr uint32_t O_COL = SHORT ? 64 : 256, O_STEP = SHORT ? 128 : DP;
    static constexpr int MMA_WARPS = APART ? 2 : 1;
    static constexpr int SMEM = (Q_BUFS * TILES + (O_OVER_Q ? 0 : TILES) + STAGES) * TILE_BYTES + 2 * ROWS * 8 + MAX_LENS * 4 + 320;     // Q, O on its way out, K and V; (reference, sum) of the rows
};
struct Bars {
    uint64_t q_full[2], q_empty[2], full[6], empty[6], s_full[2], s_free[2], p_part[2][2], pv_done[2], o_full[2], drained[2], shown[2], seen[2], o_left;
    uint32_t tmem_base, abort_flag, lost[2];                 // lost: a wait at a meeting of tile s gave up
};
static_assert(sizeof(Bars) <= 320 && Cfg<256>::SMEM <= 232448 && Cfg<128>::SMEM <= 232448 && Cfg<64>::SMEM <= 232448 && 2 * (Cfg<64, true>::SMEM + 1024) <= 233472, "shared memory of one CTA");

struct Params {
    const int32_t* lens;
    int Tq, Tk, B, Hkv, g, D, nt;    // nt: tokens of a tile
    int q_items;                     // items of a (batch item, key head)
    int dq, dh, db;                  // from one item of a CTA to its next: the grid as (items, heads, batch items)
    int kb, vb, kh, vh;              // 0: the batch (head) coordinate of k or v stays 0
    uint32_t items, whole;           // the first `whole` items are a CTA's each, the others a cluster's, whose CTAs divide the keys
    int splits;                      // CTAs of a cluster
    __nv_bfloat16* o;
    int64_t o_batch, o_token, o_head;
    float scale_log2, scale_far;     // scale_far: the power of two at or above it (Scaled)
    long long wait_limit;            // cycles, where CTAs wait for one another (launch_xattn_tc)
    long long meeting_limit;         // the same at meetings; negative: they give up at once (a test's)
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {       // NaN if one is
    float y;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ void unpack2(unsigned long long v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const void* tmap, int c0, int c1, int c2, int c3, int c4, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
        ::"r"(dst), "l"(tmap), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(bar) : "memory");
}
// A from tensor memory, predicated like umma_bf16_split_on
__device__ __forceinline__ void umma_bf16_ts_on(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t idesc,
                                                uint32_t accumulate, uint32_t on) {
    asm volatile(
        "{\n.reg .pred p, q;\n.reg .b64 db;\nsetp.ne.b32 p, %5, 0;\nsetp.ne.b32 q, %6, 0;\nmov.b64 db, {%2, %3};\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n}\n"
        ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate), "r"(on) : "memory");
}

__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// of a wait within a CTA, which may be for a role or a tile that is at a meeting
template <bool SPLIT> __device__ __forceinline__ long long limit(const Params& a) { return SPLIT ? a.wait_limit : WAIT_LIMIT_CYCLES; }
// Scores become exponents by one fused multiply-add, score * scale - reference, whose product is not rounded while the reference is one
// that was: half a step of the reference is left over, a common factor, which beyond 2^31 is an exponent of hundreds. So scores
// beyond FAR are scaled by a power of two instead, which rounds nothing. They lie 32 or more apart there (a step of fp32), so nothing but the largest
// weighs in, with either scale; and the scaling stays monotonic, so that maxima, references and their differences mean what they do elsewhere.
constexpr float FAR = 536870912.f;                           // 2^29: the factor of half a step below it is 2^16
struct Scaled {
    float near, far;
    __device__ __forceinline__ float score(float s) const { return fabsf(s * near) > FAR ? s * far : s * near; }
};
// N = 32 or 16 scores into as many numbers of P: 2^(score * scale - reference), their sums, bf16
template <int N = 32>
__device__ __forceinline__ void exp_chunk(const uint32_t (&r)[32], uint32_t t_p, unsigned long long sc, unsigned long long mr,
                                          unsigned long long& sum, unsigned long long& sum_b) {
    uint32_t pk[16];
#pragma unroll
    for (int q = 0; q < N; q += 2) {
        float e0, e1;
        unpack2(fmaf2(pack2(__uint_as_float(r[q]), __uint_as_float(r[q + 1])), sc, mr), e0, e1);
        e0 = ex2(e0);
        e1 = ex2(e1);
        if (q & 2) sum_b = add2(sum_b, pack2(e0, e1));
        else sum = add2(sum, pack2(e0, e1));
        pk[q >> 1] = pack_bf16(e0, e1);
    }
    if (N == 32) tmem_st16(t_p, pk);
    else tmem_st8(t_p, pk);
}
__device__ __forceinline__ float max_of(const uint32_t (&r)[32], float m) {
    float a = max3(__uint_as_float(r[0]), __uint_as_float(r[1]), m), b = max3(__uint_as_float(r[2]), __uint_as_float(r[3]), __uint_as_float(r[4]));
#pragma unroll
    for (int q = 5; q < 29; q += 4) {
        a = max3(a, __uint_as_float(r[q]), __uint_as_float(r[q + 1]));
        b = max3(b, __uint_as_float(r[q + 2]), __uint_as_float(r[q + 3]));
    }
    a = max3(a, __uint_as_float(r[29]), __uint_as_float(r[30]));
    return max3(a, b, __uint_as_float(r[31]));
}
// P as far as it is written (scores as far as they are read) is the tensor core's
__device__ __forceinline__ void hand_over(uint64_t* bar, int lane) {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(bar));
}
// One row's tile of scores: exponentials into P.  Where P lies over the scores, 32 of them make 16 columns of it, so those still to be read
// are not touched.
template <int DP, bool SPLIT> struct Tile {
    const Params& params;
    Scaled to_log2;
    uint32_t t_s, t_p, t_o;
    bool rescale;                // O holds something
    uint64_t* s_free;            // to be told when the scores have been read, or null
    uint64_t* pv_done;           // to be waited for before P is written or O rescaled, or null
    uint32_t pv_parity;
    volatile uint32_t* abort_flag;
    int lane;
    float m_ref;
    unsigned long long sum, sum_b;       // of even and odd pairs of keys
    bool ok = true;

    __device__ __forceinline__ float scale() const { return fabsf(m_ref) > FAR ? to_log2.far : to_log2.near; }
    // What the exponentials are relative to: at first the maximum itself, whose P is then 1 and is not rounded (a row that one key has, or all
    // but has, is that key's value).  It stays unless a score exceeds it by more than the threshold, and moves by a whole number, so
    // that what has been summed (O, the sums, P as far as it is written) is rescaled by a power of two, without rounding.
    __device__ __forceinline__ void move_reference(float score, uint32_t p_cols) {
        // (a far reference, or none yet: every score is looked at closely; score() for every tile: 5400 x 14400, 16 heads of 128 540 us instead of 522)
        if (!__any_sync(0xffffffffu, score * to_log2.near > (fabsf(m_ref) > FAR ? -INFINITY : m_ref + RESCALE_THRESHOLD))) return;
        const float top = to_log2.score(score);
        const bool grow = top > m_ref + RESCALE_THRESHOLD;
        float factor = 1.f;
        if (grow) {
            const float by = ceilf(top - m_ref);             // (infinite at the first tile)
            factor = by < 127.f ? __int_as_float((127 - (int)by) << 23) : 0.f;
            m_ref = by < 127.f ? m_ref + by : top;
        }
        if (!__any_sync(0xffffffffu, grow)) return;
        sum = fmaf2(sum, pack2(factor, factor), 0ull);
        sum_b = fmaf2(sum_b, pack2(factor, factor), 0ull);
        if (p_cols) tmem_st_wait();
#pragma unroll 1
        for (uint32_t c = 0; c < p_cols; c += 16u) {
            uint32_t v[16];
            tmem_ld16(t_p + c, v);
            tmem_ld_wait();
            const __nv_bfloat162 f = __floats2bfloat162_rn(factor, factor);
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&v[q]), f);
                v[q] = *reinterpret_cast<const uint32_t*>(&x);
            }
            tmem_st16(t_p + c, v);
        }
        if (rescale) {
#pragma unroll 1
            for (uint32_t c = 0; c < (uint32_t)DP; c += 16u) {
                uint32_t o[16];
                tmem_ld16(t_o + c, o);
                tmem_ld_wait();
#pragma unroll
                for (int q = 0; q < 16; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * factor);
                tmem_st16(t_o + c, o);
            }
        }
    }
    __device__ __forceinline__ unsigned long long minus_ref() const {
        const float ref = m_ref == -INFINITY ? 0.f : m_ref;
        return pack2(-ref, -ref);
    }
    // (Without a barrier to wait for: the scores were issued behind the last product into O and of P, which is complete then.)
    __device__ __forceinline__ void wait_pv() {
        if (!pv_done) return;
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(pv_done), pv_parity, abort_flag, limit<SPLIT>(params))) && ok;
        tc_fence_after();
    }
    // All 128 keys count.  The maximum is only needed to see that the reference may stay, so it is taken half a tile at a time in front
    // of the exponentials, and the first half of P goes to the tensor core while the second one is made.  Returns the tile's maximum, NaN if
    // a score is.
    __device__ __forceinline__ float full(uint64_t* first_half) {
        uint32_t a[32], b[32], c[32];
        tmem_ld32(t_s, a);
        tmem_ld32(t_s + 32u, b);
        tmem_ld32(t_s + 64u, c);
        tmem_ld_wait();
        const float t0 = max_of(b, max_of(a, -INFINITY));
        wait_pv();
        move_reference(t0, 0u);
        unsigned long long sc = pack2(scale(), scale()), mr = minus_ref();
        exp_chunk(a, t_p, sc, mr, sum, sum_b);
        tmem_ld32(t_s + 96u, a);
        exp_chunk(b, t_p + 16u, sc, mr, sum, sum_b);
        tmem_ld_wait();
        if (s_free) hand_over(s_free, lane);
        const float t1 = max_of(a, max_of(c, t0));
        move_reference(t1, 32u);
        tmem_st_wait();
        hand_over(first_half, lane);
        sc = pack2(scale(), scale());
        mr = minus_ref();
        exp_chunk(c, t_p + 32u, sc, mr, sum, sum_b);
        exp_chunk(a, t_p + 48u, sc, mr, sum, sum_b);
        return t1;
    }
    // The same where only the first `valid` <= 96 keys count: the others leave before the maximum, 16 keys are the least that is worked on.
    __device__ __forceinline__ float most(int valid, uint64_t* first_half) {
        uint32_t a[32], b[32], c[32];
        tmem_ld32(t_s, a);
        tmem_ld32(t_s + 32u, b);
        tmem_ld32(t_s + 64u, c);
        tmem_ld_wait();
        if (valid < 32) mask(a, valid);
        float top = max_of(a, -INFINITY);
        if (valid > 32) {
            if (valid < 64) mask(b, valid - 32);
            top = max_of(b, top);
        }
        if (valid > 64) {
            if (valid < 96) mask(c, valid - 64);
            top = max_of(c, top);
        }
        wait_pv();
        move_reference(top, 0u);
        const unsigned long long sc = pack2(scale(), scale()), mr = minus_ref();
        if (valid > 16) exp_chunk(a, t_p, sc, mr, sum, sum_b);
        else exp_chunk<16>(a, t_p, sc, mr, sum, sum_b);
        if (valid > 48) exp_chunk(b, t_p + 16u, sc, mr, sum, sum_b);
        else if (valid > 32) exp_chunk<16>(b, t_p + 16u, sc, mr, sum, sum_b);
        tmem_st_wait();
        hand_over(first_half, lane);
        if (valid > 80) exp_chunk(c, t_p + 32u, sc, mr, sum, sum_b);
        else if (valid > 64) exp_chunk<16>(c, t_p + 32u, sc, mr, sum, sum_b);
        return top;
    }
    // The same for any number of them, 32 at a time.  (The code of full() with masks spills.)
    __device__ __forceinline__ float part(int valid, uint64_t* first_half) {
        uint32_t r[32];
        float top = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < valid; c += 32) {
            tmem_ld32(t_s + (uint32_t)c, r);
            tmem_ld_wait();
            if (valid - c < 32) mask(r, valid - c);
            top = max_of(r, top);
        }
        wait_pv();
        move_reference(top, 0u);
        const unsigned long long sc = pack2(scale(), scale()), mr = minus_ref();
#pragma unroll 1
        for (int c = 0; c < valid; c += 32) {
            tmem_ld32(t_s + (uint32_t)c, r);
            tmem_ld_wait();
            if (valid - c < 32) mask(r, valid - c);
            exp_chunk(r, t_p + (uint32_t)(c >> 1), sc, mr, sum, sum_b);
        }
        tmem_st_wait();
        hand_over(first_half, lane);
        return top;
    }
    // The only tile of a row: its maximum is the reference.  Two passes, 32 scores at a time, since two CTAs share the registers.
    __device__ __forceinline__ float only(int valid) {
        uint32_t r[32];
        float top = -INFINITY;
#pragma unroll
        for (int c = 0; c < KEYS; c += 32)
            if (c < valid) {
                tmem_ld32(t_s + (uint32_t)c, r);
                tmem_ld_wait();
                if (valid - c < 32) mask(r, valid - c);
                top = max_of(r, top);
            }
        m_ref = to_log2.score(top);
        const unsigned long long sc = pack2(scale(), scale()), mr = minus_ref();
#pragma unroll
        for (int c = 0; c < KEYS; c += 32)
            if (c < valid) {
                tmem_ld32(t_s + (uint32_t)c, r);
                tmem_ld_wait();
                if (valid - c > 16) {
                    if (valid - c < 32) mask(r, valid - c);
                    exp_chunk(r, t_p + (uint32_t)(c >> 1), sc, mr, sum, sum_b);
                } else {
                    mask<16>(r, valid - c);
                    exp_chunk<16>(r, t_p + (uint32_t)(c >> 1), sc, mr, sum, sum_b);
                }
            }
        return top;
    }
    template <int N = 32> static __device__ __forceinline__ void mask(uint32_t (&r)[32], int valid) {
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (q >= valid) r[q] = __float_as_uint(-INFINITY);
    }
};

// A CTA's items: of the whole ones those one grid apart (no divisions on the way), then its share of the keys of its cluster's.
template <bool SPLIT, int TILES = 2> struct Items {
    int b, kvh, qt, t0, streams, len, tiles;     // tiles of the item, of which [j0, j0 + n) are this CTA's
    int j0, n;
    uint32_t at;
    bool first = true, split = false;        // (without SPLIT all items are whole)
    __device__ __forceinline__ void place(const Params& a) {
        const uint32_t bh = at / (uint32_t)a.q_items;
        qt = (int)(at - bh * (uint32_t)a.q_items);
        b = (int)(bh / (uint32_t)a.Hkv);
        kvh = (int)(bh - (uint32_t)b * (uint32_t)a.Hkv);
    }
    __device__ __forceinline__ Items(const Params& a) : at(blockIdx.x) { place(a); }
    __device__ __forceinline__ bool take(const Params& a, const int* lens) {
        if (!SPLIT || !split) {
            if (!first) {
                at += gridDim.x;
                qt += a.dq; kvh += a.dh; b += a.db;
                if (qt >= a.q_items) { qt -= a.q_items; ++kvh; }
                if (kvh >= a.Hkv) { kvh -= a.Hkv; ++b; }
            }
            first = false;
            if (SPLIT && at >= a.whole) {
                split = true;
                at = a.whole + blockIdx.x / (uint32_t)a.splits;
                place(a);
            }
        } else {
            at += gridDim.x / (uint32_t)a.splits;
            place(a);
        }
        if (at >= a.items) return false;
        t0 = qt * TILES * a.nt;
        streams = TILES == 2 && t0 + a.nt < a.Tq ? 2 : 1;
        len = !a.lens ? a.Tk : min(max(b < MAX_LENS ? lens[b] : a.lens[b], 0), a.Tk);
        tiles = (len + KEYS - 1) / KEYS;
        j0 = 0;
        n = tiles;
        if (SPLIT && split) {                                // (at most 2^23 tiles, 8 shares)
            const int rank = (int)(blockIdx.x % (uint32_t)a.splits);
            j0 = tiles * rank / a.splits;
            n = tiles * (rank + 1) / a.splits - j0;
        }
        return true;
    }
};
__device__ __forceinline__ void arrive_release_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
// cc::wait_cluster with a limit of the call's
__device__ __forceinline__ bool heard(const Params& a, uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
    const long long t0 = clock64();
    while (a.meeting_limit < 0 || !cc::try_wait_cluster(smem_u32(bar), parity))
        if (a.meeting_limit < 0 || clock64() - t0 > a.meeting_limit) {
            *abort_flag = 1;
            return false;
        }
    return true;
}
// The CTAs of a cluster have each taken a share of an item's keys: they show one another half of the channels at a time, in fp32, and each
// adds up (in the order of the shares) and writes its part of the tile's rows.  By the 128 threads of tile s; `rounds` counts what these
// have shown so far.  Once a wait gave up the others are told nothing more, so that they give up too and nobody takes old or half-written shares
// for an item's: what a CTA still writes is NaN.  A load of another CTA's memory takes 900 cycles.  FAST: a thread has a row, its weights in
// registers and all shares' loads under way at once (18000 instead of 29000 cycles a meeting), which crowds the softmax's registers: calls with
// whole items besides take the loops, out of line (5400 x 14400, 16 heads of 128 519 us, FAST 546).
template <int DP, bool FAST>
__device__ __forceinline__ void meet_inline(const Params& a, const Items<true>& it, Bars* bars, uint8_t* show, float2* ml, float2 mine, uint32_t t_o, int s, int row, uint32_t rounds) {
    constexpr int COLS = DP / 2, PIECES = COLS / 4;          // of a round; 16-byte pieces of them
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int rank = (int)cluster_ctarank();
    volatile uint32_t* lost = &bars->lost[s];
    bool ok = true;
    auto tell = [&](uint64_t* bar) {
        if (!ok) *lost = 1;                                  // (read behind the barrier; as barrier.red of `ok` the meetings took 2 us more)
        named_barrier_sync(1 + s, ROWS);
        if (row < a.splits && !*lost) arrive_release_cluster(map_to_cta(smem_u32(bar), (uint32_t)row));
    };
    auto hear = [&](uint64_t* bar, uint32_t parity) { ok = __all_sync(0xffffffffu, ok && !*lost && heard(a, bar, parity, abort_flag)); };
    const int r0 = ROWS * rank / a.splits, r1 = ROWS * (rank + 1) / a.splits;
    // FAST: this thread's row of the CTA's part, and how many threads it has
    const int per_row = ROWS / ((ROWS + a.splits - 1) / a.splits), r = r0 + row / per_row, tt = r / a.g, t = it.t0 + s * a.nt + tt;
    const bool mine_to_write = r < r1 && tt < a.nt && t < a.Tq;
    __nv_bfloat16* out = a.o + it.b * a.o_batch + t * a.o_token + (it.kvh * a.g + r - tt * a.g) * a.o_head;
    float f[MAX_SPLITS];                                     // the shares' weights
    for (int round = 0; round < 2; ++round, ++rounds) {
        if (rounds > 0) hear(&bars->seen[s], (rounds - 1) & 1);      // everybody has read what was shown last
        if (ok) {                                           // (the same for a warp)
            if (round == 0) ml[row] = mine;
#pragma unroll
            for (int c = 0; c < COLS; c += 32) {
                uint32_t v[32];
                if (it.n) {
                    tmem_ld32(t_o + (uint32_t)(round * COLS + c), v);
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int q = 0; q < 32; ++q) v[q] = 0u;
                }
#pragma unroll
                for (int q = 0; q < 32; q += 4)
                    *(uint4*)(show + row * (COLS * 4) + ((((c + q) >> 2) ^ (row & (PIECES - 1))) << 4)) = make_uint4(v[q], v[q + 1], v[q + 2], v[q + 3]);
            }
        }
        tell(&bars->shown[s]);
        hear(&bars->shown[s], rounds & 1);
        if (FAST && mine_to_write) {
            if (round == 0) {
                const uint32_t at = smem_u32(ml + r);
                float2 w[MAX_SPLITS];
#pragma unroll
                for (int k = 0; k < MAX_SPLITS; ++k)
                    if (k < a.splits) w[k] = ld_cluster2(map_to_cta(at, (uint32_t)k));
                float top = -INFINITY, l = 0.f;
#pragma unroll
                for (int k = 0; k < MAX_SPLITS; ++k)
                    if (k < a.splits) top = fmaxf(top, w[k].x);
                const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
                for (int k = 0; k < MAX_SPLITS; ++k)
                    if (k < a.splits) { f[k] = ex2(w[k].x - ref); l = fmaf(f[k], w[k].y, l); }
#pragma unroll
                for (int k = 0; k < MAX_SPLITS; ++k)
                    if (k < a.splits) f[k] /= l;
            }
            if (!ok)
#pragma unroll
                for (int k = 0; k < MAX_SPLITS; ++k) f[k] = __int_as_float(0x7fffffff);
            for (int piece = row % per_row; piece < PIECES; piece += per_row) {
                const int d = round * COLS + piece * 4;
                if (d >= a.D) break;
                const uint32_t at = smem_u32(show + r * (COLS * 4) + ((piece ^ (r & (PIECES - 1))) << 4));
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k0 = 0; k0 < MAX_SPLITS; k0 += 4) {
                    float4 v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k0 + k < a.splits) v[k] = ld_cluster4(map_to_cta(at, (uint32_t)(k0 + k)));
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k0 + k < a.splits) { const float g = f[k0 + k]; o.x = fmaf(g, v[k].x, o.x); o.y = fmaf(g, v[k].y, o.y); o.z = fmaf(g, v[k].z, o.z); o.w = fmaf(g, v[k].w, o.w); }
                }
                *(uint2*)(out + d) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
            }
        }
        for (int i = FAST ? r1 * PIECES : r0 * PIECES + row; i < r1 * PIECES; i += ROWS) {
            const int r = i / PIECES, piece = i % PIECES, tt = r / a.g, t = it.t0 + s * a.nt + tt, d = round * COLS + piece * 4;
            if (tt >= a.nt || t >= a.Tq || d >= a.D) continue;
            const uint32_t at = smem_u32(show + r * (COLS * 4) + ((piece ^ (r & (PIECES - 1))) << 4)), at_ml = smem_u32(ml + r);
            float top = -INFINITY;
#pragma unroll 4
            for (int k = 0; k < a.splits; ++k) top = fmaxf(top, ld_cluster2(map_to_cta(at_ml, (uint32_t)k)).x);
            const float ref = top == -INFINITY ? 0.f : top;
            float l = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
            for (int k = 0; k < a.splits; ++k) {
                const float2 w = ld_cluster2(map_to_cta(at_ml, (uint32_t)k));
                const float4 v = ld_cluster4(map_to_cta(at, (uint32_t)k));
                const float f = ex2(w.x - ref);
                l = fmaf(f, w.y, l);
                o.x = fmaf(f, v.x, o.x); o.y = fmaf(f, v.y, o.y); o.z = fmaf(f, v.z, o.z); o.w = fmaf(f, v.w, o.w);
            }
            const float inv = ok ? 1.f / l : __int_as_float(0x7fffffff);
            *(uint2*)(a.o + it.b * a.o_batch + t * a.o_token + (it.kvh * a.g + r - tt * a.g) * a.o_head + d) =
                make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
        }
        __syncwarp();
        tell(&bars->seen[s]);
    }
}
template <int DP>
__device__ __noinline__ void meet_out_of_line(const Params& a, const Items<true>& it, Bars* bars, uint8_t* show, float2* ml, float2 mine, uint32_t t_o, int s, int row, uint32_t rounds) {
    meet_inline<DP, false>(a, it, bars, show, ml, mine, t_o, s, row, rounds);
}
// Before the rows of a divided item without keys: what was shown at the last meeting has been read.  If it may not have been, they leave straight
// from the threads: false.
__device__ __noinline__ bool seen_or_zeros(const Params& a, const Items<true>& it, Bars* bars, int s, int row, uint32_t rounds) {
    bool ok = !*(volatile uint32_t*)&bars->lost[s];
    ok = __all_sync(0xffffffffu, ok && heard(a, &bars->seen[s], (rounds - 1) & 1, &bars->abort_flag));
    if (named_barrier_all(1 + s, ROWS, ok)) return true;
    bars->lost[s] = 1;
    const int tt = row / a.g, t = it.t0 + s * a.nt + tt;
    if (tt < a.nt && t < a.Tq)
        for (int d = 0; d < a.D; d += 8)
            *(uint4*)(a.o + it.b * a.o_batch + t * a.o_token + (it.kvh * a.g + row - tt * a.g) * a.o_head + d) = make_uint4(0, 0, 0, 0);
    return false;
}

// DIVIDED: by keys among the CTAs of a cluster are no items, those that whole rounds leave over, or all (builds of their own: the code costs
// short items 20 % even where it is not reached).  SHORT: contexts of one tile with heads of up to 64 channels.  An item is then a chain of
// loads, scores, softmax, output and store with nothing to overlap, so two CTAs share an SM, each with half of its tensor memory (P and O
// both lie over the scores, which are read twice, 32 at a time: 80 registers a thread): 2 x 10800 x 77, 30 heads of 64 52 -> 41 us (3.2 -> 4.0
// TB/s), 8 x 1350 x 32, 16 heads 18.7 -> 15.8.
enum { NONE = 0, REST = 1, ALL = 2, SHORT = 3 };
template <int DP, int DIVIDED>
__global__ void __launch_bounds__(NUM_THREADS, DIVIDED == SHORT ? 2 : 1)
xattn_tc_kernel(const __grid_constant__ Params a, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_o) {
    constexpr bool ONE_TILE = DIVIDED == SHORT, SPLIT = DIVIDED == REST || DIVIDED == ALL;
    using C = Cfg<DP, ONE_TILE>;
    extern __shared__ __align__(1024) uint8_t smem_q[];
    if (smem_u32(smem_q) & 1023u) return;                    // (it is: the swizzle needs it)
    uint8_t* smem_o = smem_q + (C::O_OVER_Q ? 0 : C::Q_BUFS * C::TILES * C::TILE_BYTES);
    uint8_t* smem_st = smem_o + C::TILES * C::TILE_BYTES;
    float2* ml = (float2*)(smem_st + C::STAGES * C::TILE_BYTES);         // [2][ROWS]
    int* lens = (int*)(ml + 2 * ROWS);
    Bars* bars = (Bars*)(lens + MAX_LENS);
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars->q_full[i]), 1); mbar_init(smem_u32(&bars->q_empty[i]), C::MMA_WARPS);
            mbar_init(smem_u32(&bars->s_full[i]), 1); mbar_init(smem_u32(&bars->s_free[i]), SOFTMAX_WARPS / 2);
            for (int h = 0; h < 2; ++h) mbar_init(smem_u32(&bars->p_part[i][h]), SOFTMAX_WARPS / 2);
            mbar_init(smem_u32(&bars->pv_done[i]), 1); mbar_init(smem_u32(&bars->o_full[i]), 1); mbar_init(smem_u32(&bars->drained[i]), 1);
            mbar_init(smem_u32(&bars->shown[i]), (uint32_t)a.splits); mbar_init(smem_u32(&bars->seen[i]), (uint32_t)a.splits);
        }
        for (int i = 0; i < C::STAGES; ++i) { mbar_init(smem_u32(&bars->full[i]), 1); mbar_init(smem_u32(&bars->empty[i]), C::MMA_WARPS); }
        mbar_init(smem_u32(&bars->o_left), 1);
        bars->abort_flag = bars->lost[0] = bars->lost[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async_smem();
    }
    if (a.lens && tid < min(a.B, MAX_LENS)) lens[tid] = a.lens[tid];
    if (warp == MMA_WARP) tmem_alloc(smem_u32(&bars->tmem_base), C::TMEM);
    tc_fence_before();
    __syncthreads();
    if (SPLIT) cluster_sync_all();                    // every CTA's barriers exist before another one arrives on them
    tc_fence_after();
    const uint32_t tmem = bars->tmem_base;

    if (warp < SOFTMAX_WARPS) {
        // ------------------------------------------------------------ softmax: a thread per row
        const int s = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, t_s = tmem + lanes + (uint32_t)s * 128u, t_o = tmem + lanes + C::O_COL + (uint32_t)s * C::O_STEP, t_p = tmem + lanes + C::P_COL + (uint32_t)s * C::P_STEP;
        uint8_t* out = smem_o + s * C::TILE_BYTES + row * 128;
        const bool out_thread = (tid & (ROWS - 1)) == 0;
        uint32_t n_s = 0, n_o = 0, n_pv = 0, n_meet = 0;     // tiles, items, waited-for products and rounds of meetings so far
        bool ok = true;
        for (Items<SPLIT, C::TILES> it(a); it.take(a, lens);) {
            if (s >= it.streams || (SPLIT && it.split && it.tiles == 0 && blockIdx.x % (uint32_t)a.splits != 0)) continue;
            float m_ref = -INFINITY;
            unsigned long long sum = 0, sum_b = 0;           // of even and odd pairs of keys
            bool bad = false;
            for (int j = 0; j < it.n; ++j, ++n_s) {
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->s_full[s]), n_s & 1, abort_flag, limit<SPLIT>(a))) && ok;
                tc_fence_after();
                const int valid = it.len - (it.j0 + j) * KEYS;
                Tile<DP, SPLIT> tile{a, {a.scale_log2, a.scale_far}, t_s, t_p, t_o, j > 0, C::APART && j + 1 < it.n ? &bars->s_free[s] : nullptr,
                              C::APART && j > 0 ? &bars->pv_done[s] : nullptr, n_pv & 1, abort_flag, lane, m_ref, sum, sum_b};
                if (C::APART && j > 0) ++n_pv;
                float tmax;
                if constexpr (ONE_TILE) tmax = tile.only(valid);
                else tmax = valid >= KEYS ? tile.full(&bars->p_part[s][0]) : valid <= 96 ? tile.most(valid, &bars->p_part[s][0])
                                                                                            : tile.part(valid, &bars->p_part[s][0]);
                m_ref = tile.m_ref; sum = tile.sum; sum_b = tile.sum_b;
                ok = ok && tile.ok;
                bad = bad || !(tmax < INFINITY);             // a NaN or an infinity among the scores
                tmem_st_wait();
                hand_over(&bars->p_part[s][1], lane);
            }
            if (it.n) {
                ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars->o_full[s]), n_o & 1, abort_flag, limit<SPLIT>(a))) && ok;
                tc_fence_after();
                ++n_o;
            }
            const float l = ok && !bad ? sum2(add2(sum, sum_b)) : __int_as_float(0x7fffffff);
            if constexpr (SPLIT) {
                if (it.split && it.tiles) {
                    if (out_thread) bulk_wait_group_read<0>();
                    named_barrier_sync(1 + s, ROWS);
                    const float2 mine = make_float2(m_ref, it.n ? l : 0.f);
                    if constexpr (DIVIDED == ALL) meet_inline<DP, true>(a, it, bars, smem_o + s * C::TILE_BYTES, ml + s * ROWS, mine, t_o, s, row, n_meet);
                    else meet_out_of_line<DP>(a, it, bars, smem_o + s * C::TILE_BYTES, ml + s * ROWS, mine, t_o, s, row, n_meet);
                    n_meet += 2;
                    tc_fence_before();
                    continue;
                }
            }
            const float inv = it.tiles ? 1.f / l : 0.f;
            // the rows through shared memory (swizzled like the operands), out by a bulk tensor store that the next item's softmax does not wait
            // for: rows written straight from the threads, a line each, held the load/store unit for 2000 cycles an item
            if (out_thread) bulk_wait_group_read<0>();       // the last item's rows have left
            if constexpr (SPLIT) {
                if (n_meet && !seen_or_zeros(a, it, bars, s, row, n_meet)) continue;
            }
            named_barrier_sync(1 + s, ROWS);
#pragma unroll
            for (int c = 0; c < DP; c += 32)
                if (c < a.D) {
                    uint32_t v[32];
                    if (it.tiles) {
                        tmem_ld32(t_o + (uint32_t)c, v);
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int q = 0; q < 32; ++q) v[q] = 0u;
                    }
                    if (ONE_TILE && it.tiles && c + 32 >= a.D) hand_over(&bars->s_free[s], lane);      // O, where the next scores come, has been read
#pragma unroll
                    for (int q = 0; q < 32; q += 8) {
                        float f[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(v[q + e]) * inv;
                        *(uint4*)(out + (c / 64) * (ROWS * 128) + (((uint32_t)((c % 64 + q) / 8) ^ (uint32_t)(row & 7)) << 4)) =
                            make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
                    }
                }
            fence_proxy_async_smem();
            named_barrier_sync(1 + s, ROWS);
            if (out_thread) {
                for (int c = 0; c < C::CHUNKS && c * CHUNK < a.D; ++c)
                    tma_store_5d(&tm_o, smem_u32(smem_o + s * C::TILE_BYTES + c * (ROWS * 128)), c * CHUNK, 0, it.t0 + s * a.nt, it.kvh, it.b);
                bulk_commit_group();
                if (C::O_OVER_Q) {
                    bulk_wait_group_read<0>();
                    mbar_arrive(smem_u32(&bars->o_left));
                }
            }
            tc_fence_before();                               // (the next product into O waits for this warp's next P)
        }
        if (out_thread) bulk_wait_group_read<0>();           // before the CTA's memory goes
    } else if (warp == LOAD_WARP) {
        // ------------------------------------------------------------ loads: Q, then K and V of each tile in turn
        if (lane == 0) {
            uint32_t st = 0, ph = 0;
            int issued = 0, q_issued = 0, items = 0;
            bool ok = true;
            for (Items<SPLIT, C::TILES> it(a); ok && it.take(a, lens);) {
                if (C::O_OVER_Q && items++ > 0) ok = mbar_wait(smem_u32(&bars->o_left), items & 1, abort_flag);
                if (!ok) break;
                if (!it.n) continue;
                const int buf = q_issued % C::Q_BUFS;
                ok = mbar_wait(smem_u32(&bars->q_empty[buf]), ((q_issued / C::Q_BUFS) & 1) ^ 1, abort_flag, limit<SPLIT>(a));
                if (!ok) break;
                const uint32_t qf = smem_u32(&bars->q_full[buf]);
                mbar_arrive_expect_tx(qf, (uint32_t)(it.streams * C::CHUNKS * a.g * a.nt * 128));
                for (int s = 0; s < it.streams; ++s)
                    for (int c = 0; c < C::CHUNKS; ++c)
                        tma_load_5d(smem_u32(smem_q + (buf * 2 + s) * C::TILE_BYTES + c * (ROWS * 128)), &tm_q, c * CHUNK, 0, it.t0 + s * a.nt, it.kvh, it.b, qf);
                ++q_issued;
                for (int j = 0; j < 2 * it.n && ok; ++j) {
                    ok = mbar_wait(smem_u32(&bars->empty[st]), ph ^ 1, abort_flag, limit<SPLIT>(a));
                    if (!ok) break;
                    const uint32_t full = smem_u32(&bars->full[st]);
                    mbar_arrive_expect_tx(full, C::TILE_BYTES);
                    // K0, V0, K1, V1, ...; APART: K0, K1, V0, K2, V1, ...
                    const bool is_v = C::APART ? j > 0 && ((j & 1) == 0 || (j + 1) / 2 == it.n) : (j & 1) != 0;
                    const int tile = it.j0 + (!C::APART ? j >> 1 : (j & 1) == 0 ? max(j / 2 - 1, 0) : is_v ? it.n - 1 : (j + 1) / 2);
                    for (int c = 0; c < C::CHUNKS; ++c) {
                        const uint32_t dst = smem_u32(smem_st + st * C::TILE_BYTES + c * (KEYS * 128));
                        if (is_v) tma_load_4d(dst, &tm_v, c * CHUNK, tile * KEYS, it.kvh * a.vh, it.b * a.vb, full);
                        else tma_load_4d(dst, &tm_k, c * CHUNK, tile * KEYS, it.kvh * a.kh, it.b * a.kb, full);
                    }
                    ++issued;
                    if (++st == C::STAGES) { st = 0; ph ^= 1; }
                }
            }
            // Everything has landed once it has been multiplied; if a wait gave up anywhere, before the CTA's memory goes.
            for (int k = 0; k < C::STAGES && ok; ++k) {
                ok = mbar_wait(smem_u32(&bars->empty[st]), ph ^ 1, abort_flag, limit<SPLIT>(a));
                if (ok && ++st == C::STAGES) { st = 0; ph ^= 1; }
            }
            if (!ok) {
                cc::land_loads(bars->q_full, C::Q_BUFS, q_issued);
                cc::land_loads(bars->full, C::STAGES, issued);
            }
        }
    } else if (warp < MMA_WARP + C::MMA_WARPS) {
        // ------------------------------------------------------------ MMA issue: the whole warp, instructions predicated on one lane.  Where P lies
        // over the scores one warp issues for both tiles, in turn: each tile's products come between the other's, which keeps the tiles half a
        // period apart (with a warp each they fall into step and wait for the same things: 9472 x 8192 of 128 477 -> 595 us).  Where P is apart a
        // warp each (64: 465 -> 410).
        const uint32_t on = elect_one();
        const uint32_t n_pv = (uint32_t)((a.D + 15) & ~15);
        const uint32_t idesc_qk = make_idesc_bf16(128, KEYS), idesc_pv = make_idesc_bf16(128, n_pv) | (1u << 16);      // (bit 16: B is MN-major)
        const uint32_t hi = desc_hi(1024, 2);
        const int ksteps = (int)(n_pv >> 4);                 // of Q K^T
        uint32_t st = 0, ph = 0, n_q = 0;
        auto wait_on = [&](uint64_t* bar, uint32_t parity) {
            const uint32_t p = smem_u32(bar);
            if (!mbar_try_wait(p, parity)) (void)mbar_wait(p, parity, abort_flag, limit<SPLIT>(a));
            tc_fence_after();
        };
        auto commit = [&](uint64_t* bar) { umma_commit_on(smem_u32(bar), on); };
        auto step = [&]() { if (++st == C::STAGES) { st = 0; ph ^= 1; } };
        auto issue_qk = [&](int s, uint32_t stage, uint32_t idesc_qk) {
            const uint32_t q_lo = desc_lo(smem_u32(smem_q + ((n_q % C::Q_BUFS) * 2 + s) * C::TILE_BYTES)), k_lo = desc_lo(smem_u32(smem_st + stage * C::TILE_BYTES));
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
                if (k >= ksteps) break;
                const uint32_t at = (uint32_t)((k >> 2) * (ROWS * 128 >> 4) + (k & 3) * 2);
                umma_bf16_split_on(tmem + (uint32_t)s * 128u, q_lo + at, hi, k_lo + at, hi, idesc_qk, k ? 1u : 0u, on);
            }
            commit(&bars->s_full[s]);
            __syncwarp();
        };
        auto issue_pv = [&](int s, uint32_t stage, int from, int steps, bool first) {
            const uint32_t v_lo = desc_lo(smem_u32(smem_st + stage * C::TILE_BYTES)) | (((KEYS * 128u) >> 4) << 16);
            const uint32_t d = tmem + C::O_COL + (uint32_t)s * C::O_STEP, p = tmem + C::P_COL + (uint32_t)s * C::P_STEP;
#pragma unroll
            for (int i = 0; i < HALF / 16; ++i) {
                const int k = from + i;
                if (k >= steps) break;
                umma_bf16_ts_on(d, p + (uint32_t)k * 8u, v_lo + (uint32_t)k * (2048u >> 4), hi, idesc_pv, first && k == 0 ? 0u : 1u, on);
            }
            __syncwarp();
        };
        // rows of V that count for nothing but are read by the last product
        auto clear_rows = [&](uint32_t stage, int valid, int steps) {
            if ((valid & 15) == 0) return;
            for (int c = lane; c < (steps * 16 - valid) * 8; c += 32)
#pragma unroll
                for (int x = 0; x < C::CHUNKS; ++x)
                    *(uint4*)(smem_st + stage * C::TILE_BYTES + x * (KEYS * 128) + valid * 128 + c * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
        };
        if constexpr (C::APART) {
            const int s = warp - MMA_WARP;
            uint32_t n_p = 0, n_f = 0;
            for (Items<SPLIT, C::TILES> it(a); it.take(a, lens);) {
                if (!it.n) continue;
                if (*abort_flag) break;
                wait_on(&bars->q_full[n_q % C::Q_BUFS], (n_q / C::Q_BUFS) & 1);
                if (s >= it.streams) {                       // nothing to do but to hand the stages back
                    for (int j = 0; j < 2 * it.n; ++j) {
                        wait_on(&bars->full[st], ph);
                        if (lane == 0) mbar_arrive(smem_u32(&bars->empty[st]));
                        step();
                    }
                    if (lane == 0) mbar_arrive(smem_u32(&bars->q_empty[n_q % C::Q_BUFS]));
                    __syncwarp();
                    ++n_q;
                    continue;
                }
                auto scores = [&](bool last) {               // of the next K stage
                    wait_on(&bars->full[st], ph);
                    issue_qk(s, st, ONE_TILE ? make_idesc_bf16(128, (uint32_t)((it.len + 15) & ~15)) : idesc_qk);
                    commit(&bars->empty[st]);
                    if (last) commit(&bars->q_empty[n_q % C::Q_BUFS]);
                    step();
                };
                if (ONE_TILE && n_p > 0) wait_on(&bars->s_free[s], (n_p - 1) & 1);
                scores(it.n == 1);
                for (int j = 0; j < it.n; ++j) {
                    const int valid = min(KEYS, it.len - (it.j0 + j) * KEYS), steps = (valid + 15) >> 4;
                    const bool last = j + 1 == it.n;
                    if (!last) {
                        wait_on(&bars->s_free[s], n_f & 1);
                        ++n_f;
                        scores(j + 2 == it.n);
                    }
                    wait_on(&bars->full[st], ph);
                    clear_rows(st, valid, steps);            // (both warps write the same zeros)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (!ONE_TILE || h == 1) wait_on(&bars->p_part[s][h], n_p & 1);
                        if (ONE_TILE && h == 1) issue_pv(s, st, 0, steps, j == 0);
                        if (!ONE_TILE || h == 1) issue_pv(s, st, h * (HALF / 16), steps, j == 0);
                    }
                    ++n_p;
                    commit(&bars->empty[st]);
                    commit(last ? &bars->o_full[s] : &bars->pv_done[s]);
                    step();
                    __syncwarp();
                }
                ++n_q;
            }
        } else {
            uint32_t n_p[2] = {0, 0};
            for (Items<SPLIT, C::TILES> it(a); it.take(a, lens);) {
                if (!it.n) continue;
                if (*abort_flag) break;
                wait_on(&bars->q_full[n_q % C::Q_BUFS], (n_q / C::Q_BUFS) & 1);
                wait_on(&bars->full[st], ph);
                for (int s = 0; s < it.streams; ++s) issue_qk(s, st, idesc_qk);
                commit(&bars->empty[st]);
                if (it.n == 1) commit(&bars->q_empty[n_q % C::Q_BUFS]);
                step();
                for (int j = 0; j < it.n; ++j) {
                    const uint32_t v_st = st;
                    const int valid = min(KEYS, it.len - (it.j0 + j) * KEYS), steps = (valid + 15) >> 4;
                    const bool last = j + 1 == it.n;
                    wait_on(&bars->full[st], ph);
                    step();
                    clear_rows(v_st, valid, steps);
                    for (int s = 0; s < it.streams; ++s) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            wait_on(&bars->p_part[s][h], n_p[s] & 1);
                            issue_pv(s, v_st, h * (HALF / 16), steps, j == 0);
                        }
                        ++n_p[s];
                        if (s + 1 == it.streams) commit(&bars->empty[v_st]);
                        if (last) {
                            commit(&bars->o_full[s]);
                        } else {
                            if (s == 0) wait_on(&bars->full[st], ph);
                            issue_qk(s, st, idesc_qk);
                            if (s + 1 == it.streams) {
                                commit(&bars->empty[st]);
                                if (j + 2 == it.n) commit(&bars->q_empty[n_q % C::Q_BUFS]);
                            }
                        }
                        __syncwarp();
                    }
                    if (!last) step();
                }
                ++n_q;
            }
        }
        if (*abort_flag) {                                   // nobody else waits for the products under way
            commit(&bars->drained[warp - MMA_WARP]);
            __syncwarp();
            (void)cc::wait_cluster(smem_u32(&bars->drained[warp - MMA_WARP]), 0, abort_flag);
            __syncwarp();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (SPLIT) cluster_sync_all();                    // nobody leaves while others read its memory
    if (warp == MMA_WARP) {
        tc_fence_after();
        tmem_dealloc(tmem, C::TMEM);
    }
}

// q or o as [D, heads of a key head, tokens, key heads, batch], in boxes of nt tokens
bool encode_rows(CUtensorMap* tm, const XAttnArgs& a, const void* p, const Strides& s, int nt) {
    const int g = a.H / a.Hkv;
    const uint64_t dims[5] = {(uint64_t)a.D, (uint64_t)g, (uint64_t)a.Tq, (uint64_t)a.Hkv, (uint64_t)a.B};
    uint64_t st[4];
    const uint32_t box[5] = {CHUNK, (uint32_t)g, (uint32_t)nt, 1, 1};
    return stride_ok(s.head, g, &st[0]) && stride_ok(s.token, a.Tq, &st[1]) && stride_ok(s.head * g, a.Hkv, &st[2]) && stride_ok(s.batch, a.B, &st[3]) &&
           encode_map(tm, p, 5, dims, st, box);
}

// How the items are shared out: as many rounds of whole ones as fill every CTA, and the rest (all, where there are few) divided by keys within
// clusters.  The fewest tiles in a row, counting what an item (a meeting) costs besides its tiles.
template <int DP> XAttnDivision divide(uint32_t items, int Tk, int sms) {
    const int64_t tiles = (Tk + KEYS - 1) / KEYS;
    XAttnDivision best{1, items, items, std::min(items, (uint32_t)sms)};
    if (DP == 64 && Tk <= KEYS) {
        best.grid = std::min(items, 2u * (uint32_t)sms);
        return best;
    }
    if constexpr (DP < 256) {                                // (wider heads: not divided)
        double cost = (double)((items + best.grid - 1) / best.grid) * (double)(tiles + 1);
        for (int n = 2; n <= MAX_SPLITS && n <= tiles; ++n) {
            const int held = xa::clusters_held<xattn_tc_kernel<DP, ALL>>(NUM_THREADS, Cfg<DP>::SMEM, n);      // (REST has the same shape)
            if (held < 1) continue;
            const uint32_t ctas = (uint32_t)(held * n), whole = items / ctas * ctas, left = items - whole;
            if (left == 0) continue;
            const double c = (double)(whole / ctas) * (double)(tiles + 1) +
                             (double)((left + held - 1) / held) * ((double)((tiles + n - 1) / n) + (whole ? MEET_REST : MEET_ALL));
            if (c < cost) { cost = c; best = {n, items, whole, whole ? ctas : std::min(left, (uint32_t)held) * (uint32_t)n}; }
        }
    }
    return best;
}

template <int DP, int DIVIDED> cudaError_t launch_as(const XAttnDivision& d, const Params& p, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& to, cudaStream_t s) {
    constexpr int smem = Cfg<DP, DIVIDED == SHORT>::SMEM;
    return cc::launch_clusters<xattn_tc_kernel<DP, DIVIDED>>({d.grid, NUM_THREADS, smem, smem, d.splits}, s, p, tq, tk, tv, to);
}
template <int DP> cudaError_t launch(const XAttnDivision& d, const Params& p, const CUtensorMap& tq, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& to, cudaStream_t s) {
    if constexpr (DP < 256) {
        if (d.splits > 1) return d.whole ? launch_as<DP, REST>(d, p, tq, tk, tv, to, s) : launch_as<DP, ALL>(d, p, tq, tk, tv, to, s);
    }
    if constexpr (DP == 64) {
        if (p.Tk <= KEYS) return launch_as<DP, SHORT>(d, p, tq, tk, tv, to, s);
    }
    return launch_as<DP, NONE>(d, p, tq, tk, tv, to, s);
}

std::atomic<long long> meeting_limit{0};                      // a test's; 0: by the call

int items_of_head(const XAttnArgs& a) {                      // tiles of nt tokens, two to an item (one beyond 128 channels)
    const int tokens = (a.D > 128 ? 1 : 2) * (ROWS / (a.H / a.Hkv));
    return (a.Tq + tokens - 1) / tokens;
}

}  // namespace

bool xattn_tc_supported(const XAttnArgs& a) {
    const int g = a.H / a.Hkv;
    uint64_t unused;
    const auto rows_ok = [&](const void* p, const Strides& s) {
        return ((uintptr_t)p & 15) == 0 && stride_ok(s.head, a.H, &unused) && stride_ok(s.token, a.Tq, &unused) && stride_ok(s.batch, a.B, &unused) &&
               s.head < (1ll << 38) / std::max(g, 1);
    };
    return kv_maps_supported(a, 256) && g <= ROWS && rows_ok(a.q, a.sq) && rows_ok(a.o, a.so);
}

void xattn_tc_meeting_limit(long long cycles) { meeting_limit.store(cycles, std::memory_order_relaxed); }

cudaError_t xattn_tc_division(const XAttnArgs& a, XAttnDivision* d) {
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const uint32_t items = (uint32_t)((int64_t)items_of_head(a) * a.Hkv * a.B);      // (rows are at most 2^30)
    *d = a.D <= 64 ? divide<64>(items, a.Tk, sms) : a.D <= 128 ? divide<128>(items, a.Tk, sms) : divide<256>(items, a.Tk, sms);
    return cudaSuccess;
}

cudaError_t launch_xattn_tc(const XAttnArgs& a, cudaStream_t s) {
    CUtensorMap tq, tk, tv, to;
    Params p;
    p.o = (__nv_bfloat16*)a.o; p.o_batch = a.so.batch; p.o_token = a.so.token; p.o_head = a.so.head;
    p.lens = a.kv_lens;
    p.Tq = a.Tq; p.Tk = a.Tk; p.B = a.B; p.Hkv = a.Hkv; p.g = a.H / a.Hkv; p.D = a.D; p.nt = ROWS / p.g;
    p.q_items = items_of_head(a);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    int exponent;
    p.scale_far = frexpf(p.scale_log2, &exponent) == 0.5f ? p.scale_log2 : ldexpf(1.f, exponent);
    if (!encode_rows(&tq, a, a.q, a.sq, p.nt) || !encode_rows(&to, a, a.o, a.so, p.nt) || !encode_kv(&tk, a, a.k, a.sk, KEYS, &p.kh, &p.kb) ||
        !encode_kv(&tv, a, a.v, a.sv, KEYS, &p.vh, &p.vb))
        return cudaErrorInvalidValue;
    XAttnDivision d;
    const cudaError_t e = xattn_tc_division(a, &d);
    if (e != cudaSuccess) return e;
    p.items = d.items;
    p.whole = d.whole;
    p.splits = d.splits;
    // A CTA may come to its first meeting behind all its whole items while another of its cluster had none with keys, and its other roles wait meanwhile:
    // the limit grows by what as many tiles may take, at 16384 cycles each (2000 to 3000 as measured).
    const int64_t rounds = d.splits > 1 ? d.whole / d.grid + 1 : 0, tiles = (a.Tk + KEYS - 1) / KEYS;
    p.wait_limit = tc::WAIT_LIMIT_CYCLES + rounds * tiles * 16384;
    const long long asked = meeting_limit.load(std::memory_order_relaxed);
    p.meeting_limit = asked ? asked : p.wait_limit;
    const uint32_t heads = d.grid / (uint32_t)p.q_items;
    p.dq = (int)(d.grid % (uint32_t)p.q_items);
    p.dh = (int)(heads % (uint32_t)p.Hkv);
    p.db = (int)(heads / (uint32_t)p.Hkv);
    if (a.D <= 64) return launch<64>(d, p, tq, tk, tv, to, s);
    return a.D <= 128 ? launch<128>(d, p, tq, tk, tv, to, s) : launch<256>(d, p, tq, tk, tv, to, s);
}

}  // namespace vd
