// cache_attend_rows.cu -- attention over the paged 8-bit cache for many rows that share a K/V head's tokens (chunks
// of prompts, drafts of several tokens): bound by the tensor cores and the exp2s, not by HBM.
//
// An item is up to 256 rows (tokens times the group's heads) of one sequence and K/V head, in two tiles of 128
// rows; it visits its sequence's tiles of 128 tokens (two pages):
//   S_u = Q_u K^T   tcgen05.mma kind::f8f6f4, M = 128, N = 128, K = D, twice (K's bytes as they are)
//   O_u += P_u V    tcgen05.mma kind::f16, M = 128, N = D, K = 128 (fp16, P from tensor memory, V MN-major)
// Q is the sum of two 8-bit numbers, whose products go into one sum: a row is brought below 448 by a power of two, and
// x = hi + lo with hi = e4m3(x), lo = e5m2(x - hi). Of a bf16 value's 8 bits hi takes four, and what it leaves is at most 8
// steps of the value's last bit, a number of three bits: exact from 2^-6 on, where hi is normal. Below, lo's steps end at
// 2^-16 and half of one of 2^-13 is the most that is lost: 2^-14, the row's largest being above 224. So a value is exact
// down to 2^-13 of that and within 2^-21 of it below, as with few rows. (A lo in e4m3, whose steps end at 2^-9, costs
// the same and loses up to 2^-10, 3 % of a value of 2^-5; fp16 needs K converted too, 92 us against 89 in the last case below.)
// An e4m3 value is an fp16 value, so V is converted without rounding, once for both row tiles, and the
// pages' scales stay out of the products: K's multiplies the scores, V's is added to their exponent,
//   P = 2^(s + log2 v_scale - m),   l = sum P / v_scale,   O = sum P (bytes of V) / l,
// v_scale relative to the sequence's first page (within 2^+-100 of it). P is rounded to fp16's
// 11 bits; m begins 8 below the largest exponent, so P's smallest step is 2^-32 of the largest weight.
//
// One CTA an SM, 16 warps: a producer (TMA of the pages' bytes), an issuer, four converters (half a page of V each: bytes to
// fp16 in the swizzled layout of the products), one that walks the items for the softmax, one that counts off a part
// while the next items run, and a softmax warpgroup for each row tile (a thread is a row). An item of up to 128
// rows has one row tile: both pipelines take its rows, and its tiles in turn.
// P overwrites the lower half of its S, so of one row tile PV_g comes before QK_{g + 1}; while one row tile
// is with the tensor cores the other is with its softmax. A tile's maximum is taken first, but the row's reference is
// raised (and O rescaled in tensor memory) only where P would pass 2^14. The softmax's code is loops over 32 scores: it
// has to stay in the SM's instruction cache beside the other roles' (unrolled, a tile takes 2.5 us instead of 2.2).
//
// Work is shared out and joined as in cache_attend_tc.cu, but a part is 130 KB: CTA c ends with the item that CTA c + 1
// began with, finds that one's part there and keeps its own in shared memory. (4 sequences of 4000 tokens, 1000 rows in
// all, 8 K/V heads of 128: 81 us; 90 with every part written, 110 with parts laid out by row, whose 16 bytes a thread
// fill half a sector.) Results are written 32 bytes a thread for that reason too: 82 us against 85.
// What bounds it, at that size: a tile of 256 rows takes 2.2 us, a chain of QK, softmax (1.2 us a row tile, one warp a
// scheduler, so latencies show) and PV in two pipelines; the four products alone would take 1.1 at the full rate. Two S of
// 64 tokens a pipeline, so that softmax never waits, were slower (89 us): products of 64 columns read Q twice as often.
// PV of a tile's first half while the second is in the softmax changed nothing (84). Some 24 tiles a CTA are 52 us; 10 us
// pass before the first S (dependent loads of table, scales and Q, cold instructions), 7 in the join, the rest in
// changes of items (2.7 us each) and shares of unequal cost. 64 rows of 16 sequences of up to 8000 tokens, one row tile
// each: 74 us (92 with K converted to fp16 as V is, 89 with unrolled products in the issuer, 85 where lanes and warps without
// a row were masked like rows that see nothing).
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstddef>
#include <cstring>

#include "cache_items.cuh"

namespace ssba {
namespace cache {
namespace {

constexpr int kThreads = 512;
constexpr int kRowTile = 128;
constexpr int kItemRows = 2 * kRowTile;
constexpr int kK = 3, kCv = 2, kRaw = 2, kMetas = 8;  // tiles of K; of V, converted and as bytes
constexpr float kTop = 8.f;         // log2 of the largest P against a new reference
constexpr float kMost = 14.f;       // log2 of the largest P that is let stand (fp16 ends at 65504)
constexpr int kConverters = 4;
constexpr float kSpan = 100.f;      // log2 of V scales, relative to the first page's
// The same for a page whose V is all zero. Its P meet zeros, so they count in the sum of weights alone: low enough not to raise the
// row's reference above what the other pages' values need (with 0, V scales of 2^-30 behind a first page of zeros left P
// two bits), and not so low that 2^(s + it - m) vanishes where the weight counts: for other pages from 2^-60 to 2^30, weights down
// to 2^-36 of the largest.
constexpr float kNoV = -60.f;
enum Role { kLoad = 0, kIssue = 1, kConvert = 2, kItems = 6, kSoftmax = 8 };
constexpr uint32_t kTmemCols = 512;

constexpr uint32_t idesc_f16_f32(int M, int N, bool b_mn_major) { return idesc_e4m3_f32(M, N, false, b_mn_major); }  // formats 0: fp16

constexpr uint32_t kAE5m2 = 1u << 7;  // of an instruction descriptor of kind::f8f6f4: A is e5m2 (B's type is its own)

constexpr int kItemRing = 4;

// An item's share as the softmax warps get it, which have no registers for the walk.
struct Item {
    Rows rows;
    Seq s;
    int tb, te, tiles, two;
    long long start;
};

struct Meta {
    float ks, lv, inv;  // K scale; log2 of the V scale (relative); 2^-lv
    int pos;            // token position of the page
};

template <int D>
struct __align__(1024) Smem {
    uint8_t q[2][2][kRowTile][D];          // a row tile's high (e4m3) and low (e5m2) parts, swizzled as K is
    uint8_t cv[kCv][D / 64][kTile][128];   // fp16 V, 64 channels a 128-byte row, 128-byte swizzle
    uint8_t kraw[kK][kTile * D];           // K's bytes (rows of 128 or 64 bytes, that swizzle)
    uint8_t raw[kRaw][kTile * D];          // V's bytes
    // by item parity and converter: first token whose V is NaN, of those that not every row sees
    int nan_at[2][kConverters][D];
    int nan_any[2][kConverters];
    float qf[2][kRowTile];  // scale of a row's scores
    float2 ml[kRowTile];    // (tiles in turn) reference and sum of the second pipeline's rows
    float first_lv[2];      // by item parity: log2 of the V scale that the item's are relative to
    Meta meta[kMetas][2];
    uint64_t k_full[kK], k_empty[kK], raw_full[kRaw], raw_empty[kRaw], cv_full[kCv], cv_empty[kCv], m_full[kMetas];
    uint64_t q_full[2], s_full[2], p_full[2], o_full[2], n_full[2], n_empty[2], x_full, x_empty, drain;
    long long w0, w1, total;
    int first_b, ctas;
    Seq first_s;
    long long first_at;
    uint32_t tmem_base;
    Item item[kItemRing];  // te = 0: no more
    uint64_t i_full[kItemRing], i_empty[kItemRing];
    // of the items that are shared with other CTAs: one that began before the share, one that goes on behind it
    Rows rows[2];
    float base[2];
    long long start[2];
    int tiles[2];
    int abort_flag, last[2], last_c0[2];
    uint64_t t_full, d_full;  // the first item's part is written; the last item's products are done and `direct` is set
    int direct;               // the last item's other parts were there already: the CTA's own stays in shared memory
};

__device__ __forceinline__ bool soft_any(bool x)  // over the softmax warps
{
    uint32_t r;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.u32 p, %1, 0;\n"
        "bar.red.or.pred q, 1, 256, p;\n"
        "selp.u32 %0, 1, 0, q;\n"
        "}\n"
        : "=r"(r)
        : "r"(x ? 1u : 0u)
        : "memory");
    return r != 0;
}

__device__ __forceinline__ uint32_t half2_of(uint32_t e4m3x2)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(e4m3x2)));
    return h;
}

// Two floats to two e5m2 bytes, as to_e4m3x2.
__device__ __forceinline__ uint32_t to_e5m2x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ uint32_t pack_half(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
}

__device__ __forceinline__ void store32(void* to, const uint32_t (&y)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]),
                 "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7])
                 : "memory");
}

// A part of a shared item: O as [D / 4][256 rows] of four channels, so that a warp, whose threads are rows, writes and reads
// 512 bytes in a row; behind it the rows' references and sums.
template <int D>
struct Part {
    float4 o[D / 4][kItemRows];
    float2 ml[kItemRows];
};

// Joins the np parts of an item that begins in CTA c0, in order, and writes its rows: a warp takes 32 rows and 4 kC
// channels at a time, kP parts in flight. The first part may be the CTA's own, in shared memory.
template <int D, int kC, int kP>
__device__ __noinline__ void join(const Params& p, const Rows rows, float base, int c0, int np, const Part<D>* own)
{
    constexpr int kChunks = D / 4 / kC;
    const int lane = threadIdx.x & 31, tasks = (rows.n * p.gc + 31) / 32 * kChunks, first = own ? 1 : 0;
    // part 0 is slot 1 of CTA c0, part k slot 0 of CTA c0 + k
    auto part = [&](int k) { return reinterpret_cast<const Part<D>*>(p.parts) + (size_t)(c0 + k) * 2 + (k == 0); };
#pragma unroll 1
    for (int task = threadIdx.x >> 5; task < tasks; task += kThreads / 32) {
        const int r = task / kChunks * 32 + lane, c = task % kChunks * kC;
        int head;
        const int row = rows.of(p, r, head);
        const float2 mine = own ? own->ml[r] : make_float2(-INFINITY, 0.f);
        float m = mine.x, l = mine.y;
#pragma unroll 1
        for (int k0 = first; k0 < np; k0 += kP) {
            float2 ml[kP];
#pragma unroll
            for (int k = 0; k < kP; ++k) ml[k] = k0 + k < np ? __ldcg(&part(k0 + k)->ml[r]) : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int k = 0; k < kP; ++k) {
                const float top = fmaxf(m, ml[k].x), at0 = top == -INFINITY ? 0.f : top;
                l = fmaf(ml[k].y, fast_exp2(ml[k].x - at0), l * fast_exp2(m - at0));
                m = top;
            }
        }
        const float at0 = m == -INFINITY ? 0.f : m, inv = l != 0.f ? exp2f(base) / l : 0.f, f_own = fast_exp2(mine.x - at0);
        const size_t at = (size_t)max(row, 0) * p.pl.heads + head;
        float4 o[kC];
#pragma unroll
        for (int i = 0; i < kC; ++i) {
            o[i] = own ? own->o[c + i][r] : make_float4(0.f, 0.f, 0.f, 0.f);
            o[i] = make_float4(fmaf(o[i].x, f_own, 0.f), fmaf(o[i].y, f_own, 0.f), fmaf(o[i].z, f_own, 0.f), fmaf(o[i].w, f_own, 0.f));
        }
#pragma unroll 1
        for (int k0 = first; k0 < np; k0 += kP) {
            float4 v[kP][kC];
            float f[kP];
#pragma unroll
            for (int k = 0; k < kP; ++k) {
                const bool real = k0 + k < np;
#pragma unroll
                for (int i = 0; i < kC; ++i) v[k][i] = real ? __ldcg(&part(k0 + k)->o[c + i][r]) : make_float4(0.f, 0.f, 0.f, 0.f);
                f[k] = real ? fast_exp2(__ldcg(&part(k0 + k)->ml[r]).x - at0) : 0.f;
            }
#pragma unroll
            for (int k = 0; k < kP; ++k)
#pragma unroll
                for (int i = 0; i < kC; ++i) {
                    o[i].x = fmaf(v[k][i].x, f[k], o[i].x);
                    o[i].y = fmaf(v[k][i].y, f[k], o[i].y);
                    o[i].z = fmaf(v[k][i].z, f[k], o[i].z);
                    o[i].w = fmaf(v[k][i].w, f[k], o[i].w);
                }
        }
        if (row < 0) continue;
#pragma unroll
        for (int i = 0; i < kC; i += 4) {
            uint32_t y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[2 * e] = pack_bf16(o[i + e].x * inv, o[i + e].y * inv);
                y[2 * e + 1] = pack_bf16(o[i + e].z * inv, o[i + e].w * inv);
            }
            store32(p.O + at * D + (c + i) * 4, y);
        }
        if (c == 0) p.lse[at] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
    }
}

// Many rows of two or three parts, or few rows of many parts: the way that takes fewer round trips to L2.
template <int D>
__device__ __forceinline__ void join(const Params& p, const Rows& rows, float base, int c0, int np, const Part<D>* own)
{
    const int blocks = (rows.n * p.gc + 31) / 32, others = np - (own ? 1 : 0);
    const int wide = (blocks * (D / 32) + 15) / 16 * others, deep = (blocks * (D / 16) + 15) / 16 * ((others + 3) / 4);
    if (wide <= deep) join<D, 8, 1>(p, rows, base, c0, np, own);
    else join<D, 4, 4>(p, rows, base, c0, np, own);
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) ssba_cache_attend_rows_kernel(const __grid_constant__ Maps maps,
                                                                             const __grid_constant__ Params p)
{
    extern __shared__ uint8_t smem_raw[];
    Smem<D>& sm = *reinterpret_cast<Smem<D>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        sm.abort_flag = sm.direct = sm.last[0] = sm.last[1] = sm.tiles[0] = sm.tiles[1] = 0;
        for (int i = 0; i < kItemRing; ++i) {
            mbar_init(smem_u32(&sm.i_full[i]), 1);
            mbar_init(smem_u32(&sm.i_empty[i]), 8);
        }
        for (int i = 0; i < kK; ++i) {
            mbar_init(smem_u32(&sm.k_full[i]), 1);
            mbar_init(smem_u32(&sm.k_empty[i]), 1);
        }
        for (int i = 0; i < kRaw; ++i) {
            mbar_init(smem_u32(&sm.raw_full[i]), 1);
            mbar_init(smem_u32(&sm.raw_empty[i]), kConverters);
        }
        for (int i = 0; i < kCv; ++i) {
            mbar_init(smem_u32(&sm.cv_full[i]), kConverters);
            mbar_init(smem_u32(&sm.cv_empty[i]), 1);
        }
        for (int i = 0; i < kMetas; ++i) mbar_init(smem_u32(&sm.m_full[i]), 2);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sm.q_full[i]), 4);
            mbar_init(smem_u32(&sm.s_full[i]), 1);
            mbar_init(smem_u32(&sm.p_full[i]), 4);
            mbar_init(smem_u32(&sm.o_full[i]), 1);
            mbar_init(smem_u32(&sm.n_full[i]), kConverters);
            mbar_init(smem_u32(&sm.n_empty[i]), 8);
        }
        mbar_init(smem_u32(&sm.x_full), 4);
        mbar_init(smem_u32(&sm.x_empty), 4);
        mbar_init(smem_u32(&sm.drain), 1);
        mbar_init(smem_u32(&sm.t_full), 8);
        mbar_init(smem_u32(&sm.d_full), 8);
        fence_mbar_init();
    }
    if (warp == kIssue) {
        tmem_alloc(smem_u32(&sm.tmem_base), kTmemCols);
        tmem_relinquish();
    }
    if (warp == kLoad && lane == 0) {
        tma_prefetch_desc(&maps.k);
        tma_prefetch_desc(&maps.v);
    }
    tc_fence_before();
    // everything above reads no input (programmatic dependent launch: it may run beside the last grid's end)
    grid_dep_wait();
    if (warp == kIssue) grid_dep_launch();  // by the warp that has taken tensor memory: the next grid's CTAs may then take theirs
    make_share<false, kThreads>(p, sm);  // ends in a barrier
    tc_fence_after();
    const uint32_t tbase = sm.tmem_base;
    volatile int* abortf = &sm.abort_flag;
    const uint32_t abort_at = smem_u32(&sm.abort_flag);
    const uint32_t rfull0 = smem_u32(&sm.raw_full[0]), rempty0 = smem_u32(&sm.raw_empty[0]);
    const uint32_t cfull0 = smem_u32(&sm.cv_full[0]), cempty0 = smem_u32(&sm.cv_empty[0]);
    bool dead = false;
    const uint32_t kfull0 = smem_u32(&sm.k_full[0]), kempty0 = smem_u32(&sm.k_empty[0]);
    constexpr uint32_t kSwizzle = D == 128 ? 2 : 4;  // of Q's and K's rows (see sdesc)
    uint32_t kloads = 0, vloads = 0;  // of the producer
    // an item of up to 128 rows has no second row tile: both pipelines take its rows, and its tiles in turn
    auto both = [&](const Walk<false>& w) { return w.rows().n * p.gc > kRowTile; };

    if (warp == kLoad) {
        // ------------------------------------------------------------ producer
        Walk<false> it(p, sm);
        auto copy = [&](const CUtensorMap* map, uint32_t empty, uint32_t full, uint32_t to, uint32_t turn, int p0, int p1) {
            if (!mbar_wait(empty, (turn & 1) ^ 1, abortf, p.budget_ns)) {
                dead = true;
                return;
            }
            mbar_arrive_expect_tx(full, ((p0 >= 0) + (p1 >= 0)) * (uint32_t)(kPage * D));
            if (p.withhold && blockIdx.x == 0) {
                dead = true;
                return;
            }
            if (p0 >= 0) tma_load_3d(to, map, full, 0, 0, p0);
            if (p1 >= 0) tma_load_3d(to + kPage * D, map, full, 0, 0, p1);
        };
        auto copy_k = [&](int p0, int p1) {
            const uint32_t x = kloads % kK;
            copy(&maps.k, kempty0 + 8 * x, kfull0 + 8 * x, smem_u32(&sm.kraw[x][0]), kloads / kK, p0, p1);
            if (!dead) ++kloads;
        };
        auto copy_v = [&](int p0, int p1) {
            const uint32_t x = vloads % kRaw;
            copy(&maps.v, rempty0 + 8 * x, rfull0 + 8 * x, smem_u32(&sm.raw[x][0]), vloads / kRaw, p0, p1);
            if (!dead) ++vloads;
        };
        // K_0, then K_{i + 1} and V_i
        for (; it.more() && !dead; it.next()) {
            const int h = it.hv / p.chunks;
            int v0 = -1, v1 = -1;  // the last tile's pages
            for (int c0 = 2 * it.tb; c0 < 2 * it.te && !dead; c0 += 32) {  // 32 pages at a time
                int j, page = -1;
                if (c0 + lane < 2 * it.te) page = it.page(c0 + lane, j);
                const int unit = page >= 0 ? page * p.pl.kv_heads + h : -1;
                const int n = min(16, it.te - c0 / 2);
                for (int i = 0; i < n && !dead; ++i) {
                    const int p0 = __shfl_sync(0xffffffffu, unit, 2 * i), p1 = __shfl_sync(0xffffffffu, unit, 2 * i + 1);
                    if (lane == 0) {
                        copy_k(p0, p1);
                        if (!dead && c0 / 2 + i > it.tb) copy_v(v0, v1);
                    }
                    v0 = p0;
                    v1 = p1;
                    dead = __shfl_sync(0xffffffffu, (int)dead, 0) != 0;
                }
            }
            if (!dead) {
                if (lane == 0) copy_v(v0, v1);
                dead = __shfl_sync(0xffffffffu, (int)dead, 0) != 0;
            }
        }
        __syncwarp();
    } else if (warp == kIssue) {
        // ------------------------------------------------------------ issuer
        Walk<false> it(p, sm);
        // One loop, one copy of each product's code and no unrolling, so that it stays in the instruction cache beside the other
        // roles' (with a copy for each way through it, a jump back waited 0.5 us for its code).
        uint32_t done0 = 0, done1 = 0, q0 = 0, q1 = 0, base = 0;  // QKs and items of each pipeline; tiles before the item
        for (; it.more(); it.next()) {
            const int n = it.te - it.tb;
            const bool two = both(it);
            wait_phase(smem_u32(&sm.q_full[0]), q0++ & 1, abort_at, p.budget_ns);
            if (two || n > 1) wait_phase(smem_u32(&sm.q_full[1]), q1++ & 1, abort_at, p.budget_ns);
            // A step is PV of a tile and QK of a later one in one pipeline, which take the steps in turn. Two row tiles: PV_{i-1} and
            // QK_i in both; tiles in turn: PV_{i-2} and QK_i.
            const int steps = two ? 2 * (n + 1) : n + 2;
#pragma unroll 1
            for (int s = 0; s < steps; ++s) {
                const int u = s & 1, i = two ? s >> 1 : s, t = two ? i - 1 : i - 2;
                const bool release = !two || u == 1;  // (the last to read the tile)
                if (t >= 0) {
                    const uint32_t tile = base + t, slot = tile % kCv;
                    wait_phase(smem_u32(&sm.p_full[u]), ((u ? done1 : done0) - 1) & 1, abort_at, p.budget_ns);
                    wait_phase(cfull0 + 8 * slot, (tile / kCv) & 1, abort_at, p.budget_ns);
                    tc_fence_after();
                    if (elect_one_sync()) {
                        uint64_t b = sdesc_sw128(smem_u32(&sm.cv[slot][0][0][0]), kTile * 128, 1024);
                        uint32_t more = two ? t > 0 : t > 1;
#pragma unroll 1
                        for (int k = 0; k < kTile / 16; ++k) {
                            mma_ts(tbase + 256 + u * D, tbase + u * 128 + k * 8, b, idesc_f16_f32(128, D, true), more);
                            b += 128;
                            more = 1;
                        }
                        if (t >= (two ? n - 1 : n - 2)) mma_commit(smem_u32(&sm.o_full[u]));
                        if (release) mma_commit(cempty0 + 8 * slot);
                    }
                    __syncwarp();
                }
                if (i < n) {
                    const uint32_t tile = base + i, slot = tile % kK;
                    wait_phase(kfull0 + 8 * slot, (tile / kK) & 1, abort_at, p.budget_ns);
                    tc_fence_after();
                    if (elect_one_sync()) {
                        uint64_t a = sdesc(smem_u32(&sm.q[u][0][0][0]), 16, 8 * D, kSwizzle);
                        const uint64_t b = sdesc(smem_u32(&sm.kraw[slot][0]), 16, 8 * D, kSwizzle);
#pragma unroll 1
                        for (int k = 0; k < 2 * (D / 32); ++k) {  // the high parts, then the low ones
                            mma_f8_ss(tbase + u * 128, a, b + (uint64_t)(2 * (k & (D / 32 - 1))),
                                      idesc_e4m3_f32(128, 128, false, false) | (k < D / 32 ? 0u : kAE5m2), k > 0 ? 1u : 0u);
                            a += k == D / 32 - 1 ? kRowTile * D / 16 - 2 * (D / 32 - 1) : 2;
                        }
                        mma_commit(smem_u32(&sm.s_full[u]));
                        if (release) mma_commit(kempty0 + 8 * slot);
                    }
                    __syncwarp();
                    done0 += u == 0;
                    done1 += u;
                }
            }
            base += n;
        }
        dead = *abortf != 0;
    } else if (warp >= kItems && warp < kSoftmax) {
        // ------------------------------------------------------------ items for the softmax warps
        if (warp == kItems) {
            Walk<false> it(p, sm);
            for (int seg = 0;; ++seg) {
                const int k = seg % kItemRing;
                wait_phase(smem_u32(&sm.i_empty[k]), ((seg / kItemRing) & 1) ^ 1, abort_at, p.budget_ns);
                const bool more = it.more();
                if (lane == 0) {
                    sm.item[k].te = 0;
                    if (more) sm.item[k] = Item{it.rows(), it.s, it.tb, it.te, it.tiles, both(it) ? 1 : 0, it.start};
                    mbar_arrive(smem_u32(&sm.i_full[k]));
                }
                if (!more) break;
                it.next();
            }
        } else {
            // counts the part of an item that began in an earlier CTA as soon as it is written, beside the next items: the fence
            // takes microseconds, and the earlier CTA, which ends with that item, finds the part there and need not write its own
            wait_phase(smem_u32(&sm.t_full), 0, abort_at, p.budget_ns);
            if (lane == 0 && !*abortf && sm.tiles[0] > 0) {
                const int c0 = cta_of(sm.start[0], sm), np = cta_of(sm.start[0] + sm.tiles[0] - 1, sm) - c0 + 1;
                unsigned seen;
                asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(seen) : "l"(p.tickets + c0) : "memory");
                if (seen == (unsigned)(np - 1)) {
                    p.tickets[c0] = 0;
                    sm.last_c0[0] = c0;
                    sm.last[0] = np;
                }
            }
        }
        dead = *abortf != 0;
    } else if (warp < kSoftmax) {
        // ------------------------------------------------------------ converters: half a page of every tile of V
        constexpr int kLanes = D / 16, kRows = 32 / kLanes, kIts = 32 / kRows;  // lanes of a row (16 bytes each), rows at a time
        const int w = warp - kConvert, c = lane % kLanes, row0 = w * 32 + lane / kLanes;
        uint32_t g = 0;  // tiles
        int seg = 0;
        Walk<false> it(p, sm);
        for (; it.more(); it.next(), ++seg) {
            const int h = it.hv / p.chunks;
            const Rows rows = it.rows();
            const int lo_lim = it.limit(rows.row), hi_lim = it.limit(rows.row + max(rows.n, 1) - 1);
            float base = 0.f;
            for (int c0 = it.tb; c0 < it.te; c0 += 32) {  // 32 tiles' pages at a time
                int j, j0, page = -1;
                const int page0 = it.page(0, j0);
                if (c0 + lane < it.te) page = it.page(2 * (c0 + lane) + w / 2, j);
                float my_ks = 0.f, my_lv = 0.f, vs = 0.f;
                const float vs0 = page0 >= 0 ? ld(p.pl.v_scale + (size_t)page0 * p.pl.kv_heads + h) : 0.f;
                if (page >= 0) {
                    const size_t unit = (size_t)page * p.pl.kv_heads + h;
                    my_ks = ld(p.pl.k_scale + unit);
                    vs = ld(p.pl.v_scale + unit);
                }
                if (c0 == it.tb) {
                    // V scales are taken relative to the sequence's first page's
                    base = vs0 > 0.f && vs0 < INFINITY ? log2f(vs0) : 0.f;
                    wait_phase(smem_u32(&sm.n_empty[seg & 1]), ((seg >> 1) & 1) ^ 1, abort_at, p.budget_ns);
                    for (int i = lane; i < D; i += 32) sm.nan_at[seg & 1][w][i] = INT_MAX;
                    if (lane == 0) {
                        sm.nan_any[seg & 1][w] = 0;
                        sm.first_lv[seg & 1] = base;
                    }
                    __syncwarp();
                }
                if (page >= 0) {
                    my_lv = vs > 0.f ? fminf(fmaxf(log2f(vs) - base, -kSpan), kSpan) : isnan(vs) ? vs : kNoV;
                }
                const int my_pos = page >= 0 ? j * kPage : kNowhere;
                const int n = min(32, it.te - c0);
                for (int i = 0; i < n; ++i, ++g) {
                    const int pos = __shfl_sync(0xffffffffu, my_pos, i);
                    const float ks = __shfl_sync(0xffffffffu, my_ks, i), lv = __shfl_sync(0xffffffffu, my_lv, i);
                    if ((w & 1) == 0 && lane == 0) {  // (what the softmax needs to know of the tile)
                        sm.meta[g % kMetas][w / 2] = Meta{ks, lv, exp2f(-lv), pos};
                        mbar_arrive(smem_u32(&sm.m_full[g % kMetas]));
                    }
                    {
                        const uint32_t rs = g % kRaw, cs = g % kCv;
                        wait_phase(rfull0 + 8 * rs, (g / kRaw) & 1, abort_at, p.budget_ns);
                        const int first = pos + (w & 1) * 32;  // token of the first row
                        if (first + 31 >= lo_lim) {
                            // tokens that no row sees: their V is whatever the page holds, and 0 * NaN would reach
                            // every row; tokens that some rows see: a NaN is taken out and kept for those rows
#pragma unroll 1
                            for (int k = 0; k < kIts; ++k) {
                                uint32_t* word = reinterpret_cast<uint32_t*>(&sm.raw[rs][(row0 + k * kRows) * D + c * 16]);
                                const int at = first + lane / kLanes + k * kRows;
#pragma unroll 1
                                for (int m = 0; m < 4 && at >= lo_lim; ++m) {
                                    uint32_t b = at >= hi_lim ? 0u : word[m];
                                    if ((((b & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0) {  // a byte of 0x7f
                                        for (int e = 0; e < 4; ++e)
                                            if (((b >> (8 * e)) & 0x7f) == 0x7f) {
                                                atomicMin(&sm.nan_at[seg & 1][w][c * 16 + m * 4 + e], at);
                                                sm.nan_any[seg & 1][w] = 1;
                                                b &= ~(0xffu << (8 * e));
                                            }
                                    }
                                    word[m] = b;
                                }
                            }
                        }
                        uint4 in[kIts];
#pragma unroll
                        for (int k = 0; k < kIts; ++k)
                            in[k] = *reinterpret_cast<const uint4*>(&sm.raw[rs][(row0 + k * kRows) * D + c * 16]);
                        wait_phase(cempty0 + 8 * cs, ((g / kCv) & 1) ^ 1, abort_at, p.budget_ns);
#pragma unroll
                        for (int k = 0; k < kIts; ++k) {
                            const int row = row0 + k * kRows;
                            const uint32_t x4[4] = {in[k].x, in[k].y, in[k].z, in[k].w};
                            uint32_t y[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] = half2_of(e & 1 ? x4[e / 2] >> 16 : x4[e / 2] & 0xffff);
                            const uint4 a = make_uint4(y[0], y[1], y[2], y[3]), b = make_uint4(y[4], y[5], y[6], y[7]);
                            uint8_t* to = &sm.cv[cs][c / 4][row][0];
                            const int q = (c % 4) * 2;
                            // lanes of the second 64 channels write their second half first: no bank conflicts
                            const bool turn = c / 4;
                            *reinterpret_cast<uint4*>(to + ((q + turn) ^ (row & 7)) * 16) = turn ? b : a;
                            *reinterpret_cast<uint4*>(to + ((q + !turn) ^ (row & 7)) * 16) = turn ? a : b;
                        }
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(rempty0 + 8 * rs);
                            mbar_arrive(cfull0 + 8 * cs);
                        }
                    }
                }
            }
            if (lane == 0) mbar_arrive(smem_u32(&sm.n_full[seg & 1]));
        }
        dead = *abortf != 0;
    } else {
        // ------------------------------------------------------------ softmax and output: a thread is a row
        const int u = (warp - kSoftmax) / 4, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
        const uint32_t scol = tbase + u * 128 + lanes, ocol = tbase + 256 + u * D + lanes;
        uint32_t cnt = 0, g = 0;        // tiles of this pipeline, of the CTA
        uint32_t outs0 = 0, outs1 = 0;  // results of both pipelines so far
        uint32_t handed = 0;            // of them, second ones that went through the first
        int seg = 0;
        int lim = 0;     // tokens that the thread's row sees
        float qf = 0.f;  // scale of its scores
        auto limit = [&](const Item& w, int row) {
            return row >= 0 ? min(max(w.s.len - w.s.n + row - w.s.row + 1, 0), w.s.len) : 0;
        };
        // the warp's 32 rows of Q to shared memory
        auto load_q = [&](const Item& w) {
            constexpr int kLanes = D / 8, kRows = 32 / kLanes;  // lanes of a row (8 values each), rows at a time
            const int c = lane % kLanes, top = w.two ? u * kRowTile : 0;
            const Rows rows = w.rows;
            // where the lane's 16 bytes of a row wait to be split: the row's own two parts
            auto staged = [&](int row) { return &sm.q[u][c / (kLanes / 2)][row][(c % (kLanes / 2) ^ (row & (kLanes / 2 - 1))) * 16]; };
#pragma unroll 2
            for (int k = 0; k < 32 / kRows; ++k) {
                const int at = quad * 32 + k * kRows + lane / kLanes;
                int hd;
                const int rr = rows.of(p, top + at, hd);
                const __nv_bfloat16* src = p.q + ((size_t)max(rr, 0) * p.pl.heads + (rr >= 0 ? hd : 0)) * D + c * 8;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(staged(at))), "l"(src), "r"(rr >= 0 ? 16 : 0)
                             : "memory");
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            // each lane what it has copied itself: 8 values of a row, which is scaled by a power of two and split
            // (four rows at a time, their shuffles side by side)
            constexpr int kB = 4;
#pragma unroll 1
            for (int k0 = 0; k0 < 32 / kRows; k0 += kB) {
                uint4 w[kB];
                uint32_t big[kB];
                auto at = [&](int k) { return quad * 32 + (k0 + k) * kRows + lane / kLanes; };
#pragma unroll
                for (int k = 0; k < kB; ++k) w[k] = *reinterpret_cast<const uint4*>(staged(at(k)));
#pragma unroll
                for (int k = 0; k < kB; ++k) {
                    const uint32_t a = 0x7fff7fffu;
                    big[k] = __vmaxu2(__vmaxu2(w[k].x & a, w[k].y & a), __vmaxu2(w[k].z & a, w[k].w & a));
                    if (__vcmpgeu2(big[k], 0x7f807f80u)) {  // an infinity or NaN: the finite ones' largest
                        const uint32_t v[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
                        big[k] = 0;
#pragma unroll 1
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t b = ((e < 4 ? (e < 2 ? v[0] : v[1]) : (e < 6 ? v[2] : v[3])) >> (16 * (e & 1))) & 0x7fffu;
                            if (b < 0x7f80u) big[k] = max(big[k], b);
                        }
                    }
                    big[k] = max(big[k] & 0xffffu, big[k] >> 16);
                }
#pragma unroll
                for (int o = kLanes / 2; o; o >>= 1) {
#pragma unroll
                    for (int k = 0; k < kB; ++k) big[k] = max(big[k], __shfl_xor_sync(0xffffffffu, big[k], o));
                }
                __syncwarp();  // (a row's parts take the place of its values)
#pragma unroll
                for (int k = 0; k < kB; ++k) {
                    const float scale = scale_for(__uint_as_float(big[k] << 16));
                    // (a power of two from 2^-126 to 2^120: its inverse by its exponent)
                    const float inv = scale > 0.f ? __uint_as_float(0x7f000000u - __float_as_uint(scale)) : 1.f;
                    const uint32_t v[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {  // (an infinity times 0 is NaN: it makes its row's scores NaN, as in any softmax)
                        const float a = __uint_as_float(v[e] << 16), b = __uint_as_float(v[e] & 0xffff0000u);
                        const float x = fmaf(a, 0.f, a * inv), y = fmaf(b, 0.f, b * inv);
                        hi[e] = to_e4m3x2(x, y);
                        const float2 back = from_e4m3x2(hi[e]);
                        lo[e] = to_e5m2x2(x - back.x, y - back.y);
                    }
                    const int row = at(k), chunk = D == 128 ? (c / 2) ^ (row & 7) : (c / 2) ^ ((row >> 1) & 3);
                    *reinterpret_cast<uint2*>(&sm.q[u][0][row][chunk * 16 + (c & 1) * 8]) = make_uint2(hi[0] | (hi[1] << 16), hi[2] | (hi[3] << 16));
                    *reinterpret_cast<uint2*>(&sm.q[u][1][row][chunk * 16 + (c & 1) * 8]) = make_uint2(lo[0] | (lo[1] << 16), lo[2] | (lo[3] << 16));
                    if (c == 0) sm.qf[u][row] = scale * p.scale_log2;
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.q_full[u]));
            int head;
            const int row = rows.of(p, top + r, head);
            lim = limit(w, row);
            // a lane without a row sees what the warp's rows see, so that it makes no tile one to be masked (0.7 us each)
            const int most = __reduce_max_sync(0xffffffffu, lim);
            if (row < 0) lim = most;
            qf = sm.qf[u][r];
            __syncwarp();
        };
        // the next item, its rows of Q under way
        auto begin = [&](int k) -> bool {
            wait_phase(smem_u32(&sm.i_full[k % kItemRing]), (k / kItemRing) & 1, abort_at, p.budget_ns);
            const Item& w = sm.item[k % kItemRing];
            if (w.te == 0) return false;
            if (u == 0 || w.two || w.te - w.tb > 1) load_q(w);  // (the second pipeline has nothing of a single tile)
            return true;
        };
        bool more = begin(0);
        while (more && !*abortf) {
            const Item& it = sm.item[seg % kItemRing];
            const int nt = it.te - it.tb;
            // two row tiles: each pipeline has its rows and every tile; else both have the same rows, and tiles in turn
            const int two = it.two, own = two ? 0 : u, step = two ? 1 : 2;
            float m = -INFINITY, l = 0.f;
            if (u == 1 && handed) {  // (what the first pipeline takes over is this one's O, which the next P replaces)
                wait_phase(smem_u32(&sm.x_empty), (handed - 1) & 1, abort_at, p.budget_ns);
            }
            for (int i = own; i < nt; i += step, ++cnt) {
                const uint32_t gt = g + i;
                wait_phase(smem_u32(&sm.m_full[gt % kMetas]), (gt / kMetas) & 1, abort_at, p.budget_ns);
                const Meta ma = sm.meta[gt % kMetas][0], mb = sm.meta[gt % kMetas][1];
                // (a factor of 0 would make a masked score NaN)
                const float fa = ma.ks * qf, fb = mb.ks * qf, ca = fa == 0.f ? 1e-30f : fa, cb = fb == 0.f ? 1e-30f : fb;
                const int la = min(max(lim - ma.pos, 0), kPage), lb = min(max(lim - mb.pos, 0), kPage);
                const bool cut = __any_sync(0xffffffffu, la < kPage || lb < kPage);
                wait_phase(smem_u32(&sm.s_full[u]), cnt & 1, abort_at, p.budget_ns);
                tc_fence_after();
                if (!__any_sync(0xffffffffu, la + lb > 0)) {
                    // none of the warp's rows sees any of it (in an item of few rows most warps have none): its weights are zero
                    const uint32_t zero[16] = {};
#pragma unroll 1
                    for (int ch = 0; ch < 4; ++ch) tmem_st_32x32b_x16(scol + 16 * ch, zero);
                } else {
                    uint32_t x[32];
                    auto get = [&](int ch) {  // chunk ch of the scores, what the row does not see at -inf
                        tmem_ld_32x32b_x32(scol + 32 * ch, x);
                        tmem_wait_ld();
                        if (cut) {
                            const int left = (ch < 2 ? la : lb) - (ch & 1) * 32;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (e >= left) x[e] = 0xff800000u;
                        }
                    };
                    // the tile's largest exponent: factors of scores are not negative
                    float mx = -INFINITY;
#pragma unroll 1
                    for (int ch = 0; ch < 4; ++ch) {
                        get(ch);
                        float top = __uint_as_float(x[0]);
#pragma unroll
                        for (int e = 1; e < 31; e += 2) top = max3(top, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                        top = fmaxf(top, __uint_as_float(x[31]));
                        mx = fmaxf(mx, fmaf(top, ch < 2 ? ca : cb, ch < 2 ? ma.lv : mb.lv));
                    }
                    const bool up = m == -INFINITY ? mx > -INFINITY : mx > m + kMost;
                    if (__any_sync(0xffffffffu, up)) {
                        const float now = up ? mx - kTop : m, f = up ? fast_exp2(m - now) : 1.f;
                        l *= f;
                        m = now;
                        if (i > own) {  // O holds the tiles so far: QK of this one was issued behind their PV
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tmem_ld_32x32b_x16(ocol + c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st_32x32b_x16(ocol + c, o);
                            }
                        }
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
                    // P of a chunk goes over scores that have been read
#pragma unroll 1
                    for (int ch = 0; ch < 4; ++ch) {
                        get(ch);
                        const float cc = ch < 2 ? ca : cb, off = (ch < 2 ? ma.lv : mb.lv) - ref;
                        const float2 c2 = make_float2(cc, cc), o2 = make_float2(off, off);
                        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float2 y = __ffma2_rn(make_float2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), c2, o2);
                            y = make_float2(fast_exp2(y.x), fast_exp2(y.y));
                            sum[e & 1] = __fadd2_rn(sum[e & 1], y);
                            pk[e] = pack_half(y.x, y.y);
                        }
                        tmem_st_32x32b_x16(scol + 16 * ch, pk);
                        l = fmaf((sum[0].x + sum[1].x) + (sum[0].y + sum[1].y), ch < 2 ? ma.inv : mb.inv, l);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm.p_full[u]));
            }
            g += nt;
            // the next item's rows first: its QK can run beside this one's output (nothing reads Q's memory any more: the
            // last S has come)
            const int lim0 = lim;
            more = begin(seg + 1);
            const bool whole = it.tb == 0 && it.te == it.tiles, head_part = it.tb == 0;
            wait_phase(smem_u32(&sm.n_full[seg & 1]), (seg >> 1) & 1, abort_at, p.budget_ns);
            const float base = sm.first_lv[seg & 1];
            if (!whole && threadIdx.x == kSoftmax * 32) {
                sm.rows[head_part] = it.rows;
                sm.base[head_part] = base;
                sm.start[head_part] = it.start;
                sm.tiles[head_part] = it.tiles;
            }
            const bool hand = !two && nt > 1;  // the second pipeline's result goes to the first
            const bool shared = head_part && !whole;  // (with later CTAs: the share's last item)
            if (shared && threadIdx.x == kSoftmax * 32) {
                const int c0 = blockIdx.x, np = cta_of(it.start + it.tiles - 1, sm) - c0 + 1;
                unsigned seen;
                asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(p.tickets + c0) : "memory");
                if (seen == (unsigned)(np - 1)) {
                    p.tickets[c0] = 0;
                    sm.direct = 1;
                    sm.last_c0[1] = c0;
                    sm.last[1] = np;
                }
            }
            if (hand && u == 1) {
                sm.ml[r] = make_float2(m, l);
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm.x_full));
            }
            if (two || u == 0) {
                wait_phase(smem_u32(&sm.o_full[u]), (u ? outs1 : outs0) & 1, abort_at, p.budget_ns);
                if (hand) wait_phase(smem_u32(&sm.o_full[1]), outs1 & 1, abort_at, p.budget_ns);
            }
            if (shared) {  // a part in shared memory takes the place of Q, K and V: no product may be left that reads them
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm.d_full));
                wait_phase(smem_u32(&sm.d_full), 0, abort_at, p.budget_ns);
            }
            if (two || u == 0) {
                float f = 1.f, f1 = 0.f;  // factors of the two pipelines' O
                if (hand) {
                    wait_phase(smem_u32(&sm.x_full), handed & 1, abort_at, p.budget_ns);
                    const float2 other = sm.ml[r];
                    const float top = fmaxf(m, other.x), at0 = top == -INFINITY ? 0.f : top;
                    f = fast_exp2(m - at0);
                    f1 = fast_exp2(other.x - at0);
                    m = top;
                    l = fmaf(l, f, other.y * f1);
                }
                tc_fence_after();
                bool nan = false;
#pragma unroll
                for (int k = 0; k < kConverters; ++k) nan |= sm.nan_any[seg & 1][k] != 0;
                Part<D>* part = shared && sm.direct ? reinterpret_cast<Part<D>*>(sm.q)
                                                    : reinterpret_cast<Part<D>*>(p.parts) + (size_t)blockIdx.x * 2 + head_part;
                const float inv = l != 0.f ? exp2f(base) / l : 0.f;
                int head0;
                const int row0 = it.rows.of(p, (two ? u * kRowTile : 0) + r, head0);
                const size_t at = (size_t)max(row0, 0) * p.pl.heads + head0;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld_32x32b_x32(ocol + c, o);
                    tmem_wait_ld();
                    if (hand) {
#pragma unroll
                        for (int e = 0; e < 32; e += 16) {
                            uint32_t x[16];
                            tmem_ld_32x32b_x16(ocol + D + c + e, x);
                            tmem_wait_ld();
#pragma unroll
                            for (int k = 0; k < 16; ++k)
                                o[e + k] = __float_as_uint(fmaf(__uint_as_float(o[e + k]), f, __uint_as_float(x[k]) * f1));
                        }
                    }
                    if (nan) {
#pragma unroll 1
                        for (int e = 0; e < 32; ++e) {
                            int at = INT_MAX;
#pragma unroll
                            for (int k = 0; k < kConverters; ++k) at = min(at, sm.nan_at[seg & 1][k][c + e]);
                            if (at < lim0) {
#pragma unroll
                                for (int k = 0; k < 32; ++k)
                                    if (k == e) o[k] = 0x7fc00000u;
                            }
                        }
                    }
                    if (whole && row0 >= 0) {
#pragma unroll
                        for (int e = 0; e < 32; e += 16) {
                            uint32_t y[8];
#pragma unroll
                            for (int k = 0; k < 8; ++k)
                                y[k] = pack_bf16(__uint_as_float(o[e + 2 * k]) * inv, __uint_as_float(o[e + 2 * k + 1]) * inv);
                            store32(p.O + at * D + c + e, y);
                        }
                    } else if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            *reinterpret_cast<uint4*>(&part->o[(c + e) / 4][u * kRowTile + r]) =
                                make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    }
                }
                if (whole && row0 >= 0) p.lse[at] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
                if (!whole) part->ml[u * kRowTile + r] = make_float2(m, l);
                tc_fence_before();
            }
            __syncwarp();
            if (hand && u == 0 && lane == 0) mbar_arrive(smem_u32(&sm.x_empty));
            outs0 += 1;
            outs1 += two || hand;
            handed += hand;
            if (lane == 0) {
                mbar_arrive(smem_u32(&sm.n_empty[seg & 1]));
                mbar_arrive(smem_u32(&sm.i_empty[seg % kItemRing]));
            }
            if (seg == 0 && lane == 0) mbar_arrive(smem_u32(&sm.t_full));
            ++seg;
        }
        if (seg == 0 && lane == 0) mbar_arrive(smem_u32(&sm.t_full));
        // the part of the last item, where it was written for another CTA
        const bool bad = soft_any(*abortf != 0);  // (else every warp has been through every item)
        if (!bad && threadIdx.x == kSoftmax * 32 && sm.tiles[1] > 0 && !sm.direct) {
            const int c0 = cta_of(sm.start[1], sm), np = cta_of(sm.start[1] + sm.tiles[1] - 1, sm) - c0 + 1;
            unsigned seen;
            asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(seen) : "l"(p.tickets + c0) : "memory");
            if (seen == (unsigned)(np - 1)) {
                p.tickets[c0] = 0;
                sm.last_c0[1] = c0;
                sm.last[1] = np;
            }
        }
        dead = *abortf != 0;
    }
    if (__syncthreads_or(dead)) {
        // a wait ran out: nothing more is issued, but copies and products may be in flight
        if (warp == kLoad && lane == 0) {
            for (uint32_t x = kloads > kK ? kloads - kK : 0; x < kloads; ++x) wait_raw(kfull0 + 8 * (x % kK), (x / kK) & 1, p.budget_ns);
            for (uint32_t x = vloads > kRaw ? vloads - kRaw : 0; x < vloads; ++x)
                wait_raw(rfull0 + 8 * (x % kRaw), (x / kRaw) & 1, p.budget_ns);
        }
        if (warp == kIssue && elect_one_sync()) {
            mma_commit(smem_u32(&sm.drain));
            wait_raw(smem_u32(&sm.drain), 0, p.budget_ns);
        }
        if (threadIdx.x == 0) atomicExch(p.pl.status, SSBA_ERR_TIMEOUT);
    } else {
        for (int i = 0; i < 2; ++i)
            if (sm.last[i])
                join<D>(p, sm.rows[i], sm.base[i], sm.last_c0[i], sm.last[i],
                        i && sm.direct ? reinterpret_cast<const Part<D>*>(sm.q) : nullptr);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kIssue) tmem_dealloc(tbase, kTmemCols);
}

template <int D>
int launch(const Maps& maps, const Params& p, cudaStream_t st)
{
    const size_t smem = sizeof(Smem<D>) + 1024;
    static_assert(offsetof(Smem<D>, raw) >= sizeof(Part<D>), "a part in the place of Q, K and V");
    static_assert(sizeof(Smem<D>) + 1024 + 128 <= 232448, "shared memory of one CTA (227 KB opt-in limit)");
    static PerDeviceOnce once;
    once.run([smem] {
        cudaFuncSetAttribute(ssba_cache_attend_rows_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    const cudaError_t e = launch_dependent(ssba_cache_attend_rows_kernel<D>, dim3(std::min(device_sm_count(), kMaxGrid)),
                                           kThreads, smem, st, maps, p);
    if (e == cudaSuccess) return SSBA_OK;
    set_error("ssba_cache_attend: %s", cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

}  // namespace
}  // namespace cache

size_t cache_attend_rows_workspace()
{
    return SSBA_CACHE_TICKET_BYTES +
           (size_t)2 * std::min(device_sm_count(), cache::kMaxGrid) * cache::kItemRows * (128 + 2) * sizeof(float);
}

int launch_cache_attend_rows(const cache::Pool& pl, const cache::Batch& bt, int head_dim, float scale, const void* q,
                             void* O, float* lse, void* ws, cudaStream_t st, uint64_t budget_ns, int withhold)
{
    using namespace cache;
    Maps maps;
    memset(&maps, 0, sizeof(maps));
    const long long tiles = (long long)pl.pages * pl.kv_heads;
    if (!encode_page_map(&maps.k, pl.K, tiles, head_dim, head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B) ||
        !encode_page_map(&maps.v, pl.V, tiles, head_dim, CU_TENSOR_MAP_SWIZZLE_NONE)) {
        set_error("ssba_cache_attend: cuTensorMapEncodeTiled failed");
        return SSBA_ERR_CUDA;
    }
    Params p;
    memset(&p, 0, sizeof(p));
    p.pl = pl;
    p.bt = bt;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.scale_log2 = scale * kLog2e;
    p.O = static_cast<__nv_bfloat16*>(O);
    p.lse = lse;
    p.tickets = static_cast<unsigned*>(ws);
    p.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + SSBA_CACHE_TICKET_BYTES);
    p.G = pl.heads / pl.kv_heads;
    p.budget_ns = budget_ns;
    p.withhold = withhold;
    p.chunks = (p.G + kItemRows - 1) / kItemRows;
    p.gc = (p.G + p.chunks - 1) / p.chunks;
    p.gc_inv = (65536 + p.gc - 1) / p.gc;
    p.tq = 1;
    while (2 * p.tq * p.gc <= kItemRows) p.tq *= 2;
    return head_dim == 64 ? launch<64>(maps, p, st) : launch<128>(maps, p, st);
}

}  // namespace ssba
