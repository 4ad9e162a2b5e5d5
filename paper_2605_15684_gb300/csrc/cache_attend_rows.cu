// cache_attend_rows.cu -- attention over the paged 8-bit cache for many rows that share a K/V head's tokens (chunks
// of prompts, drafts of several tokens): bound by the tensor cores and the exp2s, not by HBM.
//
// An item is up to 256 rows (tokens times the group's heads) of one sequence and K/V head, in two tiles of 128
// rows; it visits its sequence's tiles of 128 tokens (two pages):
//   S_u = Q_u K^T   tcgen05.mma kind::f16, M = 128, N = 128, K = D   (fp16 operands, K-major)
//   O_u += P_u V    M = 128, N = D, K = 128                          (P from tensor memory, V MN-major)
// An e4m3 value is an fp16 value, so K and V are converted without rounding, once for both row tiles, and their
// page's scale stays out of the products: K's multiplies the scores, V's is added to their exponent,
//   P = 2^(s + log2 v_scale - m),   l = sum P / v_scale,   O = sum P (bytes of V) / l,
// v_scale relative to the sequence's first page (within 2^+-100 of it). Rows of Q are brought below 448 by a
// power of two; their 8 bits of significand are exact in fp16 down to 2^-25 of the row's largest. P is rounded to fp16's
// 11 bits; m is 8 below the largest exponent, so P's smallest step is 2^-32 of the largest weight.
//
// One CTA an SM, 12 warps: a producer (TMA of the pages' bytes), an issuer, two converters (a page each: bytes to
// fp16 in the swizzled layout of the products), and a softmax warpgroup for each row tile (a thread is a row). P
// overwrites the upper half of its S, so of one row tile PV_g comes before QK_{g + 1}; while one row tile
// is with the tensor cores the other is with its softmax. Against a reference maximum that is raised only
// where a tile's sum passes 2^14 (O is then rescaled in tensor memory), as in the other kernels of this library.
// Work is shared out and joined as in cache_attend_tc.cu.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "cache_items.cuh"

namespace ssba {
namespace cache {
namespace {

constexpr int kThreads = 384;
constexpr int kRowTile = 128;
constexpr int kItemRows = 2 * kRowTile;
constexpr int kCv = 3, kRaw = 3, kMetas = 8;
constexpr float kTop = 8.f;         // log2 of the largest P against a new reference
constexpr float kMost = 16384.f;    // row sum of a tile above which the reference is raised (fp16 ends at 65504)
constexpr float kSpan = 100.f;      // log2 of V scales, relative to the first page's
enum Role { kLoad = 0, kIssue = 1, kConvert = 2, kSoftmax = 4 };
constexpr uint32_t kTmemCols = 512;

constexpr uint32_t idesc_f16_f32(int M, int N, bool b_mn_major) { return idesc_e4m3_f32(M, N, false, b_mn_major); }

struct Meta {
    float ks, lv, inv;  // K scale; log2 of the V scale (relative); 2^-lv
    int pos;            // token position of the page
};

template <int D>
struct __align__(1024) Smem {
    uint8_t q[2][D / 64][kRowTile][128];   // fp16, 64 channels a 128-byte row, 128-byte swizzle
    uint8_t cv[kCv][D / 64][kTile][128];
    uint8_t raw[kRaw][kTile * D];
    int nan_at[2][2][D];  // by item parity and converter: first token whose V is NaN, of those that not every row sees
    int nan_any[2][2];
    Meta meta[kMetas][2];
    uint64_t raw_full[kRaw], raw_empty[kRaw], cv_full[kCv], cv_empty[kCv], m_full[kMetas];
    uint64_t q_full[2], s_full[2], p_full[2], o_full[2], n_full[2], n_empty[2], drain;
    long long w0, w1, total;
    int first_b, ctas;
    long long first_at;
    uint32_t tmem_base;
    Rows rows[2];
    float base[2];
    int abort_flag, last[2], last_c0[2];
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

__device__ __forceinline__ uint32_t pack_half(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// log2 of the V scale that an item's P is relative to: its sequence's first page's.
template <class W>
__device__ __forceinline__ float base_of(const Params& p, const W& it)
{
    int j;
    const int page = it.page(0, j);
    const float vs = page >= 0 ? __ldg(p.pl.v_scale + (size_t)page * p.pl.kv_heads + it.hv / p.chunks) : 0.f;
    return vs > 0.f && vs < INFINITY ? log2f(vs) : 0.f;
}

// Joins the np parts of an item that begins in CTA c0, in order, and writes its rows: a softmax warp takes every
// eighth row, a lane D / 32 channels, with eight parts' loads in flight.
template <int D>
__device__ __noinline__ void join(const Params& p, const Rows rows, float base, int c0, int np, int w, int lane)
{
    constexpr int kAhead = 8, kE = D / 32;
    const size_t size = (size_t)kItemRows * (D + 2);
#pragma unroll 1
    for (int r = w; r < kItemRows; r += 8) {
        int head;
        const int row = rows.of(p, r, head);
        if (row < 0) continue;
        float m = -INFINITY, l = 0.f, o[kE] = {};
#pragma unroll 1
        for (int k0 = 0; k0 < np; k0 += kAhead) {
            float2 ml[kAhead];
            float v[kAhead][kE];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const float* at = p.parts + ((size_t)(c0 + k0 + k) * 2 + (k0 + k == 0)) * size;
                const bool real = k0 + k < np;
                ml[k] = real ? __ldcg(reinterpret_cast<const float2*>(at + kItemRows * D) + r) : make_float2(-INFINITY, 0.f);
#pragma unroll
                for (int e = 0; e < kE; ++e) v[k][e] = real ? __ldcg(at + (size_t)r * D + e * 32 + lane) : 0.f;
            }
            float top = m;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) top = fmaxf(top, ml[k].x);
            const float at0 = top == -INFINITY ? 0.f : top, f = fast_exp2(m - at0);
            m = top;
            l *= f;
#pragma unroll
            for (int e = 0; e < kE; ++e) o[e] *= f;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const float fk = fast_exp2(ml[k].x - at0);
                l = fmaf(ml[k].y, fk, l);
#pragma unroll
                for (int e = 0; e < kE; ++e) o[e] = fmaf(v[k][e], fk, o[e]);
            }
        }
        const size_t at = (size_t)row * p.pl.heads + head;
        const float inv = l != 0.f ? exp2f(base) / l : 0.f;
#pragma unroll
        for (int e = 0; e < kE; ++e) p.O[at * D + e * 32 + lane] = __float2bfloat16_rn(o[e] * inv);
        if (lane == 0) p.lse[at] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) ssba_cache_attend_rows_kernel(const __grid_constant__ Maps maps,
                                                                             const __grid_constant__ Params p)
{
    extern __shared__ uint8_t smem_raw[];
    Smem<D>& sm = *reinterpret_cast<Smem<D>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        sm.abort_flag = 0;
        for (int i = 0; i < kRaw; ++i) {
            mbar_init(smem_u32(&sm.raw_full[i]), 1);
            mbar_init(smem_u32(&sm.raw_empty[i]), 2);
        }
        for (int i = 0; i < kCv; ++i) {
            mbar_init(smem_u32(&sm.cv_full[i]), 2);
            mbar_init(smem_u32(&sm.cv_empty[i]), 1);
        }
        for (int i = 0; i < kMetas; ++i) mbar_init(smem_u32(&sm.m_full[i]), 2);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sm.q_full[i]), 4);
            mbar_init(smem_u32(&sm.s_full[i]), 1);
            mbar_init(smem_u32(&sm.p_full[i]), 4);
            mbar_init(smem_u32(&sm.o_full[i]), 1);
            mbar_init(smem_u32(&sm.n_full[i]), 2);
            mbar_init(smem_u32(&sm.n_empty[i]), 8);
        }
        mbar_init(smem_u32(&sm.drain), 1);
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
    grid_dep_launch();
    make_share<false, kThreads>(p, sm);  // ends in a barrier
    tc_fence_after();
    const uint32_t tbase = sm.tmem_base;
    volatile int* abortf = &sm.abort_flag;
    const uint32_t abort_at = smem_u32(&sm.abort_flag);
    const uint32_t rfull0 = smem_u32(&sm.raw_full[0]), rempty0 = smem_u32(&sm.raw_empty[0]);
    const uint32_t cfull0 = smem_u32(&sm.cv_full[0]), cempty0 = smem_u32(&sm.cv_empty[0]);
    bool dead = false;
    uint32_t loads = 0;  // of the producer
    Walk<false> it(p, sm);
    // an item of up to 128 rows has no second row tile
    auto both = [&](const Walk<false>& w) { return w.rows().n * p.gc > kRowTile; };

    if (warp == kLoad) {
        // ------------------------------------------------------------ producer: K_0, V_0, K_1, ...
        for (; it.more() && !dead; it.next()) {
            const int h = it.hv / p.chunks;
            for (int c0 = 2 * it.tb; c0 < 2 * it.te && !dead; c0 += 32) {  // 32 pages at a time
                int j, page = -1;
                if (c0 + lane < 2 * it.te) page = it.page(c0 + lane, j);
                const int unit = page >= 0 ? page * p.pl.kv_heads + h : -1;
                const int n = min(16, it.te - c0 / 2);
                for (int i = 0; i < n && !dead; ++i) {
                    const int p0 = __shfl_sync(0xffffffffu, unit, 2 * i), p1 = __shfl_sync(0xffffffffu, unit, 2 * i + 1);
                    if (lane == 0) {
                        for (int v = 0; v < 2; ++v) {
                            const uint32_t slot = loads % kRaw;
                            if (!mbar_wait(rempty0 + 8 * slot, ((loads / kRaw) & 1) ^ 1, abortf, p.budget_ns)) {
                                dead = true;
                                break;
                            }
                            const uint32_t bar = rfull0 + 8 * slot, to = smem_u32(&sm.raw[slot][0]);
                            const CUtensorMap* map = v ? &maps.v : &maps.k;
                            mbar_arrive_expect_tx(bar, ((p0 >= 0) + (p1 >= 0)) * (uint32_t)(kPage * D));
                            if (p0 >= 0) tma_load_3d(to, map, bar, 0, 0, p0);
                            if (p1 >= 0) tma_load_3d(to + kPage * D, map, bar, 0, 0, p1);
                            ++loads;
                        }
                    }
                    dead = __shfl_sync(0xffffffffu, (int)dead, 0) != 0;
                }
            }
        }
        __syncwarp();
    } else if (warp == kIssue) {
        // ------------------------------------------------------------ issuer
        uint32_t cnt[2] = {0, 0}, qs[2] = {0, 0};  // tiles, items of each row tile
        bool pend[2] = {false, false}, p_first[2] = {}, p_last[2] = {};  // PV still to come: first, last tile of its item's share
        uint32_t vslot = 0;
        auto slot_full = [&](uint32_t x) { wait_phase(cfull0 + 8 * (x % kCv), (x / kCv) & 1, abort_at, p.budget_ns); };
        auto pv = [&](int u) {
            wait_phase(smem_u32(&sm.p_full[u]), (cnt[u] - 1) & 1, abort_at, p.budget_ns);
            slot_full(vslot);
            tc_fence_after();
            if (elect_one_sync()) {
                const uint64_t b = sdesc_sw128(smem_u32(&sm.cv[vslot % kCv][0][0][0]), kTile * 128, 1024);
#pragma unroll
                for (int k = 0; k < kTile / 16; ++k)
                    mma_ts(tbase + 256 + u * D, tbase + u * 128 + 64 + k * 8, b + (uint64_t)(k * 128),
                           idesc_f16_f32(128, D, true), (!p_first[u] || k > 0) ? 1u : 0u);
                if (p_last[u]) mma_commit(smem_u32(&sm.o_full[u]));
                if (u == 1 || !pend[1]) mma_commit(cempty0 + 8 * (vslot % kCv));
            }
            __syncwarp();
        };
        uint32_t g = 0;
        for (; it.more(); it.next()) {
            const bool two = both(it);
            for (int i = it.tb; i < it.te; ++i, ++g) {
                const uint32_t kslot = 2 * g;
                vslot = 2 * g - 1;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (pend[u]) pv(u);
                    if (u == 1 && !two) continue;
                    if (i == it.tb) wait_phase(smem_u32(&sm.q_full[u]), qs[u]++ & 1, abort_at, p.budget_ns);
                    slot_full(kslot);
                    tc_fence_after();
                    if (elect_one_sync()) {
                        const uint64_t a = sdesc_sw128(smem_u32(&sm.q[u][0][0][0]), 16, 1024);
                        const uint64_t b = sdesc_sw128(smem_u32(&sm.cv[kslot % kCv][0][0][0]), 16, 1024);
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint64_t at = (uint64_t)((k / 4) * (kTile * 128 / 16) + (k % 4) * 2);
                            mma_ss(tbase + u * 128, a + at, b + at, idesc_f16_f32(128, 128, false), k > 0 ? 1u : 0u);
                        }
                        mma_commit(smem_u32(&sm.s_full[u]));
                        if (u == 1 || !two) mma_commit(cempty0 + 8 * (kslot % kCv));
                    }
                    __syncwarp();
                    ++cnt[u];
                }
                pend[0] = true;
                pend[1] = two;
                p_first[0] = p_first[1] = i == it.tb;
                p_last[0] = p_last[1] = i == it.te - 1;
            }
        }
        if (g > 0) {
            vslot = 2 * g - 1;
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (pend[u]) pv(u);
        }
        dead = *abortf != 0;
    } else if (warp < kSoftmax) {
        // ------------------------------------------------------------ converters: page `w` of every tile
        constexpr int kLanes = D / 16, kRows = 32 / kLanes;  // lanes of a row (16 bytes each), rows at a time
        const int w = warp - kConvert, c = lane % kLanes;
        uint32_t use = 0, g = 0;
        int seg = 0;
        for (; it.more(); it.next(), ++seg) {
            const int h = it.hv / p.chunks;
            const Rows rows = it.rows();
            const int lo_lim = it.limit(rows.row), hi_lim = it.limit(rows.row + max(rows.n, 1) - 1);
            const float base = base_of(p, it);
            wait_phase(smem_u32(&sm.n_empty[seg & 1]), ((seg >> 1) & 1) ^ 1, abort_at, p.budget_ns);
            for (int i = lane; i < D; i += 32) sm.nan_at[seg & 1][w][i] = INT_MAX;
            if (lane == 0) sm.nan_any[seg & 1][w] = 0;
            __syncwarp();
            for (int c0 = it.tb; c0 < it.te; c0 += 32) {  // 32 tiles' pages at a time
                int j, page = -1;
                if (c0 + lane < it.te) page = it.page(2 * (c0 + lane) + w, j);
                float my_ks = 0.f, my_lv = 0.f;
                if (page >= 0) {
                    const size_t unit = (size_t)page * p.pl.kv_heads + h;
                    my_ks = __ldg(p.pl.k_scale + unit);
                    const float vs = __ldg(p.pl.v_scale + unit);
                    my_lv = vs > 0.f ? fminf(fmaxf(log2f(vs) - base, -kSpan), kSpan) : isnan(vs) ? vs : 0.f;
                }
                const int my_pos = page >= 0 ? j * kPage : kNowhere;
                const int n = min(32, it.te - c0);
                for (int i = 0; i < n; ++i, ++g) {
                    const int pos = __shfl_sync(0xffffffffu, my_pos, i);
                    const float ks = __shfl_sync(0xffffffffu, my_ks, i), lv = __shfl_sync(0xffffffffu, my_lv, i);
#pragma unroll
                    for (int v = 0; v < 2; ++v, ++use) {
                        const uint32_t rs = use % kRaw, cs = use % kCv;
                        wait_phase(rfull0 + 8 * rs, (use / kRaw) & 1, abort_at, p.budget_ns);
                        wait_phase(cempty0 + 8 * cs, ((use / kCv) & 1) ^ 1, abort_at, p.budget_ns);
                        const uint8_t* from = &sm.raw[rs][w * kPage * D];
                        if (pos != kNowhere || v) {
#pragma unroll 4
                            for (int r0 = 0; r0 < kPage; r0 += kRows) {
                                const int r = r0 + lane / kLanes, row = w * kPage + r;
                                uint4 x = *reinterpret_cast<const uint4*>(from + r * D + c * 16);
                                if (v && pos + r >= lo_lim) {
                                    // tokens that no row sees: their V is whatever the page holds, and 0 * NaN would
                                    // reach every row; tokens that some rows see: a NaN is taken out and kept for those
                                    if (pos + r >= hi_lim) {
                                        x = make_uint4(0, 0, 0, 0);
                                    } else {
                                        uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                                        for (int k = 0; k < 4; ++k) {
                                            const uint32_t m = word[k] & 0x7f7f7f7fu;
                                            if (((m + 0x01010101u) & 0x80808080u) == 0) continue;  // no byte of 0x7f
                                            for (int e = 0; e < 4; ++e)
                                                if (((word[k] >> (8 * e)) & 0x7f) == 0x7f) {
                                                    atomicMin(&sm.nan_at[seg & 1][w][c * 16 + k * 4 + e], pos + r);
                                                    sm.nan_any[seg & 1][w] = 1;
                                                    word[k] &= ~(0xffu << (8 * e));
                                                }
                                        }
                                        x = make_uint4(word[0], word[1], word[2], word[3]);
                                    }
                                }
                                const uint4 a = make_uint4(half2_of(x.x & 0xffff), half2_of(x.x >> 16), half2_of(x.y & 0xffff), half2_of(x.y >> 16));
                                const uint4 b = make_uint4(half2_of(x.z & 0xffff), half2_of(x.z >> 16), half2_of(x.w & 0xffff), half2_of(x.w >> 16));
                                uint8_t* to = &sm.cv[cs][c / 4][row][0];
                                const int k = (c % 4) * 2;
                                // lanes of the second 64 channels write their second half first: no bank conflicts
                                const bool turn = c / 4;
                                *reinterpret_cast<uint4*>(to + ((k + turn) ^ (row & 7)) * 16) = turn ? b : a;
                                *reinterpret_cast<uint4*>(to + ((k + !turn) ^ (row & 7)) * 16) = turn ? a : b;
                            }
                        }
                        if (!v && lane == 0) sm.meta[g % kMetas][w] = Meta{ks, lv, exp2f(-lv), pos};
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            mbar_arrive(rempty0 + 8 * rs);
                            mbar_arrive(cfull0 + 8 * cs);
                            if (!v) mbar_arrive(smem_u32(&sm.m_full[g % kMetas]));
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
        const uint32_t scol = tbase + u * 128 + lanes, pcol = scol + 64, ocol = tbase + 256 + u * D + lanes;
        long long start0 = 0, start1 = 0;
        int tiles0 = 0, tiles1 = 0;
        uint32_t cnt = 0, items = 0, g = 0;  // tiles and items of this row tile; tiles of the CTA
        int seg = 0;
        // the row's query to shared memory; its row of the batch, head, tokens it sees and factor of scores
        int row = -1, head = 0, lim = 0;
        float qf = 0.f, base = 0.f;
        auto load_q = [&](const Walk<false>& w) {
            base = base_of(p, w);
            row = w.rows().of(p, u * kRowTile + r, head);
            lim = row >= 0 ? w.limit(row) : 0;
            uint4 in[D / 8];
            float amax = 0.f;
#pragma unroll
            for (int c = 0; c < D / 8; ++c)
                in[c] = row >= 0 ? __ldg(reinterpret_cast<const uint4*>(p.q + ((size_t)row * p.pl.heads + head) * D) + c)
                                 : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const uint32_t x[4] = {in[c].x, in[c].y, in[c].z, in[c].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float a = fabsf(__uint_as_float(x[e] << 16)), b = fabsf(__uint_as_float(x[e] & 0xffff0000u));
                    if (a < INFINITY) amax = fmaxf(amax, a);
                    if (b < INFINITY) amax = fmaxf(amax, b);
                }
            }
            const float scale = scale_for(amax), inv = scale > 0.f ? 1.f / scale : 1.f;
            qf = scale * p.scale_log2;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                const uint32_t x[4] = {in[c].x, in[c].y, in[c].z, in[c].w};
                uint32_t y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // an infinity makes its row's scores NaN, as it would a softmax's
                    const float a = __uint_as_float(x[e] << 16), b = __uint_as_float(x[e] & 0xffff0000u);
                    y[e] = pack_half(fabsf(a) < INFINITY ? a * inv : NAN, fabsf(b) < INFINITY ? b * inv : NAN);
                }
                *reinterpret_cast<uint4*>(&sm.q[u][c / 8][r][((c % 8) ^ (r & 7)) * 16]) = make_uint4(y[0], y[1], y[2], y[3]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.q_full[u]));
        };
        if (it.more() && (u == 0 || both(it))) load_q(it);
        while (it.more() && !*abortf) {
            const bool active = u == 0 || both(it);
            float m = -INFINITY, l = 0.f;
            for (int i = it.tb; i < it.te && active; ++i, ++cnt) {
                const uint32_t gt = g + (i - it.tb);
                wait_phase(smem_u32(&sm.m_full[gt % kMetas]), (gt / kMetas) & 1, abort_at, p.budget_ns);
                const Meta ma = sm.meta[gt % kMetas][0], mb = sm.meta[gt % kMetas][1];
                const float ca = ma.ks * qf, cb = mb.ks * qf;
                const int la = min(max(lim - ma.pos, 0), kPage), lb = min(max(lim - mb.pos, 0), kPage);
                const bool cut = __any_sync(0xffffffffu, la < kPage || lb < kPage);
                wait_phase(smem_u32(&sm.s_full[u]), cnt & 1, abort_at, p.budget_ns);
                tc_fence_after();
                uint32_t pk[64];
                float sa = 0.f, sb = 0.f;
                bool raise = __any_sync(0xffffffffu, m == -INFINITY && la + lb > 0);
#pragma unroll 1
                for (bool again = true; again;) {
                    if (raise) {
                        float mx = -INFINITY;
#pragma unroll
                        for (int ch = 0; ch < 4; ++ch) {
                            uint32_t x[32];
                            tmem_ld_32x32b_x32(scol + 32 * ch, x);
                            tmem_wait_ld();
                            const float cc = ch < 2 ? ca : cb, lv = ch < 2 ? ma.lv : mb.lv;
                            const int left = (ch < 2 ? la : lb) - (ch & 1) * 32;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (e < left) mx = fmaxf(mx, fmaf(__uint_as_float(x[e]), cc, lv));
                        }
                        const float now = mx == -INFINITY ? m : fmaxf(m, mx - kTop);
                        const float f = m == -INFINITY ? 0.f : fast_exp2(m - now);
                        l *= f;
                        m = now;
                        if (i > it.tb) {  // O holds the tiles so far: QK of this one was issued behind their PV
#pragma unroll
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tmem_ld_32x32b_x16(ocol + c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st_32x32b_x16(ocol + c, o);
                            }
                            tmem_wait_st();
                        }
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
                    sa = sb = 0.f;
#pragma unroll
                    for (int ch = 0; ch < 4; ++ch) {
                        uint32_t x[32];
                        tmem_ld_32x32b_x32(scol + 32 * ch, x);
                        tmem_wait_ld();
                        const float cc = ch < 2 ? ca : cb, off = (ch < 2 ? ma.lv : mb.lv) - ref;
                        const int left = (ch < 2 ? la : lb) - (ch & 1) * 32;
                        const float2 c2 = make_float2(cc, cc), o2 = make_float2(off, off);
                        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float2 y = __ffma2_rn(make_float2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), c2, o2);
                            if (cut) {
                                if (2 * e >= left) y.x = -INFINITY;
                                if (2 * e + 1 >= left) y.y = -INFINITY;
                            }
                            y = make_float2(fast_exp2(y.x), fast_exp2(y.y));
                            sum = __fadd2_rn(sum, y);
                            pk[16 * ch + e] = pack_half(y.x, y.y);
                        }
                        if (ch < 2) sa += sum.x + sum.y;
                        else sb += sum.x + sum.y;
                    }
                    again = !raise && __any_sync(0xffffffffu, sa + sb > kMost);
                    raise = again;
                }
                l += sa * ma.inv + sb * mb.inv;
#pragma unroll
                for (int ch = 0; ch < 4; ++ch) tmem_st_32x32b_x16(pcol + 16 * ch, *reinterpret_cast<uint32_t(*)[16]>(&pk[16 * ch]));
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm.p_full[u]));
            }
            g += it.te - it.tb;
            // the next item's rows first: its QK can run beside this one's output (no wait is under way on Q's memory:
            // the last S has come)
            const int row0 = row, head0 = head, lim0 = lim;
            const float base0 = base;
            const bool whole = it.tb == 0 && it.te == it.tiles, head_part = it.tb == 0;
            if (!whole) {
                if (head_part) {
                    start1 = it.start;
                    tiles1 = it.tiles;
                } else {
                    start0 = it.start;
                    tiles0 = it.tiles;
                }
                if (threadIdx.x == kSoftmax * 32) {
                    sm.rows[head_part] = it.rows();
                    sm.base[head_part] = base0;
                }
            }
            it.next();
            if (it.more() && (u == 0 || both(it))) load_q(it);
            wait_phase(smem_u32(&sm.n_full[seg & 1]), (seg >> 1) & 1, abort_at, p.budget_ns);
            if (active) {
                wait_phase(smem_u32(&sm.o_full[u]), items & 1, abort_at, p.budget_ns);
                ++items;
                tc_fence_after();
                const bool nan = sm.nan_any[seg & 1][0] || sm.nan_any[seg & 1][1];
                float* part = p.parts + ((size_t)blockIdx.x * 2 + head_part) * kItemRows * (D + 2);
                const float inv = l != 0.f ? exp2f(base0) / l : 0.f;
                const size_t at = (size_t)max(row0, 0) * p.pl.heads + head0;
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld_32x32b_x32(ocol + c, o);
                    tmem_wait_ld();
                    if (nan) {
#pragma unroll 1
                        for (int e = 0; e < 32; ++e)
                            if (min(sm.nan_at[seg & 1][0][c + e], sm.nan_at[seg & 1][1][c + e]) < lim0) {
#pragma unroll
                                for (int k = 0; k < 32; ++k)
                                    if (k == e) o[k] = 0x7fc00000u;
                            }
                    }
                    if (whole && row0 >= 0) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t y[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(o[e + 2 * k]) * inv, __uint_as_float(o[e + 2 * k + 1]) * inv);
                                y[k] = *reinterpret_cast<const uint32_t*>(&b);
                            }
                            *reinterpret_cast<uint4*>(p.O + at * D + c + e) = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    } else if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            *reinterpret_cast<uint4*>(part + (size_t)(u * kRowTile + r) * D + c + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    }
                }
                if (whole && row0 >= 0) p.lse[at] = l != 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
                if (!whole) reinterpret_cast<float2*>(part + kItemRows * D)[u * kRowTile + r] = make_float2(m, l);
                tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.n_empty[seg & 1]));
            ++seg;
        }
        // the items that are shared with other CTAs, counted off once all is written (see cache_attend_tc.cu)
        const bool bad = soft_any(*abortf != 0);  // (else every warp has been through every item)
        if (tiles0 + tiles1 > 0 && !bad) {
            const int tid = threadIdx.x - kSoftmax * 32;
            if (tid < 2) {
                const long long start = tid ? start1 : start0;
                const int tiles = tid ? tiles1 : tiles0;
                int c0 = 0, np = 0;
                if (tiles > 0) {
                    c0 = cta_of(start, sm);
                    np = cta_of(start + tiles - 1, sm) - c0 + 1;
                    unsigned seen;
                    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(seen) : "l"(p.tickets + c0) : "memory");
                    if (seen == (unsigned)(np - 1)) p.tickets[c0] = 0;
                    else np = 0;
                }
                sm.last_c0[tid] = c0;
                sm.last[tid] = np;
            }
            soft_any(false);
            for (int i = 0; i < 2; ++i)
                if (sm.last[i]) join<D>(p, sm.rows[i], sm.base[i], sm.last_c0[i], sm.last[i], warp - kSoftmax, lane);
        }
        dead = *abortf != 0;
    }
    if (__syncthreads_or(dead)) {
        // a wait ran out: nothing more is issued, but copies and products may be in flight
        if (warp == kLoad && lane == 0)
            for (uint32_t x = loads > kRaw ? loads - kRaw : 0; x < loads; ++x)
                wait_raw(rfull0 + 8 * (x % kRaw), (x / kRaw) & 1, p.budget_ns);
        if (warp == kIssue && elect_one_sync()) {
            mma_commit(smem_u32(&sm.drain));
            wait_raw(smem_u32(&sm.drain), 0, p.budget_ns);
        }
        if (threadIdx.x == 0) atomicExch(p.pl.status, SSBA_ERR_TIMEOUT);
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
    static_assert(sizeof(Smem<D>) + 1024 + 128 <= 232448, "shared memory of one CTA (227 KB opt-in limit)");
    static PerDeviceOnce once;
    once.run([smem] {
        cudaFuncSetAttribute(ssba_cache_attend_rows_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(std::min(device_sm_count(), kMaxGrid), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, ssba_cache_attend_rows_kernel<D>, maps, p);
    if (e == cudaSuccess) e = cudaGetLastError();
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
                             void* O, float* lse, void* ws, cudaStream_t st)
{
    using namespace cache;
    Maps maps;
    memset(&maps, 0, sizeof(maps));
    const long long tiles = (long long)pl.pages * pl.kv_heads;
    if (!encode_page_map(&maps.k, pl.K, tiles, head_dim, CU_TENSOR_MAP_SWIZZLE_NONE) ||
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
    p.budget_ns = kWaitBudgetNs;
    p.chunks = (p.G + kItemRows - 1) / kItemRows;
    p.gc = (p.G + p.chunks - 1) / p.chunks;
    p.tq = 1;
    while (2 * p.tq * p.gc <= kItemRows) p.tq *= 2;
    return head_dim == 64 ? launch<64>(maps, p, st) : launch<128>(maps, p, st);
}

}  // namespace ssba
