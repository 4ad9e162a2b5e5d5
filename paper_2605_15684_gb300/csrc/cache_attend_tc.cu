// cache_attend_tc.cu -- attention over the paged 8-bit cache on the sm_103a tensor cores (bf16 queries).
//
// A served token reads its sequence's whole cache once for a handful of query heads, so the kernel is
// to be bound by HBM: K and V go from the pool to shared memory by TMA and from there to the tensor
// cores as the bytes they are, with tokens (for S) and channels (for O) as the products' 128 rows and the
// queries as their few columns. With R rows (query heads of some tokens) and tiles of 128 tokens:
//   S^T = K Q^T   tcgen05.mma kind::f8f6f4, M = 128 tokens, N = 2R, K = D   (A = K tile, K-major)
//   O^T = V^T P^T M = 128 channels, N = 2R, K = 128 tokens                  (A = V tile, MN-major)
// Q and P are not 8-bit values: each is the sum of two e4m3 numbers, x = hi + lo / 16 with hi = e4m3(x) and
// lo = e4m3(16 (x - hi)), 4 + 4 bits of significand, in two columns whose products are added in fp32. A row
// of Q is first brought below 448 by a power of two; its 8-bit significands then split without rounding
// down to 2^-13 of the row's largest, and to within 2^-21 of it below. P is rounded to 8 bits as a bf16 P would be.
//
// A CTA takes an equal share of the batch's tiles, whole items (one sequence, one K/V head, R rows) and
// parts of them, in order. Warps of a CTA (all walk the same items):
//   producer   TMA of K and V tiles (two pages) into one ring, in the order they are used
//   issuer     QK of tile g, then PV of tile g - 1
//   Q loader   an item's rows of Q, split, and each row's limit (tokens it sees)
//   meta       page scales and token positions of 32 pages at a time
//   softmax    four warps, two a page. For S a thread is a token; warps reduce a tile's row maxima, and lane r
//              works out row r's references. For O a thread is a channel: every tile's O^T comes out of
//              tensor memory and is added to registers.
// P is formed against the tile's own maximum, of scores plus log2 of their page's V scale, as 2^(s - max + 8): what e4m3
// cannot hold is then below 2^-22 of the tile's largest term, however large an earlier token's weight was (against
// a running maximum, the small weights behind one dominating token would be lost, which many together are
// not). O takes the tile's factor 2^(max - 8 - reference) as it is added, the sum of weights is kept apart.
// An item that several CTAs share leaves parts (O, reference, sum) in the workspace; the CTA that comes
// last joins them in order, so that the result does not depend on which it was.
//
// Bound by HBM where sequences are long: 64 of up to 16000 tokens, 8 K/V heads of 128 for 64 query heads (1.33 GB):
// 210 us, 0.93 of the copy rate (a first version on the CUDA cores took 996). Some 10 us
// do not depend on the size: shares, table, scales and first tiles at the start, the last tile's chain and the join at
// the end; they are what 16 sequences of up to 8000 tokens (35.7 us) take beyond the 24 at the copy rate, and nearly all of one
// of 700 tokens (9.1 us). The tensor pipe is busy for 3 % of the time: N = 2R columns of 128 rows.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "cache_items.cuh"

namespace ssba {
namespace cache {
namespace {

constexpr int kThreads = 256;
constexpr int kSoft = 128;           // softmax threads
constexpr int kMeta = 32;            // pages of a meta chunk
constexpr float kTop = 8.f;          // log2 of a tile's largest P: 2^8 < 448
enum Role { kLoad = 0, kIssue = 1, kLoadQ = 2, kLoadMeta = 3 };

constexpr size_t kPartFloats = (size_t)16 * (128 + 2) * 2 * kMaxGrid;  // two parts a CTA of up to 16 rows

template <int R, int D>
struct Cfg {
    static constexpr int N = 2 * R;
    static constexpr int kCtas = 2;  // of an SM
    static constexpr uint32_t kSlotBytes = kTile * D;
    static constexpr int kRing = (R == 8 ? 96 : 80) * 1024 / kSlotBytes, kSlots = kRing < 12 ? kRing : 12;
    static constexpr uint32_t kTmemCols = 4 * N;
    static constexpr uint32_t kColS = 0, kColO = 2 * N;  // two buffers of N each
    static constexpr uint32_t kIdescQK = idesc_e4m3_f32(128, N, false, false);
    static constexpr uint32_t kIdescPV = idesc_e4m3_f32(128, N, true, true);
    static constexpr uint32_t kSwizzle = D == 128 ? 2 : 4;
};

template <int R, int D>
struct __align__(1024) Smem {
    using C = Cfg<R, D>;
    uint8_t ring[C::kSlots][C::kSlotBytes];
    uint8_t p[2][C::N / 16][kTile][16];
    uint8_t q[2][D / 16][C::N][16];
    float qf[2][R];   // scale of a row of Q, times the softmax scale
    int lim[2][R];    // tokens that a row sees; -1: no such row
    float top[2][4][R];   // the softmax warps' row maxima, by tile parity
    float red[4][R];
    float4 row[4][2][R];  // per softmax warp and tile parity: tile's maximum - 8, reference, and the factors of o and O
    int nan_at[D];    // first token of the item whose V is NaN at this channel, of those that not every row sees
    float ks[2][kMeta], lv[2][kMeta];  // K scale; log2 of the V scale
    int pos[2][kMeta];
    uint64_t full[C::kSlots], empty[C::kSlots];
    uint64_t s_full[2], p_full[2], o_full[2], q_full[2], q_empty[2], m_full[2], m_empty[2], drain;
    long long w0, w1, total;
    int first_b, ctas;
    Seq first_s;
    long long first_at;
    uint32_t tmem_base;
    Rows rows[2];          // of the items that are shared with other CTAs
    int abort_flag, last[2], last_c0[2];
};

__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// Largest of the warp's values (NaN are passed over).
__device__ __forceinline__ float warp_max(float x)
{
    const int i = __float_as_int(x);  // an order of ints that is the floats', negative ones turned round
    const int m = __reduce_max_sync(0xffffffffu, isnan(x) ? INT_MIN : i ^ ((i >> 31) & 0x7fffffff));
    return m == INT_MIN ? -INFINITY : __int_as_float(m ^ ((m >> 31) & 0x7fffffff));
}

__device__ __forceinline__ bool soft_any(bool x)
{
    uint32_t r;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.u32 p, %1, 0;\n"
        "bar.red.or.pred q, 1, 128, p;\n"
        "selp.u32 %0, 1, 0, q;\n"
        "}\n"
        : "=r"(r)
        : "r"(x ? 1u : 0u)
        : "memory");
    return r != 0;
}

// Joins the np parts of an item that begins in CTA c0, in order, and writes its rows: four warps an item, a warp takes every
// fourth row, two at a time, a lane four channels, with eight parts' loads in flight.
template <int R, int D>
__device__ __noinline__ void join(const Params& p, const Rows rows, int c0, int np, int quad, int lane)
{
    constexpr int kAhead = 8;
#pragma unroll 1
    for (int r0 = quad; r0 < R; r0 += 8) {
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {}, o[2][4] = {};
        int row[2], head[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) row[u] = rows.of(p, r0 + 4 * u, head[u]);
#pragma unroll 1
        for (int k0 = 0; k0 < np; k0 += kAhead) {
            float2 ml[2][kAhead];
            float4 v[2][kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                // part 0 is slot 1 of CTA c0, part k slot 0 of CTA c0 + k
                const float* at = p.parts + ((size_t)(c0 + k0 + k) * 2 + (k0 + k == 0)) * R * (D + 2);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    ml[u][k] = make_float2(-INFINITY, 0.f);
                    v[u][k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (k0 + k < np && row[u] >= 0) {
                        ml[u][k] = __ldcg(reinterpret_cast<const float2*>(at + R * D) + r0 + 4 * u);
                        if (lane < D / 4) v[u][k] = __ldcg(reinterpret_cast<const float4*>(at + (r0 + 4 * u) * D) + lane);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float top = m[u];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) top = fmaxf(top, ml[u][k].x);
                const float at0 = top == -INFINITY ? 0.f : top, f = fast_exp2(m[u] - at0);
                m[u] = top;
                l[u] *= f;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[u][e] *= f;
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const float fk = fast_exp2(ml[u][k].x - at0);
                    l[u] = fmaf(ml[u][k].y, fk, l[u]);
                    o[u][0] = fmaf(v[u][k].x, fk, o[u][0]);
                    o[u][1] = fmaf(v[u][k].y, fk, o[u][1]);
                    o[u][2] = fmaf(v[u][k].z, fk, o[u][2]);
                    o[u][3] = fmaf(v[u][k].w, fk, o[u][3]);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (row[u] < 0) continue;
            const size_t at = (size_t)row[u] * p.pl.heads + head[u];
            const float inv = l[u] != 0.f ? 1.f / l[u] : 0.f;
            if (lane < D / 4) {
                __nv_bfloat162 a = __floats2bfloat162_rn(o[u][0] * inv, o[u][1] * inv);
                __nv_bfloat162 b = __floats2bfloat162_rn(o[u][2] * inv, o[u][3] * inv);
                *reinterpret_cast<uint2*>(p.O + at * D + lane * 4) =
                    make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
            }
            if (lane == 0) p.lse[at] = l[u] != 0.f ? (m[u] + log2f(l[u])) * kLn2 : -INFINITY;
        }
    }
}

template <int R, int D, bool kList>
__global__ void __launch_bounds__(kThreads, Cfg<R, D>::kCtas) ssba_cache_attend_tc_kernel(const __grid_constant__ Maps maps,
                                                                                          const __grid_constant__ Params p)
{
    using C = Cfg<R, D>;
    constexpr int N = C::N;
    extern __shared__ uint8_t smem_raw[];
    Smem<R, D>& sm = *reinterpret_cast<Smem<R, D>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                    ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        sm.abort_flag = sm.last[0] = sm.last[1] = 0;
        for (int i = 0; i < C::kSlots; ++i) {
            mbar_init(smem_u32(&sm.full[i]), 1);
            mbar_init(smem_u32(&sm.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sm.s_full[i]), 1);
            mbar_init(smem_u32(&sm.p_full[i]), 4);
            mbar_init(smem_u32(&sm.o_full[i]), 1);
            mbar_init(smem_u32(&sm.q_full[i]), 1);
            mbar_init(smem_u32(&sm.q_empty[i]), 5);  // the item's last QK and the softmax warps
            mbar_init(smem_u32(&sm.m_full[i]), 1);
            mbar_init(smem_u32(&sm.m_empty[i]), 4);
        }
        mbar_init(smem_u32(&sm.drain), 1);
        fence_mbar_init();
    }
    if (warp == kIssue) {
        tmem_alloc(smem_u32(&sm.tmem_base), C::kTmemCols);
        tmem_relinquish();
    }
    if (warp == kLoad && lane == 0) {
        tma_prefetch_desc(&maps.k);
        tma_prefetch_desc(&maps.v);
    }
    if (threadIdx.x >= kSoft) {
        for (int i = threadIdx.x - kSoft; i < D; i += kSoft) sm.nan_at[i] = INT_MAX;
    }
    tc_fence_before();
    // everything above reads no input (programmatic dependent launch: it may run beside the last grid's end)
    grid_dep_wait();
    grid_dep_launch();
    make_share<kList, kThreads>(p, sm);  // ends in a barrier
    tc_fence_after();
    const uint32_t tbase = sm.tmem_base;
    volatile int* abortf = &sm.abort_flag;
    const uint32_t abort_at = smem_u32(&sm.abort_flag);
    const uint32_t full0 = smem_u32(&sm.full[0]), empty0 = smem_u32(&sm.empty[0]), ring0 = smem_u32(&sm.ring[0][0]);
    bool dead = false;
    uint32_t loads = 0;  // of the producer
    const int tiles_all = (int)(sm.w1 - sm.w0);
    Walk<kList> it(p, sm);

    if (warp == kLoad) {
        // ------------------------------------------------------------ producer
        // order of use: K_0, then K_g, V_{g-1} for every further tile, then the last V
        int vp0 = 0, vp1 = 0;  // (page, head) tiles of the last V that is still to come, -1: none
        auto copy = [&](const CUtensorMap* map, int p0, int p1) {
            const uint32_t slot = loads % C::kSlots;
            if (!mbar_wait(empty0 + 8 * slot, ((loads / C::kSlots) & 1) ^ 1, abortf, p.budget_ns)) {
                dead = true;
                return;
            }
            const uint32_t bar = full0 + 8 * slot, to = ring0 + slot * C::kSlotBytes;
            mbar_arrive_expect_tx(bar, ((p0 >= 0) + (p1 >= 0)) * (uint32_t)(kPage * D));
            if (p.withhold && blockIdx.x == 0) {
                dead = true;
                return;
            }
            if (p0 >= 0) tma_load_3d(to, map, bar, 0, 0, p0);
            if (p1 >= 0) tma_load_3d(to + kPage * D, map, bar, 0, 0, p1);
            ++loads;
        };
        int g = 0;
        for (; it.more() && !dead; it.next()) {
            const int h = it.hv / p.chunks;
            for (int c0 = 2 * it.tb; c0 < 2 * it.te && !dead; c0 += 32) {  // 32 pages at a time
                int j, page = -1;
                if (c0 + lane < 2 * it.te) page = it.page(c0 + lane, j);
                const int unit = page >= 0 ? page * p.pl.kv_heads + h : -1;
                const int n = min(16, it.te - c0 / 2);
                for (int i = 0; i < n && !dead; ++i, ++g) {
                    const int p0 = __shfl_sync(0xffffffffu, unit, 2 * i), p1 = __shfl_sync(0xffffffffu, unit, 2 * i + 1);
                    if (lane == 0) {
                        copy(&maps.k, p0, p1);
                        if (g > 0 && !dead) copy(&maps.v, vp0, vp1);
                    }
                    vp0 = p0;
                    vp1 = p1;
                    dead = __shfl_sync(0xffffffffu, (int)dead, 0) != 0;
                }
            }
        }
        if (lane == 0 && g > 0 && !dead) copy(&maps.v, vp0, vp1);
        __syncwarp();
    } else if (warp == kIssue) {
        // ------------------------------------------------------------ issuer
        uint32_t use = 0;  // ring slots used
        auto pv = [&](int g) {
            const uint32_t slot = use % C::kSlots;
            wait_phase(full0 + 8 * slot, (use / C::kSlots) & 1, abort_at, p.budget_ns);
            wait_phase(smem_u32(&sm.p_full[g & 1]), (g >> 1) & 1, abort_at, p.budget_ns);
            tc_fence_after();
            if (elect_one_sync()) {
                // 64 channels fill half of the 128 rows: the other half reads the next eight tokens' and goes unused
                const uint64_t a = sdesc(ring0 + slot * C::kSlotBytes, 8 * D, 8 * D, C::kSwizzle);
                const uint64_t b = sdesc(smem_u32(&sm.p[g & 1][0][0][0]), 128, kTile * 16, 0);
#pragma unroll
                for (int k = 0; k < kTile / 32; ++k)
                    mma_f8_ss(tbase + C::kColO + (g & 1) * N, a + (uint64_t)(k * 32 * D / 16), b + (uint64_t)(k * 32),
                              C::kIdescPV, k > 0 ? 1u : 0u);
                mma_commit(smem_u32(&sm.o_full[g & 1]));
                mma_commit(empty0 + 8 * slot);
            }
            __syncwarp();
            ++use;
        };
        int g = 0, seg = 0;
        for (; it.more(); it.next(), ++seg) {
            wait_phase(smem_u32(&sm.q_full[seg & 1]), (seg >> 1) & 1, abort_at, p.budget_ns);
            for (int i = it.tb; i < it.te; ++i, ++g) {
                const uint32_t slot = use % C::kSlots;
                wait_phase(full0 + 8 * slot, (use / C::kSlots) & 1, abort_at, p.budget_ns);
                tc_fence_after();
                if (elect_one_sync()) {
                    const uint64_t a = sdesc(ring0 + slot * C::kSlotBytes, 16, 8 * D, C::kSwizzle);
                    const uint64_t b = sdesc(smem_u32(&sm.q[seg & 1][0][0][0]), N * 16, 128, 0);
#pragma unroll
                    for (int k = 0; k < D / 32; ++k)
                        mma_f8_ss(tbase + C::kColS + (g & 1) * N, a + (uint64_t)(k * 2), b + (uint64_t)(k * 2 * N),
                                  C::kIdescQK, k > 0 ? 1u : 0u);
                    mma_commit(smem_u32(&sm.s_full[g & 1]));
                    mma_commit(empty0 + 8 * slot);
                    if (i == it.te - 1) mma_commit(smem_u32(&sm.q_empty[seg & 1]));
                }
                __syncwarp();
                ++use;
                if (g > 0) pv(g - 1);
            }
        }
        if (g > 0) pv(g - 1);
        dead = *abortf != 0;
    } else if (warp == kLoadQ) {
        // ------------------------------------------------------------ rows of Q
        constexpr int kLanes = D / 8, kRows = 32 / kLanes;  // lanes of a row (8 values each), rows at a time
        const int c = lane % kLanes;
        int seg = 0;
        for (; it.more(); it.next(), ++seg) {
            const int st = seg & 1;
            wait_phase(smem_u32(&sm.q_empty[st]), ((seg >> 1) & 1) ^ 1, abort_at, p.budget_ns);
            for (int r0 = 0; r0 < R; r0 += 4 * kRows) {
                uint4 in[4];
                int row[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int r = r0 + u * kRows + lane / kLanes;
                    int head;
                    row[u] = r < R ? it.row_of(r, head) : -1;
                    in[u] = row[u] >= 0 ? ld(reinterpret_cast<const uint4*>(p.q + ((size_t)row[u] * p.pl.heads + head) * D) + c)
                                        : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int r = r0 + u * kRows + lane / kLanes;
                    const uint32_t w[4] = {in[u].x, in[u].y, in[u].z, in[u].w};
                    float f[8], amax = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        f[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
                        const float a = fabsf(f[e]);
                        if (a < INFINITY) amax = fmaxf(amax, a);
                    }
#pragma unroll
                    for (int o = kLanes / 2; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                    const float scale = scale_for(amax), inv = scale > 0.f ? 1.f / scale : 1.f;
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        // an infinity makes its row's scores NaN, as it would a softmax's
                        const float x = fabsf(f[2 * e]) < INFINITY ? f[2 * e] * inv : NAN;
                        const float y = fabsf(f[2 * e + 1]) < INFINITY ? f[2 * e + 1] * inv : NAN;
                        hi[e] = to_e4m3x2(x, y);
                        const float2 back = from_e4m3x2(hi[e]);
                        lo[e] = to_e4m3x2((x - back.x) * 16.f, (y - back.y) * 16.f);
                    }
                    if (r < R) {
                        uint8_t* at = &sm.q[st][c / 2][r][(c & 1) * 8];
                        *reinterpret_cast<uint2*>(at) = make_uint2(hi[0] | (hi[1] << 16), hi[2] | (hi[3] << 16));
                        *reinterpret_cast<uint2*>(at + R * 16) = make_uint2(lo[0] | (lo[1] << 16), lo[2] | (lo[3] << 16));
                        if (c == 0) {
                            sm.qf[st][r] = scale * p.scale_log2;
                            sm.lim[st][r] = row[u] >= 0 ? it.limit(row[u]) : -1;
                        }
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.q_full[st]));
        }
    } else if (warp == kLoadMeta) {
        // ------------------------------------------------------------ scales and positions of pages
        int ch = 0;
        for (; it.more(); it.next()) {
            const int h = it.hv / p.chunks;
            for (int c0 = 2 * it.tb; c0 < 2 * it.te; c0 += kMeta, ++ch) {
                int j, page = -1;
                if (c0 + lane < 2 * it.te) page = it.page(c0 + lane, j);
                float ks = 0.f, vs = 0.f;
                if (page >= 0) {
                    const size_t unit = (size_t)page * p.pl.kv_heads + h;
                    ks = ld(p.pl.k_scale + unit);
                    vs = ld(p.pl.v_scale + unit);
                }
                wait_phase(smem_u32(&sm.m_empty[ch & 1]), ((ch >> 1) & 1) ^ 1, abort_at, p.budget_ns);
                sm.ks[ch & 1][lane] = ks;
                sm.lv[ch & 1][lane] = log2f(vs);
                sm.pos[ch & 1][lane] = page >= 0 ? j * kPage : kNowhere;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm.m_full[ch & 1]));
            }
        }
    } else {
        // ------------------------------------------------------------ softmax and O
        const int quad = warp & 3, tok = quad * 32 + lane;  // the thread's token of a tile, and its channel of O
        const uint32_t tq = tbase + (static_cast<uint32_t>(quad * 32) << 16);
        float l[R], o[R];
        float ref = -INFINITY;  // of row `lane`: the largest score so far
        int g = 0, seg = 0, ch = 0;
        bool pending = false;   // O of tile g - 1 is still to be added
        auto add_o = [&]() {
            const uint32_t buf = (g - 1) & 1;
            wait_phase(smem_u32(&sm.o_full[buf]), ((g - 1) >> 1) & 1, abort_at, p.budget_ns);
            tc_fence_after();
#pragma unroll
            for (int r0 = 0; r0 < R; r0 += 16) {
                uint32_t x[16], y[16];
                tmem_ld_32x32b_x16(tq + C::kColO + buf * N + r0, x);
                if (R > 8) tmem_ld_32x32b_x16(tq + C::kColO + buf * N + R + r0, y);
                tmem_wait_ld();
#pragma unroll
                for (int r = 0; r < 16 && r0 + r < R; ++r) {
                    const float4 w = sm.row[quad][buf][r0 + r];
                    const float v = fmaf(__uint_as_float(R > 8 ? y[r] : x[(8 + r) & 15]), 0.0625f, __uint_as_float(x[r]));
                    o[r0 + r] = fmaf(v, w.w, o[r0 + r] * w.z);
                }
            }
            pending = false;
        };
        // items shared with other CTAs: one that began before the share, one that goes on behind it
        long long start0 = 0, start1 = 0;
        int tiles0 = 0, tiles1 = 0;
        // (the four warps meet in barriers, so they give up together)
        for (; it.more() && !soft_any(*abortf != 0); ++seg) {
            const int st = seg & 1;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                l[r] = 0.f;
                o[r] = 0.f;
            }
            ref = -INFINITY;
            wait_phase(smem_u32(&sm.q_full[st]), (seg >> 1) & 1, abort_at, p.budget_ns);
            int lo_lim = INT_MAX, hi_lim = 0;  // over the item's rows
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int x = sm.lim[st][r];
                if (x >= 0) lo_lim = min(lo_lim, x);
                hi_lim = max(hi_lim, x);
            }
            for (int i = it.tb; i < it.te; ++i) {
                const int c = 2 * (i - it.tb) % kMeta;
                if (c == 0) wait_phase(smem_u32(&sm.m_full[ch & 1]), (ch >> 1) & 1, abort_at, p.budget_ns);
                const float ks = sm.ks[ch & 1][c + tok / kPage];
                const float lva = sm.lv[ch & 1][c], lvb = sm.lv[ch & 1][c + 1];
                const int at = sm.pos[ch & 1][c + tok / kPage] + tok % kPage;
                if (c == kMeta - 2 || i == it.te - 1) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sm.m_empty[ch & 1]));
                    ++ch;
                }
                wait_phase(smem_u32(&sm.s_full[g & 1]), (g >> 1) & 1, abort_at, p.budget_ns);
                tc_fence_after();
                float s[R];
#pragma unroll
                for (int r0 = 0; r0 < R; r0 += 16) {
                    uint32_t x[16], y[16];
                    tmem_ld_32x32b_x16(tq + C::kColS + (g & 1) * N + r0, x);
                    if (R > 8) tmem_ld_32x32b_x16(tq + C::kColS + (g & 1) * N + R + r0, y);
                    tmem_wait_ld();
#pragma unroll
                    for (int r = 0; r < 16 && r0 + r < R; ++r) {
                        const float lo = __uint_as_float(R > 8 ? y[r] : x[(8 + r) & 15]);
                        s[r0 + r] = fmaf(lo, 0.0625f, __uint_as_float(x[r])) * (ks * sm.qf[st][r0 + r]);
                    }
                }
                if (at >= lo_lim) {
#pragma unroll
                    for (int r = 0; r < R; ++r)
                        if (at >= sm.lim[st][r]) s[r] = -INFINITY;
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float m = warp_max(s[r]);
                    if (lane == 0) sm.top[g & 1][quad][r] = m;
                }
                soft_sync();
                if (lane < R) {
                    const float(&top)[4][R] = sm.top[g & 1];
                    const float ma = fmaxf(top[0][lane], top[1][lane]), mb = fmaxf(top[2][lane], top[3][lane]);
                    const float mv = fmaxf(ma + lva, mb + lvb) - kTop;
                    const float now = fmaxf(ref, fmaxf(ma, mb)), at0 = now == -INFINITY ? 0.f : now;
                    sm.row[quad][g & 1][lane] =
                        make_float4(mv == -INFINITY ? 0.f : mv, at0, fast_exp2(ref - at0), fast_exp2(mv - at0));
                    ref = now;
                }
                __syncwarp();
                const float lv = tok < kPage ? lva : lvb;
                // P = 2^(s + lv - max + 8) as two e4m3 numbers, and the sum of 2^(s - reference)
#pragma unroll
                for (int r0 = 0; r0 < R; r0 += 16) {
                    uint32_t hi[8], lo[8];
#pragma unroll
                    for (int r = 0; r < 16 && r0 + r < R; r += 2) {
                        float w[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float4 t = sm.row[quad][g & 1][r0 + r + e];
                            const float x = s[r0 + r + e];
                            l[r0 + r + e] = fmaf(l[r0 + r + e], t.z, fast_exp2(x - t.y));
                            w[e] = fast_exp2(x + lv - t.x);
                        }
                        hi[r / 2] = to_e4m3x2(w[0], w[1]);
                        const float2 back = from_e4m3x2(hi[r / 2]);
                        lo[r / 2] = to_e4m3x2((w[0] - back.x) * 16.f, (w[1] - back.y) * 16.f);
                    }
                    auto put = [&](int plane, const uint32_t* a, const uint32_t* b) {  // 16 columns
                        *reinterpret_cast<uint4*>(&sm.p[g & 1][plane][tok][0]) =
                            make_uint4(a[0] | (a[1] << 16), a[2] | (a[3] << 16), b[0] | (b[1] << 16), b[2] | (b[3] << 16));
                    };
                    if (R == 8) {
                        put(0, hi, lo);
                    } else {
                        put(r0 / 16, hi, hi + 4);
                        put(R / 16 + r0 / 16, lo, lo + 4);
                    }
                }
                if (__any_sync(0xffffffffu, at >= lo_lim)) {
                    // tokens that no row sees: their V is whatever the page holds, and 0 * NaN would reach every
                    // row; tokens that some rows see: a NaN is taken out of V and kept for those rows
                    const uint32_t use = g + 1 < tiles_all ? 2 * (g + 1) : 2 * g + 1;
                    const uint32_t slot = use % C::kSlots;
                    wait_phase(full0 + 8 * slot, (use / C::kSlots) & 1, abort_at, p.budget_ns);
                    uint4* v = reinterpret_cast<uint4*>(&sm.ring[slot][tok * D]);
                    if (at >= hi_lim) {
#pragma unroll
                        for (int e = 0; e < D / 16; ++e) v[e] = make_uint4(0, 0, 0, 0);
                    } else if (at >= lo_lim) {
                        for (int e = 0; e < D / 16; ++e) {
                            const uint4 u = v[e];
                            uint32_t w[4] = {u.x, u.y, u.z, u.w};
                            bool any = false;
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t m = w[k] & 0x7f7f7f7fu;
                                any |= ((m + 0x01010101u) & 0x80808080u) != 0;  // a byte of 0x7f
                            }
                            if (any) {
                                const int chunk = D == 128 ? e ^ (tok & 7) : e ^ ((tok >> 1) & 3);  // of the swizzle
                                for (int k = 0; k < 16; ++k) {
                                    const uint32_t byte = (w[k / 4] >> (8 * (k & 3))) & 0x7f;
                                    if (byte == 0x7f) {
                                        atomicMin(&sm.nan_at[chunk * 16 + k], at);
                                        w[k / 4] &= ~(0xffu << (8 * (k & 3)));
                                    }
                                }
                                v[e] = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        }
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before();
                if (pending) add_o();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&sm.p_full[g & 1]));
                ++g;
                pending = true;
            }
            add_o();
            tc_fence_before();
            // The sums over tokens: lanes halve what they hold with every exchange, so that row r ends in lane r * 32 / R.
            // Lane r then works out row r's factor and place. (All of this runs once an item, when the code has to
            // come from memory: as short as can be.)
            constexpr int kEach = 32 / R;
#pragma unroll
            for (int n = R / 2, d = 16; d; d >>= 1) {
                if (n) {
#pragma unroll
                    for (int r = 0; r < R / 2; ++r)
                        if (r < n) {
                            const float keep = lane & d ? l[r + n] : l[r], send = lane & d ? l[r] : l[r + n];
                            l[r] = keep + __shfl_xor_sync(0xffffffffu, send, d);
                        }
                    n /= 2;
                } else {
                    l[0] += __shfl_xor_sync(0xffffffffu, l[0], d);
                }
            }
            if (lane % kEach == 0) sm.red[quad][lane / kEach] = l[0];
            soft_sync();
            const int nan_at = tok < D ? sm.nan_at[tok] : INT_MAX;
            if (nan_at != INT_MAX) {
                sm.nan_at[tok] = INT_MAX;
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (nan_at < sm.lim[st][r]) o[r] = NAN;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sm.q_empty[st]));
            const bool whole = it.tb == 0 && it.te == it.tiles;
            // parts: slot 1 of the CTA that the item starts in, slot 0 of the others
            float* part = p.parts + ((size_t)blockIdx.x * 2 + (it.tb == 0)) * R * (D + 2);
            if (lane < R) {
                const float sum = (sm.red[0][lane] + sm.red[1][lane]) + (sm.red[2][lane] + sm.red[3][lane]);
                int head;
                const int row = it.row_of(lane, head);
                const long long at = row >= 0 ? (long long)row * p.pl.heads + head : -1;
                sm.row[quad][0][lane] =
                    make_float4(sum != 0.f ? 1.f / sum : 0.f, 0.f, __int_as_float((int)at), __int_as_float((int)(at >> 32)));
                if (quad == 0) {
                    if (!whole) reinterpret_cast<float2*>(part + R * D)[lane] = make_float2(ref, sum);
                    else if (row >= 0) p.lse[at] = sum != 0.f ? (ref + log2f(sum)) * kLn2 : -INFINITY;
                }
            }
            __syncwarp();
            if (tok < D) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float4 w = sm.row[quad][0][r];
                    const int hi = __float_as_int(w.w);
                    const size_t at = ((size_t)(uint32_t)hi << 32) | (uint32_t)__float_as_int(w.z);
                    if (!whole) part[r * D + tok] = o[r];
                    else if (hi >= 0) p.O[at * D + tok] = __float2bfloat16_rn(o[r] * w.x);
                }
            }
            __syncwarp();
            if (!whole) {
                const int which = it.tb == 0;
                if (which) {
                    start1 = it.start;
                    tiles1 = it.tiles;
                } else {
                    start0 = it.start;
                    tiles0 = it.tiles;
                }
                if (tok == 0) sm.rows[which] = it.rows();
            }
            if (it.start + it.te >= it.w1) break;  // (the walk stays at its last item)
            it.next();
        }
        // The items that are shared with other CTAs, counted off once all is written: a fence beside the loads of
        // every CTA takes 10 us and more, in which this one would issue none (16 sequences of up to 8000 tokens:
        // 43 us with a fence behind each item, 40 like this).
        if (tiles0 + tiles1 > 0 && !soft_any(*abortf != 0)) {
            if (tok < 2) {  // (everyone's stores lie before the barrier, and with it before the counting)
                const long long start = tok ? start1 : start0;
                const int tiles = tok ? tiles1 : tiles0;
                int c0 = 0, np = 0;
                if (tiles > 0) {
                    c0 = cta_of(start, sm);
                    np = cta_of(start + tiles - 1, sm) - c0 + 1;
                    unsigned seen;
                    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(seen) : "l"(p.tickets + c0) : "memory");
                    if (seen == (unsigned)(np - 1)) p.tickets[c0] = 0;
                    else np = 0;
                }
                sm.last_c0[tok] = c0;
                sm.last[tok] = np;
            }
        }
        dead = *abortf != 0;
    }
    if (__syncthreads_or(dead)) {
        // a wait ran out: nothing more is issued, but copies and products may be in flight
        if (warp == kLoad && lane == 0)
            for (uint32_t x = loads > C::kSlots ? loads - C::kSlots : 0; x < loads; ++x)
                wait_raw(full0 + 8 * (x % C::kSlots), (x / C::kSlots) & 1, p.budget_ns);
        if (warp == kIssue && elect_one_sync()) {
            mma_commit(smem_u32(&sm.drain));
            wait_raw(smem_u32(&sm.drain), 0, p.budget_ns);
        }
        if (threadIdx.x == 0) atomicExch(p.pl.status, SSBA_ERR_TIMEOUT);
    } else if (sm.last[warp / 4]) {
        join<R, D>(p, sm.rows[warp / 4], sm.last_c0[warp / 4], sm.last[warp / 4], warp & 3, lane);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kIssue) tmem_dealloc(tbase, C::kTmemCols);
}

template <int R, int D, bool kList>
int launch(const Maps& maps, const Params& p, cudaStream_t st)
{
    using C = Cfg<R, D>;
    const size_t smem = sizeof(Smem<R, D>) + 1024;
    static_assert((sizeof(Smem<R, D>) + 1024 + 1024 + 256) * C::kCtas <= 233472, "shared memory of an SM (228 KB)");
    static PerDeviceOnce once;
    once.run([smem] {
        cudaFuncSetAttribute(ssba_cache_attend_tc_kernel<R, D, kList>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    const cudaError_t e = launch_dependent(ssba_cache_attend_tc_kernel<R, D, kList>,
                                           dim3(std::min(device_sm_count() * C::kCtas, kMaxGrid)), kThreads, smem, st, maps, p);
    if (e == cudaSuccess) return SSBA_OK;
    set_error("ssba_cache_attend: %s", cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

template <int R>
int launch_rows(const Maps& maps, const Params& p, int D, cudaStream_t st)
{
    if (p.idx) return D == 64 ? launch<R, 64, true>(maps, p, st) : launch<R, 128, true>(maps, p, st);
    return D == 64 ? launch<R, 64, false>(maps, p, st) : launch<R, 128, false>(maps, p, st);
}

}  // namespace
}  // namespace cache

size_t cache_attend_tc_workspace() { return SSBA_CACHE_TICKET_BYTES + cache::kPartFloats * sizeof(float); }

int launch_cache_attend_tc(const cache::Pool& pl, const cache::Batch& bt, int head_dim, float scale, const void* q,
                           const int32_t* idx, const int32_t* cnt, int keep, void* O, float* lse, void* ws,
                           cudaStream_t st, uint64_t budget_ns, int withhold)
{
    using namespace cache;
    Maps maps;
    memset(&maps, 0, sizeof(maps));
    const long long tiles = (long long)pl.pages * pl.kv_heads;
    const CUtensorMapSwizzle swizzle = head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
    if (!encode_page_map(&maps.k, pl.K, tiles, head_dim, swizzle) || !encode_page_map(&maps.v, pl.V, tiles, head_dim, swizzle)) {
        set_error("ssba_cache_attend: cuTensorMapEncodeTiled failed");
        return SSBA_ERR_CUDA;
    }
    Params p;
    p.pl = pl;
    p.bt = bt;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.idx = idx;
    p.cnt = cnt;
    p.keep = keep;
    p.scale_log2 = scale * kLog2e;
    p.O = static_cast<__nv_bfloat16*>(O);
    p.lse = lse;
    p.tickets = static_cast<unsigned*>(ws);
    p.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + SSBA_CACHE_TICKET_BYTES);
    p.G = pl.heads / pl.kv_heads;
    p.budget_ns = budget_ns;
    p.withhold = withhold;
    // rows of an item: a group's heads, of several tokens where the sequences have them (16 rows cost the
    // softmax warps twice what 8 do: 16 sequences of up to 8000 tokens 37 us with 8 rows, 62 with 16)
    const long long each = idx ? 1 : ((long long)bt.T + bt.B - 1) / bt.B;  // rows of a sequence, on average
    const int R = (long long)p.G * each <= 8 ? 8 : 16;
    p.chunks = (p.G + R - 1) / R;
    p.gc = (p.G + p.chunks - 1) / p.chunks;
    p.gc_inv = (65536 + p.gc - 1) / p.gc;
    p.tq = 1;
    while (!idx && 2 * p.tq * p.gc <= R) p.tq *= 2;
    return R == 8 ? launch_rows<8>(maps, p, head_dim, st) : launch_rows<16>(maps, p, head_dim, st);
}

}  // namespace ssba
