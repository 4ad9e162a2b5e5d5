// linear_pair.cu -- products of many rows with what follows them, on pairs of CTAs.
//
//   y = act(a b^T xs ws + bias) + r          a [M][K], b [N][K], bf16 or e4m3 with row scales xs, ws
//   gated: y = act(g) u,  g = a b_0^T xs ws_0,  u = a b_1^T xs ws_1
//   backward, in one launch: dx = dz W, dW = dz^T x
//
// A tile is 256 rows x kBN columns (gated: 128 columns of g beside 128 of u) of a pair of CTAs, cta_group::2: each CTA
// holds 128 rows of a and half of b's rows, so that a k step of 128 bytes brings 32 KB into an SM for 512 tensor
// cycles of bf16 (one CTA alone would take 48 KB; shared memory moves 128 bytes a cycle and products read it too).
// Gated, the first CTA holds gate rows and the second the matching up rows, so that a row's g and u meet in one
// thread of the epilogue. Operands along K are 128-byte rows; operands along their rows ("mn": dW's both, dx's b) come as
// boxes of 64 columns x 64 k. e4m3 takes the same bytes: a step has 128 values of K in place of 64.
// Persistent, one CTA an SM:
//   warp 0   TMA of this CTA's operands, counted on the first CTA's barriers
//   warp 1   (first CTA) tcgen05.mma M = 256, N = kBN into one of two accumulators; commits reach both CTAs
//   the rest epilogue of this CTA's 128 rows, a warp a quadrant of TMEM lanes and 64 columns (16 warps at 256 columns; gated 8
//            warps with 64 columns of g and of u): a lane has a row; results go to 32 x 64 boxes in shared memory
//            (128-byte swizzle, so that neither the rows' stores nor the copy out conflict) and out by TMA, which
//            also clips ragged edges. The residual comes the same way, before the products are done.
// What bounds a tile: the products, whose operands take nearly all that shared memory moves (64 KB in and out a step
// of 512 cycles; 600 measured). An epilogue of eight warps took longer than 12 steps of it, waiting for its loads
// and for the special function units in turn.
// Sums are fp32 in TMEM; z and y are rounded once each. Tiles go through the rows in bands of eight tiles, so that the
// CTAs at work share operands in L2. Waits on barriers in shared memory are bounded; a timeout is written to the device status word. The
// allocation of tensor memory and the cluster's barriers have no limit of their own: each ends as the CTAs that it waits for do.
#include <cstddef>
#include <cstring>

#include "layer.cuh"

namespace ssba {
namespace layer {
namespace {

using namespace ptx;

constexpr uint32_t kABytes = 128 * 128, kBoxBytes = 32 * 128;
constexpr int kBand = 8;

enum { kPlain = 0, kGated = 1, kBare = 2 };  // kBare: y alone, nothing but the rounding

template <int kBN, int kEpi, bool kZ>
struct PairCfg {
    static constexpr uint32_t kBBytes = kBN / 2 * 128;
    static constexpr int kEpiWarps = kEpi == kGated ? 8 : kBN / 16;
    static constexpr int kThreads = (2 + kEpiWarps) * 32;
    static constexpr int kBoxes = kEpi == kGated && kZ ? 3 : 1;  // a warp
    static constexpr int kStages = kEpi == kGated ? (kZ ? 4 : 6) : kBN == 256 ? 5 : 6;
};

template <int kBN, int kEpi, bool kZ>
struct __align__(1024) PairSmem {
    using C = PairCfg<kBN, kEpi, kZ>;
    uint8_t a[C::kStages][kABytes];
    uint8_t b[C::kStages][C::kBBytes];
    uint8_t box[C::kEpiWarps][C::kBoxes][kBoxBytes];
    uint64_t full[C::kStages], empty[C::kStages];
    uint64_t acc_full[2], acc_empty[2];
    uint64_t drain;
    uint64_t res[C::kEpiWarps];
    uint32_t tmem_base;
    int abort_flag;
};

struct PairMaps {
    CUtensorMap a, b, y, z, r;  // kBare: a, b, y of dx; dW's below
    CUtensorMap a2, b2, y2;
};

// Tiles of a product; with split, each is cut along K into `split` (tiles counts them all).
struct Tiles {
    int m_tiles, n_tiles, tiles, ksteps, split;
};

// A launch has one set of tiles, or (kBare) two, dx's and dW's: set `first`, then the other. Pair q of P takes
// tiles q, q + P ... of the first set; those of the second are dealt out so that the pairs with a tile more of the
// first (q < over) take fewer: n_over each, the others n_rest.
struct PairParams {
    int M, N;
    int M2, N2;
    Tiles set[2];
    int first, pairs, over, n_over, n_rest;
    int first_tiles, other_tiles, rounds;  // rounds: whole ones of the first set
    int act;
    int has_r;
    const float *xs, *ws, *bias;
    int* status;
    uint64_t budget_ns;
    int withhold;
};

// The k-th tile of pair q: which set, the tile's row and column of tiles, and its steps of K. Within a set (and part of K),
// tiles go through the rows in bands of kBand.
struct Item {
    int set, m, n, part, k0, k1;
};

__device__ __forceinline__ bool item_at(const PairParams& p, int q, int k, Item& o)
{
    o.set = p.first;
    int t = q + k * p.pairs;
    if (t >= p.first_tiles) {
        const bool over = q < p.over;
        const int j = k - p.rounds - (over ? 1 : 0);
        if (j >= (over ? p.n_over : p.n_rest)) return false;
        o.set = 1 - p.first;
        t = over ? p.n_rest * (p.pairs - p.over) + j * p.over + q : j * (p.pairs - p.over) + q - p.over;
        if (t >= p.other_tiles) return false;
    }
    const int n_tiles = o.set ? p.set[1].n_tiles : p.set[0].n_tiles, m_tiles = o.set ? p.set[1].m_tiles : p.set[0].m_tiles;
    const int ksteps = o.set ? p.set[1].ksteps : p.set[0].ksteps, split = o.set ? p.set[1].split : 1;
    o.part = 0;
    if (split > 1) {
        o.part = t / (m_tiles * n_tiles);
        t -= o.part * m_tiles * n_tiles;
    }
    o.k0 = (int)((long long)ksteps * o.part / split);
    o.k1 = (int)((long long)ksteps * (o.part + 1) / split);
    const int band = t / (kBand * n_tiles), in = t - band * kBand * n_tiles;
    const int rows = min(kBand, m_tiles - band * kBand);
    o.n = in / rows;
    o.m = band * kBand + in - o.n * rows;
    return true;
}

// Values of z to act(z), with the branch on the activation outside the loop.
template <int kAct, int n>
__device__ __forceinline__ void apply(float (&v)[n])
{
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = act_fn<kAct>(v[i]);
}

template <int n>
__device__ __forceinline__ void activate(float (&v)[n], int act)
{
    if (act == SSBA_ACT_SILU)
        apply<SSBA_ACT_SILU>(v);
    else if (act == SSBA_ACT_GELU)
        apply<SSBA_ACT_GELU>(v);
    else if (act == SSBA_ACT_RELU)
        apply<SSBA_ACT_RELU>(v);
}

// Unit j (16 bytes, eight columns) of a row of a 32 x 64 box, 128-byte swizzle.
__device__ __forceinline__ uint4* unit(uint8_t* box, int row, int j)
{
    return reinterpret_cast<uint4*>(box + row * 128 + ((j ^ (row & 7)) << 4));
}

// n values (a multiple of 8) from unit j on, rounded.
template <int n>
__device__ __forceinline__ void put(uint8_t* box, int row, int j, const float (&v)[n])
{
#pragma unroll
    for (int i = 0; i < n / 8; ++i)
        *unit(box, row, j + i) = make_uint4(pack2(v[8 * i], v[8 * i + 1]), pack2(v[8 * i + 2], v[8 * i + 3]),
                                            pack2(v[8 * i + 4], v[8 * i + 5]), pack2(v[8 * i + 6], v[8 * i + 7]));
}

template <int n>
__device__ __forceinline__ void add(uint8_t* box, int row, int j, float (&v)[n])
{
#pragma unroll
    for (int i = 0; i < n / 8; ++i) {
        const uint4 w = *unit(box, row, j + i);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = unpack2(u[e]);
            v[8 * i + 2 * e] += f.x;
            v[8 * i + 2 * e + 1] += f.y;
        }
    }
}

// Columns from c on of a row of N values of fp32 (N a multiple of 8), all under way at once: a load behind a branch of its
// own would wait for each, some 250 cycles where L1 is left 28 KB. Past N they repeat the last; nothing reads those.
template <int n4>
__device__ __forceinline__ void cols(float4 (&w)[n4], const float* from, int c, int N)
{
#pragma unroll
    for (int j = 0; j < n4; ++j) w[j] = __ldg(reinterpret_cast<const float4*>(from + min(c + 4 * j, N - 4)));
}

template <int n4>
__device__ __forceinline__ void scale(float (&v)[4 * n4], float xs, const float4 (&w)[n4])
{
#pragma unroll
    for (int j = 0; j < n4; ++j) {
        v[4 * j] *= xs * w[j].x;
        v[4 * j + 1] *= xs * w[j].y;
        v[4 * j + 2] *= xs * w[j].z;
        v[4 * j + 3] *= xs * w[j].w;
    }
}

template <int n4>
__device__ __forceinline__ void plus(float (&v)[4 * n4], const float4 (&w)[n4])
{
#pragma unroll
    for (int j = 0; j < n4; ++j) {
        v[4 * j] += w[j].x;
        v[4 * j + 1] += w[j].y;
        v[4 * j + 2] += w[j].z;
        v[4 * j + 3] += w[j].w;
    }
}

__device__ __forceinline__ void tmem_get(float (&v)[32], uint32_t at)
{
    tmem_ld_32x32b_x32(at, reinterpret_cast<uint32_t*>(v));
}

__device__ __forceinline__ void tmem_get(float (&v)[16], uint32_t at)
{
    tmem_ld_32x32b_x16(at, reinterpret_cast<uint32_t(&)[16]>(v));
}

template <int kBN, bool kF8, int kEpi, bool kZ>
__global__ void __launch_bounds__(PairCfg<kBN, kEpi, kZ>::kThreads, 1)
    ssba_product_pair_kernel(const __grid_constant__ PairMaps maps, const PairParams p)
{
    using C = PairCfg<kBN, kEpi, kZ>;
    constexpr int kStages = C::kStages, kEpiWarps = C::kEpiWarps;
    constexpr int kBK = kF8 ? 128 : 64;                    // values of K a step
    constexpr int kCols = kEpi == kGated ? kBN / 2 : kBN;  // output columns of a tile
    constexpr uint32_t kStep = kABytes + C::kBBytes;
    extern __shared__ uint8_t smem_raw[];
    using Smem = PairSmem<kBN, kEpi, kZ>;
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1;
    volatile int* abortf = &sm.abort_flag;

    if (threadIdx.x == 0) {
        sm.abort_flag = 0;
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&sm.full[s]), 1);
            mbar_init(smem_u32(&sm.empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&sm.acc_full[b]), 1);
            mbar_init(smem_u32(&sm.acc_empty[b]), 2 * kEpiWarps);
        }
        mbar_init(smem_u32(&sm.drain), 1);
        for (int w = 0; w < kEpiWarps; ++w) mbar_init(smem_u32(&sm.res[w]), 1);
        fence_mbar_init();
        tma_prefetch_desc(&maps.a);
        tma_prefetch_desc(&maps.b);
        tma_prefetch_desc(&maps.y);
    }
    if (warp == 1) tmem_alloc_pair(smem_u32(&sm.tmem_base), 2 * kBN);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();  // both CTAs' barriers stand
    tc_fence_after();
    const uint32_t tbase = sm.tmem_base;
    bool dead = false;
    Item o;

    if (warp == 0) {
        // ------------------------------------------------------------ this CTA's operands
        uint32_t g = 0;
        if (lane == 0) {
            for (int it = 0; !dead && item_at(p, pair, it, o); ++it) {
                const int m0 = o.m * 256 + (int)rank * 128;
                const int n0 = kEpi == kGated ? o.n * kCols : o.n * kBN + (int)rank * (kBN / 2);
                const int plane = kEpi == kGated ? (int)rank : 0;
                const bool second = kEpi == kBare && o.set == 1;
                const CUtensorMap *ma = second ? &maps.a2 : &maps.a, *mb = second ? &maps.b2 : &maps.b;
                for (int k = o.k0; k < o.k1; ++k, ++g) {
                    const uint32_t s = g % kStages;
                    if (!mbar_wait(smem_u32(&sm.empty[s]), ((g / kStages) & 1) ^ 1, abortf, p.budget_ns)) {
                        dead = true;
                        break;
                    }
                    // the first CTA's barrier counts the copies of both
                    const uint32_t bar = at_rank(smem_u32(&sm.full[s]), 0);
                    if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sm.full[s]), 2 * kStep);
                    if (p.withhold && blockIdx.x == 0 && g == 0) continue;
                    const uint32_t a = smem_u32(&sm.a[s][0]), b = smem_u32(&sm.b[s][0]);
                    if (second) {
                        tma_load_pair(a, ma, bar, m0, k * kBK, 0);
                        tma_load_pair(a + 8192, ma, bar, m0 + 64, k * kBK, 0);
                    } else {
                        tma_load_pair(a, ma, bar, k * kBK, m0, 0);
                    }
                    if constexpr (kEpi == kBare) {
#pragma unroll
                        for (int i = 0; i < kBN / 128; ++i)
                            tma_load_pair(b + 8192 * i, mb, bar, n0 + 64 * i, k * kBK, 0);
                    } else {
                        tma_load_pair(b, mb, bar, k * kBK, n0, plane);
                    }
                }
            }
            const uint32_t last = g > kStages ? g - kStages : 0;
            // the products' arrivals on this CTA's barriers come from the first CTA: none may be under way when this one ends
            for (uint32_t x = last; !dead && x < g; ++x) dead = !mbar_wait(smem_u32(&sm.empty[x % kStages]), (x / kStages) & 1, abortf, p.budget_ns);
            if (dead && rank == 0) {
                // drain: the copies of the last stages issued may still be under way
                for (uint32_t x = last; x < g; ++x) wait_raw(smem_u32(&sm.full[x % kStages]), (x / kStages) & 1, p.budget_ns);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ products, by the first CTA
        if (rank == 0 && elect_one_sync()) {
            constexpr bool kBmn = kEpi == kBare;
            uint32_t g = 0;
            const uint32_t a0 = smem_u32(&sm.a[0][0]), b0 = smem_u32(&sm.b[0][0]);
            for (uint32_t it = 0; !dead && item_at(p, pair, (int)it, o); ++it) {
                const uint32_t acc = it & 1;
                if (!mbar_wait(smem_u32(&sm.acc_empty[acc]), ((it >> 1) & 1) ^ 1, abortf, p.budget_ns)) {
                    dead = true;
                    break;
                }
                tc_fence_after();
                const uint32_t d = tbase + acc * kBN;
                // 16 k are 2 KB of an operand along its rows, 32 bytes of one along K
                const bool amn = kEpi == kBare && o.set == 1;
                const uint32_t idesc = amn ? idesc_of(kF8, 256, kBN, true, kBmn) : idesc_of(kF8, 256, kBN, false, kBmn);
                const uint32_t a_lbo = amn ? 8192 : 16;
                const uint64_t a_step = amn ? 128 : 2;
                for (int k = o.k0; k < o.k1; ++k, ++g) {
                    const uint32_t s = g % kStages;
                    if (!mbar_wait(smem_u32(&sm.full[s]), (g / kStages) & 1, abortf, p.budget_ns)) {
                        dead = true;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t ad = sdesc_sw128(a0 + s * kABytes, a_lbo, 1024);
                    const uint64_t bd = sdesc_sw128(b0 + s * C::kBBytes, kBmn ? 8192 : 16, 1024);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mma<kF8, true>(d, ad + i * a_step, bd + (uint64_t)(i * (kBmn ? 128 : 2)), idesc, k > o.k0 || i > 0 ? 1u : 0u);
                    commit_pair(smem_u32(&sm.empty[s]));
                    if (k == o.k1 - 1) commit_pair(smem_u32(&sm.acc_full[acc]));
                }
            }
            if (dead) {
                commit_pair(smem_u32(&sm.drain));
                wait_raw(smem_u32(&sm.drain), 0, p.budget_ns);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ epilogue
        const int w = warp - 2, quad = warp & 3, part = w >> 2;  // part: which 64 columns of the tile (gated: of g and of u)
        uint8_t(*box)[kBoxBytes] = sm.box[w];
        const uint32_t empty0 = at_rank(smem_u32(&sm.acc_empty[0]), 0), empty1 = at_rank(smem_u32(&sm.acc_empty[1]), 0);
        uint32_t nres = 0;
        for (uint32_t it = 0; item_at(p, pair, (int)it, o); ++it) {
            const bool second = kEpi == kBare && o.set == 1;
            const int M = second ? p.M2 : p.M, N = second ? p.N2 : p.N;
            const CUtensorMap* my = second ? &maps.y2 : &maps.y;
            const bool parts = second && p.set[1].split > 1;
            const int row0 = o.m * 256 + (int)rank * 128 + 32 * quad, row = row0 + lane, col = o.n * kCols + part * 64;
            const uint32_t acc = it & 1;
            const bool live = row0 < M && col < N;
            const bool res = kEpi == kPlain && p.has_r && live;
            if (live) {  // the boxes are free once the last tile's have been read
                if (lane == 0) {
                    store_wait_read<0>();
                    if (res) {
                        mbar_arrive_expect_tx(smem_u32(&sm.res[w]), kBoxBytes);
                        tma_load_3d(smem_u32(box[0]), &maps.r, smem_u32(&sm.res[w]), col, row0, 0);
                    }
                }
                __syncwarp();
            }
            const float xs = kF8 && row < M ? p.xs[row] : 1.f;
            bool ok = mbar_wait(smem_u32(&sm.acc_full[acc]), (it >> 1) & 1, abortf, p.budget_ns);
            tc_fence_after();
            if (res) {  // waited for in any case: the copy must not outlive the CTA
                ok = wait_raw(smem_u32(&sm.res[w]), nres & 1, p.budget_ns) && ok;
                ++nres;
            }
            if (!__all_sync(0xffffffffu, ok)) {
                dead = true;
                break;
            }
            const uint32_t taddr = tbase + ((uint32_t)(32 * quad) << 16) + acc * kBN + part * 64;
            auto read = [&] {  // the accumulator has been read
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_cluster(acc ? empty1 : empty0);
            };
            if constexpr (kEpi == kGated) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float v[32], u[32];
                    float4 sv[8], su[8];
                    tmem_get(v, taddr + 32 * i);
                    tmem_get(u, taddr + kBN / 2 + 32 * i);
                    if (kF8) cols(sv, p.ws, col + 32 * i, N);
                    if (kF8) cols(su, p.ws + N, col + 32 * i, N);
                    tmem_wait_ld();
                    if (i == 1) read();
                    if (kF8) {
                        scale(v, xs, sv);
                        scale(u, xs, su);
                    }
                    if (kZ && live) {
                        put(box[1], lane, 4 * i, v);
                        put(box[2], lane, 4 * i, u);
                    }
                    activate(v, p.act);
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] *= u[e];
                    if (live) put(box[0], lane, 4 * i, v);
                }
            } else {
                uint32_t late[kZ ? 32 : 1];  // with z: y's bits, until z has left the box
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[16];
                    float4 sw[4], sb[4];
                    tmem_get(v, taddr + 16 * i);
                    if (kEpi == kPlain && kF8) cols(sw, p.ws, col + 16 * i, N);
                    if (kEpi == kPlain && p.bias) cols(sb, p.bias, col + 16 * i, N);
                    tmem_wait_ld();
                    if (i == 3) read();
                    if constexpr (kEpi == kPlain) {
                        if (kF8) scale(v, xs, sw);
                        if (p.bias) plus(v, sb);
                        if constexpr (kZ) {
                            float z[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) z[e] = v[e];
                            activate(v, p.act);
                            if (res) add(box[0], lane, 2 * i, v);
                            if (live) put(box[0], lane, 2 * i, z);
#pragma unroll
                            for (int e = 0; e < 8; ++e) late[8 * i + e] = pack2(v[2 * e], v[2 * e + 1]);
                        } else {
                            activate(v, p.act);
                            if (res) add(box[0], lane, 2 * i, v);
                        }
                    }
                    if (kEpi == kBare && parts) {  // a part of K: fp32, 32 columns a box
                        if (live) {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                *reinterpret_cast<float4*>(unit(box[0], lane, 4 * (i & 1) + j)) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                            if (i == 1) {
                                fence_proxy_async_smem();
                                __syncwarp();
                                if (lane == 0) {
                                    tma_store(my, smem_u32(box[0]), col, row0, o.part);
                                    store_commit();
                                    store_wait_read<0>();
                                }
                                __syncwarp();
                            }
                        }
                    } else if (!kZ && live) {
                        put(box[0], lane, 2 * i, v);
                    }
                }
                if (kZ && live) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store(&maps.z, smem_u32(box[0]), col, row0, 0);
                        store_commit();
                        store_wait_read<0>();
                    }
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j) *unit(box[0], lane, j) = make_uint4(late[4 * j], late[4 * j + 1], late[4 * j + 2], late[4 * j + 3]);
                }
            }
            if (live) {
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if (!(kEpi == kBare && parts))
                        tma_store(my, smem_u32(box[0]), col, row0, 0);
                    else if (col + 32 < N)
                        tma_store(my, smem_u32(box[0]), col + 32, row0, o.part);
                    if (kZ && kEpi == kGated) {
                        tma_store(&maps.z, smem_u32(box[1]), col, row0, 0);
                        tma_store(&maps.z, smem_u32(box[2]), col, row0, 1);
                    }
                    store_commit();
                }
            }
        }
        if (lane == 0) store_wait_all();
        __syncwarp();
    }

    if (dead) atomicExch(p.status, SSBA_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();  // neither CTA's barriers and operands are in use by the other
    tc_fence_after();
    if (warp == 1) tmem_free_pair(tbase, 2 * kBN);
}

// Pairs of CTAs of a kernel that run at once on the current device, kept for each kernel by itself (they are one type).
template <auto kernel>
int pairs_at_once(int threads, size_t smem)
{
    static int cache[kMaxDevices] = {};
    static std::mutex m;
    const int dev = current_device();
    std::lock_guard<std::mutex> lock(m);
    if (dev >= 0 && dev < kMaxDevices && cache[dev] > 0) return cache[dev];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (device_sm_count() / 2), 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeClusterDimension;
    la[0].val.clusterDim.x = 2;
    la[0].val.clusterDim.y = la[0].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return device_sm_count() / 2 > 0 ? device_sm_count() / 2 : 1;
    }
    if (dev >= 0 && dev < kMaxDevices) cache[dev] = n;
    return n;
}

// Pairs, and how the second set's tiles go to them: the last pair to end ends as early as it can. Returns its steps of K.
long long plan(PairParams& p, int most)
{
    const long long all = (long long)p.set[0].tiles + p.set[1].tiles;
    const int P = p.pairs = (int)(all < most ? all : most);
    long long best = -1;
    for (int f = 0; f < 2; ++f) {
        const Tiles &a = p.set[f], &b = p.set[1 - f];
        if (!a.tiles) continue;
        const int over = a.tiles % P, c = a.tiles / P;
        const int top = over ? (b.tiles + P - 1) / P : 0;
        for (int n = 0; n <= top; ++n) {
            const long long left = (long long)b.tiles - (long long)n * over;
            const int rest = left > 0 ? (int)((left + P - over - 1) / (P - over)) : 0;
            const long long sa = (a.ksteps + a.split - 1) / a.split, sb = b.tiles ? (b.ksteps + b.split - 1) / b.split : 0;
            const long long t0 = over ? (c + 1ll) * sa + n * sb : 0, t1 = c * sa + rest * sb;
            const long long end = t0 > t1 ? t0 : t1;
            if (best < 0 || end < best) {
                best = end;
                p.first = f;
                p.over = over;
                p.n_over = n;
                p.n_rest = rest;
            }
        }
    }
    p.first_tiles = p.set[p.first].tiles;
    p.other_tiles = p.set[1 - p.first].tiles;
    p.rounds = p.first_tiles / P;
    return best;
}

template <int kBN, bool kF8, int kEpi, bool kZ>
int launch_pairs(PairMaps& maps, PairParams& p, const char* who, cudaStream_t st)
{
    constexpr auto kernel = ssba_product_pair_kernel<kBN, kF8, kEpi, kZ>;
    constexpr int kThreads = PairCfg<kBN, kEpi, kZ>::kThreads;
    const size_t smem = sizeof(PairSmem<kBN, kEpi, kZ>) + 1024;
    static PerDeviceOnce attr;
    attr.run([=] { cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
    p.status = device_status_word();
    if (!p.status) {
        set_error("%s: could not resolve the device status word", who);
        return SSBA_ERR_CUDA;
    }
    plan(p, pairs_at_once<kernel>(kThreads, smem));
    const int P = p.pairs;
    // In stream order, neither beginning before the grid in front has ended nor letting the next one begin. Pairs that
    // were set up beside the last waves of another grid (a gated block's backward pass, many calls queued)
    // did not end; the cause is not known. A launch of its own costs about 2 us.
    const cudaError_t err = launch_on(false, kernel, dim3(2 * P), kThreads, smem, st, 2, maps, p);
    if (err == cudaSuccess) return SSBA_OK;
    set_error("%s: ssba_product_pair_kernel launch: %s", who, cudaGetErrorString(err));
    return SSBA_ERR_CUDA;
}

Tiles tiles_of(long long M, long long N, long long K, int cols, int bk)
{
    Tiles t;
    t.split = 1;
    t.m_tiles = (int)((M + 255) / 256);
    t.n_tiles = (int)((N + cols - 1) / cols);
    t.tiles = t.m_tiles * t.n_tiles;
    t.ksteps = (int)((K + bk - 1) / bk);
    return t;
}

int no_maps(const char* who)
{
    set_error("%s: cuTensorMapEncodeTiled failed", who);
    return SSBA_ERR_CUDA;
}

template <int kBN, bool kF8, int kEpi, bool kZ>
int launch_as(const Product& q, const char* who, cudaStream_t st)
{
    constexpr int kBK = kF8 ? 128 : 64, kCols = kEpi == kGated ? kBN / 2 : kBN;
    const int e = kF8 ? 1 : 2;
    PairMaps maps;
    memset(&maps, 0, sizeof(maps));
    const uint64_t M = q.M, N = q.N, K = q.K, planes = kEpi == kGated ? 2 : 1;
    bool ok = encode_map(&maps.a, q.a, kF8 ? kE4m3 : kBf16, K, M, 1, K * e, 0, kBK, 128) &&
              encode_map(&maps.b, q.b, kF8 ? kE4m3 : kBf16, K, N, planes, K * e, N * K * e, kBK, kBN / 2) &&
              encode_map(&maps.y, q.y, kBf16, N, M, 1, N * 2, 0, 64, 32);
    if (kZ) ok = ok && encode_map(&maps.z, q.z, kBf16, N, M, planes, planes * N * 2, N * 2, 64, 32);
    if (q.r) ok = ok && encode_map(&maps.r, q.r, kBf16, N, M, 1, N * 2, 0, 64, 32);
    if (!ok) return no_maps(who);
    PairParams p = {};
    p.M = q.M;
    p.N = q.N;
    p.set[0] = tiles_of(q.M, q.N, q.K, kCols, kBK);
    p.act = q.act;
    p.has_r = q.r != nullptr;
    p.xs = q.xs;
    p.ws = q.ws;
    p.bias = q.bias;
    p.budget_ns = q.budget_ns;
    p.withhold = q.withhold;
    return launch_pairs<kBN, kF8, kEpi, kZ>(maps, p, who, st);
}

}  // namespace

namespace {

long long rounds(long long M, long long N, long long cols)
{
    const long long pairs = device_sm_count() / 2 > 0 ? device_sm_count() / 2 : 1;
    return (((M + 255) / 256) * ((N + cols - 1) / cols) + pairs - 1) / pairs;
}

// 256 columns a tile, or 128 where that needs no more rounds over the SMs: a 128-column step brings three quarters of
// the bytes for half the products, and takes 0.9 of the time (dx of 5001 rows, 2048 columns, K 11264).
bool narrow(long long M, long long N) { return 9 * rounds(M, N, 128) < 10 * rounds(M, N, 256); }

}  // namespace

int launch_product_pair(const Product& q, const char* who, cudaStream_t st)
{
    if (q.gated) {
        if (q.f8) return q.z ? launch_as<256, true, kGated, true>(q, who, st) : launch_as<256, true, kGated, false>(q, who, st);
        return q.z ? launch_as<256, false, kGated, true>(q, who, st) : launch_as<256, false, kGated, false>(q, who, st);
    }
    if (q.z) return q.f8 ? launch_as<256, true, kPlain, true>(q, who, st) : launch_as<256, false, kPlain, true>(q, who, st);
    const bool half = narrow(q.M, q.N);
    if (q.f8) return half ? launch_as<128, true, kPlain, false>(q, who, st) : launch_as<256, true, kPlain, false>(q, who, st);
    return half ? launch_as<128, false, kPlain, false>(q, who, st) : launch_as<256, false, kPlain, false>(q, who, st);
}

// A start and an end of 5.6 us in all and 0.25 a step of K and round of tiles (measured 7 to 45 us within a tenth).
double product_pair_us(long long M, long long N, long long K, bool f8, bool gated)
{
    const long long ksteps = (K + (f8 ? 127 : 63)) / (f8 ? 128 : 64), wide = gated ? 128 : 256;
    return 5.6 + 0.25 * ksteps * rounds(M, N, wide);
}

namespace {

constexpr int kMaxParts = 32;

// dx and dW of a backward pass: dx with the weights as rows or in dW's launch, and the parts that dW's sum over the tokens is
// cut into (where its tiles are too few for the SMs). By the sizes alone, whether or not both are wanted, so that
// neither changes with the other.
struct GradientPlan {
    bool rows;
    int parts;
};

// Steps of 0.33 us (operands along their rows, few pairs at work); parts add a join, some 3 us and their bytes.
GradientPlan gradient_plan(int T, int N, int K)
{
    const int most = device_sm_count() / 2 > 0 ? device_sm_count() / 2 : 1;
    const Tiles of_dx = tiles_of(T, K, N, 256, 64), of_dW = tiles_of(N, K, T, 256, 64);
    const double rows_us = product_rows_us(T, K, N, false, false);
    GradientPlan best = {T <= 64, 1};
    double best_us = -1.;
    for (int parts = 1; parts <= kMaxParts; parts *= 2) {
        if (parts > 1 && (of_dW.ksteps < 8 * parts || (long long)of_dW.tiles * parts > 2 * most)) break;
        for (int rows = T <= 64 ? 1 : 0; rows < 2; ++rows) {
            PairParams p = {};
            if (!rows) p.set[0] = of_dx;
            p.set[1] = of_dW;
            p.set[1].split = parts;
            p.set[1].tiles *= parts;
            const double us = 0.33 * plan(p, most) + (rows ? rows_us : 0.) + (parts > 1 ? 3. + 2e-6 * parts * N * K : 0.);
            if (best_us < 0. || us < best_us) {
                best_us = us;
                best = {rows != 0, parts};
            }
        }
    }
    return best;
}

// dW = the parts' sum, in their order, rounded. n4: fours of a part.
__global__ void __launch_bounds__(256) ssba_join_parts_kernel(const float4* part, int parts, long long n4, uint2* dW)
{
    grid_dep_wait();
    grid_dep_launch();
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n4; i += (long long)gridDim.x * 256) {
        float4 s = part[i];
#pragma unroll 4
        for (int k = 1; k < parts; ++k) {
            const float4 v = part[k * n4 + i];
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
        dW[i] = make_uint2(pack2(s.x, s.y), pack2(s.z, s.w));
    }
}

}  // namespace

size_t gradients_workspace_bytes(int T, int N, int K)
{
    const int parts = gradient_plan(T, N, K).parts;
    return parts > 1 ? sizeof(float) * parts * (size_t)N * K : 0;
}

int launch_gradients(const void* dz, const void* x, const void* W, void* dx, void* dW, float* parts, int T, int N, int K,
                     const char* who, cudaStream_t st)
{
    const GradientPlan g = gradient_plan(T, N, K);
    if (dx && g.rows) {
        Product q{};
        q.a = dz;
        q.b = W;
        q.y = dx;
        q.M = T;
        q.N = K;
        q.K = N;
        q.b_mn = true;
        const int rc = launch_product_rows(q, who, st);
        if (rc != SSBA_OK || !dW) return rc;
        dx = nullptr;
    }
    PairMaps maps;
    memset(&maps, 0, sizeof(maps));
    PairParams p = {};
    p.budget_ns = kWaitBudgetNs;
    const uint64_t t = T, n = N, k = K;
    bool ok = true;
    if (dx) {
        ok = encode_map(&maps.a, dz, kBf16, n, t, 1, n * 2, 0, 64, 128) && encode_map(&maps.b, W, kBf16, k, n, 1, k * 2, 0, 64, 64) &&
             encode_map(&maps.y, dx, kBf16, k, t, 1, k * 2, 0, 64, 32);
        p.M = T;
        p.N = K;
        p.set[0] = tiles_of(T, K, N, 256, 64);
    }
    if (dW) {
        ok = ok && encode_map(&maps.a2, dz, kBf16, n, t, 1, n * 2, 0, 64, 64) && encode_map(&maps.b2, x, kBf16, k, t, 1, k * 2, 0, 64, 64) &&
             (g.parts > 1 ? encode_map(&maps.y2, parts, kF32, k, n, g.parts, k * 4, n * k * 4, 32, 32)
                          : encode_map(&maps.y2, dW, kBf16, k, n, 1, k * 2, 0, 64, 32));
        p.M2 = N;
        p.N2 = K;
        p.set[1] = tiles_of(N, K, T, 256, 64);
        p.set[1].split = g.parts;
        p.set[1].tiles *= g.parts;
    }
    if (!ok) return no_maps(who);
    const int rc = launch_pairs<256, false, kBare, false>(maps, p, who, st);
    if (rc != SSBA_OK || !dW || g.parts == 1) return rc;
    const long long n4 = (long long)N * K / 4, ctas = (n4 + 255) / 256, most = 16ll * device_sm_count();
    const cudaError_t e = launch_early(ssba_join_parts_kernel, dim3((unsigned)(ctas < most ? ctas : most)), 256, 0, st, 1,
                                       reinterpret_cast<const float4*>(parts), g.parts, n4, static_cast<uint2*>(dW));
    if (e == cudaSuccess) return SSBA_OK;
    set_error("%s: ssba_join_parts_kernel launch: %s", who, cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

}  // namespace layer
}  // namespace ssba
