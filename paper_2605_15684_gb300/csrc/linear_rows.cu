// linear_rows.cu -- the products of linear_pair.cu where rows are few: the weights are the tensor cores' rows.
//
// With few tokens a product is the reading of its weights, and the tiles of many tokens would leave most SMs without
// work. So the weights take the 128 rows of a tile, kNT tokens its columns, and K is split over the CTAs of a cluster:
//   D[128 weight rows][kNT] = sum over this CTA's share of K,   then   y[t][n] = act(sum of the CTAs' D ...) + r
// Gated, a tile is 64 gate rows over the 64 matching up rows. For dx = dz W the weights come along their rows ("mn").
// The partial tiles stay in shared memory (fp32, where the operands were) and each CTA of the cluster adds up and
// finishes a share of the outputs through distributed shared memory: no workspace, no atomics, one order.
// Bound by HBM (the weights once; tokens come from L2): some 200 KB of operands are under way in an SM, of two CTAs.
// 192 threads: warp 0 TMA, warp 1 tcgen05.mma M = 128, N = kNT, warps 2-5 take D out of TMEM, and all finish.
// Waits on barriers in shared memory are bounded; a timeout is written to the device status word. The allocation of tensor memory, the
// cluster's barrier and the wait for the grid in front have no limit of their own: each ends as the CTAs that it
// waits for do. No CTA holds tensor memory while it waits for another grid, and none lets the next grid in before it has its own.
#include <algorithm>
#include <cstddef>
#include <cstring>

#include "layer.cuh"

namespace ssba {
namespace layer {
namespace {

using namespace ptx;

constexpr int kThreads = 192;
constexpr uint32_t kABytes = 128 * 128;
constexpr int kPitch = 132;  // floats of a column of D: 128 and a shift of banks
constexpr int kMaxSplit = 8;

// Two CTAs an SM. (Three with shorter rings, where that let K be cut once more, took 1 to 12 % longer with tensor memory taken behind
// the wait, and half as long again where clusters of eight then needed a second round: 12 tokens, K 4096: gated N 11008 28.1 us
// against 29.3, N 7168 11.2 against 15.6; 16 tokens, 1536 x 6144 6.1 against 7.1; 32, 8-bit gated 4096 x 12288 19.4 against 20.)
template <int kNT>
struct RowsCfg {
    static constexpr uint32_t kBBytes = kNT * 128;
    static constexpr int kStages = kNT == 16 ? 6 : kNT == 32 ? 5 : kNT == 64 ? 4 : 3;
};

template <int kNT>
struct __align__(1024) RowsSmem {
    using C = RowsCfg<kNT>;
    union {
        struct {
            uint8_t a[C::kStages][kABytes];
            uint8_t b[C::kStages][C::kBBytes];
        };
        float part[kNT][kPitch];  // [token][weight row], when the products are done
    };
    uint64_t full[C::kStages], empty[C::kStages];
    uint64_t done;
    uint32_t tmem_base;
    int abort_flag;
};

struct RowsMaps {
    CUtensorMap w, x;
};

struct RowsParams {
    __nv_bfloat16 *y, *z;
    const __nv_bfloat16* r;
    const float *xs, *ws, *bias;
    int T, N;  // tokens; outputs a token (gated: of either half)
    int ksteps, split, act;
    int* status;
    uint64_t budget_ns;
    int withhold;
};

template <int kAct>
__device__ __forceinline__ float4 act4(float4 v)
{
    return make_float4(act_fn<kAct>(v.x), act_fn<kAct>(v.y), act_fn<kAct>(v.z), act_fn<kAct>(v.w));
}

__device__ __forceinline__ float4 activate4(float4 v, int act)
{
    if (act == SSBA_ACT_SILU) return act4<SSBA_ACT_SILU>(v);
    if (act == SSBA_ACT_GELU) return act4<SSBA_ACT_GELU>(v);
    if (act == SSBA_ACT_RELU) return act4<SSBA_ACT_RELU>(v);
    return v;
}

__device__ __forceinline__ void put4(__nv_bfloat16* to, float4 v)
{
    *reinterpret_cast<uint2*>(to) = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
}

// Four rows of D of a token: the cluster's partial sums in the order of its CTAs. All loads are under way before the
// first is needed (one after the other they took 2 us of a join of eight).
__device__ __forceinline__ float4 joined(uint32_t at, int split)
{
    float4 v[kMaxSplit];
#pragma unroll
    for (int c = 0; c < kMaxSplit; ++c) v[c] = c < split ? ld_cluster4(at_rank(at, c)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int c = 1; c < kMaxSplit; ++c) {
        v[0].x += v[c].x;
        v[0].y += v[c].y;
        v[0].z += v[c].z;
        v[0].w += v[c].w;
    }
    return v[0];
}

__device__ __forceinline__ float4 scaled(float4 v, const RowsParams& p, int t, const float* ws)
{
    if (!p.xs) return v;
    const float x = p.xs[t];
    const float4 w = *reinterpret_cast<const float4*>(ws);  // plain loads: the grid in front may have written these
    return make_float4(v.x * (x * w.x), v.y * (x * w.y), v.z * (x * w.z), v.w * (x * w.w));
}

template <int kNT, bool kF8, bool kWmn, bool kGated>
__global__ void __launch_bounds__(kThreads) ssba_product_rows_kernel(const __grid_constant__ RowsMaps maps, const RowsParams p)
{
    using C = RowsCfg<kNT>;
    using Smem = RowsSmem<kNT>;
    constexpr int kStages = C::kStages, kBK = kF8 ? 128 : 64;
    constexpr int kOut = kGated ? 64 : 128;  // outputs a token of a tile
    constexpr uint32_t kIdesc = idesc_of(kF8, 128, kNT, kWmn, false);
    constexpr uint32_t kTmem = kNT < 32 ? 32 : kNT;
    extern __shared__ uint8_t smem_raw[];
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank();
    const int n0 = (int)(blockIdx.x / p.split) * kOut, t0 = (int)blockIdx.y * kNT;
    const int k0 = (int)((long long)p.ksteps * rank / p.split), k1 = (int)((long long)p.ksteps * (rank + 1) / p.split);
    volatile int* abortf = &sm.abort_flag;

    if (threadIdx.x == 0) {
        sm.abort_flag = 0;
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&sm.full[s]), 1);
            mbar_init(smem_u32(&sm.empty[s]), 1);
        }
        mbar_init(smem_u32(&sm.done), 1);
        fence_mbar_init();
        tma_prefetch_desc(&maps.w);
        tma_prefetch_desc(&maps.x);
    }
    bool dead = false;
    // Its first weights to L2 while the grid in front ends: a prefetch takes nothing that may yet be written. With the next
    // grid let in once a CTA's last operands are asked for, that fills the time of its joins: one token, gated 4096 x
    // 11008 31.3 -> 29.4 us, 128 tokens, 4096 x 4096 14.5 -> 13.8. (Let in at once, its prefetches took from this grid's loads.)
    if (warp == 0 && lane == 0) {
        for (int k = k0; k < min(k1, k0 + kStages); ++k) {
            if constexpr (kWmn) {
                tma_prefetch_3d(&maps.w, n0, k * kBK, 0);
                tma_prefetch_3d(&maps.w, n0 + 64, k * kBK, 0);
            } else {
                tma_prefetch_3d(&maps.w, k * kBK, n0, 0);
                if (kGated) tma_prefetch_3d(&maps.w, k * kBK, n0, 1);
            }
        }
    }
    grid_dep_wait();

    // the g-th step's operands
    auto load = [&](int g) {
        const int s = g % kStages, k = k0 + g;
        const uint32_t bar = smem_u32(&sm.full[s]), a = smem_u32(&sm.a[s][0]);
        mbar_arrive_expect_tx(bar, kABytes + C::kBBytes);
        if (p.withhold && blockIdx.x == 0 && blockIdx.y == 0 && g == 0) return;
        if constexpr (kWmn) {
            tma_load_3d(a, &maps.w, bar, n0, k * kBK, 0);
            tma_load_3d(a + 8192, &maps.w, bar, n0 + 64, k * kBK, 0);
        } else if constexpr (kGated) {
            tma_load_3d(a, &maps.w, bar, k * kBK, n0, 0);
            tma_load_3d(a + 8192, &maps.w, bar, k * kBK, n0, 1);
        } else {
            tma_load_3d(a, &maps.w, bar, k * kBK, n0, 0);
        }
        tma_load_3d(smem_u32(&sm.b[s][0]), &maps.x, bar, k * kBK, t0, 0);
    };
    // The ring is filled while tensor memory is allocated: behind the wait, so that no grid holds any while it waits for another. (In
    // front of it, calls back to back took 0.1 to 0.9 us less: 32 tokens, 4096 x 4096 8.6 us, now 9.4.)
    if (warp == 0 && lane == 0)
        for (int g = 0; g < min(k1 - k0, kStages); ++g) load(g);
    if (warp == 1) {
        tmem_alloc(smem_u32(&sm.tmem_base), kTmem);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tbase = sm.tmem_base;

    if (warp == 0) {
        if (lane == 0) {
            int g = min(k1 - k0, kStages);
            for (; g < k1 - k0; ++g) {
                if (!mbar_wait(smem_u32(&sm.empty[g % kStages]), ((g / kStages) & 1) ^ 1, abortf, p.budget_ns)) {
                    dead = true;
                    break;
                }
                load(g);
            }
            grid_dep_launch();  // the next grid may set up, and prefetch, while this one's last operands come in
            if (dead) {
                for (int x = g > kStages ? g - kStages : 0; x < g; ++x)
                    wait_raw(smem_u32(&sm.full[x % kStages]), (x / kStages) & 1, p.budget_ns);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one_sync()) {
            const uint32_t a0 = smem_u32(&sm.a[0][0]), b0 = smem_u32(&sm.b[0][0]);
            int g = 0;
            for (int k = k0; k < k1; ++k, ++g) {
                const int s = g % kStages;
                if (!mbar_wait(smem_u32(&sm.full[s]), (g / kStages) & 1, abortf, p.budget_ns)) {
                    dead = true;
                    break;
                }
                tc_fence_after();
                const uint64_t ad = sdesc_sw128(a0 + s * kABytes, kWmn ? 8192 : 16, 1024);
                const uint64_t bd = sdesc_sw128(b0 + s * C::kBBytes, 16, 1024);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mma<kF8, false>(tbase, ad + (uint64_t)(i * (kWmn ? 128 : 2)), bd + (uint64_t)(i * 2), kIdesc, (g | i) != 0 ? 1u : 0u);
                mma_commit(smem_u32(&sm.empty[s]));
            }
            mma_commit(smem_u32(&sm.done));  // given up or not: nothing of this CTA's products is under way after it
        }
        __syncwarp();
    }
    // all: the products are done, so the operands' memory is free for D
    {
        const bool ok = wait_raw(smem_u32(&sm.done), 0, 2 * p.budget_ns);
        tc_fence_after();
        if (!__all_sync(0xffffffffu, ok)) dead = true;
    }
    if (warp >= 2) {
        const int quad = warp & 3;
        const uint32_t at = tbase + ((uint32_t)(32 * quad) << 16);
#pragma unroll
        for (int c = 0; c < kNT; c += 16) {
            uint32_t v[16];
            tmem_ld_32x32b_x16(at + c, v);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) sm.part[c + i][32 * quad + lane] = __uint_as_float(v[i]);
        }
        tc_fence_before();
    }
    __syncwarp();
    cluster_sync_all();

    // outputs of the tile in fours, those of a token in a row, dealt out over the cluster's threads
    const int tokens = min(kNT, p.T - t0);
    for (int e = rank * kThreads + (int)threadIdx.x; e < tokens * (kOut / 4); e += p.split * kThreads) {
        const int t = e / (kOut / 4), i = (e - t * (kOut / 4)) * 4, n = n0 + i;
        if (n >= p.N) continue;
        const size_t o = (size_t)(t0 + t) * p.N + n;
        const uint32_t at = smem_u32(&sm.part[t][i]);
        float4 v = joined(at, p.split);
        if constexpr (kGated) {
            float4 u = joined(at + 64 * 4, p.split);
            v = scaled(v, p, t0 + t, p.ws + n);
            u = scaled(u, p, t0 + t, p.ws + p.N + n);
            if (p.z) {
                put4(p.z + (size_t)(t0 + t) * 2 * p.N + n, v);
                put4(p.z + (size_t)(t0 + t) * 2 * p.N + p.N + n, u);
            }
            v = activate4(v, p.act);
            v = make_float4(v.x * u.x, v.y * u.y, v.z * u.z, v.w * u.w);
        } else {
            v = scaled(v, p, t0 + t, p.ws + n);
            if (p.bias) {
                const float4 w = *reinterpret_cast<const float4*>(p.bias + n);
                v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
            }
            if (p.z) put4(p.z + o, v);
            v = activate4(v, p.act);
            if (p.r) {
                const uint2 w = *reinterpret_cast<const uint2*>(p.r + o);
                const float2 a = unpack2(w.x), b = unpack2(w.y);
                v = make_float4(v.x + a.x, v.y + a.y, v.z + b.x, v.w + b.y);
            }
        }
        put4(p.y + o, v);
    }
    if (dead) atomicExch(p.status, SSBA_ERR_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();  // the others have read this CTA's part
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tbase, kTmem);
}

// CTAs that share a tile's K: as many as the SMs hold (two each), with two steps each at least.
int split_of(long long tiles, int ksteps)
{
    int split = 1;
    while (split < kMaxSplit && tiles * split * 2 <= 2ll * device_sm_count() && ksteps >= split * 4) split *= 2;
    return split;
}

template <int kNT, bool kF8, bool kWmn, bool kGated>
int launch_as(const Product& q, const char* who, cudaStream_t st)
{
    constexpr int kBK = kF8 ? 128 : 64, kOut = kGated ? 64 : 128;
    auto kernel = ssba_product_rows_kernel<kNT, kF8, kWmn, kGated>;
    const size_t smem = sizeof(RowsSmem<kNT>) + 1024;
    static PerDeviceOnce attr;
    attr.run([=] { cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
    const int e = kF8 ? 1 : 2;
    const uint64_t T = q.M, N = q.N, K = q.K;
    RowsMaps maps;
    memset(&maps, 0, sizeof(maps));
    bool ok = kWmn ? encode_map(&maps.w, q.b, kF8 ? kE4m3 : kBf16, N, K, 1, N * e, N * K * e, 64, 64)
                   : encode_map(&maps.w, q.b, kF8 ? kE4m3 : kBf16, K, N, kGated ? 2 : 1, K * e, N * K * e, kBK, kOut);
    ok = ok && encode_map(&maps.x, q.a, kF8 ? kE4m3 : kBf16, K, T, 1, K * e, T * K * e, kBK, kNT);
    if (!ok) {
        set_error("%s: cuTensorMapEncodeTiled failed", who);
        return SSBA_ERR_CUDA;
    }
    RowsParams p = {};
    p.y = static_cast<__nv_bfloat16*>(q.y);
    p.z = static_cast<__nv_bfloat16*>(q.z);
    p.r = static_cast<const __nv_bfloat16*>(q.r);
    p.xs = q.xs;
    p.ws = q.ws;
    p.bias = q.bias;
    p.T = q.M;
    p.N = q.N;
    p.ksteps = (q.K + kBK - 1) / kBK;
    p.act = q.act;
    p.budget_ns = q.budget_ns;
    p.withhold = q.withhold;
    p.status = device_status_word();
    if (!p.status) {
        set_error("%s: could not resolve the device status word", who);
        return SSBA_ERR_CUDA;
    }
    const long long tiles = (q.N + kOut - 1) / kOut, cols = (q.M + kNT - 1) / kNT;
    const int split = p.split = split_of(tiles * cols, p.ksteps);
    const cudaError_t err = launch_early(kernel, dim3((unsigned)(tiles * split), (unsigned)cols), kThreads, smem, st, split, maps, p);
    if (err == cudaSuccess) return SSBA_OK;
    set_error("%s: ssba_product_rows_kernel launch: %s", who, cudaGetErrorString(err));
    return SSBA_ERR_CUDA;
}

template <int kNT>
int launch_tokens(const Product& q, const char* who, cudaStream_t st)
{
    if (q.b_mn) return launch_as<kNT, false, true, false>(q, who, st);
    if (q.gated) return q.f8 ? launch_as<kNT, true, false, true>(q, who, st) : launch_as<kNT, false, false, true>(q, who, st);
    return q.f8 ? launch_as<kNT, true, false, false>(q, who, st) : launch_as<kNT, false, false, false>(q, who, st);
}

}  // namespace

namespace {

// Microseconds of a call of more than 64 tokens: a start and an end (the join of the parts among them), and a step of K, with
// two CTAs an SM. 64 tokens a tile cost less of either and have twice the tiles, which read the weights from L2 the
// second time: 128 tokens, 4096 x 4096 11.8 us (16 steps) against 13.8 (8); 256, 1536 x 1536 7.7 against 10.4; but 128, gated
// 4096 x 4096 19.6 (32) against 17.9 (16). Within a fifth of 7 to 32 us measured of 100 to 1024 tokens.
double rows_us(int nt, long long M, long long N, long long K, bool f8, bool gated)
{
    const long long cols = (M + nt - 1) / nt, tiles = ((N + (gated ? 63 : 127)) / (gated ? 64 : 128)) * cols, slots = 2ll * device_sm_count();
    if (cols > 65535) return 1e30;  // tiles of tokens are the grid's y
    const int ksteps = (int)((K + (f8 ? 127 : 63)) / (f8 ? 128 : 64)), split = split_of(tiles, ksteps);
    return (nt == 64 ? 6.4 : 8.4) + (nt == 64 ? 0.30 : 0.37) * ((ksteps + split - 1) / split) * ((tiles * split + slots - 1) / slots);
}

}  // namespace

double product_rows_us(long long M, long long N, long long K, bool f8, bool gated)
{
    return std::min(rows_us(64, M, N, K, f8, gated), rows_us(128, M, N, K, f8, gated));
}

int launch_product_rows(const Product& q, const char* who, cudaStream_t st)
{
    if (q.M <= 16) return launch_tokens<16>(q, who, st);
    if (q.M <= 32) return launch_tokens<32>(q, who, st);
    const bool narrow = q.M <= 64 || rows_us(64, q.M, q.N, q.K, q.f8, q.gated) <= rows_us(128, q.M, q.N, q.K, q.f8, q.gated);
    return narrow ? launch_tokens<64>(q, who, st) : launch_tokens<128>(q, who, st);
}

int launch_product(const Product& q, const char* who, cudaStream_t st)
{
    // Up to 64 tokens the weights are the rows; above, whichever is expected to end first.
    const bool rows = q.M <= 64 || product_rows_us(q.M, q.N, q.K, q.f8, q.gated) < product_pair_us(q.M, q.N, q.K, q.f8, q.gated);
    return rows ? launch_product_rows(q, who, st) : launch_product_pair(q, who, st);
}

}  // namespace layer
}  // namespace ssba
