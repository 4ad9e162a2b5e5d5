// linear_pair.cu -- products of many rows with what follows them, on pairs of CTAs.
//
//   y = act(a b^T xs ws + bias) + r          a [M][K], b [N][K], bf16 or e4m3 with row scales xs, ws
//   gated: y = act(g) u,  g = a b_0^T xs ws_0,  u = a b_1^T xs ws_1
//   backward: dx = dz W (b along its rows, "b_mn"), dW = dz^T x (both along their rows)
//
// A tile is 256 rows x kBN columns (gated: 128 columns of g beside 128 of u) of a pair of CTAs, cta_group::2: each CTA
// holds 128 rows of a and half of b's rows, so that a k step of 128 bytes brings 32 KB into an SM for 512 tensor
// cycles of bf16 (one CTA alone would take 48 KB; shared memory moves 128 bytes a cycle and products read it too).
// Gated, the first CTA holds gate rows and the second the matching up rows, so that a row's g and u meet in one
// thread of the epilogue. Operands along K are 128-byte rows; operands along their rows ("mn") come as boxes of 64
// columns x 64 k. e4m3 takes the same bytes: a step has 128 values of K in place of 64.
// Persistent, one CTA an SM, 320 threads:
//   warp 0     TMA of this CTA's operands, counted on the first CTA's barriers
//   warp 1     (first CTA) tcgen05.mma M = 256, N = kBN into one of two accumulators; commits reach both CTAs
//   warps 2-9  epilogue of this CTA's 128 rows, two warps a quadrant of TMEM lanes, 64 columns at a time: a lane has a
//              row; results go to 32 x 64 boxes in shared memory (128-byte swizzle, so that neither the
//              rows' stores nor the copy out conflict) and out by TMA, which also clips ragged edges. The residual
//              comes the same way, before the products are done.
// Sums are fp32 in TMEM; z and y are rounded once each. Tiles go through the rows in bands of eight tiles, so that the
// CTAs at work share operands in L2. Every wait is bounded; a timeout is written to the device status word.
#include <cstddef>
#include <cstring>

#include "layer.cuh"

namespace ssba {
namespace layer {
namespace {

using namespace ptx;

constexpr int kEpiWarps = 8, kThreads = (2 + kEpiWarps) * 32;
constexpr uint32_t kABytes = 128 * 128, kBoxBytes = 32 * 128;
constexpr int kBand = 8;

enum { kPlain = 0, kGated = 1, kBare = 2 };  // kBare: y alone, nothing but the rounding

template <int kBN, bool kZ>
struct PairCfg {
    static constexpr uint32_t kBBytes = kBN / 2 * 128;
    static constexpr int kBoxes = kZ ? 3 : 2;
    static constexpr int kStages = kZ ? (kBN == 256 ? 4 : 5) : (kBN == 256 ? 5 : 6);
};

template <int kBN, bool kZ>
struct __align__(1024) PairSmem {
    using C = PairCfg<kBN, kZ>;
    uint8_t a[C::kStages][kABytes];
    uint8_t b[C::kStages][C::kBBytes];
    uint8_t box[kEpiWarps][C::kBoxes][kBoxBytes];
    uint64_t full[C::kStages], empty[C::kStages];
    uint64_t acc_full[2], acc_empty[2];
    uint64_t drain;
    uint64_t res[kEpiWarps];
    uint32_t tmem_base;
    int abort_flag;
};

struct PairMaps {
    CUtensorMap a, b, y, z, r;
};

struct PairParams {
    int M, N, K;
    int m_tiles, n_tiles, tiles, ksteps;
    int act;
    int has_r;
    const float *xs, *ws, *bias;
    int* status;
    uint64_t budget_ns;
};

__device__ __forceinline__ void tile_at(const PairParams& p, int t, int& m, int& n)
{
    const int band = t / (kBand * p.n_tiles), in = t - band * kBand * p.n_tiles;
    const int rows = min(kBand, p.m_tiles - band * kBand);
    n = in / rows;
    m = band * kBand + in - n * rows;
}

// 32 values of z to act(z), with the branch on the activation outside the loop.
template <int kAct>
__device__ __forceinline__ void apply32(float (&v)[32])
{
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = act_fn<kAct>(v[i]);
}

__device__ __forceinline__ void activate(float (&v)[32], int act)
{
    if (act == SSBA_ACT_SILU)
        apply32<SSBA_ACT_SILU>(v);
    else if (act == SSBA_ACT_GELU)
        apply32<SSBA_ACT_GELU>(v);
    else if (act == SSBA_ACT_RELU)
        apply32<SSBA_ACT_RELU>(v);
}

// Half a row (32 values, 64 bytes) of a 32 x 64 box, 128-byte swizzle.
__device__ __forceinline__ void put_half(uint8_t* box, int row, int half, const float (&v)[32])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint4 w = make_uint4(pack2(v[8 * j], v[8 * j + 1]), pack2(v[8 * j + 2], v[8 * j + 3]),
                                   pack2(v[8 * j + 4], v[8 * j + 5]), pack2(v[8 * j + 6], v[8 * j + 7]));
        *reinterpret_cast<uint4*>(box + row * 128 + (((4 * half + j) ^ (row & 7)) << 4)) = w;
    }
}

__device__ __forceinline__ void add_half(const uint8_t* box, int row, int half, float (&v)[32])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint4 w = *reinterpret_cast<const uint4*>(box + row * 128 + (((4 * half + j) ^ (row & 7)) << 4));
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(u[i]);
            v[8 * j + 2 * i] += f.x;
            v[8 * j + 2 * i + 1] += f.y;
        }
    }
}

// v *= xs ws[c ..], v += bias[c ..]; N, a multiple of 8, bounds the columns.
__device__ __forceinline__ void scale_bias(float (&v)[32], float xs, const float* ws, const float* bias, int c, int N)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (c + 4 * j >= N) break;
        if (ws) {
            const float4 w = __ldg(reinterpret_cast<const float4*>(ws + c) + j);
            v[4 * j] *= xs * w.x;
            v[4 * j + 1] *= xs * w.y;
            v[4 * j + 2] *= xs * w.z;
            v[4 * j + 3] *= xs * w.w;
        }
        if (bias) {
            const float4 w = __ldg(reinterpret_cast<const float4*>(bias + c) + j);
            v[4 * j] += w.x;
            v[4 * j + 1] += w.y;
            v[4 * j + 2] += w.z;
            v[4 * j + 3] += w.w;
        }
    }
}

__device__ __forceinline__ void tmem_get(float (&v)[32], uint32_t at)
{
    tmem_ld_32x32b_x32(at, reinterpret_cast<uint32_t*>(v));
}

template <int kBN, bool kF8, bool kAmn, bool kBmn, int kEpi, bool kZ>
__global__ void __launch_bounds__(kThreads, 1) ssba_product_pair_kernel(const __grid_constant__ PairMaps maps, const PairParams p)
{
    using C = PairCfg<kBN, kZ>;
    constexpr int kStages = C::kStages;
    constexpr int kBK = kF8 ? 128 : 64;               // values of K a step
    constexpr int kCols = kEpi == kGated ? kBN / 2 : kBN;  // output columns of a tile
    constexpr uint32_t kStep = kABytes + C::kBBytes;
    constexpr uint32_t kIdesc = idesc_of(kF8, 256, kBN, kAmn, kBmn);
    extern __shared__ uint8_t smem_raw[];
    PairSmem<kBN, kZ>& sm = *reinterpret_cast<PairSmem<kBN, kZ>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                                  ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int first = blockIdx.x >> 1, step = gridDim.x >> 1;
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

    if (warp == 0) {
        // ------------------------------------------------------------ this CTA's operands
        uint32_t g = 0;
        if (lane == 0) {
            for (int t = first; t < p.tiles && !dead; t += step) {
                int m, n;
                tile_at(p, t, m, n);
                const int m0 = m * 256 + (int)rank * 128;
                const int n0 = kEpi == kGated ? n * kCols : n * kBN + (int)rank * (kBN / 2);
                const int plane = kEpi == kGated ? (int)rank : 0;
                for (int k = 0; k < p.ksteps; ++k, ++g) {
                    const uint32_t s = g % kStages;
                    if (!mbar_wait(smem_u32(&sm.empty[s]), ((g / kStages) & 1) ^ 1, abortf, p.budget_ns)) {
                        dead = true;
                        break;
                    }
                    // the first CTA's barrier counts the copies of both
                    const uint32_t bar = at_rank(smem_u32(&sm.full[s]), 0);
                    if (rank == 0) mbar_arrive_expect_tx(smem_u32(&sm.full[s]), 2 * kStep);
                    const uint32_t a = smem_u32(&sm.a[s][0]), b = smem_u32(&sm.b[s][0]);
                    if constexpr (kAmn) {
                        tma_load_pair(a, &maps.a, bar, m0, k * kBK, 0);
                        tma_load_pair(a + 8192, &maps.a, bar, m0 + 64, k * kBK, 0);
                    } else {
                        tma_load_pair(a, &maps.a, bar, k * kBK, m0, 0);
                    }
                    if constexpr (kBmn) {
#pragma unroll
                        for (int i = 0; i < kBN / 128; ++i)
                            tma_load_pair(b + 8192 * i, &maps.b, bar, n0 + 64 * i, k * kBK, 0);
                    } else {
                        tma_load_pair(b, &maps.b, bar, k * kBK, n0, plane);
                    }
                }
            }
            if (dead && rank == 0) {
                // drain: the copies of the last stages issued may still be under way
                for (uint32_t x = g > kStages ? g - kStages : 0; x < g; ++x)
                    wait_raw(smem_u32(&sm.full[x % kStages]), (x / kStages) & 1, p.budget_ns);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------ products, by the first CTA
        if (rank == 0 && elect_one_sync()) {
            uint32_t g = 0, it = 0;
            const uint32_t a0 = smem_u32(&sm.a[0][0]), b0 = smem_u32(&sm.b[0][0]);
            for (int t = first; t < p.tiles && !dead; t += step, ++it) {
                const uint32_t acc = it & 1;
                if (!mbar_wait(smem_u32(&sm.acc_empty[acc]), ((it >> 1) & 1) ^ 1, abortf, p.budget_ns)) {
                    dead = true;
                    break;
                }
                tc_fence_after();
                const uint32_t d = tbase + acc * kBN;
                for (int k = 0; k < p.ksteps; ++k, ++g) {
                    const uint32_t s = g % kStages;
                    if (!mbar_wait(smem_u32(&sm.full[s]), (g / kStages) & 1, abortf, p.budget_ns)) {
                        dead = true;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t ad = sdesc_sw128(a0 + s * kABytes, kAmn ? 8192 : 16, 1024);
                    const uint64_t bd = sdesc_sw128(b0 + s * C::kBBytes, kBmn ? 8192 : 16, 1024);
#pragma unroll
                    for (int i = 0; i < 4; ++i)  // 16 k along rows are 2 KB, along K 32 bytes
                        mma<kF8, true>(d, ad + (uint64_t)(i * (kAmn ? 128 : 2)), bd + (uint64_t)(i * (kBmn ? 128 : 2)),
                                       kIdesc, (k | i) != 0 ? 1u : 0u);
                    commit_pair(smem_u32(&sm.empty[s]));
                    if (k == p.ksteps - 1) commit_pair(smem_u32(&sm.acc_full[acc]));
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
        const int w = warp - 2, quad = warp & 3, half = w >> 2;
        constexpr int kChunks = kEpi == kGated ? 1 : kBN / 128;  // of 64 columns a warp
        uint8_t(*box)[kBoxBytes] = sm.box[w];
        const uint32_t empty0 = at_rank(smem_u32(&sm.acc_empty[0]), 0), empty1 = at_rank(smem_u32(&sm.acc_empty[1]), 0);
        uint32_t it = 0, nres = 0, nbox = 0;
        for (int t = first; t < p.tiles && !dead; t += step, ++it) {
            int m, n;
            tile_at(p, t, m, n);
            const int row0 = m * 256 + (int)rank * 128 + 32 * quad, row = row0 + lane;
            const int col0 = n * kCols + half * (kCols / 2);
            const uint32_t acc = it & 1;
            bool res = false;
            if constexpr (kEpi == kPlain) {
                res = p.has_r && row0 < p.M && col0 < p.N;
                if (res) {
                    if (lane == 0) {
                        store_wait_read<0>();
                        const int boxes = kChunks == 2 && col0 + 64 < p.N ? 2 : 1;
                        mbar_arrive_expect_tx(smem_u32(&sm.res[w]), boxes * kBoxBytes);
                        for (int c = 0; c < boxes; ++c)
                            tma_load_3d(smem_u32(box[c]), &maps.r, smem_u32(&sm.res[w]), col0 + 64 * c, row0, 0);
                    }
                    __syncwarp();
                }
            }
            const float xs = kEpi != kBare && p.xs && row < p.M ? p.xs[row] : 1.f;
            bool ok = mbar_wait(smem_u32(&sm.acc_full[acc]), (it >> 1) & 1, abortf, p.budget_ns);
            tc_fence_after();
            if constexpr (kEpi == kPlain) {
                if (res) {  // waited for in any case: the copy must not outlive the CTA
                    ok = wait_raw(smem_u32(&sm.res[w]), nres & 1, p.budget_ns) && ok;
                    ++nres;
                }
            }
            if (!__all_sync(0xffffffffu, ok)) {
                dead = true;
                break;
            }
            const uint32_t taddr = tbase + ((uint32_t)(32 * quad) << 16) + acc * kBN;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                const int col = col0 + 64 * c;
                const bool live = row0 < p.M && col < p.N;
                // the chunk's boxes: with a residual, or with z, by chunk; else in turn
                uint8_t *by, *bz, *bu;
                if (kZ) {
                    by = box[kEpi == kGated ? 0 : c];
                    bz = box[kEpi == kGated ? 1 : 2];
                    bu = box[2];
                    if (live) {
                        if (lane == 0) store_wait_read<0>();
                        __syncwarp();
                    }
                } else {
                    by = box[kEpi == kPlain && p.has_r ? c : (nbox & 1)];
                    bz = bu = nullptr;
                    if (live && !(kEpi == kPlain && p.has_r)) {
                        ++nbox;
                        if (lane == 0) store_wait_read<1>();
                        __syncwarp();
                    }
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float v[32];
                    if constexpr (kEpi == kGated) {
                        float u[32];
                        tmem_get(v, taddr + half * 64 + 32 * q);
                        tmem_get(u, taddr + kBN / 2 + half * 64 + 32 * q);
                        tmem_wait_ld();
                        if (p.ws) {
                            scale_bias(v, xs, p.ws, nullptr, col + 32 * q, p.N);
                            scale_bias(u, xs, p.ws + p.N, nullptr, col + 32 * q, p.N);
                        }
                        if (kZ && live) {
                            put_half(bz, lane, q, v);
                            put_half(bu, lane, q, u);
                        }
                        activate(v, p.act);
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] *= u[i];
                    } else {
                        tmem_get(v, taddr + half * (kBN / 2) + 64 * c + 32 * q);
                        tmem_wait_ld();
                        if constexpr (kEpi == kPlain) {
                            scale_bias(v, xs, p.ws, p.bias, col + 32 * q, p.N);
                            if (kZ && live) put_half(bz, lane, q, v);
                            activate(v, p.act);
                            if (res && live) add_half(by, lane, q, v);
                        }
                    }
                    if (c == kChunks - 1 && q == 1) {  // the accumulator has been read
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) arrive_cluster(acc ? empty1 : empty0);
                    }
                    if (live) put_half(by, lane, q, v);
                }
                if (live) {
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        tma_store(&maps.y, smem_u32(by), col, row0, 0);
                        if (kZ) {
                            tma_store(&maps.z, smem_u32(bz), col, row0, 0);
                            if (kEpi == kGated) tma_store(&maps.z, smem_u32(bu), col, row0, 1);
                        }
                        store_commit();
                    }
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

// Pairs of CTAs that run at once on the current device.
template <class Kernel>
int pairs_at_once(Kernel k, size_t smem)
{
    static int cache[kMaxDevices] = {};
    static std::mutex m;
    const int dev = current_device();
    std::lock_guard<std::mutex> lock(m);
    if (dev >= 0 && dev < kMaxDevices && cache[dev] > 0) return cache[dev];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (device_sm_count() / 2), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute la[1];
    la[0].id = cudaLaunchAttributeClusterDimension;
    la[0].val.clusterDim.x = 2;
    la[0].val.clusterDim.y = la[0].val.clusterDim.z = 1;
    cfg.attrs = la;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, k, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return device_sm_count() / 2 > 0 ? device_sm_count() / 2 : 1;
    }
    if (dev >= 0 && dev < kMaxDevices) cache[dev] = n;
    return n;
}

template <int kBN, bool kF8, bool kAmn, bool kBmn, int kEpi, bool kZ>
int launch_as(const Product& q, const char* who, cudaStream_t st)
{
    constexpr int kBK = kF8 ? 128 : 64, kCols = kEpi == kGated ? kBN / 2 : kBN;
    auto kernel = ssba_product_pair_kernel<kBN, kF8, kAmn, kBmn, kEpi, kZ>;
    const size_t smem = sizeof(PairSmem<kBN, kZ>) + 1024;
    static PerDeviceOnce attr;
    attr.run([=] { cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
    const int e = kF8 ? 1 : 2;
    PairMaps maps;
    memset(&maps, 0, sizeof(maps));
    const uint64_t M = q.M, N = q.N, K = q.K, planes = kEpi == kGated ? 2 : 1;
    bool ok = kAmn ? encode_map(&maps.a, q.a, kF8, M, K, 1, M * e, M * K * e, 64, 64)
                   : encode_map(&maps.a, q.a, kF8, K, M, 1, K * e, M * K * e, kBK, 128);
    ok = ok && (kBmn ? encode_map(&maps.b, q.b, kF8, N, K, 1, N * e, N * K * e, 64, 64)
                     : encode_map(&maps.b, q.b, kF8, K, N, planes, K * e, N * K * e, kBK, kBN / 2));
    ok = ok && encode_map(&maps.y, q.y, false, N, M, 1, N * 2, M * N * 2, 64, 32);
    if (kZ) ok = ok && encode_map(&maps.z, q.z, false, N, M, planes, planes * N * 2, N * 2, 64, 32);
    if (q.r) ok = ok && encode_map(&maps.r, q.r, false, N, M, 1, N * 2, M * N * 2, 64, 32);
    if (!ok) {
        set_error("%s: cuTensorMapEncodeTiled failed", who);
        return SSBA_ERR_CUDA;
    }
    PairParams p = {};
    p.M = q.M;
    p.N = q.N;
    p.K = q.K;
    p.m_tiles = (q.M + 255) / 256;
    p.n_tiles = (q.N + kCols - 1) / kCols;
    p.tiles = p.m_tiles * p.n_tiles;
    p.ksteps = (q.K + kBK - 1) / kBK;
    p.act = q.act;
    p.has_r = q.r != nullptr;
    p.xs = q.xs;
    p.ws = q.ws;
    p.bias = q.bias;
    p.budget_ns = kWaitBudgetNs;
    p.status = device_status_word();
    if (!p.status) {
        set_error("%s: could not resolve the device status word", who);
        return SSBA_ERR_CUDA;
    }
    const int most = pairs_at_once(kernel, smem);
    const int pairs = p.tiles < most ? p.tiles : most;
    // In stream order, neither beginning before the grid in front has ended nor letting the next one begin. Pairs that
    // were set up beside the last waves of another grid (a gated block's backward pass, many calls queued)
    // did not end; a launch of its own costs about 2 us.
    const cudaError_t err = launch_on(false, kernel, dim3(2 * pairs), kThreads, smem, st, 2, maps, p);
    if (err == cudaSuccess) return SSBA_OK;
    set_error("%s: ssba_product_pair_kernel launch: %s", who, cudaGetErrorString(err));
    return SSBA_ERR_CUDA;
}

}  // namespace

int launch_product_pair(const Product& q, const char* who, cudaStream_t st)
{
    if (q.gated) {
        if (q.f8) return q.z ? launch_as<256, true, false, false, kGated, true>(q, who, st) : launch_as<256, true, false, false, kGated, false>(q, who, st);
        return q.z ? launch_as<256, false, false, false, kGated, true>(q, who, st) : launch_as<256, false, false, false, kGated, false>(q, who, st);
    }
    // 256 columns a tile, or 128 where their rounds over the SMs are shorter in all (a 128-column step takes the
    // same bytes of a for half the products)
    const long long pairs = device_sm_count() / 2 > 0 ? device_sm_count() / 2 : 1, mt = (q.M + 255) / 256;
    const long long wide = (mt * ((q.N + 255) / 256) + pairs - 1) / pairs, narrow = (mt * ((q.N + 127) / 128) + pairs - 1) / pairs;
    const bool half = 11 * narrow < 20 * wide;
    if (q.a_mn) return half ? launch_as<128, false, true, true, kBare, false>(q, who, st) : launch_as<256, false, true, true, kBare, false>(q, who, st);
    if (q.b_mn) return half ? launch_as<128, false, false, true, kBare, false>(q, who, st) : launch_as<256, false, false, true, kBare, false>(q, who, st);
    if (q.f8) {
        if (q.z) return launch_as<256, true, false, false, kPlain, true>(q, who, st);
        return half ? launch_as<128, true, false, false, kPlain, false>(q, who, st) : launch_as<256, true, false, false, kPlain, false>(q, who, st);
    }
    if (q.z) return launch_as<256, false, false, false, kPlain, true>(q, who, st);
    return half ? launch_as<128, false, false, false, kPlain, false>(q, who, st) : launch_as<256, false, false, false, kPlain, false>(q, who, st);
}

}  // namespace layer
}  // namespace ssba
