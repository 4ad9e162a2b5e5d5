// layer.cuh -- what the kernels of a layer around its attention share: the norm, the products with their
// epilogues, rotary positions (norm.cu, linear_pair.cu, linear_rows.cu, linear_bwd.cu, rope.cu, layer_api.cu).
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"
#include "ptx.cuh"

namespace ssba {
namespace layer {

// ------------------------------------------------------------------ activations
// silu(z) = z sigma(z); gelu(z) = z sigma(2 sqrt(2/pi) (z + 0.044715 z^3)), which is its tanh form. sigma(t) is formed as
// 1 / (1 + 2^u), u = -log2(e) t: two units of the special function pipe, whose rate (16 a cycle and SM) bounds
// an epilogue that can hide behind short products, and three to five of the others.
constexpr float kLog2e = 1.4426950408889634f, kGelu = 1.5957691216057308f, kGelu3 = 0.044715f;

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// sigma(t(z)): 0 where the power overflows, which is z sigma to fp32's least numbers.
template <int kAct>
__device__ __forceinline__ float sigma(float z)
{
    const float u = kAct == SSBA_ACT_GELU ? z * fmaf(z * z, -kLog2e * kGelu * kGelu3, -kLog2e * kGelu) : z * -kLog2e;
    return rcp(1.f + ex2(u));
}

template <int kAct>
__device__ __forceinline__ float act_fn(float z)
{
    if (kAct == SSBA_ACT_NONE) return z;
    if (kAct == SSBA_ACT_RELU) return z < 0.f ? 0.f : z;  // a NaN stays one
    return z * sigma<kAct>(z);
}

// act'(z) and act(z). With p = sigma(t(z)): act' = p + z p (1 - p) t'(z) = p (1 + z t' (1 - p)). z is held within 10^6 in the
// second term, where 1 - p or p is 0 long before, so that no infinity meets a 0.
template <int kAct>
__device__ __forceinline__ float act_slope(float z, float& value)
{
    if (kAct == SSBA_ACT_RELU) {
        value = z < 0.f ? 0.f : z;
        return z > 0.f ? 1.f : (z == z ? 0.f : z);  // a NaN stays one
    }
    const float p = sigma<kAct>(z), c = fminf(fmaxf(z, -1e6f), 1e6f);
    value = z * p;
    const float t = kAct == SSBA_ACT_GELU ? c * fmaf(c * c, 3.f * kGelu * kGelu3, kGelu) : c;
    return p * fmaf(t, 1.f - p, 1.f);
}

// ------------------------------------------------------------------ small pieces
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}

__device__ __forceinline__ float2 unpack2(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}

__device__ __forceinline__ bool wait_raw(uint32_t bar, uint32_t parity, uint64_t budget_ns)
{
    const uint64_t t0 = ptx::globaltimer_ns();
    while (!ptx::mbar_try_wait(bar, parity))
        if (ptx::globaltimer_ns() - t0 > budget_ns) return false;
    return true;
}

// ------------------------------------------------------------------ clusters
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The address of this CTA's shared address `a` in the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t at_rank(uint32_t a, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}

__device__ __forceinline__ void arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ float4 ld_cluster4(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(a));
    return v;
}

// ------------------------------------------------------------------ products, one CTA or a pair
// The instruction descriptor: bf16 operands (K 16 a step) or e4m3 (K 32), fp32 accumulators; fields as in idesc_bf16_f32.
__host__ __device__ constexpr uint32_t idesc_of(bool f8, int M, int N, bool a_mn, bool b_mn)
{
    return (1u << 4) | (f8 ? 0u : (1u << 7) | (1u << 10)) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// D[tmem] (+)= A[smem] B[smem]^T, one instruction (32 bytes of K), by one thread.
template <bool kF8, bool kPair>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
#define SSBA_MMA(group, kind)                                                                              \
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::" group ".kind::" kind    \
                 " [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)         \
                 : "memory")
    if constexpr (kPair && kF8)
        SSBA_MMA("2", "f8f6f4");
    else if constexpr (kPair)
        SSBA_MMA("2", "f16");
    else if constexpr (kF8)
        SSBA_MMA("1", "f8f6f4");
    else
        SSBA_MMA("1", "f16");
#undef SSBA_MMA
}

// Arrives once on `bar` of both CTAs of a pair when the pair's products issued so far are done.
__device__ __forceinline__ void commit_pair(uint32_t bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"((uint16_t)3)
        : "memory");
}

__device__ __forceinline__ void tmem_alloc_pair(uint32_t dst, uint32_t ncols)
{
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_free_pair(uint32_t base, uint32_t ncols)
{
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(ncols) : "memory");
}

// A tile into this CTA's shared memory, counted on a barrier of either CTA of the pair (a cluster address).
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const void* map, uint32_t bar, int c0, int c1, int c2)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}

__device__ __forceinline__ void tma_store(const void* map, uint32_t src, int c0, int c1, int c2)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(src), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}

// A tile to L2 alone.
__device__ __forceinline__ void tma_prefetch_3d(const void* map, int c0, int c1, int c2)
{
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global [%0, {%1, %2, %3}];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0),
                 "r"(c1), "r"(c2)
                 : "memory");
}

__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// At most n of this thread's groups of stores still read shared memory / are still under way.
template <int n>
__device__ __forceinline__ void store_wait_read()
{
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(n) : "memory");
}
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// ------------------------------------------------------------------ host side
// What a product and its epilogue work on: y[t][n] = act(sum_k a b xs[t] ws[n] + bias[n]) + r[t][n], or, gated,
// act(g) u of the products with b's first and last N rows.
struct Product {
    const void* a;      // rows [M][K]
    const void* b;      // weights [N][K] ([2][N][K] gated), or [K][N] (b_mn: linear_rows.cu alone)
    void* y;            // [M][N] bf16
    void* z;            // [M][N] ([M][2 N] gated) bf16, or null
    const void* r;      // [M][N] bf16, or null
    const float* xs;    // [M], or null (both or none)
    const float* ws;    // [N] ([2 N])
    const float* bias;  // [N], or null
    int M, N, K;
    int act;
    bool f8, b_mn, gated;
    uint64_t budget_ns = kWaitBudgetNs;  // of each wait
    int withhold = 0;                    // the failure-detection test hook: CTA 0 announces its first copies and leaves them
};

// Rows as CTA pairs' 256-row tiles / weights as rows and tokens as columns, K split over a cluster.
int launch_product_pair(const Product& p, const char* who, cudaStream_t st);
int launch_product_rows(const Product& p, const char* who, cudaStream_t st);
int launch_product(const Product& p, const char* who, cudaStream_t st);
// What either is expected to take, in microseconds.
double product_pair_us(long long M, long long N, long long K, bool f8, bool gated);
double product_rows_us(long long M, long long N, long long K, bool f8, bool gated);
// dx = dz W and dW = dz^T x; either may be null. parts: gradients_workspace_bytes (only dW needs them).
size_t gradients_workspace_bytes(int T, int N, int K);
int launch_gradients(const void* dz, const void* x, const void* W, void* dx, void* dW, float* parts, int T, int N, int K,
                     const char* who, cudaStream_t st);

// dz = dy act'(z) ([T][N]; gated: dy [T][N], z and dz [T][2 N]), and with db its column sums by way of part.
int launch_act_backward(const void* dy, const void* z, void* dz, float* db, float* part, int T, int N, int act, bool gated,
                        const char* who, cudaStream_t st);
int act_backward_parts(int T, int N);  // rows of part, [parts][N]

int launch_rms_norm(const void* x, const void* r, const float* w, int T, int D, int dtype, float eps, void* h, void* y,
                    bool e4m3, float* scale, float* rstd, cudaStream_t st);
int launch_rms_norm_backward(const void* dy, const void* h, const float* w, const float* rstd, const void* dh, int T, int D,
                             int dtype, void* dx, float* dw, float* part, cudaStream_t st);
int rms_norm_backward_parts(int T, int D, int dtype);
// out[c] = sum over p of part[p][c], in one order
int launch_column_sum(const float* part, int parts, int N, float* out, const char* who, cudaStream_t st);

int launch_rope(const ssba_rope_desc& d, const void* x, const int64_t* xs, const int32_t* pos, int64_t pos_batch, void* out,
                const int64_t* os, cudaStream_t st);

// A launch on st. early: it may begin before the grid in front has ended (the kernel waits for that itself).
template <class... P, class... A>
cudaError_t launch_on(bool early, void (*k)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, A... a)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute la[2];
    if (early) {
        la[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        la[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        la[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        la[cfg.numAttrs].val.clusterDim.x = (unsigned)cluster;
        la[cfg.numAttrs].val.clusterDim.y = 1;
        la[cfg.numAttrs++].val.clusterDim.z = 1;
    }
    cfg.attrs = la;
    cudaError_t e = cudaLaunchKernelEx(&cfg, k, a...);
    const cudaError_t last = cudaGetLastError();
    return e == cudaSuccess ? last : e;
}

template <class... P, class... A>
cudaError_t launch_early(void (*k)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, A... a)
{
    return launch_on(true, k, grid, threads, smem, st, cluster, a...);
}

// A tensor of `depth` planes of rows, its boxes box_rows rows of `box_cols` elements.
enum Element { kBf16, kE4m3, kF32 };

inline bool encode_map(CUtensorMap* m, const void* base, Element type, uint64_t cols, uint64_t rows, uint64_t depth,
                       uint64_t row_bytes, uint64_t plane_bytes, uint32_t box_cols, uint32_t box_rows)
{
    EncodeTiledFn fn = tensor_map_encoder();
    if (!fn) return false;
    cuuint64_t dims[3] = {cols, rows, depth}, strides[2] = {row_bytes, depth > 1 ? plane_bytes : row_bytes};
    cuuint32_t box[3] = {box_cols, box_rows, 1}, es[3] = {1, 1, 1};
    return fn(m, type == kE4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : type == kF32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims,
              strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace layer
}  // namespace ssba
