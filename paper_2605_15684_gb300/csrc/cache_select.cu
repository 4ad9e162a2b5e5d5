// cache_select.cu -- the pages that each query of a served sequence attends to: Sec. 2.2's gate (score
// blocks by their mean key, keep the best) over a paged cache, for causal single-token queries with
// grouped heads.
//
// Row (t, kv head) sees L tokens in P = ceil(L / 64) pages. Page P - 1, which may not be full, and the
// first `first` pages are kept; of the others, all full, those with the highest
//   score_j = max over the group's heads of q_h . k_mean_j
// are, ties going to the lower label and NaN lowest, until min(keep, P) are. The scores are fp32 sums.
#include <algorithm>
#include <cmath>

#include "cache.cuh"
#include "select.cuh"

namespace ssba {
namespace cache {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// Sum of v over the CTA, to every thread.
__device__ __forceinline__ int block_sum(int v, int* buf)
{
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) t += buf[w];
    return t;
}

// One CTA per row: scores to shared memory as ordered keys, then the threshold by a radix walk of 8 bits
// at a time, then the kept labels in order.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) ssba_cache_select_kernel(const Pool pl, const Batch bt, const T* q, int keep,
                                                                     int first, int32_t* idx, int32_t* cnt)
{
    extern __shared__ uint8_t smem[];
    const int G = pl.heads / pl.kv_heads;
    float* qs = reinterpret_cast<float*>(smem);             // [G][D]
    uint32_t* keys = reinterpret_cast<uint32_t*>(qs + G * D);  // [P - 1 - first]
    __shared__ int hist[256];
    __shared__ int wbuf[kWarps];
    __shared__ int pick[2];
    const int t = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = find_seq(bt, t, lane);
    if (b < 0) return;
    const Seq s = load_seq(bt, b, pl.status);
    const size_t row = (size_t)t * pl.kv_heads + h;
    int32_t* out = idx + row * keep;
    const int L = visible(s, t, pl.status);
    const int P = (L + kPage - 1) / kPage;
    const int m = min(keep, P);
    if (tid == 0) cnt[row] = m;
    for (int i = m + tid; i < keep; i += kThreads) out[i] = -1;
    if (P <= keep) {
        for (int i = tid; i < P; i += kThreads) out[i] = i;
        return;
    }
    for (int i = tid; i < G * D; i += kThreads) qs[i] = to_float(q[((size_t)t * pl.heads + h * G) * D + i]);
    __syncthreads();
    const int n = P - 1 - first, want = keep - 1 - first;  // scored labels are first + [0, n)
    // eight lanes a page, each with every eighth chunk of four channels
    constexpr int kC = D / 32;
    const int sub = lane & 7;
    for (int i0 = warp * 4; i0 < n; i0 += kWarps * 4) {
        const int i = i0 + (lane >> 3);
        int page = -1;
        if (i < n) page = page_of(bt, pl, b, first + i);
        float4 km[kC];
#pragma unroll
        for (int c = 0; c < kC; ++c)
            km[c] = page >= 0 ? __ldg(reinterpret_cast<const float4*>(pl.k_mean + ((size_t)page * pl.kv_heads + h) * D) + c * 8 + sub)
                              : make_float4(NAN, NAN, NAN, NAN);
        float best = -INFINITY;
        bool nan = false;
        for (int g = 0; g < G; ++g) {
            float a = 0.f;
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                const float4 x = *reinterpret_cast<const float4*>(qs + g * D + (c * 8 + sub) * 4);
                a = fmaf(x.x, km[c].x, a);
                a = fmaf(x.y, km[c].y, a);
                a = fmaf(x.z, km[c].z, a);
                a = fmaf(x.w, km[c].w, a);
            }
#pragma unroll
            for (int o = 4; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
            nan |= isnan(a);
            best = fmaxf(best, a);
        }
        if (i < n && sub == 0) keys[i] = nan ? 0u : sel::order_key(best);
    }
    __syncthreads();
    // the want-th largest key: digits from the top, `above` keys lie over the prefix so far
    uint32_t prefix = 0;
    int left = want;  // still to take among the keys with the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kThreads) hist[i] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
        for (int i = tid; i < n; i += kThreads) {
            const uint32_t u = keys[i];
            if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift) & 255], 1);
        }
        __syncthreads();
        if (warp == 0) {  // lane l owns digits 255 - 8 l ... 248 - 8 l
            int c[8], sum = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += c[e] = hist[255 - 8 * lane - e];
            int inc = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= o) inc += x;
            }
            int over = inc - sum;
            if (over < left && inc >= left) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (over < left && over + c[e] >= left) {
                        pick[0] = 255 - 8 * lane - e;
                        pick[1] = left - over;
                    }
                    over += c[e];
                }
            }
        }
        __syncthreads();
        if (want > 0) {
            prefix |= static_cast<uint32_t>(pick[0]) << shift;
            left = pick[1];
        }
        __syncthreads();
    }
    // keys above the threshold, and the first `left` equal to it
    int base = 0, eq_base = 0;
    for (int i0 = 0; i0 < n && want > 0; i0 += kThreads) {
        const int i = i0 + tid;
        const uint32_t u = i < n ? keys[i] : 0u;
        const bool eq = i < n && u == prefix, gt = i < n && u > prefix;
        const unsigned em = __ballot_sync(0xffffffffu, eq);
        const unsigned below = (1u << lane) - 1u;
        __syncthreads();
        if (lane == 0) wbuf[warp] = __popc(em);
        __syncthreads();
        int before = eq_base, total = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += wbuf[w];
            total += wbuf[w];
        }
        const bool kept = gt || (eq && before + __popc(em & below) < left);
        eq_base += total;
        const unsigned km = __ballot_sync(0xffffffffu, kept);
        __syncthreads();
        if (lane == 0) wbuf[warp] = __popc(km);
        __syncthreads();
        int at = base;
        total = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) at += wbuf[w];
            total += wbuf[w];
        }
        if (kept) out[first + at + __popc(km & below)] = first + i;
        base += total;
    }
    if (tid < first) out[tid] = tid;
    if (tid == 0) out[keep - 1] = P - 1;
}

template <typename T, int D>
int select_as(const Pool& pl, const Batch& bt, const void* q, int keep, int first, int32_t* idx, int32_t* cnt,
              cudaStream_t st)
{
    const size_t smem = ((size_t)(pl.heads / pl.kv_heads) * D + bt.width) * 4;
    static PerDeviceOnce once;
    cudaError_t e = cudaSuccess;
    once.run([&] {
        e = cudaFuncSetAttribute(ssba_cache_select_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kSelectSmem);
    });
    if (e == cudaSuccess) {
        ssba_cache_select_kernel<T, D>
            <<<dim3(bt.T, pl.kv_heads), kThreads, smem, st>>>(pl, bt, static_cast<const T*>(q), keep, first, idx, cnt);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) return SSBA_OK;
    set_error("ssba_cache_select: %s", cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

}  // namespace
}  // namespace cache

int launch_cache_select(const cache::Pool& pl, const cache::Batch& bt, int head_dim, int dtype, const void* q, int keep,
                        int first, int32_t* idx, int32_t* cnt, cudaStream_t st)
{
    if (dtype == SSBA_BF16)
        return head_dim == 64 ? cache::select_as<__nv_bfloat16, 64>(pl, bt, q, keep, first, idx, cnt, st)
                              : cache::select_as<__nv_bfloat16, 128>(pl, bt, q, keep, first, idx, cnt, st);
    return head_dim == 64 ? cache::select_as<float, 64>(pl, bt, q, keep, first, idx, cnt, st)
                          : cache::select_as<float, 128>(pl, bt, q, keep, first, idx, cnt, st);
}

}  // namespace ssba
