// cache_select.cu -- the pages that each query of a served sequence attends to: Sec. 2.2's gate (score
// blocks by their mean key, keep the best) over a paged cache, for causal single-token queries with
// grouped heads.
//
// Row (t, kv head) sees L tokens in P = ceil(L / 64) pages. Page P - 1, which may not be full, and the
// first `first` pages are kept; of the others, all full, those with the highest
//   score_j = max over the group's heads of q_h . k_mean_j
// are, ties going to the lower label and NaN lowest, until min(keep, P) are. The scores are fp32 sums.
//
// Bound by the means, which are read once, where sequences are long: 32 rows of up to 65000 tokens, 8 heads of 128
// (84 MB): 24.6 us, 12.4 at the copy rate. What is left over: 2 us of dependent loads before the first mean, rows of unequal
// length (the median CTA has scored after 12 us, the last one after 18), and 3.5 us of histogram, ranks and lists in a row's
// first CTA. (One CTA of 1024 threads a row 51 us, clusters 28, 128-thread CTAs of one wave 25.) One row each of
// four sequences of up to 8000 tokens: 5.3 us, latencies.
#include <algorithm>
#include <cmath>

#include "cache.cuh"
#include "ptx.cuh"
#include "select.cuh"

namespace ssba {
namespace cache {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ uint32_t score_key(float s) { return isnan(s) ? 0u : sel::order_key(s); }

// Exclusive prefix of v over the CTA's threads; the CTA's sum to `total`.
__device__ __forceinline__ int block_prefix(int v, int* buf, int& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += x;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = inc;
    __syncthreads();
    int before = inc - v;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += buf[w];
        total += buf[w];
    }
    return before;
}

constexpr int kBins = 1024, kCand = kThreads, kSlice = 512;

struct Scratch {
    int hist[kBins];
    int pages[kSlice];
    uint32_t cand_key[kCand];
    int cand_at[kCand];
    int buf[kWarps];
    float lo[kWarps], hi[kWarps];
    int pick[2], ncand;
};

// Kept labels where scores are not all finite, or many tie at the cut: a radix walk of 8 bits at a time for
// the want-th largest key, then the keys above it and the first of those equal to it, in order.
__device__ void select_radix(const float* score, int n, int want, int first, int32_t* out, Scratch& sc)
{
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    int left = want;  // still to take among the keys with the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kThreads) sc.hist[i] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
        for (int i = tid; i < n; i += kThreads) {
            const uint32_t u = score_key(score[i]);
            if ((u & mask) == prefix) atomicAdd(&sc.hist[(u >> shift) & 255], 1);
        }
        __syncthreads();
        int total;
        const int c1 = sc.hist[255 - 2 * tid], c0 = sc.hist[254 - 2 * tid];
        int over = block_prefix(c1 + c0, sc.buf, total);  // keys of higher digits
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int c = e ? c0 : c1;
            if (over < left && over + c >= left) {
                sc.pick[0] = 255 - 2 * tid - e;
                sc.pick[1] = left - over;
            }
            over += c;
        }
        __syncthreads();
        prefix |= static_cast<uint32_t>(sc.pick[0]) << shift;
        left = sc.pick[1];
        __syncthreads();
    }
    int base = 0, eq_base = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + tid;
        const uint32_t u = i < n ? score_key(score[i]) : 0u;
        const bool eq = i < n && u == prefix, gt = i < n && u > prefix;
        int total;
        const int eq_before = eq_base + block_prefix(eq, sc.buf, total);
        const bool kept = gt || (eq && eq_before < left);
        eq_base += total;
        const int at = base + block_prefix(kept, sc.buf, total);
        if (kept) out[at] = first + i;
        base += total;
    }
}

// The want largest of n finite scores, ties to the lower label, as labels first + i in order; 0 < want < n. `kept` holds
// a bit a label. Scores fall into equal steps between the lowest and the highest; those above the step
// that holds the want-th are kept, and those in it are ranked by counting.
__device__ void select_top(const float* score, uint32_t* kept, int n, int want, int first, int32_t* out, Scratch& sc)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    float lo = INFINITY, hi = -INFINITY;
    bool odd = false;
    for (int i = tid; i < n; i += kThreads) {
        const float s = score[i];
        odd |= !(fabsf(s) < INFINITY);
        lo = fminf(lo, s);
        hi = fmaxf(hi, s);
    }
    for (int i = tid; i < kBins; i += kThreads) sc.hist[i] = 0;
    if (tid == 0) sc.ncand = 0;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    if (lane == 0) {
        sc.lo[warp] = lo;
        sc.hi[warp] = hi;
    }
    odd = __syncthreads_or(odd);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        lo = fminf(lo, sc.lo[w]);
        hi = fmaxf(hi, sc.hi[w]);
    }
    const float per = (kBins - 1) / (hi - lo);
    if (odd || !(per > 0.f && per < INFINITY)) {
        select_radix(score, n, want, first, out, sc);
        return;
    }
    // (s - lo) * per does not decrease with s, rounded or not, so steps are in the scores' order
    auto step = [&](float s) { return min((int)((s - lo) * per), kBins - 1); };
    for (int i = tid; i < n; i += kThreads) atomicAdd(&sc.hist[step(score[i])], 1);
    __syncthreads();
    int c[kBins / kThreads], sum = 0, total;
#pragma unroll
    for (int e = 0; e < kBins / kThreads; ++e) sum += c[e] = sc.hist[kBins - 1 - (tid * (kBins / kThreads) + e)];
    int over = block_prefix(sum, sc.buf, total);
    if (over < want && over + sum >= want) {
#pragma unroll
        for (int e = 0; e < kBins / kThreads; ++e) {
            if (over < want && over + c[e] >= want) {
                sc.pick[0] = kBins - 1 - (tid * (kBins / kThreads) + e);
                sc.pick[1] = want - over;
            }
            over += c[e];
        }
    }
    __syncthreads();
    const int cut = sc.pick[0], left = sc.pick[1], nc = sc.hist[cut];
    if (nc > kCand) {
        __syncthreads();  // everyone has read its step's count: the walk clears the histogram for its own
        select_radix(score, n, want, first, out, sc);
        return;
    }
    for (int i0 = warp * 32; i0 < n; i0 += kThreads) {
        const int i = i0 + lane, b = i < n ? step(score[i]) : -1;
        const unsigned m = __ballot_sync(0xffffffffu, b > cut || (b == cut && nc == left));
        if (lane == 0) kept[i0 / 32] = m;
        if (b == cut && nc != left) {
            const int k = atomicAdd(&sc.ncand, 1);
            sc.cand_key[k] = sel::order_key(score[i]);
            sc.cand_at[k] = i;
        }
    }
    __syncthreads();
    if (nc != left && tid < nc) {
        const uint32_t u = sc.cand_key[tid];
        const int at = sc.cand_at[tid];
        int rank = 0;
        for (int k = 0; k < nc; ++k) {
            const uint32_t x = sc.cand_key[k];
            rank += x > u || (x == u && sc.cand_at[k] < at);
        }
        if (rank < left) atomicOr(&kept[at / 32], 1u << (at % 32));
    }
    __syncthreads();
    int base = 0;
    for (int w0 = 0; w0 < (n + 31) / 32; w0 += kThreads) {
        uint32_t m = w0 + tid < (n + 31) / 32 ? kept[w0 + tid] : 0u;
        int at = base + block_prefix(__popc(m), sc.buf, total);
        for (; m; m &= m - 1) out[at++] = first + (w0 + tid) * 32 + __ffs(m) - 1;
        base += total;
    }
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}

// A cluster of 1 to 8 CTAs per row: each scores its share of the pages, into the first CTA's shared memory; that
// one then selects. kU: pages that eight lanes have in flight.
template <typename T, int D, int kU>
__global__ void __launch_bounds__(kThreads) ssba_cache_select_kernel(const Pool pl, const Batch bt, const T* q, int keep,
                                                                     int first, int32_t* idx, int32_t* cnt)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ Scratch sc;
    const int G = pl.heads / pl.kv_heads;
    float* qs = reinterpret_cast<float*>(smem);       // [G][D]
    float* score = qs + G * D;                        // [width], of the scored labels
    uint32_t* kept = reinterpret_cast<uint32_t*>(score + bt.width);
    const int ranks = cluster_size(), rank = cluster_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int t = blockIdx.x / ranks, h = blockIdx.y;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    Seq s;
    const int b = seq_of(bt, pl, t, lane, s);
    if (b < 0) return;  // (the whole cluster)
    const size_t row = (size_t)t * pl.kv_heads + h;
    int32_t* out = idx + row * keep;
    const int L = visible(s, t, pl.status);
    const int P = (L + kPage - 1) / kPage;
    if (P <= keep) {
        if (rank == 0) {
            if (tid == 0) cnt[row] = P;
            for (int i = tid; i < keep; i += kThreads) out[i] = i < P ? i : -1;
        }
        return;
    }
    const int n = P - 1 - first, want = keep - 1 - first;  // scored labels are first + [0, n)
    const int share = (n + ranks - 1) / ranks, i_end = min(n, (rank + 1) * share);
    for (int i = tid; i < G * D; i += kThreads) qs[i] = to_float(q[((size_t)t * pl.heads + h * G) * D + i]);
    // (the first CTA has to run before its memory is written: waited for below)
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    uint32_t score_at;  // of the first CTA's scores
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(score_at) : "r"(ptx::smem_u32(score)));
    // eight lanes a page, each with every eighth chunk of four channels; 4 kU pages of a warp in flight
    constexpr int kC = D / 32;
    const int sub = lane & 7;
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    for (int s0 = rank * share; s0 < i_end; s0 += kSlice) {
        const int ns = min(kSlice, i_end - s0);
        __syncthreads();
        for (int i = tid; i < ns; i += kThreads) sc.pages[i] = page_of(bt, pl, b, first + s0 + i);
        __syncthreads();
        for (int i0 = warp * 4 * kU; i0 < ns; i0 += kWarps * 4 * kU) {
            float4 km[kU][kC];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int i = i0 + 4 * u + (lane >> 3), page = i < ns ? sc.pages[i] : -1;
                const float4* at = reinterpret_cast<const float4*>(pl.k_mean + ((size_t)max(page, 0) * pl.kv_heads + h) * D) + sub;
#pragma unroll
                for (int c = 0; c < kC; ++c) km[u][c] = page >= 0 ? ld(at + c * 8) : make_float4(NAN, NAN, NAN, NAN);
            }
            float best[kU];
            bool nan[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                best[u] = -INFINITY;
                nan[u] = false;
            }
#pragma unroll 2
            for (int g = 0; g < G; ++g) {
                float a[kU] = {};
#pragma unroll
                for (int c = 0; c < kC; ++c) {
                    const float4 x = *reinterpret_cast<const float4*>(qs + g * D + (c * 8 + sub) * 4);
#pragma unroll
                    for (int u = 0; u < kU; ++u) {
                        a[u] = fmaf(x.x, km[u][c].x, a[u]);
                        a[u] = fmaf(x.y, km[u][c].y, a[u]);
                        a[u] = fmaf(x.z, km[u][c].z, a[u]);
                        a[u] = fmaf(x.w, km[u][c].w, a[u]);
                    }
                }
#pragma unroll
                for (int u = 0; u < kU; ++u) {
#pragma unroll
                    for (int o = 4; o; o >>= 1) a[u] += __shfl_xor_sync(0xffffffffu, a[u], o);
                    nan[u] |= isnan(a[u]);
                    best[u] = fmaxf(best[u], a[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int i = i0 + 4 * u + (lane >> 3);
                if (sub == 0 && i < ns)
                    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(score_at + 4 * (s0 + i)), "f"(nan[u] ? NAN : best[u])
                                 : "memory");
            }
        }
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank != 0) return;
    if (want > 0) select_top(score, kept, n, want, first, out + first, sc);
    for (int i = tid; i < first; i += kThreads) out[i] = i;
    if (tid == 0) {
        out[keep - 1] = P - 1;
        cnt[row] = keep;
    }
}

template <typename T, int D, int kU>
cudaError_t select_with(const Pool& pl, const Batch& bt, const void* q, int keep, int first, int32_t* idx, int32_t* cnt,
                        int ranks, cudaStream_t st)
{
    const size_t smem = ((size_t)(pl.heads / pl.kv_heads) * D + bt.width + (bt.width + 31) / 32) * 4;
    static PerDeviceOnce once;
    once.run([&] {
        cudaFuncSetAttribute(ssba_cache_select_kernel<T, D, kU>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSelectSmem);
    });
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(bt.T * ranks, pl.kv_heads, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, ssba_cache_select_kernel<T, D, kU>, pl, bt, static_cast<const T*>(q), keep,
                                             first, idx, cnt);
    return e == cudaSuccess ? cudaGetLastError() : e;
}

template <typename T, int D>
int select_as(const Pool& pl, const Batch& bt, const void* q, int keep, int first, int32_t* idx, int32_t* cnt,
              cudaStream_t st)
{
    // CTAs a row: as many as run at once (eight an SM), and no share of fewer than 32 pages
    const long long rows = (long long)bt.T * pl.kv_heads;
    int ranks = 1;
    while (ranks < 8 && 2 * rows * ranks <= 8LL * device_sm_count() && bt.width > 64 * ranks) ranks *= 2;
    // Twice the pages in flight takes registers for four or five CTAs an SM: where no more are to run. (8 heads of 128, up
    // to 8000 tokens: 4 rows 6.3 us with two, 5.3 with four, 16 rows 6.6, 5.7; up to 65000: 8 rows 10.5, 9.1, 12 rows
    // 14.3, 14.2, 16 rows, where more run, 16.2, 18.0, 32 rows 24.6, 25.9.)
    const cudaError_t e = rows * ranks <= 5LL * device_sm_count() ? select_with<T, D, 4>(pl, bt, q, keep, first, idx, cnt, ranks, st)
                                                                  : select_with<T, D, 2>(pl, bt, q, keep, first, idx, cnt, ranks, st);
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
