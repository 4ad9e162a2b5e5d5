// cache_append.cu -- new tokens into the paged 8-bit cache, and copies of its pages.
//
// For every page and head that new tokens of a sequence fall into: s = the smallest power of two with
// max |x| / s <= 448 over the new finite values, or the page's own scale where that is larger and the page
// holds older tokens; a new value becomes e4m3(x / s); where s has grown, older bytes become
// e4m3(byte * s_old / s). Scales being powers of two, x / s is exact, a value is rounded once in 32 bits'
// exponent range, and a change of scale rounds again only what falls below the smallest normal e4m3.
// A page that becomes full gets its mean key, s * (sum of the 64 bytes' values) / 64: at most 64 * 448 in
// steps of 2^-9 are 24 bits, so that sum is exact in any order.
//
// Bound by HBM where there is much to append: every value is read once, kept in shared memory between its maximum
// and its rounding, and written as a byte. 16384 tokens of 8 prompts, 8 heads of 128: 101 MB, 24 us, of which 15 are
// those bytes at the copy rate; the rest is the start (cu and lens, table, scale: three loads in a row) and the last of
// some five units a CTA. (One unit at a time 45 us; the next one's inputs under way 33; consecutive units a CTA and whole
// pages without checks 24.) One token of each of 32 sequences: 4.7 us, all latencies of that chain.
#include <algorithm>
#include <climits>
#include <cmath>

#include "cache.cuh"
#include "ptx.cuh"

namespace ssba {
namespace cache {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kStages = 2;

// 16 bytes of input: running largest magnitude of finite values (as bits that are ordered like them), and e4m3
// bytes of the values times a power of two (an infinity times 0 is NaN, so it is held as NaN).
template <typename T>
struct Chunk;
template <>
struct Chunk<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ uint32_t largest(const uint4& u, uint32_t top, bool& odd)
    {
        const uint32_t m = 0x7fff7fffu, a[4] = {u.x & m, u.y & m, u.z & m, u.w & m};
        const uint32_t t = __vmaxu2(__vmaxu2(a[0], a[1]), __vmaxu2(a[2], a[3]));
        if (__vcmpgeu2(t, 0x7f807f80u) == 0) return __vmaxu2(top, t);
        odd = true;
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const uint32_t b = ((e < 4 ? (e < 2 ? a[0] : a[1]) : (e < 6 ? a[2] : a[3])) >> (16 * (e & 1))) & 0x7fffu;
            if (b < 0x7f80u) top = __vmaxu2(top, b);
        }
        return top;
    }
    static __device__ __forceinline__ float value(uint32_t top) { return __uint_as_float(max(top & 0xffffu, top >> 16) << 16); }
    template <bool kOdd>
    static __device__ __forceinline__ void round(const uint4& u, float inv, uint32_t* w)
    {
        const uint32_t x[4] = {u.x, u.y, u.z, u.w};
        const __nv_bfloat162 s = __float2bfloat162_rn(inv), zero = __float2bfloat162_rn(0.f);  // a power of two: exact
        uint32_t r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(&x[i]);
            const __nv_bfloat162 y = kOdd ? __hfma2(v, zero, __hmul2(v, s)) : __hmul2(v, s);
            const uint32_t b = *reinterpret_cast<const uint32_t*>(&y);
            r[i] = to_e4m3x2(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u));
        }
        w[0] = r[0] | (r[1] << 16);
        w[1] = r[2] | (r[3] << 16);
    }
};
template <>
struct Chunk<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ uint32_t largest(const uint4& u, uint32_t top, bool& odd)
    {
        const uint32_t a[4] = {u.x & 0x7fffffffu, u.y & 0x7fffffffu, u.z & 0x7fffffffu, u.w & 0x7fffffffu};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (a[i] < 0x7f800000u) top = max(top, a[i]);
            else odd = true;
        }
        return top;
    }
    static __device__ __forceinline__ float value(uint32_t top) { return __uint_as_float(top); }
    template <bool kOdd>
    static __device__ __forceinline__ void round(const uint4& u, float inv, uint32_t* w)
    {
        float y[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = kOdd ? fmaf(y[i], 0.f, y[i] * inv) : y[i] * inv;
        w[0] = to_e4m3x2(y[0], y[1]) | (to_e4m3x2(y[2], y[3]) << 16);
    }
};

// Touched pages of sequences [b0, b0 + kEach * kThreads): ends[i] is how many those up to b0 + i have; returns their sum.
template <int kEach>
__device__ int count_pages(const Batch& bt, int b0, int* status, int* ends, int* buf)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int cnt[kEach], sum = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int b = b0 + tid * kEach + e;
        cnt[e] = 0;
        if (b < bt.B) {
            const Seq s = load_seq(bt, b, status);
            const int room = bt.width * kPage - s.len;
            if (s.n > room) flag(status);  // the rest has no place in the table and is left out
            const int n = min(s.n, room);
            cnt[e] = n > 0 ? (s.len + n - 1) / kPage - s.len / kPage + 1 : 0;
        }
        sum += cnt[e];
    }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += x;
    }
    __syncthreads();
    if (lane == 31) buf[warp] = inc;
    __syncthreads();
    int at = inc - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) at += buf[w];
        total += buf[w];
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) ends[tid * kEach + e] = at += cnt[e];
    __syncthreads();
    return total;
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}

// A unit is a touched page, a head, and K or V. A CTA takes consecutive ones, so that it seldom has to look for a page;
// the inputs of the next one are under way (each thread copies to shared memory what it will read itself) while
// one is worked on.
// kEach: sequences that a thread counts, 1 for batches of up to 128.
template <typename T, int D, int kEach>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 5 : 2) ssba_cache_append_kernel(const Pool pl, const Batch bt, const T* k,
                                                                     const T* v)
{
    constexpr int kN = Chunk<T>::n, kRowChunks = D / kN, kRows = kThreads / kRowChunks, kPass = kPage / kRows;
    constexpr int kSeqs = kEach * kThreads;
    extern __shared__ uint4 stage[];  // [kStages][kPass][kThreads]
    __shared__ int ends[kSeqs];
    __shared__ int buf[kWarps];
    __shared__ uint32_t red[2][kWarps];
    __shared__ float sums[kWarps][D];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row0 = tid / kRowChunks, c = tid % kRowChunks;

    struct Unit {
        int s0, s1;       // new slots
        size_t tile;      // page * kv_heads + head
        bool v, real;
        float was;
    };
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    int turn = 0, phase = 0;
    for (int b0 = 0; b0 < bt.B; b0 += kSeqs) {
        const int pages = count_pages<kEach>(bt, b0, pl.status, ends, buf), each = 2 * pl.kv_heads;
        const long long units = (long long)pages * each;
        const bool small = units < INT_MAX / 65536;  // (32-bit division where it does)
        long long u = small ? (int)units * (int)blockIdx.x / (int)gridDim.x : units * blockIdx.x / gridDim.x;
        const long long u_end = small ? (int)units * (int)(blockIdx.x + 1) / (int)gridDim.x : units * (blockIdx.x + 1) / gridDim.x;
        // the touched page that the next unit lies in, its sequence, and the unit's place among the page's
        int pg = small ? (int)u / each : (int)(u / each), hv = (int)(u - (long long)pg * each), b = 0, page = -1, s0 = 0, s1 = 0;
        ptrdiff_t first = 0;  // row of the page's slot 0
        bool found = false;
        {
            int hi = kSeqs - 1;  // the first sequence with ends > pg
            while (b < hi) {
                const int mid = (b + hi) / 2;
                if (ends[mid] > pg) hi = mid;
                else b = mid + 1;
            }
        }
        // the next unit, its copies under way into stage st
        auto begin = [&](long long i, int st) {
            Unit x{0, 0, 0, false, false, 0.f};
            if (i < u_end) {
                if (!found) {
                    while (ends[b] <= pg) ++b;
                    const Seq s = load_seq(bt, b0 + b, pl.status);
                    const int j = s.len / kPage + pg - (b ? ends[b - 1] : 0), n = min(s.n, bt.width * kPage - s.len);
                    page = page_of(bt, pl, b0 + b, j);
                    s0 = max(s.len - j * kPage, 0);
                    s1 = min(s.len + n - j * kPage, kPage);
                    first = (ptrdiff_t)s.row + j * kPage - s.len;
                    found = true;
                }
                if (page >= 0) {
                    const int h = hv >> 1;
                    x.real = true;
                    x.v = hv & 1;
                    x.s0 = s0;
                    x.s1 = s1;
                    x.tile = (size_t)page * pl.kv_heads + h;
                    if (s0 > 0) x.was = (x.v ? pl.v_scale : pl.k_scale)[x.tile];
                    const T* src = (x.v ? v : k) + (first * pl.kv_heads + h) * D + c * kN;
#pragma unroll
                    for (int i = 0; i < kPass; ++i) {
                        const int slot = row0 + i * kRows;
                        const bool in = slot >= s0 && slot < s1;
                        copy16(static_cast<uint32_t>(__cvta_generic_to_shared(stage + (st * kPass + i) * kThreads + tid)),
                               in ? src + (ptrdiff_t)slot * pl.kv_heads * D : k, in);
                    }
                }
                if (++hv == each) {
                    hv = 0;
                    ++pg;
                    found = false;
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            return x;
        };
        Unit next = begin(u, turn % kStages);
        for (; u < u_end; ++u, ++turn) {
            const Unit x = next;
            next = begin(u + 1, (turn + 1) % kStages);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            if (!x.real) continue;
            phase ^= 1;
            const uint4* in = stage + (turn % kStages) * kPass * kThreads + tid;
            uint32_t top = 0;
            bool odd = false;
#pragma unroll
            for (int i = 0; i < kPass; ++i) top = Chunk<T>::largest(in[i * kThreads], top, odd);
            const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(Chunk<T>::value(top)));
            if (lane == 0) red[phase][warp] = most;
            __syncthreads();
            const float amax = __uint_as_float(max(max(red[phase][0], red[phase][1]), max(red[phase][2], red[phase][3])));
            const float scale = fmaxf(x.was, scale_for(amax));
            const float inv = scale > 0.f ? 1.f / scale : 1.f;
            const float shrink = x.was < scale ? x.was * inv : 1.f;  // of the older bytes
            const bool full = !x.v && x.s1 == kPage;
            uint8_t* dst = (x.v ? pl.V : pl.K) + x.tile * kPage * D + c * kN;
            float sum[kN] = {};
            auto put = [&](uint32_t* at, const uint32_t* w) {
                if (kN == 8) *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[kN / 4 - 1]);
                else at[0] = w[0];
                if (full) {
#pragma unroll
                    for (int e = 0; e < kN; e += 4) {
                        float y[4];
                        from_e4m3x4(w[e / 4], y);
#pragma unroll
                        for (int r = 0; r < 4; ++r) sum[e + r] += y[r];
                    }
                }
            };
            if (x.s0 == 0 && x.s1 == kPage && !odd) {  // a whole page, as most of a prompt's are
#pragma unroll
                for (int i = 0; i < kPass; ++i) {
                    uint32_t w[kN / 4];
                    Chunk<T>::template round<false>(in[i * kThreads], inv, w);
                    put(reinterpret_cast<uint32_t*>(dst + (row0 + i * kRows) * D), w);
                }
            } else {
                // older bytes, where they are needed, all under way at once
                const bool older = full || shrink != 1.f;
                uint32_t w[kPass][kN / 4];
#pragma unroll
                for (int i = 0; i < kPass; ++i) {
                    const int slot = row0 + i * kRows;
                    const uint32_t* at = reinterpret_cast<const uint32_t*>(dst + slot * D);
                    if (older && slot < x.s0) {
#pragma unroll
                        for (int e = 0; e < kN / 4; ++e) w[i][e] = at[e];
                    }
                }
#pragma unroll
                for (int i = 0; i < kPass; ++i) {
                    const int slot = row0 + i * kRows;
                    if (slot >= x.s0 && slot < x.s1) {
                        Chunk<T>::template round<true>(in[i * kThreads], inv, w[i]);
                    } else if (older && slot < x.s0) {
                        if (shrink != 1.f) {
#pragma unroll
                            for (int e = 0; e < kN / 4; ++e) {
                                float y[4];
                                from_e4m3x4(w[i][e], y);
                                w[i][e] = to_e4m3x2(y[0] * shrink, y[1] * shrink) | (to_e4m3x2(y[2] * shrink, y[3] * shrink) << 16);
                            }
                        }
                    } else {
                        continue;
                    }
                    put(reinterpret_cast<uint32_t*>(dst + slot * D), w[i]);
                }
            }
            if (tid == 0) (x.v ? pl.v_scale : pl.k_scale)[x.tile] = scale;
            if (full) {
                // rows of a warp by shuffles (where it holds several), the warps through shared memory
#pragma unroll
                for (int e = 0; e < kN; ++e) {
#pragma unroll
                    for (int o = 16; o >= kRowChunks; o >>= 1) sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], o);
                    if (lane < kRowChunks) sums[warp][c * kN + e] = sum[e];
                }
                __syncthreads();
                if (tid < D) {
                    const float m = (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]);
                    pl.k_mean[x.tile * D + tid] = m * (scale * (1.f / kPage));
                }
                __syncthreads();
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
    }
}

// Pages src[i] -> dst[i]; the kv_heads * 64 * D bytes of a page are contiguous in K and in V. A CTA a page and head, all of
// its loads under way at once. Bound by HBM: 2048 pages of 8 heads of 128 (554 MB both ways) take 90.5 us, 6.1 TB/s.
constexpr int kCopyThreads = 256;

__global__ void __launch_bounds__(kCopyThreads) ssba_cache_copy_kernel(const Pool pl, int D, const int32_t* src,
                                                                   const int32_t* dst)
{
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int i = blockIdx.x, h = blockIdx.y;
    const int a = ld(src + i), b = ld(dst + i);
    if (a < 0 || a >= pl.pages || b < 0 || b >= pl.pages) {
        if (threadIdx.x == 0) flag(pl.status);
        return;
    }
    const size_t from = (size_t)a * pl.kv_heads + h, to = (size_t)b * pl.kv_heads + h;
    const int n16 = kPage * D / 16;
    const uint4 *ks = reinterpret_cast<const uint4*>(pl.K) + from * n16, *vs = reinterpret_cast<const uint4*>(pl.V) + from * n16;
    uint4 *kd = reinterpret_cast<uint4*>(pl.K) + to * n16, *vd = reinterpret_cast<uint4*>(pl.V) + to * n16;
    uint4 kr[2], vr[2];  // D <= 128: at most 512 chunks a tensor
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int at = threadIdx.x + u * kCopyThreads;
        if (at < n16) {
            kr[u] = __ldcs(ks + at);
            vr[u] = __ldcs(vs + at);
        }
    }
    if (threadIdx.x < D) pl.k_mean[to * D + threadIdx.x] = pl.k_mean[from * D + threadIdx.x];
    if (threadIdx.x == 0) pl.k_scale[to] = pl.k_scale[from];
    if (threadIdx.x == 32) pl.v_scale[to] = pl.v_scale[from];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int at = threadIdx.x + u * kCopyThreads;
        if (at < n16) {
            __stcs(kd + at, kr[u]);
            __stcs(vd + at, vr[u]);
        }
    }
}

int launched(const char* who, cudaError_t e)
{
    if (e == cudaSuccess) return SSBA_OK;
    set_error("%s: %s", who, cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

template <typename T, int D, int kEach>
int append_as(const Pool& pl, const Batch& bt, const void* k, const void* v, cudaStream_t st)
{
    const size_t smem = (size_t)kStages * kPage * D * sizeof(T);
    static PerDeviceOnce once;
    once.run([smem] {
        cudaFuncSetAttribute(ssba_cache_append_kernel<T, D, kEach>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    // every touched page takes a new token, and a run of n tokens touches at most n / 64 + 2 pages
    const long long units = std::min<long long>(bt.T, bt.T / kPage + 2LL * bt.B) * pl.kv_heads * 2;
    const int fit = (int)std::min<size_t>(8, (size_t)200 * 1024 / (smem + 8192));  // CTAs of an SM
    const dim3 grid((unsigned)std::min<long long>(units, (long long)fit * device_sm_count()));
    return launched("ssba_cache_append", launch_dependent(ssba_cache_append_kernel<T, D, kEach>, grid, kThreads, smem, st, pl, bt,
                                                          static_cast<const T*>(k), static_cast<const T*>(v)));
}

template <typename T, int D>
int append_any(const Pool& pl, const Batch& bt, const void* k, const void* v, cudaStream_t st)
{
    return bt.B <= kThreads ? append_as<T, D, 1>(pl, bt, k, v, st) : append_as<T, D, 8>(pl, bt, k, v, st);
}

}  // namespace
}  // namespace cache

int launch_cache_append(const cache::Pool& pl, const cache::Batch& bt, int head_dim, int dtype, const void* k,
                        const void* v, cudaStream_t st)
{
    if (dtype == SSBA_BF16)
        return head_dim == 64 ? cache::append_any<__nv_bfloat16, 64>(pl, bt, k, v, st)
                              : cache::append_any<__nv_bfloat16, 128>(pl, bt, k, v, st);
    return head_dim == 64 ? cache::append_any<float, 64>(pl, bt, k, v, st)
                          : cache::append_any<float, 128>(pl, bt, k, v, st);
}

int launch_cache_copy(const cache::Pool& pl, int head_dim, const int32_t* src, const int32_t* dst, int n,
                      cudaStream_t st)
{
    return cache::launched("ssba_cache_copy", cache::launch_dependent(cache::ssba_cache_copy_kernel, dim3(n, pl.kv_heads),
                                                                      cache::kCopyThreads, 0, st, pl, head_dim, src, dst));
}

}  // namespace ssba
