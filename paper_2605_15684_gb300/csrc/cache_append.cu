// cache_append.cu -- new tokens into the paged 8-bit cache, and copies of its pages.
//
// For every page and head that new tokens of a sequence fall into: s = the smallest power of two with
// max |x| / s <= 448 over the new finite values, or the page's own scale where that is larger and the page
// holds older tokens; a new value becomes e4m3(x / s); where s has grown, older bytes become
// e4m3(byte * s_old / s). Scales being powers of two, x / s is exact, a value is rounded once in 32 bits'
// exponent range, and a change of scale rounds again only what falls below the smallest normal e4m3.
// A page that becomes full gets its mean key, s * (sum of the 64 bytes' values) / 64: at most 64 * 448 in
// steps of 2^-9 are 24 bits, so that sum is exact in any order.
#include <algorithm>
#include <cmath>

#include "cache.cuh"

namespace ssba {
namespace cache {
namespace {

constexpr int kThreads = 256;  // half of them K, half V
constexpr int kHalf = kThreads / 2;

template <typename T>
struct Chunk;  // 16 bytes of input
template <>
struct Chunk<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void get(const uint4& u, float* f)
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
template <>
struct Chunk<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void get(const uint4& u, float* f)
    {
        f[0] = __uint_as_float(u.x);
        f[1] = __uint_as_float(u.y);
        f[2] = __uint_as_float(u.z);
        f[3] = __uint_as_float(u.w);
    }
};

// The unit-th (sequence, page label) that the batch touches, pages of a sequence in order; false if
// there are fewer. Called by the whole CTA.
__device__ bool find_unit(const Batch& bt, int unit, int* status, int& b_out, int& j_out, Seq& s_out)
{
    __shared__ int wsum[kThreads / 32];
    __shared__ int found[2];
    __shared__ Seq fseq;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) found[0] = -1;
    int base = 0;
    for (int b0 = 0; b0 < bt.B; b0 += kThreads) {
        const int b = b0 + tid;
        int cnt = 0;
        Seq s{0, 0, 0};
        if (b < bt.B) {
            s = load_seq(bt, b, status);
            const int end = s.len + min(s.n, bt.width * kPage - s.len);
            if (end < s.len + s.n) flag(status);  // no room in the table: the rest is left out
            s.n = end - s.len;
            cnt = s.n > 0 ? (end - 1) / kPage - s.len / kPage + 1 : 0;
        }
        int inc = cnt;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += x;
        }
        if (lane == 31) wsum[warp] = inc;
        __syncthreads();
        int before = base, total = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before += wsum[w];
            total += wsum[w];
        }
        const int from = before + inc - cnt;
        if (unit >= from && unit < from + cnt) {
            found[0] = b;
            found[1] = s.len / kPage + (unit - from);
            fseq = s;
        }
        base += total;
        __syncthreads();
        if (found[0] >= 0 || unit < base) break;
    }
    b_out = found[0];
    j_out = found[1];
    s_out = fseq;
    return b_out >= 0;
}

// One CTA per (touched page, head); threads [0, 128) take K, the others V. A thread keeps its chunks of
// 16 input bytes in registers between the maximum and the rounding, so that inputs are read once.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) ssba_cache_append_kernel(const Pool pl, const Batch bt, const T* k,
                                                                     const T* v)
{
    constexpr int kN = Chunk<T>::n, kRowChunks = D / kN, kRows = kHalf / kRowChunks, kPass = kPage / kRows;
    __shared__ float red[2][kHalf / 32];
    __shared__ float sums[kRows][D];
    int b, j;
    Seq s;
    if (!find_unit(bt, blockIdx.x, pl.status, b, j, s)) return;
    const int page = page_of(bt, pl, b, j);
    if (page < 0) return;
    const int h = blockIdx.y, half = threadIdx.x / kHalf, tid = threadIdx.x % kHalf;
    const int row0 = tid / kRowChunks, c = tid % kRowChunks;
    const int s0 = max(s.len - j * kPage, 0), s1 = min(s.len + s.n - j * kPage, kPage);  // new slots
    const T* x = half ? v : k;
    const T* src = x + ((size_t)(s.row + j * kPage - s.len) * pl.kv_heads + h) * D + c * kN;
    uint8_t* dst = (half ? pl.V : pl.K) + ((size_t)page * pl.kv_heads + h) * kPage * D + c * kN;
    float* scale_at = (half ? pl.v_scale : pl.k_scale) + (size_t)page * pl.kv_heads + h;

    uint4 in[kPass];
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < kPass; ++i) {
        const int slot = row0 + i * kRows;
        in[i] = make_uint4(0, 0, 0, 0);
        if (slot >= s0 && slot < s1) in[i] = __ldg(reinterpret_cast<const uint4*>(src + (size_t)slot * pl.kv_heads * D));
    }
    const float was = s0 > 0 ? *scale_at : 0.f;
#pragma unroll
    for (int i = 0; i < kPass; ++i) {
        float f[kN];
        Chunk<T>::get(in[i], f);
#pragma unroll
        for (int e = 0; e < kN; ++e) {
            const float a = fabsf(f[e]);
            if (a < INFINITY) amax = fmaxf(amax, a);
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if ((tid & 31) == 0) red[half][tid >> 5] = amax;
    __syncthreads();
    amax = fmaxf(fmaxf(red[half][0], red[half][1]), fmaxf(red[half][2], red[half][3]));
    const float scale = fmaxf(was, scale_for(amax));
    const float inv = scale > 0.f ? 1.f / scale : 1.f;
    const float shrink = was < scale ? was * inv : 1.f;  // of the older bytes
    const bool full = !half && s1 == kPage;
    float sum[kN] = {};
#pragma unroll
    for (int i = 0; i < kPass; ++i) {
        const int slot = row0 + i * kRows;
        uint8_t* at = dst + (size_t)slot * D;
        if (slot >= s0 && slot < s1) {
            float f[kN];
            Chunk<T>::get(in[i], f);
            uint32_t w[kN / 4];
#pragma unroll
            for (int e = 0; e < kN; e += 4) {
                float y[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) y[r] = fabsf(f[e + r]) < INFINITY ? f[e + r] * inv : NAN;
                w[e / 4] = to_e4m3x2(y[0], y[1]) | (to_e4m3x2(y[2], y[3]) << 16);
            }
#pragma unroll
            for (int e = 0; e < kN / 4; ++e) reinterpret_cast<uint32_t*>(at)[e] = w[e];
            if (full) {
#pragma unroll
                for (int e = 0; e < kN; e += 4) {
                    float y[4];
                    from_e4m3x4(w[e / 4], y);
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[e + r] += y[r];
                }
            }
        } else if (slot < s0 && (full || shrink != 1.f)) {
#pragma unroll
            for (int e = 0; e < kN; e += 4) {
                uint32_t w = reinterpret_cast<uint32_t*>(at)[e / 4];
                float y[4];
                from_e4m3x4(w, y);
                if (shrink != 1.f) {
                    w = to_e4m3x2(y[0] * shrink, y[1] * shrink) | (to_e4m3x2(y[2] * shrink, y[3] * shrink) << 16);
                    reinterpret_cast<uint32_t*>(at)[e / 4] = w;
                    from_e4m3x4(w, y);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[e + r] += y[r];
            }
        }
    }
    if (full) {
#pragma unroll
        for (int e = 0; e < kN; ++e) sums[row0][c * kN + e] = sum[e];
    }
    __syncthreads();
    if (tid == 0) *scale_at = scale;
    if (full && tid < D) {
        float m = 0.f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) m += sums[r][tid];
        pl.k_mean[((size_t)page * pl.kv_heads + h) * D + tid] = m * (scale * (1.f / kPage));
    }
}

// Pages src[i] -> dst[i]; the kv_heads * 64 * D bytes of a page are contiguous in K and in V.
__global__ void __launch_bounds__(kThreads) ssba_cache_copy_kernel(const Pool pl, int D, const int32_t* src,
                                                                   const int32_t* dst)
{
    const int i = blockIdx.x, h = blockIdx.y;
    const int a = __ldg(src + i), b = __ldg(dst + i);
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
        const int at = threadIdx.x + u * kThreads;
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
        const int at = threadIdx.x + u * kThreads;
        if (at < n16) {
            __stcs(kd + at, kr[u]);
            __stcs(vd + at, vr[u]);
        }
    }
}

int launched(const char* who)
{
    const cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess) return SSBA_OK;
    set_error("%s: %s", who, cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

template <typename T, int D>
int append_as(const Pool& pl, const Batch& bt, const void* k, const void* v, cudaStream_t st)
{
    // every touched page takes a new token, and a run of n tokens touches at most n / 64 + 2 pages
    const long long units = std::min<long long>(bt.T, bt.T / kPage + 2LL * bt.B);
    ssba_cache_append_kernel<T, D><<<dim3((unsigned)units, pl.kv_heads), kThreads, 0, st>>>(
        pl, bt, static_cast<const T*>(k), static_cast<const T*>(v));
    return launched("ssba_cache_append");
}

}  // namespace
}  // namespace cache

int launch_cache_append(const cache::Pool& pl, const cache::Batch& bt, int head_dim, int dtype, const void* k,
                        const void* v, cudaStream_t st)
{
    if (dtype == SSBA_BF16)
        return head_dim == 64 ? cache::append_as<__nv_bfloat16, 64>(pl, bt, k, v, st)
                              : cache::append_as<__nv_bfloat16, 128>(pl, bt, k, v, st);
    return head_dim == 64 ? cache::append_as<float, 64>(pl, bt, k, v, st)
                          : cache::append_as<float, 128>(pl, bt, k, v, st);
}

int launch_cache_copy(const cache::Pool& pl, int head_dim, const int32_t* src, const int32_t* dst, int n,
                      cudaStream_t st)
{
    cache::ssba_cache_copy_kernel<<<dim3(n, pl.kv_heads), cache::kThreads, 0, st>>>(pl, head_dim, src, dst);
    return cache::launched("ssba_cache_copy");
}

}  // namespace ssba
