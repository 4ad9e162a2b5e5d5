// cache.cuh -- what the kernels of the paged 8-bit K/V cache share: its geometry, how a batch's
// rows map to sequences and pages, and the e4m3 conversions.
//
// A cache is a pool of pages of 64 tokens. K and V are e4m3 [pages][kv_heads][64][head_dim], each
// page and head with an fp32 scale (value = byte value * scale; the library writes powers of two, so
// that a change of scale moves exponents only), and fp32 [pages][kv_heads][head_dim] holds the mean key
// of every full page. table[b][j] is the page of tokens [64 j, 64 j + 64) of sequence b.
#pragma once
#include <cstdint>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace ssba {
namespace cache {

constexpr int kPage = SSBA_CACHE_PAGE;
static_assert(kPage == 64, "the kernels' tiles are 64 tokens a page");

// The pool and the batch, as every kernel gets them. Lengths and rows are clamped to what the
// buffers hold and pages are checked before use: bad ones set SSBA_ERR_CHECK and reach no memory.
struct Pool {
    uint8_t *K, *V;
    float *k_scale, *v_scale, *k_mean;
    int pages, heads, kv_heads;
    int* status;
};

struct Batch {
    const int32_t *table, *lens, *cu;
    int B, width, T;
};

struct Seq {
    int row, n, len;  // rows [row, row + n) of the batch; tokens held
};

// A load of what an earlier grid may have written. Not the read-only path (__ldg): these kernels may start beside that
// grid's end, so what it writes is not constant for their whole time.
template <typename T>
__device__ __forceinline__ T ld(const T* p)
{
    return *p;
}

// A timeout that nobody has read yet stays: whoever reads it drops the workspaces whose counters it has left set.
__device__ __forceinline__ void flag(int* status) { atomicCAS(status, SSBA_OK, SSBA_ERR_CHECK); }

// A sequence from its entries in cu and lens, clamped.
__device__ __forceinline__ Seq make_seq(const Batch& bt, int c0, int c1, int l, int* status)
{
    Seq s;
    s.row = min(max(c0, 0), bt.T);
    const int end = min(max(c1, s.row), bt.T);
    s.n = end - s.row;
    s.len = min(max(l, 0), bt.width * kPage);
    if (s.row != c0 || end != c1 || s.len != l) flag(status);
    return s;
}

__device__ __forceinline__ Seq load_seq(const Batch& bt, int b, int* status)
{
    return make_seq(bt, ld(bt.cu + b), ld(bt.cu + b + 1), ld(bt.lens + b), status);
}

// Tokens that row t sees: those up to its own, the new tokens of a sequence being its last.
__device__ __forceinline__ int visible(const Seq& s, int t, int* status)
{
    if (t < s.row || t >= s.row + s.n) flag(status);  // rows out of order in cu
    return min(max(s.len - s.n + (t - s.row) + 1, 0), s.len);
}

// The sequence that row t belongs to: the last b with cu[b] <= t, or -1 behind the last sequence.
// Called by whole warps: 32 entries are compared at a time, so that a batch of 1024 takes two rounds.
__device__ __forceinline__ int find_seq(const Batch& bt, int t, int lane)
{
    if (t < bt.B) {  // most batches have one row a sequence: then this is it
        const int c0 = ld(bt.cu + t), c1 = ld(bt.cu + t + 1);
        if (c0 <= t && t < c1) return t;
    }
    if (t < ld(bt.cu) || t >= ld(bt.cu + bt.B)) return -1;
    int lo = 0, n = bt.B;  // the answer lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const bool le = lane * step < n && ld(bt.cu + at) <= t;
        const unsigned m = __ballot_sync(0xffffffffu, le);
        const int k = m ? 31 - __clz(m) : 0;
        n = min(step, n - k * step);
        lo += k * step;
    }
    return lo;
}

// find_seq, and the sequence itself (of no tokens where there is none): where each has one row, all of it in one round trip.
__device__ __forceinline__ int seq_of(const Batch& bt, const Pool& pl, int t, int lane, Seq& s)
{
    if (t < bt.B) {
        const int c0 = ld(bt.cu + t), c1 = ld(bt.cu + t + 1), l = ld(bt.lens + t);
        if (c0 <= t && t < c1) {
            s = make_seq(bt, c0, c1, l, pl.status);
            return t;
        }
    }
    const int b = find_seq(bt, t, lane);
    s = b >= 0 ? load_seq(bt, b, pl.status) : Seq{0, 0, 0};
    return b;
}

// Page of label j of sequence b, or -1 (flagged) when the table holds none of the pool's.
__device__ __forceinline__ int page_of(const Batch& bt, const Pool& pl, int b, int j)
{
    const int p = ld(bt.table + (size_t)b * bt.width + j);
    if (p >= 0 && p < pl.pages) return p;
    flag(pl.status);
    return -1;
}

// Dynamic shared memory of the selection: the row's scores and the group's queries.
constexpr size_t kSelectSmem = 200 * 1024;

// Two floats to two e4m3 bytes (nearest, ties to even; `lo` in the low byte; NaN stays NaN).
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ float2 from_e4m3x2(uint32_t v)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(v)));
    return __half22float2(*reinterpret_cast<__half2*>(&h));
}

__device__ __forceinline__ void from_e4m3x4(uint32_t v, float (&f)[4])
{
    const float2 a = from_e4m3x2(v & 0xffffu), b = from_e4m3x2(v >> 16);
    f[0] = a.x;
    f[1] = a.y;
    f[2] = b.x;
    f[3] = b.y;
}

// The smallest power of two s with amax / s <= 448, the largest e4m3 value: 448 = 1.75 * 2^8. 0 for
// amax = 0; at least 2^-126, so that 1 / s is finite.
__device__ __forceinline__ float scale_for(float amax)
{
    if (!(amax > 0.f)) return 0.f;
    const uint32_t u = __float_as_uint(amax);
    const int k = static_cast<int>(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float(static_cast<uint32_t>(max(k, -126) + 127) << 23);
}

// Launch in the stream's order, but allowed to start beside the last grid's end: the kernels wait for that grid before
// they touch memory that it may have written (griddepcontrol).
template <class... P, class... A>
cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, P(args)...);
    if (e == cudaSuccess) e = cudaGetLastError();
    return e;
}

}  // namespace cache

int launch_cache_append(const cache::Pool& pl, const cache::Batch& bt, int head_dim, int dtype, const void* k,
                        const void* v, cudaStream_t st);
int launch_cache_copy(const cache::Pool& pl, int head_dim, const int32_t* src, const int32_t* dst, int n,
                      cudaStream_t st);
int launch_cache_select(const cache::Pool& pl, const cache::Batch& bt, int head_dim, int dtype, const void* q,
                        int keep, int first, int32_t* idx, int32_t* cnt, cudaStream_t st);
// idx null: every page of the sequence; else [T][kv_heads][keep] with cnt [T][kv_heads].
int launch_cache_attend_simt(const cache::Pool& pl, const cache::Batch& bt, int head_dim, float scale, const void* q,
                             const int32_t* idx, const int32_t* cnt, int keep, void* O, float* lse, void* ws,
                             cudaStream_t st);
size_t cache_attend_simt_workspace();
int launch_cache_attend_tc(const cache::Pool& pl, const cache::Batch& bt, int head_dim, float scale, const void* q,
                           const int32_t* idx, const int32_t* cnt, int keep, void* O, float* lse, void* ws,
                           cudaStream_t st, uint64_t budget_ns = kWaitBudgetNs, int withhold = 0);
size_t cache_attend_tc_workspace();
int launch_cache_attend_rows(const cache::Pool& pl, const cache::Batch& bt, int head_dim, float scale, const void* q,
                             void* O, float* lse, void* ws, cudaStream_t st, uint64_t budget_ns = kWaitBudgetNs,
                             int withhold = 0);
size_t cache_attend_rows_workspace();

}  // namespace ssba
