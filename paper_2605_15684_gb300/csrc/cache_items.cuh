// cache_items.cuh -- how the tensor-core kernels of the cache attention cut a batch into work: items of rows that
// share a K/V head's tokens, tiles of 128 tokens, and an equal share of all tiles for every CTA.
#pragma once
#include <climits>

#include "cache.cuh"
#include "ptx.cuh"

namespace ssba {
namespace cache {
namespace {

using namespace ptx;

// Shared-memory matrix descriptor with any layout code (0 none, 2 128-byte, 4 64-byte swizzle); see sdesc_sw128.
__device__ __forceinline__ uint64_t sdesc(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes, uint32_t layout)
{
    return (sdesc_sw128(saddr, lbo_bytes, sbo_bytes) & ~(7ull << 61)) | (static_cast<uint64_t>(layout) << 61);
}

// Instruction descriptor for kind::f8f6f4 with e4m3 A and B (formats 0; each operand has its own field), and for kind::f16
// with fp16 ones (also 0, and the same for both),
// with an fp32 accumulator; the other fields as in idesc_bf16_f32.
__host__ __device__ constexpr uint32_t idesc_e4m3_f32(int M, int N, bool a_mn_major, bool b_mn_major)
{
    return (1u << 4) | ((a_mn_major ? 1u : 0u) << 15) | ((b_mn_major ? 1u : 0u) << 16) |
           (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// D[tmem] (+)= A[smem] * B[smem]^T of 8-bit values, K = 32, issued by one thread.
__device__ __forceinline__ void mma_f8_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                          uint32_t accumulate)
{
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n"
        "}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

constexpr int kTile = 128;           // tokens of a tile: two pages
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kNowhere = 1 << 30;    // token position of a page that is not there

constexpr int kLeast = 4;            // tiles of a share at least: below, joining costs more than the tiles
constexpr int kMaxGrid = 608;        // CTAs of a launch at most (two an SM of up to 304)
static_assert(kMaxGrid * sizeof(unsigned) <= SSBA_CACHE_TICKET_BYTES, "a counter a CTA");

struct Params {
    Pool pl;
    Batch bt;
    const __nv_bfloat16* q;
    const int32_t *idx, *cnt;  // null: all pages
    int keep;
    float scale_log2;
    __nv_bfloat16* O;
    float* lse;
    float* parts;
    unsigned* tickets;
    int G, gc, chunks, tq;  // group size; heads and tokens of an item; chunks of a group
    int gc_inv;             // ceil(2^16 / gc): r / gc for r < 256
    uint64_t budget_ns;     // of every wait
    int withhold;           // (test hook) CTA 0 announces its first copies and issues none
};

// The rows of an item: tokens [row, row + n) of the batch, each with the heads of chunk hv.
struct Rows {
    int hv, row, n;

    // Row r of the item: its row of the batch (-1: none) and head.
    __device__ __forceinline__ int of(const Params& p, int r, int& head) const
    {
        const int i = r * p.gc_inv >> 16, chunk = p.chunks == 1 ? 0 : hv % p.chunks;  // r < 256
        const int g = chunk * p.gc + r - i * p.gc;
        head = (p.chunks == 1 ? hv : hv / p.chunks) * p.G + g;
        return g < p.G && i < n ? row + i : -1;
    }
};

struct Maps {
    CUtensorMap k, v;
};

__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ bool wait_raw(uint32_t bar, uint32_t parity, uint64_t budget_ns)
{
    const uint64_t t0 = globaltimer_ns();
    while (!mbar_try_wait(bar, parity))
        if (globaltimer_ns() - t0 > budget_ns) return false;
    return true;
}

// Tiles of the row blocks of a sequence. Block t of tq tokens (a power of two) sees a + (t + 1) tq tokens,
// a = len - n, the last one len; a block takes max(1, ceil(seen / 128)) tiles. With u = ceil(a / tq) and m = 128 / tq
// that is max(1, ceil((u + t + 1) / m)), and for tq = 128 c with u = ceil(a / 128) it is max(1, u + (t + 1) c), so
// sums over blocks have closed forms.
struct Blocks {
    int a, n, len, tq, count;

    __device__ __forceinline__ Blocks(const Seq& s, int tq_) : a(s.len - s.n), n(s.n), len(s.len), tq(tq_)
    {
        count = (n + tq - 1) >> shift();
    }
    __device__ __forceinline__ int shift() const { return 31 - __clz(tq); }
    __device__ __forceinline__ int tiles(int t) const
    {
        const int seen = t + 1 < count ? a + (t + 1) * tq : len;
        return max(1, (seen + kTile - 1) / kTile);
    }
    static __device__ __forceinline__ long long upto(int k, int m)  // sum of max(1, ceil(j / m)), j = 1 .. k
    {
        if (k <= 0) return k;
        const int d = k >> (31 - __clz(m)), r = k & (m - 1);  // m is a power of two
        return (long long)m * d * (d + 1) / 2 + (long long)r * (d + 1);
    }
    __device__ __forceinline__ long long before(int t) const  // tiles of blocks 0 .. t - 1, t < count
    {
        if (tq > kTile) {
            const long long u = (a + kTile - 1) >> 7, c = tq >> 7, z = u < 0 ? min(-u / c, (long long)t) : 0;
            return z + (t - z) * u + c * ((long long)t * (t + 1) - z * (z + 1)) / 2;
        }
        const int u = (a + tq - 1) >> shift(), m = kTile >> shift();
        return upto(u + t, m) - upto(u, m);
    }
    __device__ __forceinline__ long long sum() const { return count ? before(count - 1) + tiles(count - 1) : 0; }
};

// The items of a CTA's share, in order: sequence, K/V head (and chunk of its group), block of rows. With lists an
// item is one row and K/V head, of equally many tiles for all.
template <bool kList>
struct Walk {
    const Params& p;
    long long w, w1;   // next tile of the share, its end
    long long start;   // first tile of the item, in the batch's order
    int heads;         // K/V heads times chunks
    int b, hv, t;      // t: row block of the sequence, or the row with lists
    Seq s;
    int tiles, tb, te;  // tiles of the item; those of this CTA

    template <class S>
    __device__ __forceinline__ Walk(const Params& p_, const S& sm) : p(p_), w(sm.w0), w1(sm.w1)
    {
        heads = p.pl.kv_heads * p.chunks;
        if (w >= w1) return;
        if (kList) {
            tiles = (p.keep + 1) / 2;
            const long long item = sm.total < INT_MAX ? (int)w / tiles : w / tiles;
            start = item * tiles;
            t = (int)(sm.total < INT_MAX ? (int)item / heads : item / heads);
            hv = (int)(item - (long long)t * heads);
            t += max(0, min(ld(p.bt.cu), p.bt.T));
            locate();
        } else {
            b = sm.first_b;
            s = sm.first_s;
            const Blocks bl(s, p.tq);
            const long long one = max(bl.sum(), 1LL);
            long long at = sm.first_at;
            hv = (int)min(sm.total < INT_MAX ? (int)at / (int)one : at / one, (long long)heads - 1);
            at -= (long long)hv * one;
            int lo = 0, hi = bl.count - 1;  // the last block with before(t) <= at
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (bl.before(mid) <= at) lo = mid;
                else hi = mid - 1;
            }
            t = lo;
            tiles = bl.tiles(t);
            start = w - (at - bl.before(t));
        }
        share();
    }
    __device__ __forceinline__ void locate()  // (lists) the sequence of row t
    {
        b = seq_of(p.bt, p.pl, t, threadIdx.x & 31, s);
    }
    __device__ __forceinline__ void share()
    {
        tb = (int)(w - start);
        te = (int)min((long long)tiles, tb + (w1 - w));
    }
    __device__ __forceinline__ bool more() const { return w < w1; }
    __device__ __forceinline__ void next()
    {
        w = start + te;
        if (w >= w1) return;
        start += tiles;
        if (kList) {
            if (++hv == heads) {
                hv = 0;
                ++t;
                locate();
            }
        } else {
            Blocks bl(s, p.tq);
            if (++t >= bl.count) {
                t = 0;
                if (++hv == heads) {
                    hv = 0;
                    do {
                        ++b;
                        s = load_seq(p.bt, min(b, p.bt.B - 1), p.pl.status);
                    } while (s.n == 0 && b < p.bt.B - 1);
                }
                bl = Blocks(s, p.tq);
            }
            tiles = bl.tiles(t);
        }
        share();
    }
    __device__ __forceinline__ Rows rows() const
    {
        if (kList) return Rows{hv, t, b >= 0 ? 1 : 0};
        return Rows{hv, s.row + t * p.tq, min(s.n - t * p.tq, p.tq)};
    }
    __device__ __forceinline__ int row_of(int r, int& head) const { return rows().of(p, r, head); }
    __device__ __forceinline__ int limit(int row) const { return min(max(s.len - s.n + row - s.row + 1, 0), s.len); }
    // Label of the item's k-th page, or -1: no such page, or (flagged) a listed label that the row does not see.
    __device__ __forceinline__ int label(int k) const
    {
        if (!kList) return (long long)k * kPage < s.len ? k : -1;
        if (b < 0) return -1;
        const size_t at = (size_t)t * p.pl.kv_heads + hv / p.chunks;
        int n = ld(p.cnt + at);
        if (n < 0 || n > p.keep) flag(p.pl.status);
        if (k >= min(n, p.keep)) return -1;
        const int j = ld(p.idx + at * p.keep + k);
        if (j >= 0 && (long long)j * kPage < limit(t)) return j;
        flag(p.pl.status);
        return -1;
    }
    __device__ __forceinline__ int page(int k, int& j) const
    {
        j = label(k);
        if (j < 0) return -1;
        return page_of(p.bt, p.pl, b, j);
    }
};

// The CTA's share [w0, w1) of the batch's tiles and where it starts. All threads.
template <bool kList, int kThreads, class S>
__device__ void make_share(const Params& p, S& sm)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int heads = p.pl.kv_heads * p.chunks;
    __shared__ long long wsum[kThreads / 32];
    // tiles of thread tid's sequence of those from b0 on, all heads: sum over the CTA, or that in front of the thread
    auto scan = [&](int b0, long long mine, long long& front) {
        long long inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += x;
        }
        __syncthreads();
        if (lane == 31) wsum[warp] = inc;
        __syncthreads();
        long long sum = 0;
        front = inc - mine;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) front += wsum[w];
            sum += wsum[w];
        }
        return sum;
    };
    Seq seq{0, 0, 0};  // the thread's of the last scan
    auto tiles_of = [&](int b) {
        if (b >= p.bt.B) return 0LL;
        seq = load_seq(p.bt, b, p.pl.status);
        return Blocks(seq, p.tq).sum() * heads;
    };
    long long W = 0, mine = 0, front = 0;
    if (kList) {
        const int r0 = max(0, min(ld(p.bt.cu), p.bt.T)), r1 = max(r0, min(ld(p.bt.cu + p.bt.B), p.bt.T));
        W = (long long)(r1 - r0) * heads * ((p.keep + 1) / 2);
    } else {
        for (int b0 = 0; b0 < p.bt.B; b0 += kThreads) {
            mine = tiles_of(b0 + tid);
            W += scan(b0, mine, front);
        }
    }
    const int C = (int)min((long long)gridDim.x, max(W / kLeast, 1LL)), c = blockIdx.x;
    // (32-bit division where it does)
    const bool small = W < INT_MAX / kMaxGrid;
    const long long w0 = c >= C ? W : small ? (int)W * c / C : W * c / C;
    const long long w1 = c >= C ? W : small ? (int)W * (c + 1) / C : W * (c + 1) / C;
    if (tid == 0) {
        sm.w0 = w0;
        sm.w1 = w1;
        sm.total = W;
        sm.ctas = C;
        sm.first_b = 0;
        sm.first_at = 0;
    }
    __syncthreads();
    if (!kList && w0 < w1) {
        long long base = 0;  // tiles of the sequences in front, all heads
        for (int b0 = 0; b0 < p.bt.B && base <= w0; b0 += kThreads) {
            long long sum = W;
            if (p.bt.B > kThreads) {  // else the sum's own scan
                mine = tiles_of(b0 + tid);
                sum = scan(b0, mine, front);
            }
            const long long at = base + front;
            if (w0 >= at && w0 < at + mine) {
                sm.first_b = b0 + tid;
                sm.first_s = seq;
                sm.first_at = w0 - at;
            }
            base += sum;
        }
    }
    __syncthreads();
}

// The CTA whose share tile w lies in: the last c with W c / C <= w.
template <class S>
__device__ __forceinline__ int cta_of(long long w, const S& sm)
{
    if (sm.total < INT_MAX / kMaxGrid - 1) return (int)(((int)w + 1) * sm.ctas - 1) / (int)sm.total;
    return (int)(((w + 1) * sm.ctas - 1) / sm.total);
}

// [pages * kv_heads][64][D] bytes, a box a page and head.
inline bool encode_page_map(CUtensorMap* m, const void* base, long long tiles, int D, CUtensorMapSwizzle swizzle)
{
    EncodeTiledFn fn = tensor_map_encoder();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)kPage, (cuuint64_t)tiles};
    cuuint64_t strides[2] = {(cuuint64_t)D, (cuuint64_t)kPage * D};
    cuuint32_t box[3] = {(cuuint32_t)D, (cuuint32_t)kPage, 1};
    cuuint32_t es[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace cache
}  // namespace ssba
