// cache_attend_simt.cu -- attention over the paged 8-bit cache on the CUDA cores, for fp32 queries.
//
//   s = scale * k_scale * (q . byte values of k),  O = sum softmax(s) * v_scale * byte values of v
// over the tokens that a row sees, in all pages of its sequence or in listed ones.
//
// fp32 queries serve to check a model, so the kernel is kept simple: products on the CUDA cores, a row at a time, K and V
// from L2 where rows share them. Shares of a row's pages are joined by the last of their CTAs. Eight rows of three sequences
// of up to 1500 tokens, 24 heads of 64: 11.6 us, of which 1.4 are the bytes: latencies of the page's chain (table, scale, K,
// softmax, V) and of the join. (K 16 channels and V four tokens at a time 12.9 us, eight heads a CTA whatever the group's size 30.)
#include <algorithm>
#include <cmath>

#include "cache.cuh"
#include "ptx.cuh"

namespace ssba {
namespace cache {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kHeads = 8;      // query heads that a CTA takes together at most
constexpr int kMaxParts = 608;  // CTAs that write partial results at most: four an SM

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// One CTA: row t, up to H heads of one group (1, 2, 4 or 8, by the group's size: a head costs 2 D multiply-adds a
// token whether it is there or not), and one of `parts` shares of its pages. A warp takes whole
// pages: a lane scores two tokens (their K rows in 16-byte loads, q broadcast from shared memory), then owns D / 32
// channels of O over the page's V rows. The warps' results are joined at the end; shares through the workspace.
template <int D, int H>
__global__ void __launch_bounds__(kThreads) ssba_cache_attend_simt_kernel(
    const Pool pl, const Batch bt, const float* q, const int32_t* idx, const int32_t* cnt, int keep, float scale_log2,
    float* O, float* lse, float* ws, unsigned* tickets, int parts, int chunks)
{
    constexpr int kC = D / 32;  // channels of a lane
    constexpr int kV = 16;      // tokens whose V is under way at a time (32: no faster)
    __shared__ __align__(16) float qs[H][D];
    __shared__ __align__(16) float ps[kWarps][kPage][H];
    __shared__ float ms[kWarps][H], ls[kWarps][H];
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int t = blockIdx.x, part = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int h = blockIdx.y / chunks, chunk = blockIdx.y % chunks;
    Seq s;
    const int b = seq_of(bt, pl, t, lane, s);
    if (b < 0) return;
    const int G = pl.heads / pl.kv_heads, g0 = chunk * H, ng = min(H, G - g0);
    const size_t head0 = (size_t)t * pl.heads + h * G + g0;
    const int L = visible(s, t, pl.status);
    const int P = (L + kPage - 1) / kPage;
    const size_t row = (size_t)t * pl.kv_heads + h;
    int n = P;
    if (idx) {
        n = ld(cnt + row);
        if (n < 0 || n > keep) {
            flag(pl.status);
            n = min(max(n, 0), keep);
        }
    }
    for (int i = tid; i < H * D; i += kThreads)
        qs[i / D][i % D] = i / D < ng ? q[head0 * D + i] : 0.f;
    __syncthreads();
    float m[H], l[H], o[H][kC];
#pragma unroll
    for (int g = 0; g < H; ++g) {
        m[g] = -INFINITY;
        l[g] = 0.f;
#pragma unroll
        for (int c = 0; c < kC; ++c) o[g][c] = 0.f;
    }
    for (int i = part * kWarps + warp; i < n; i += parts * kWarps) {
        int j = i;
        if (idx) {
            j = ld(idx + row * keep + i);
            if (j < 0 || j >= P) {
                flag(pl.status);
                continue;
            }
        }
        const int page = page_of(bt, pl, b, j);
        if (page < 0) continue;
        const int nt = min(kPage, L - j * kPage);  // tokens of the page that the row sees
        const size_t unit = (size_t)page * pl.kv_heads + h;
        const float ks = ld(pl.k_scale + unit) * scale_log2, vs = ld(pl.v_scale + unit);
        const uint8_t* K = pl.K + unit * kPage * D;
        const uint8_t* V = pl.V + unit * kPage * D;
        float a[2][H] = {};
        // 64 channels of the lane's two tokens under way at a time
#pragma unroll 1
        for (int c = 0; c < D; c += 64) {
            uint4 kk[4][2];
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int u = 0; u < 2; ++u) kk[x][u] = ld(reinterpret_cast<const uint4*>(K + (lane + 32 * u) * D + c + 16 * x));
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float f[2][4];
                    from_e4m3x4((&kk[x][0].x)[e], f[0]);
                    from_e4m3x4((&kk[x][1].x)[e], f[1]);
#pragma unroll
                    for (int g = 0; g < H; ++g) {
                        const float4 q4 = *reinterpret_cast<const float4*>(&qs[g][c + 16 * x + 4 * e]);
#pragma unroll
                        for (int u = 0; u < 2; ++u)
                            a[u][g] = fmaf(q4.w, f[u][3], fmaf(q4.z, f[u][2], fmaf(q4.y, f[u][1], fmaf(q4.x, f[u][0], a[u][g]))));
                    }
                }
        }
        __syncwarp();
#pragma unroll
        for (int g = 0; g < H; ++g) {
            const float s0 = lane < nt ? a[0][g] * ks : -INFINITY, s1 = lane + 32 < nt ? a[1][g] * ks : -INFINITY;
            float top = fmaxf(s0, s1);
#pragma unroll
            for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float mn = fmaxf(m[g], top), ref = mn == -INFINITY ? 0.f : mn;
            const float f = exp2f(m[g] - ref);
            m[g] = mn;
            const float p0 = lane < nt ? exp2f(s0 - ref) : 0.f, p1 = lane + 32 < nt ? exp2f(s1 - ref) : 0.f;
            l[g] = l[g] * f + (p0 + p1);
#pragma unroll
            for (int c = 0; c < kC; ++c) o[g][c] *= f;
            ps[warp][lane][g] = p0 * vs;
            ps[warp][lane + 32][g] = p1 * vs;
        }
        __syncwarp();
#pragma unroll 1
        for (int r0 = 0; r0 < nt; r0 += kV) {
            uint32_t raw[kV];
#pragma unroll
            for (int r = 0; r < kV; ++r) {
                const uint8_t* at = V + (r0 + r) * D + lane * kC;
                if (r0 + r >= nt) raw[r] = 0;
                else raw[r] = kC == 4 ? ld(reinterpret_cast<const uint32_t*>(at)) : ld(reinterpret_cast<const uint16_t*>(at));
            }
#pragma unroll
            for (int r = 0; r < kV; ++r) {
                float f[4];
                from_e4m3x4(raw[r], f);
#pragma unroll
                for (int g = 0; g < H; ++g) {
                    const float x = ps[warp][r0 + r][g];
#pragma unroll
                    for (int c = 0; c < kC; ++c) o[g][c] = fmaf(x, f[c], o[g][c]);
                }
            }
        }
    }
    // join the warps, two heads at a time through shared memory
#pragma unroll
    for (int g = 0; g < H; ++g) {
        float lg = l[g];
#pragma unroll
        for (int d = 16; d; d >>= 1) lg += __shfl_xor_sync(0xffffffffu, lg, d);
        if (lane == 0) {
            ms[warp][g] = m[g];
            ls[warp][g] = lg;
        }
    }
    __syncthreads();
    constexpr int kP = H < 2 ? 1 : 2;
    __shared__ float po[kWarps * kP * D];  // heads gp .. gp + kP - 1 of the warps
#pragma unroll
    for (int gp = 0; gp < H; gp += kP) {
#pragma unroll
        for (int g = gp; g < gp + kP; ++g)
#pragma unroll
            for (int c = 0; c < kC; ++c) po[(warp * kP + g - gp) * D + lane * kC + c] = o[g][c];
        __syncthreads();
        for (int i = tid; i < kP * D; i += kThreads) {
            const int g = gp + i / D, c = i % D;
            if (g < ng) {
                float top = -INFINITY, lt = 0.f, ot = 0.f;
                for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ms[w][g]);
                const float ref = top == -INFINITY ? 0.f : top;
                for (int w = 0; w < kWarps; ++w) {
                    const float f = exp2f(ms[w][g] - ref);
                    lt += ls[w][g] * f;
                    ot += po[(w * kP + g - gp) * D + c] * f;
                }
                if (parts == 1) {
                    O[(head0 + g) * D + c] = lt != 0.f ? ot / lt : 0.f;
                    if (c == 0) lse[head0 + g] = (ref + log2f(lt)) * kLn2;
                } else {
                    float* w = ws + (((size_t)blockIdx.x * gridDim.y + blockIdx.y) * parts + part) * H * (D + 2) + g * (D + 2);
                    w[c] = ot;
                    if (c == 0) {
                        w[D] = top;
                        w[D + 1] = lt;
                    }
                }
            }
        }
        __syncthreads();
    }
    if (parts == 1) return;
    // the CTA that comes last joins the row's shares, in order
    __shared__ bool last;
    const unsigned item = blockIdx.x * gridDim.y + blockIdx.y;
    if (tid == 0) {  // (everyone's stores lie before the last barrier)
        unsigned seen;
        asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(seen) : "l"(tickets + item) : "memory");
        last = seen == (unsigned)(parts - 1);
        if (last) tickets[item] = 0;
    }
    __syncthreads();
    if (!last) return;
    const size_t step = (size_t)H * (D + 2);
    for (int i = tid; i < ng * D; i += kThreads) {
        const int g = i / D, c = i % D;
        const float* w = ws + (size_t)item * parts * step + g * (D + 2);
        float top = -INFINITY, lt = 0.f, ot = 0.f;
#pragma unroll 4
        for (int k = 0; k < parts; ++k) top = fmaxf(top, __ldcg(w + k * step + D));
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll 4
        for (int k = 0; k < parts; ++k) {
            const float f = exp2f(__ldcg(w + k * step + D) - ref);
            lt += __ldcg(w + k * step + D + 1) * f;
            ot += __ldcg(w + k * step + c) * f;
        }
        O[(head0 + g) * D + c] = lt != 0.f ? ot / lt : 0.f;
        if (c == 0) lse[head0 + g] = (ref + log2f(lt)) * kLn2;
    }
}

template <int D, int H>
int attend_as(const Pool& pl, const Batch& bt, float scale, const void* q, const int32_t* idx, const int32_t* cnt,
              int keep, void* O, float* lse, void* ws, cudaStream_t st)
{
    const int G = pl.heads / pl.kv_heads, chunks = (G + H - 1) / H;
    float* parts_at = reinterpret_cast<float*>(static_cast<char*>(ws) + SSBA_CACHE_TICKET_BYTES);
    const long long items = (long long)bt.T * pl.kv_heads * chunks;
    const int pages = idx ? keep : bt.width;
    // shares: as many as give the SMs work, none of fewer than a page a warp
    const long long most = std::min<long long>(kMaxParts / std::max<long long>(items, 1), (pages + kWarps - 1) / kWarps);
    const int parts = (int)std::max<long long>(1, most);
    const dim3 grid(bt.T, pl.kv_heads * chunks, parts);
    const cudaError_t e = launch_dependent(ssba_cache_attend_simt_kernel<D, H>, grid, kThreads, 0, st, pl, bt,
                                           static_cast<const float*>(q), idx, cnt, keep, scale * kLog2e, static_cast<float*>(O),
                                           lse, parts_at, static_cast<unsigned*>(ws), parts, chunks);
    if (e == cudaSuccess) return SSBA_OK;
    set_error("ssba_cache_attend: %s", cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

template <int D, class... A>
int attend_heads(const Pool& pl, A... a)
{
    const int G = pl.heads / pl.kv_heads;
    if (G == 1) return attend_as<D, 1>(pl, a...);
    if (G == 2) return attend_as<D, 2>(pl, a...);
    if (G <= 4) return attend_as<D, 4>(pl, a...);
    return attend_as<D, 8>(pl, a...);
}

}  // namespace
}  // namespace cache

size_t cache_attend_simt_workspace()
{
    return SSBA_CACHE_TICKET_BYTES + (size_t)cache::kMaxParts * cache::kHeads * (128 + 2) * sizeof(float);
}

int launch_cache_attend_simt(const cache::Pool& pl, const cache::Batch& bt, int head_dim, float scale, const void* q,
                             const int32_t* idx, const int32_t* cnt, int keep, void* O, float* lse, void* ws,
                             cudaStream_t st)
{
    return head_dim == 64 ? cache::attend_heads<64>(pl, bt, scale, q, idx, cnt, keep, O, lse, ws, st)
                          : cache::attend_heads<128>(pl, bt, scale, q, idx, cnt, keep, O, lse, ws, st);
}

}  // namespace ssba
