// norm.cu -- the root-mean-square norm in front of a layer's products, with the residual's addition, and backward.
//
//   h = round(x + r)                    (x itself without a residual)
//   rstd = 1 / sqrt(mean_i h_i^2 + eps),   y_i = h_i rstd w_i
//   8-bit rows: s = the least power of two with max_i |y_i| / s <= 448, q_i = e4m3(y_i / s)
//   backward, with xh = h rstd and g = dy w:   dx = rstd (g - xh mean(g xh)) (+ dh),   dw = sum_t dy xh
//
// y is the norm of the rounded h, which is what the backward pass reads. Both kernels are bound by HBM: every tensor
// passes once, a row stays in registers (as the packed bits that were read) between its sum and its output. A row is
// one warp's or one CTA's, 16 bytes a thread and step; the 8-bit rows' maximum of |h w| goes through the same
// reduction as the sum of squares (max |y| = rstd max |h w|, so one barrier serves both). In fp32 that product is off by three
// roundings: where it lies next to a power of two times 448, the row is taken again, by the largest y as it is rounded.
// Under the 8-bit rows, y is the fp32 number nearest to the exact product: the sum of squares, rstd and the products carry
// their rounding errors along in a second fp32 (the pass is bound by HBM; the extra eight instructions a value are
// free). A plain fp32 product puts one value in a million on the other side of a tie, and so off by an eighth.
// Backward: CTAs walk over rows and keep dw of their columns in registers (fp32); the partial sums of all
// CTAs meet in a second launch, in one order.
#include "layer.cuh"

namespace ssba {
namespace layer {
namespace {

using namespace ptx;

template <class T>
struct Vec;  // 16 bytes of T
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void get(const uint4& v, float* f)
    {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = unpack2(u[i]);
            f[2 * i] = p.x;
            f[2 * i + 1] = p.y;
        }
    }
    static __device__ __forceinline__ uint4 put(const float* f)
    {
        return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
    }
};
template <>
struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void get(const uint4& v, float* f)
    {
        f[0] = __uint_as_float(v.x);
        f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z);
        f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 put(const float* f)
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

template <int n>
__device__ __forceinline__ void load_w(const float* w, float* f)
{
#pragma unroll
    for (int i = 0; i < n; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(w + i);  // plain: the grid in front may have written it
        f[i] = v.x;
        f[i + 1] = v.y;
        f[i + 2] = v.z;
        f[i + 3] = v.w;
    }
}

// A sum and the error of its roundings. a.add(b) and b.add(a) are one to the bit: the error of hi + x is exact in either order.
struct Sum {
    float hi, lo;
    __device__ __forceinline__ void add(float x, float err)
    {
        const float t = hi + x, z = t - hi;
        lo = ((hi - (t - z)) + (x - z)) + (lo + err);
        hi = t;
    }
    __device__ __forceinline__ void add_square(float x, bool bf16)
    {
        const float q = x * x;  // exact for bf16
        add(q, bf16 ? 0.f : fmaf(x, x, -q));
    }
};

// The sum of s and the maximum of m over the row's kTPR threads (a warp, or the whole CTA; `at` alternates between two
// halves of the exchange area, so that one barrier a row is enough). kExact: with the sums' errors. All of the row's threads
// end with the same bits, since each step adds the same two numbers in either lane.
template <int kTPR, bool kMax, bool kExact>
__device__ __forceinline__ void row_reduce(Sum& s, float& m, float4 (*area)[32], int at)
{
    auto step = [&](int o) {
        const float x = __shfl_xor_sync(0xffffffffu, s.hi, o);
        if (kExact)
            s.add(x, __shfl_xor_sync(0xffffffffu, s.lo, o));
        else
            s.hi += x;
        if (kMax) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    };
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) step(o);
    if constexpr (kTPR > 32) {
        constexpr int kWarps = kTPR / 32;
        const int lane = threadIdx.x & 31;
        if (lane == 0) area[at][threadIdx.x >> 5] = make_float4(s.hi, s.lo, m, 0.f);
        __syncthreads();
        const float4 v = area[at][lane % kWarps];
        s.hi = v.x;
        s.lo = v.y;
        m = v.z;
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) step(o);
    }
}

// 1 / sqrt(sum / D + eps) as a pair of fp32: the hardware's value and one step of Newton's iteration on its error.
__device__ __forceinline__ Sum exact_rstd(const Sum& s, float D, float eps)
{
    Sum m{s.hi / D, 0.f};
    m.lo = (fmaf(-m.hi, D, s.hi) + s.lo) / D;
    m.add(eps, 0.f);
    const float r = rsqrtf(m.hi);
    if (!(r > 0.f && r < __int_as_float(0x7f800000))) return Sum{r, 0.f};
    const float t = m.hi * r, off = fmaf(m.hi, r, -t) + m.lo * r;  // (m.hi + m.lo) r = t + off
    const float low = 0.5f * r * (fmaf(-t, r, 1.f) - off * r);
    const float hi = r + low;
    return Sum{hi, (r - hi) + low};
}

// f k w, rounded once.
__device__ __forceinline__ float product(float f, const Sum& k, float w)
{
    const float p = f * k.hi, pe = fmaf(f, k.lo, fmaf(f, k.hi, -p)), y = p * w;
    return y + fmaf(pe, w, fmaf(p, w, -y));
}

// Whether the scale that a row's largest |y| asks for is not certain from a = max |h w| rstd in fp32, which is off by three
// roundings: a within eight units of the last place of a border (448 times a power of two), or a or m = max |h w| where fp32
// has lost bits, or all of them (below 2^-100; NaN and infinities). A row of zeros, m = 0, is certain.
__device__ __forceinline__ bool scale_is_open(float a, float m)
{
    const uint32_t bits = __float_as_uint(a), least = (127u - 100u) << 23;
    return (((bits - (0x600000u - 8u)) & 0x7fffffu) <= 16u || bits - least >= 0x7f800000u - least || m < 0x1p-100f) && bits != 0;
}

// The least power of two s with a / s <= 448 = 1.75 * 2^8 (at least 2^-126; 1 for a = 0), and its reciprocal.
__device__ __forceinline__ float row_scale(float a, float& inverse)
{
    const uint32_t bits = __float_as_uint(a);
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    if (a == 0.f) e = 0;
    e = min(max(e, -126), 126);
    inverse = __uint_as_float((uint32_t)(127 - e) << 23);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}

__device__ __forceinline__ uint32_t pack_e4m3(const float* f)
{
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[0], f[1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[2], f[3]), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}

// Eight-bit values of n of y: 8 or 4 bytes.
template <int n>
__device__ __forceinline__ void put_e4m3(uint8_t* q, long long i, const float* f)
{
    if constexpr (n == 8)
        reinterpret_cast<uint2*>(q)[i] = make_uint2(pack_e4m3(f), pack_e4m3(f + 4));
    else
        reinterpret_cast<uint32_t*>(q)[i] = pack_e4m3(f);
}

struct NormArgs {
    const uint4 *x, *r;
    const float* w;
    uint4 *h, *y;
    uint8_t* q;
    float *scale, *rstd;
    int T, D;
    float eps;
};

constexpr int kWarpCta = 128;  // threads of a CTA whose warps take a row each

template <class T, int kTPR, int kNV, bool kRes, bool kF8>
__global__ void __launch_bounds__(kTPR == 32 ? kWarpCta : kTPR) ssba_rms_norm_kernel(const NormArgs p)
{
    constexpr int n = Vec<T>::n, kRows = kTPR == 32 ? kWarpCta / 32 : 1;
    __shared__ float4 area[2][32];
    const int nv = p.D / n, tid = threadIdx.x % kTPR;
    grid_dep_wait();
    grid_dep_launch();
    int at = 0;
    bool again = false;
    for (long long t = (long long)blockIdx.x * kRows + threadIdx.x / kTPR; t < p.T; t += (long long)gridDim.x * kRows, at ^= 1) {
        uint4 v[kNV], u[kRes ? kNV : 1];
#pragma unroll
        for (int j = 0; j < kNV; ++j) {
            const int i = tid + j * kTPR;
            v[j] = i < nv ? p.x[t * nv + i] : make_uint4(0, 0, 0, 0);
            if (kRes) u[j] = i < nv ? p.r[t * nv + i] : make_uint4(0, 0, 0, 0);
        }
        Sum s{0.f, 0.f};
        float m = 0.f;
#pragma unroll
        for (int j = 0; j < kNV; ++j) {
            const int i = tid + j * kTPR;
            float f[n];
            Vec<T>::get(v[j], f);
            if (kRes) {
                float g[n];
                Vec<T>::get(u[j], g);
#pragma unroll
                for (int e = 0; e < n; ++e) f[e] += g[e];
                v[j] = Vec<T>::put(f);
                if (i < nv) p.h[t * nv + i] = v[j];
                Vec<T>::get(v[j], f);
            }
#pragma unroll
            for (int e = 0; e < n; ++e) {
                if (kF8)
                    s.add_square(f[e], n == 8);
                else
                    s.hi = fmaf(f[e], f[e], s.hi);
            }
            if (kF8 && i < nv) {
                float w[n];
                load_w<n>(p.w + (size_t)i * n, w);
#pragma unroll
                for (int e = 0; e < n; ++e) m = fmaxf(m, fabsf(f[e] * w[e]));
            }
        }
        row_reduce<kTPR, kF8, kF8>(s, m, area, at);
        Sum rstd{0.f, 0.f};
        if (kF8)
            rstd = exact_rstd(s, (float)p.D, p.eps);
        else
            rstd.hi = 1.f / sqrtf(s.hi / (float)p.D + p.eps);
        float inverse = 1.f;
        if (kF8) {
            const float a = m * rstd.hi, scale = row_scale(a, inverse);
            const bool open = scale_is_open(a, m);
            if (tid == 0) p.scale[t] = open ? 0.f : scale;
            again = again || open;
        }
        if (tid == 0) p.rstd[t] = rstd.hi;
#pragma unroll
        for (int j = 0; j < kNV; ++j) {
            const int i = tid + j * kTPR;
            if (i >= nv) continue;
            float f[n], w[n];
            Vec<T>::get(v[j], f);
            load_w<n>(p.w + (size_t)i * n, w);
#pragma unroll
            for (int e = 0; e < n; ++e) f[e] = kF8 ? product(f[e], rstd, w[e]) * inverse : f[e] * rstd.hi * w[e];
            if (kF8)
                put_e4m3<n>(p.q, t * nv + i, f);
            else
                p.y[t * nv + i] = Vec<T>::put(f);
        }
    }
    if constexpr (kF8) {
        const bool mine = kTPR == 32 ? __any_sync(0xffffffffu, again) : __syncthreads_or(again);
        if (!mine) return;
        __syncwarp();
        // The rows left open, behind the loop (in it they took 4 % of the others' time): the scale of the largest finite y as it is
        // rounded, and the row's values. A thread reads the h that it wrote, and where all read scale[t] a barrier of
        // the sum's lies in front of its writing.
#pragma unroll 1
        for (long long t = (long long)blockIdx.x * kRows + threadIdx.x / kTPR; t < p.T; t += (long long)gridDim.x * kRows) {
            if (p.scale[t] != 0.f) continue;
            const uint4* row = (kRes ? p.h : p.x) + t * nv;
            float f[n], w[n], a = 0.f;
            Sum s{0.f, 0.f};
#pragma unroll 1
            for (int i = tid; i < nv; i += kTPR) {
                Vec<T>::get(row[i], f);
#pragma unroll
                for (int e = 0; e < n; ++e) s.add_square(f[e], n == 8);
            }
            row_reduce<kTPR, false, true>(s, a, area, at);
            at ^= 1;
            const Sum rstd = exact_rstd(s, (float)p.D, p.eps);
#pragma unroll 1
            for (int i = tid; i < nv; i += kTPR) {
                Vec<T>::get(row[i], f);
                load_w<n>(p.w + (size_t)i * n, w);
#pragma unroll
                for (int e = 0; e < n; ++e) {
                    const float y = fabsf(product(f[e], rstd, w[e]));
                    a = fmaxf(a, y < __int_as_float(0x7f800000) ? y : 0.f);
                }
            }
            Sum none{0.f, 0.f};
            row_reduce<kTPR, true, false>(none, a, area, at);
            at ^= 1;
            float inverse;
            const float scale = row_scale(a, inverse);
            if (tid == 0) p.scale[t] = scale;
#pragma unroll 1
            for (int i = tid; i < nv; i += kTPR) {
                Vec<T>::get(row[i], f);
                load_w<n>(p.w + (size_t)i * n, w);
#pragma unroll
                for (int e = 0; e < n; ++e) f[e] = product(f[e], rstd, w[e]) * inverse;
                put_e4m3<n>(p.q, t * nv + i, f);
            }
        }
    }
}

struct NormBwdArgs {
    const uint4 *dy, *h, *dh;
    const float *w, *rstd;
    uint4* dx;
    float* part;
    int T, D;
};

constexpr int kBwdWarps = 4;  // warps of a CTA whose warps take a row each

// CTAs of an SM, all of which run at once: 12 warps of 48 columns a lane (up to 168 registers with what is under way), more of fewer, or 1024
// threads of 16 columns (64 registers).
constexpr int bwd_ctas_of(int tpr, int steps)
{
    return tpr == 32 ? (steps == 1 ? 8 : steps == 2 ? 6 : steps == 4 ? 4 : 3) : 1024 / tpr;
}

template <class T, int kTPR, int kNV, bool kDh>
__global__ void __launch_bounds__(kTPR == 32 ? kBwdWarps * 32 : kTPR, bwd_ctas_of(kTPR, kNV)) ssba_rms_norm_bwd_kernel(const NormBwdArgs p)
{
    constexpr int n = Vec<T>::n, kRows = kTPR == 32 ? kBwdWarps : 1;
    __shared__ float4 area[2][32];
    extern __shared__ float cols[];  // [warps][D], where a CTA's warps add up
    const int nv = p.D / n, tid = threadIdx.x % kTPR;
    float dw[kNV][n] = {};
    grid_dep_wait();
    grid_dep_launch();
    int at = 0;
    for (long long t = (long long)blockIdx.x * kRows + threadIdx.x / kTPR; t < p.T; t += (long long)gridDim.x * kRows, at ^= 1) {
        uint4 a[kNV], b[kNV], c[kDh ? kNV : 1];
#pragma unroll
        for (int j = 0; j < kNV; ++j) {
            const int i = tid + j * kTPR;
            const bool in = i < nv;
            a[j] = in ? p.dy[t * nv + i] : make_uint4(0, 0, 0, 0);
            b[j] = in ? p.h[t * nv + i] : make_uint4(0, 0, 0, 0);
            if (kDh) c[j] = in ? p.dh[t * nv + i] : make_uint4(0, 0, 0, 0);
        }
        const float rstd = p.rstd[t];
        Sum s{0.f, 0.f};
        float none = 0.f;
#pragma unroll
        for (int j = 0; j < kNV; ++j) {
            const int i = tid + j * kTPR;
            if (i >= nv) continue;
            float d[n], h[n], w[n];
            Vec<T>::get(a[j], d);
            Vec<T>::get(b[j], h);
            load_w<n>(p.w + (size_t)i * n, w);
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float k = d[e] * (h[e] * rstd);
                s.hi = fmaf(k, w[e], s.hi);
                dw[j][e] += k;
            }
        }
        row_reduce<kTPR, false, false>(s, none, area, at);
        const float along = s.hi / (float)p.D;
#pragma unroll
        for (int j = 0; j < kNV; ++j) {
            const int i = tid + j * kTPR;
            if (i >= nv) continue;
            float d[n], h[n], w[n], g[n];
            Vec<T>::get(a[j], d);
            Vec<T>::get(b[j], h);
            load_w<n>(p.w + (size_t)i * n, w);
            if (kDh) Vec<T>::get(c[j], g);
#pragma unroll
            for (int e = 0; e < n; ++e) {
                const float o = rstd * (d[e] * w[e] - h[e] * rstd * along);
                d[e] = kDh ? o + g[e] : o;
            }
            p.dx[t * nv + i] = Vec<T>::put(d);
        }
    }
    float* out = p.part + (size_t)blockIdx.x * p.D;
    if constexpr (kTPR == 32) {
        // the warps' sums, in the order of the warps
        float* mine = cols + (threadIdx.x >> 5) * p.D;
#pragma unroll
        for (int j = 0; j < kNV; ++j) {
            const int i = tid + j * kTPR;
            if (i >= nv) continue;
#pragma unroll
            for (int e = 0; e < n; e += 4)
                *reinterpret_cast<float4*>(mine + i * n + e) = make_float4(dw[j][e], dw[j][e + 1], dw[j][e + 2], dw[j][e + 3]);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < p.D; c += kBwdWarps * 32) {
            float v = cols[c];
#pragma unroll
            for (int k = 1; k < kBwdWarps; ++k) v += cols[k * p.D + c];
            out[c] = v;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kNV; ++j) {
            const int i = tid + j * kTPR;
            if (i >= nv) continue;
#pragma unroll
            for (int e = 0; e < n; e += 4)
                *reinterpret_cast<float4*>(out + (size_t)i * n + e) =
                    make_float4(dw[j][e], dw[j][e + 1], dw[j][e + 2], dw[j][e + 3]);
        }
    }
}

// out[c] = sum_p part[p][c]: a CTA takes 32 columns, its 32 warps every 32nd part each, then the warps in order.
__global__ void __launch_bounds__(1024) ssba_column_sum_kernel(const float* part, int parts, int N, float* out)
{
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    grid_dep_wait();
    grid_dep_launch();
    float s = 0.f;
    if (c < N) {
#pragma unroll 4
        for (int p = warp; p < parts; p += 32) s += part[(size_t)p * N + c];
    }
    sums[warp][lane] = s;
    __syncthreads();
    s = sums[lane][warp];  // column `warp` of the 32, its parts over the lanes
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0 && blockIdx.x * 32 + warp < N) out[blockIdx.x * 32 + warp] = s;
}

// Threads a row and 16-byte steps a thread. Rows of up to 4 KB are a warp's (no barrier; all its loads under way at
// once), longer ones a CTA's.
template <class T, class F>
int by_width(int nv, F&& f)
{
    using std::integral_constant;
#define SSBA_ROW(tpr, steps) return f(integral_constant<int, tpr>(), integral_constant<int, steps>())
    if (nv <= 32) SSBA_ROW(32, 1);
    if (nv <= 64) SSBA_ROW(32, 2);
    if (nv <= 128) SSBA_ROW(32, 4);
    if (nv <= 192) SSBA_ROW(32, 6);
    if (nv <= 256) SSBA_ROW(128, 2);
    if (nv <= 512) SSBA_ROW(256, 2);
    if (nv <= 1024) SSBA_ROW(256, 4);
    if constexpr (sizeof(T) == 4) {
        if (nv > 2048) SSBA_ROW(1024, 4);
    }
    SSBA_ROW(512, 4);
#undef SSBA_ROW
}

int launched(cudaError_t e, const char* what)
{
    if (e == cudaSuccess) return SSBA_OK;
    set_error("%s launch: %s", what, cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

template <class T, bool kRes, bool kF8>
int norm_as(const NormArgs& p, cudaStream_t st)
{
    return by_width<T>(p.D / Vec<T>::n, [&](auto tpr, auto steps) {
        constexpr int kTPR = decltype(tpr)::value, kRows = kTPR == 32 ? kWarpCta / 32 : 1;
        const long long ctas = ((long long)p.T + kRows - 1) / kRows, most = 64ll * device_sm_count();
        return launched(launch_early(ssba_rms_norm_kernel<T, kTPR, decltype(steps)::value, kRes, kF8>,
                                     dim3((unsigned)(ctas < most ? ctas : most)), kTPR == 32 ? kWarpCta : kTPR, 0, st, 1, p),
                        "ssba_rms_norm_kernel");
    });
}

// The backward pass: threads a row and steps a thread. Its registers hold dw of the columns as well, so long rows take more
// threads of two steps (one wave of CTAs; in two, with four steps, 4096 rows of 8192 took 51 us).
template <class T, class F>
int by_width_bwd(int nv, F&& f)
{
    using std::integral_constant;
#define SSBA_ROW(tpr, steps) return f(integral_constant<int, tpr>(), integral_constant<int, steps>())
    if (nv <= 32) SSBA_ROW(32, 1);
    if (nv <= 64) SSBA_ROW(32, 2);
    if (nv <= 128) SSBA_ROW(32, 4);
    if (nv <= 192) SSBA_ROW(32, 6);
    if (nv <= 256) SSBA_ROW(128, 2);
    if (nv <= 512) SSBA_ROW(256, 2);
    if (nv <= 1024) SSBA_ROW(512, 2);
    if constexpr (sizeof(T) == 4) {
        if (nv > 2048) SSBA_ROW(1024, 4);
    }
    SSBA_ROW(1024, 2);
#undef SSBA_ROW
}

// CTAs of the backward pass: as many as run at once.
template <class T>
int bwd_ctas_as(int rows, int D)
{
    return by_width_bwd<T>(D / Vec<T>::n, [&](auto tpr, auto steps) {
        constexpr int kTPR = decltype(tpr)::value, kRows = kTPR == 32 ? kBwdWarps : 1;
        const long long need = ((long long)rows + kRows - 1) / kRows, most = (long long)device_sm_count() * bwd_ctas_of(kTPR, decltype(steps)::value);
        return (int)(need < most ? need : most);
    });
}

int bwd_ctas(int T, int D, int dtype) { return dtype == SSBA_BF16 ? bwd_ctas_as<__nv_bfloat16>(T, D) : bwd_ctas_as<float>(T, D); }

template <class T, bool kDh>
int norm_bwd_as(const NormBwdArgs& p, int ctas, cudaStream_t st)
{
    return by_width_bwd<T>(p.D / Vec<T>::n, [&](auto tpr, auto steps) {
        constexpr int kTPR = decltype(tpr)::value;
        return launched(launch_early(ssba_rms_norm_bwd_kernel<T, kTPR, decltype(steps)::value, kDh>, dim3(ctas),
                                     kTPR == 32 ? kBwdWarps * 32 : kTPR, kTPR == 32 ? sizeof(float) * kBwdWarps * p.D : 0, st, 1, p),
                        "ssba_rms_norm_bwd_kernel");
    });
}

}  // namespace

int launch_column_sum(const float* part, int parts, int N, float* out, const char* who, cudaStream_t st)
{
    return launched(launch_early(ssba_column_sum_kernel, dim3((N + 31) / 32), 1024, 0, st, 1, part, parts, N, out), who);
}

int launch_rms_norm(const void* x, const void* r, const float* w, int T, int D, int dtype, float eps, void* h, void* y,
                    bool e4m3, float* scale, float* rstd, cudaStream_t st)
{
    const NormArgs p{static_cast<const uint4*>(x), static_cast<const uint4*>(r), w, static_cast<uint4*>(h),
                     static_cast<uint4*>(y), static_cast<uint8_t*>(y), scale, rstd, T, D, eps};
    auto go = [&](auto t) {
        using E = decltype(t);
        if (r) return e4m3 ? norm_as<E, true, true>(p, st) : norm_as<E, true, false>(p, st);
        return e4m3 ? norm_as<E, false, true>(p, st) : norm_as<E, false, false>(p, st);
    };
    return dtype == SSBA_BF16 ? go(__nv_bfloat16()) : go(float());
}

int rms_norm_backward_parts(int T, int D, int dtype) { return bwd_ctas(T, D, dtype); }

int launch_rms_norm_backward(const void* dy, const void* h, const float* w, const float* rstd, const void* dh, int T, int D,
                             int dtype, void* dx, float* dw, float* part, cudaStream_t st)
{
    const int ctas = bwd_ctas(T, D, dtype);
    const bool one = ctas == 1 && reinterpret_cast<uintptr_t>(dw) % 16 == 0;  // its sums are dw
    const NormBwdArgs p{static_cast<const uint4*>(dy), static_cast<const uint4*>(h), static_cast<const uint4*>(dh), w, rstd,
                        static_cast<uint4*>(dx), one ? dw : part, T, D};
    auto go = [&](auto t) {
        using E = decltype(t);
        return dh ? norm_bwd_as<E, true>(p, ctas, st) : norm_bwd_as<E, false>(p, ctas, st);
    };
    const int rc = dtype == SSBA_BF16 ? go(__nv_bfloat16()) : go(float());
    return rc == SSBA_OK && !one ? launch_column_sum(part, ctas, D, dw, "ssba_rms_norm_backward", st) : rc;
}

}  // namespace layer
}  // namespace ssba
