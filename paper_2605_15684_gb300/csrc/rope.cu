// rope.cu -- rotary positions with several axes (time, height, width, ...), on heads at any strides.
//
// A head's first 2P dimensions are P pairs, cut into one run of pairs for each axis. Pair j of axis a turns by the
// angle pos_a theta_j: (u, v) -> (u cos - v sin, u sin + v cos); the inverse, which is the gradient, by its negative.
// Pairs are adjacent dimensions (2j, 2j + 1) or halves (j, j + P); dimensions from 2P on stay.
//
// Angles: theta_j / (2 pi) is held as a 64-bit fraction of a turn, whose product with an integer position modulo 2^64 is
// the angle modulo whole turns, without a rounding (a product in fp32 is off by a tenth of a radian at a million). Its top 24
// bits, signed, are an fp32 number of units of pi, which sincospif takes; the next 32 turn that sine and cosine on by an angle l
// below 2^-24 of a turn, sin + l cos and cos - l sin (l^2 is 2^-43). So the angle is used to 2^-48 of a turn, beside
// theta's own 53 bits, and what is left is sincospif's error, a unit of the last place, and a rounding.
//
// Bound by HBM: x is read once and written once, 16 bytes a thread and step where the strides and the cut allow it (else
// 8, 4 or 2). A thread forms the sines of its pairs of one token once and applies them to the heads of its share.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "layer.cuh"

namespace ssba {
namespace layer {
namespace {

using namespace ptx;

constexpr int kMaxPairs = SSBA_ROPE_MAX_HEAD_DIM / 2;

struct RopeArgs {
    const char* x;
    char* out;
    const int32_t* pos;
    int64_t xs[3], os[3], pos_batch;  // strides of batch, token, head in bytes; of pos's batch in elements
    long long lanes;                  // units of all tokens
    int T, heads, axes, P, D;
    int units, turned;                // units a token and head; of them those that turn
    int share;                        // heads a thread; the grid's y has the shares
    int inverse;
    uint8_t axis[kMaxPairs];
    uint64_t theta[kMaxPairs];        // turns of 2^64 a position
};

template <int kBytes>
struct Word;
template <>
struct Word<16> { using type = uint4; };
template <>
struct Word<8> { using type = uint2; };
template <>
struct Word<4> { using type = uint32_t; };
template <>
struct Word<2> { using type = uint16_t; };

// n elements of E in 16, 8, 4 or 2 bytes
template <class E, int n>
struct Pack {
    using W = typename Word<n * (int)sizeof(E)>::type;
    union U {
        W w;
        E e[n];
        __device__ U() {}
    };
    static __device__ __forceinline__ void get(const W& w, float* f)
    {
        U u;
        u.w = w;
#pragma unroll
        for (int i = 0; i < n; ++i) f[i] = (float)u.e[i];
    }
    static __device__ __forceinline__ W put(const float* f)
    {
        U u;
#pragma unroll
        for (int i = 0; i < n; ++i) u.e[i] = (E)f[i];
        return u.w;
    }
};

// w with its 32-bit words from `first` on as they are in x
template <class W>
__device__ __forceinline__ W kept(W w, const W& x, int first)
{
    uint32_t* to = reinterpret_cast<uint32_t*>(&w);
    const uint32_t* from = reinterpret_cast<const uint32_t*>(&x);
#pragma unroll
    for (int i = 0; i < (int)sizeof(W) / 4; ++i) to[i] = i >= first ? from[i] : to[i];
    return w;
}

// (u, v) turned, with the same roundings in every instantiation: widths and layouts give the same bits.
__device__ __forceinline__ void turn(float u, float v, float c, float s, float& a, float& b)
{
    a = fmaf(u, c, -__fmul_rn(v, s));
    b = fmaf(u, s, __fmul_rn(v, c));
}

// kN: elements of a piece. Halves: a unit is a piece of either half; adjacent pairs: one piece.
template <class E, int kN, bool kHalves>
__global__ void __launch_bounds__(256) ssba_rope_kernel(const __grid_constant__ RopeArgs p)
{
    constexpr int kPairs = kHalves ? kN : kN / 2, kBatch = kHalves ? 3 : 6;
    using W = typename Pack<E, kN>::W;
    grid_dep_wait();
    grid_dep_launch();
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= p.lanes) return;
    int unit;
    long long b, t;
    if (p.lanes <= 0xffffffffll) {  // 32-bit divisions where they do (a fifth of the instructions)
        const uint32_t i = (uint32_t)id, token = i / (uint32_t)p.units, seq = token / (uint32_t)p.T;
        unit = (int)(i - token * (uint32_t)p.units);
        b = seq;
        t = token - seq * (uint32_t)p.T;
    } else {
        const long long token = id / p.units;
        unit = (int)(id - token * p.units);
        b = token / p.T;
        t = token - b * p.T;
    }
    const int h0 = (int)blockIdx.y * p.share, h1 = min(h0 + p.share, p.heads);
    const char* x = p.x + b * p.xs[0] + t * p.xs[1] + h0 * p.xs[2];
    char* o = p.out + b * p.os[0] + t * p.os[1] + h0 * p.os[2];
    const int at = unit * kN * (int)sizeof(E), half = p.P * (int)sizeof(E);
    if (unit >= p.turned) {  // dimensions that stay (halves only)
        const int stay = (2 * p.P + (unit - p.turned) * kN) * (int)sizeof(E);
        for (int h = h0; h < h1; ++h, x += p.xs[2], o += p.os[2]) *reinterpret_cast<W*>(o + stay) = *reinterpret_cast<const W*>(x + stay);
        return;
    }
    // Adjacent pairs: of a unit's 32-bit words, the first that stays. The bits that were read are written there (a turn by nothing would
    // spread an infinity or a NaN over its pair); a loop of its own, without the batches below, took half as long again.
    const int first = (2 * p.P - unit * kN) * (int)sizeof(E) / 4;
    // a batch of heads is loaded at once, the first before the sines are formed
    W u[kBatch], v[kHalves ? kBatch : 1];
    auto load = [&](int left) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (k < left) {
                u[k] = *reinterpret_cast<const W*>(x + k * p.xs[2] + at);
                if (kHalves) v[k] = *reinterpret_cast<const W*>(x + k * p.xs[2] + at + half);
            }
    };
    load(h1 - h0);
    const int32_t* pos = p.pos + b * p.pos_batch + t * p.axes;
    float c[kPairs], s[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const int j = unit * kPairs + i;
        if (!kHalves && j >= p.P) {
            c[i] = 1.f;
            s[i] = 0.f;
            continue;
        }
        const uint64_t turns = (uint64_t)(int64_t)pos[p.axis[j]] * p.theta[j];
        const float l = (float)(uint32_t)(turns >> 8) * 8.719671245021580e-17f;  // 2 pi 2^-56
        float sn, cs;
        sincospif((float)((int32_t)(turns >> 32) & ~0xff) * 4.656612873077393e-10f, &sn, &cs);
        s[i] = fmaf(l, cs, sn);
        c[i] = fmaf(-l, sn, cs);
        if (p.inverse) s[i] = -s[i];
    }
    for (int h = h0;;) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (h + k >= h1) break;
            char* to = o + k * p.os[2] + at;
            float f[kN], a[kN];
            Pack<E, kN>::get(u[k], f);
            if constexpr (kHalves) {
                float g[kN], d[kN];
                Pack<E, kN>::get(v[k], g);
#pragma unroll
                for (int i = 0; i < kN; ++i) turn(f[i], g[i], c[i], s[i], a[i], d[i]);
                *reinterpret_cast<W*>(to + half) = Pack<E, kN>::put(d);
            } else {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) turn(f[2 * i], f[2 * i + 1], c[i], s[i], a[2 * i], a[2 * i + 1]);
            }
            W w = Pack<E, kN>::put(a);
            if constexpr (!kHalves) w = kept(w, u[k], first);
            *reinterpret_cast<W*>(to) = w;
        }
        h += kBatch;
        if (h >= h1) return;
        x += kBatch * p.xs[2];
        o += kBatch * p.os[2];
        load(h1 - h);
    }
}

template <class E, bool kHalves>
int rope_as(RopeArgs& p, int bytes, long long tokens, cudaStream_t st)
{
    auto go = [&](auto n_) {
        constexpr int n = decltype(n_)::value;
        p.units = kHalves ? p.P / n + (p.D - 2 * p.P) / n : p.D / n;
        p.turned = kHalves ? p.P / n : p.units;
        // Heads a thread: as many as leave some eight warps a scheduler; a thread's sines then serve them all.
        const long long full = (long long)device_sm_count() * 1024;
        p.lanes = tokens * p.units;
        const int shares = (int)std::min<long long>(std::max<long long>(full / p.lanes, 1), std::min(p.heads, 65535));
        p.share = (p.heads + shares - 1) / shares;
        const dim3 grid((unsigned)((p.lanes + 255) / 256), (unsigned)((p.heads + p.share - 1) / p.share));
        const cudaError_t e = launch_early(ssba_rope_kernel<E, n, kHalves>, grid, 256, 0, st, 1, p);
        if (e == cudaSuccess) return (int)SSBA_OK;
        set_error("ssba_rope_kernel launch: %s", cudaGetErrorString(e));
        return (int)SSBA_ERR_CUDA;
    };
    using std::integral_constant;
    constexpr int s = sizeof(E);
    if (bytes == 16) return go(integral_constant<int, 16 / s>());
    if (bytes == 8) return go(integral_constant<int, 8 / s>());
    if constexpr (kHalves || s == 2) {
        if (bytes == 4) return go(integral_constant<int, 4 / s>());
    }
    if constexpr (kHalves && s == 2) return go(integral_constant<int, 1>());
    return SSBA_ERR_INVALID;  // not reached: the caller's bytes hold a pair, or an element of halves
}

// The rates of a call's pairs and their axes follow from the rule alone. A thread keeps those of its last rule: a model's
// calls share one, and 64 powers in 64 bits take longer than a few tokens' kernel.
struct Rates {
    int32_t axes = 0, sections[SSBA_ROPE_MAX_AXES] = {}, shared = 0;
    double base = 0;
    int P = 0;
    uint8_t axis[kMaxPairs];
    uint64_t theta[kMaxPairs];

    void set(const ssba_rope_desc& d)
    {
        bool same = axes == d.axes && (shared != 0) == (d.shared != 0) && base == d.base;
        for (int a = 0; same && a < axes; ++a) same = sections[a] == d.sections[a];
        if (same) return;
        axes = d.axes;
        shared = d.shared;
        base = d.base;
        P = 0;
        for (int a = 0; a < axes; ++a) P += sections[a] = d.sections[a];
        const double two64 = 18446744073709551616.0, turn = 6.283185307179586476925286766559;
        for (int a = 0, j = 0; a < axes; ++a)
            for (int i = 0; i < sections[a]; ++i, ++j) {
                axis[j] = (uint8_t)a;
                const double e = shared ? (double)j / P : (double)i / sections[a];
                theta[j] = (uint64_t)(std::pow(base, -e) / turn * two64 + 0.5);
            }
    }
};

}  // namespace

int launch_rope(const ssba_rope_desc& d, const void* x, const int64_t* xs, const int32_t* pos, int64_t pos_batch, void* out,
                const int64_t* os, cudaStream_t st)
{
    RopeArgs p;
    const int es = d.dtype == SSBA_BF16 ? 2 : 4;
    p.x = static_cast<const char*>(x);
    p.out = static_cast<char*>(out);
    p.pos = pos;
    p.pos_batch = pos_batch;
    uint64_t all = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out);
    for (int i = 0; i < 3; ++i) {
        p.xs[i] = xs[i] * es;
        p.os[i] = os[i] * es;
        all |= (uint64_t)p.xs[i] | (uint64_t)p.os[i];
    }
    p.T = d.T;
    p.heads = d.heads;
    p.axes = d.axes;
    p.D = d.head_dim;
    static thread_local Rates rates;
    rates.set(d);
    p.P = rates.P;
    memcpy(p.axis, rates.axis, p.P);
    memcpy(p.theta, rates.theta, sizeof(uint64_t) * p.P);
    p.inverse = d.inverse != 0;
    // the widest piece that every row's start, and the cuts of halves, are multiples of
    const bool halves = d.layout == SSBA_ROPE_HALVES;
    all |= (uint64_t)p.D * es;
    if (halves) all |= (uint64_t)p.P * es;
    int bytes = 16;
    while (all & (bytes - 1)) bytes >>= 1;
    const long long tokens = (long long)d.B * d.T;
    if (d.dtype == SSBA_BF16)
        return halves ? rope_as<__nv_bfloat16, true>(p, bytes, tokens, st) : rope_as<__nv_bfloat16, false>(p, bytes, tokens, st);
    return halves ? rope_as<float, true>(p, bytes, tokens, st) : rope_as<float, false>(p, bytes, tokens, st);
}

}  // namespace layer
}  // namespace ssba
