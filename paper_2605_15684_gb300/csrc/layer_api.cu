// layer_api.cu -- the entry points of a layer around its attention (include/ssba.h): argument validation on the host and
// kernel launches on the caller's stream.
#include <cmath>
#include <utility>

#include "layer.cuh"

namespace ssba {
namespace layer {
namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

int invalid(const char* who, const char* what)
{
    set_error("%s: %s", who, what);
    return SSBA_ERR_INVALID;
}

// A range of device memory that a call reads or writes.
struct Range {
    const void* at;
    size_t bytes;
    bool meets(const Range& o) const
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(at), b = reinterpret_cast<uintptr_t>(o.at);
        return at && o.at && a < b + o.bytes && b < a + bytes;
    }
};

// Whether `out` lies on any of the others. (Where it may be one of them, the caller leaves that one out if they are the same.)
template <size_t n>
bool lies_on(const Range& out, const Range (&others)[n])
{
    for (const Range& o : others)
        if (out.meets(o)) return true;
    return false;
}

Range unless_same(const Range& r, const void* out) { return r.at == out ? Range{nullptr, 0} : r; }

// Whether two sets of heads that lie alike, `apart` elements from one another, have an element in common: apart is then a sum
// of c[i] * stride[i], |c[i]| < size[i]. Each stride steps past the dimensions inside it (given largest first), so the
// coefficients are the quotients or next to them.
bool lie_on_each_other(int64_t apart, const int64_t* size, const int64_t* stride, int dims)
{
    if (dims == 0) return apart == 0;
    if (size[0] <= 1 || stride[0] == 0) return lie_on_each_other(apart, size + 1, stride + 1, dims - 1);
    const int64_t q = apart / stride[0];
    for (int64_t c = q - 1; c <= q + 1; ++c)
        if (c < size[0] && -c < size[0] && lie_on_each_other(apart - c * stride[0], size + 1, stride + 1, dims - 1)) return true;
    return false;
}

// From the first element of heads at these strides to behind the last.
Range rope_extent(const ssba_rope_desc& d, const void* at, const int64_t* s, int64_t es)
{
    return Range{at, (size_t)(((d.B - 1) * s[0] + (d.T - 1) * s[1] + (d.heads - 1) * s[2] + d.head_dim) * es)};
}

// Whether writing `out` may change an x that is still to be read: not where out is x, nor where they share nothing.
bool rope_overlaps(const ssba_rope_desc& d, const void* x, const int64_t* xs, const void* out, const int64_t* os, int64_t es)
{
    if (!rope_extent(d, x, xs, es).meets(rope_extent(d, out, os, es))) return false;
    int64_t size[4] = {d.B, d.T, d.heads, d.head_dim}, stride[4] = {os[0], os[1], os[2], 1};
    for (int i = 0; i < 3; ++i)
        if (xs[i] != os[i] && size[i] > 1) return true;
    if (x == out) return false;
    const int64_t bytes = (int64_t)(reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(x));
    if (bytes % es) return true;
    for (int i = 1; i < 4; ++i)
        for (int j = i; j > 0 && stride[j] > stride[j - 1]; --j) {
            std::swap(stride[j], stride[j - 1]);
            std::swap(size[j], size[j - 1]);
        }
    return lie_on_each_other(bytes / es, size, stride, 4);
}

int check_norm(const char* who, int32_t T, int32_t D, int32_t dtype)
{
    if (T < 0 || D <= 0) {
        set_error("%s: T=%d must be >= 0 and D=%d positive", who, T, D);
        return SSBA_ERR_INVALID;
    }
    if (dtype != SSBA_BF16 && dtype != SSBA_FP32) {
        set_error("%s: dtype %d: SSBA_BF16 and SSBA_FP32 are supported", who, dtype);
        return SSBA_ERR_INVALID;
    }
    if (D % 8 || D > SSBA_NORM_MAX_WIDTH) {
        set_error("%s: D=%d must be a multiple of 8 and at most %d", who, D, SSBA_NORM_MAX_WIDTH);
        return SSBA_ERR_UNSUPPORTED;
    }
    return SSBA_OK;
}

int check_linear(const char* who, const ssba_linear_desc* d)
{
    if (!d) return invalid(who, "null descriptor");
    if (d->T < 0 || d->N <= 0 || d->K <= 0) {
        set_error("%s: T=%d must be >= 0, N=%d and K=%d positive", who, d->T, d->N, d->K);
        return SSBA_ERR_INVALID;
    }
    if (d->dtype != SSBA_BF16 && d->dtype != SSBA_E4M3) {
        set_error("%s: dtype %d: SSBA_BF16 and SSBA_E4M3 are supported", who, d->dtype);
        return SSBA_ERR_INVALID;
    }
    if (d->act < SSBA_ACT_NONE || d->act > SSBA_ACT_SILU || (d->gated && d->act == SSBA_ACT_NONE)) {
        set_error("%s: unknown activation %d, or none of a gated product", who, d->act);
        return SSBA_ERR_INVALID;
    }
    if (d->N % 8 || d->K % (d->dtype == SSBA_E4M3 ? 16 : 8) || d->N > SSBA_LINEAR_MAX_WIDTH || d->K > SSBA_LINEAR_MAX_WIDTH ||
        d->T > SSBA_CACHE_MAX_ROWS) {
        set_error("%s: N=%d and K=%d must be multiples of 8 (K of 16 in e4m3) and at most %d, T=%d at most %d", who, d->N, d->K,
                  SSBA_LINEAR_MAX_WIDTH, d->T, SSBA_CACHE_MAX_ROWS);
        return SSBA_ERR_UNSUPPORTED;
    }
    return SSBA_OK;
}

// ssba_linear, and its test hook with a limit of its own and copies that never come.
int linear(const char* who, const ssba_linear_desc* desc, const void* x, const void* W, const float* x_scale,
           const float* w_scale, const float* bias, const void* r, void* y, void* z, void* stream, uint64_t budget_ns, int withhold)
{
    const int rc = check_linear(who, desc);
    if (rc != SSBA_OK) return rc;
    const bool f8 = desc->dtype == SSBA_E4M3;
    if ((x_scale != nullptr) != f8 || (w_scale != nullptr) != f8)
        return invalid(who, "x_scale and w_scale are given for e4m3 and for nothing else");
    if (desc->gated && (bias || r)) return invalid(who, "a gated product has no bias and no residual");
    if (desc->T == 0) return SSBA_OK;
    if (!x || !W || !y) return invalid(who, "x, W and y must be non-null");
    if (!aligned(x, 16) || !aligned(W, 16) || !aligned(w_scale, 16) || !aligned(bias, 16) || !aligned(r, 16) ||
        !aligned(y, 16) || !aligned(z, 16) || !aligned(x_scale, 4))
        return invalid(who, "x, W, w_scale, bias, r, y and z must be 16-byte aligned, x_scale 4-byte");
    const size_t T = desc->T, N = desc->N, K = desc->K, rows = desc->gated ? 2 * N : N, e = f8 ? 1 : 2;
    const Range X{x, T * K * e}, M{W, rows * K * e}, XS{x_scale, 4 * T}, WS{w_scale, 4 * rows}, B{bias, 4 * N}, R{r, T * N * 2}, Y{y, T * N * 2};
    if (lies_on(Y, {X, M, XS, WS, B, unless_same(R, y)}) || lies_on(Range{z, T * rows * 2}, {X, M, XS, WS, B, R, Y}))
        return invalid(who, "an output lies on another tensor of the call (y may be r)");
    const Product p{x, W, y, z, r, x_scale, w_scale, bias, desc->T, desc->N, desc->K, desc->act, f8, false, desc->gated != 0, budget_ns, withhold};
    return launch_product(p, who, static_cast<cudaStream_t>(stream));
}

}  // namespace
}  // namespace layer
}  // namespace ssba

using namespace ssba;
using namespace ssba::layer;

extern "C" {

int ssba_rms_norm(const void* x, const void* r, const float* w, int32_t T, int32_t D, int32_t dtype, float eps, void* h,
                  void* y, float* scale, float* rstd, void* stream)
{
    static const char who[] = "ssba_rms_norm";
    SSBA_NVTX_RANGE(who);
    const int rc = check_norm(who, T, D, dtype);
    if (rc != SSBA_OK) return rc;
    if (!(eps >= 0.f) || std::isinf(eps)) return invalid(who, "eps must be finite and >= 0");
    if ((r != nullptr) != (h != nullptr)) return invalid(who, "r and h come together");
    if (T == 0) return SSBA_OK;
    if (!x || !w || !y || !rstd) return invalid(who, "x, w, y and rstd must be non-null");
    if (!aligned(x, 16) || !aligned(r, 16) || !aligned(w, 16) || !aligned(h, 16) || !aligned(y, 16) || !aligned(scale, 4) ||
        !aligned(rstd, 4))
        return invalid(who, "x, r, w, h and y must be 16-byte aligned, scale and rstd 4-byte");
    const size_t rows = (size_t)T * D * (dtype == SSBA_BF16 ? 2 : 4), out = scale ? (size_t)T * D : rows, each = sizeof(float) * T;
    const Range X{x, rows}, R{r, rows}, W{w, sizeof(float) * D}, H{h, rows}, Y{y, out};
    if (lies_on(H, {unless_same(X, h), unless_same(R, h), W}) || lies_on(Y, {scale ? X : unless_same(X, y), R, W, H}) ||
        lies_on(Range{rstd, each}, {X, R, W, H, Y}) || lies_on(Range{scale, scale ? each : 0}, {X, R, W, H, Y, Range{rstd, each}}))
        return invalid(who, "an output lies on another tensor of the call (h may be x or r, and y of dtype x)");
    return launch_rms_norm(x, r, w, T, D, dtype, eps, h, y, scale != nullptr, scale, rstd, static_cast<cudaStream_t>(stream));
}

size_t ssba_rms_norm_backward_workspace_bytes(int32_t T, int32_t D, int32_t dtype)
{
    if (check_norm("ssba_rms_norm_backward_workspace_bytes", T, D, dtype) != SSBA_OK) return 0;
    return round256(sizeof(float) * D * (size_t)rms_norm_backward_parts(T, D, dtype));
}

int ssba_rms_norm_backward(const void* dy, const void* h, const float* w, const float* rstd, const void* dh, int32_t T,
                           int32_t D, int32_t dtype, void* dx, float* dw, void* workspace, size_t ws_bytes, void* stream)
{
    static const char who[] = "ssba_rms_norm_backward";
    SSBA_NVTX_RANGE(who);
    const int rc = check_norm(who, T, D, dtype);
    if (rc != SSBA_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!dw || !aligned(dw, 4)) return invalid(who, "dw must be non-null and 4-byte aligned");
    if (T == 0) {
        const cudaError_t e = cudaMemsetAsync(dw, 0, sizeof(float) * D, st);
        if (e == cudaSuccess) return SSBA_OK;
        cudaGetLastError();
        set_error("%s: %s", who, cudaGetErrorString(e));
        return SSBA_ERR_CUDA;
    }
    if (!dy || !h || !w || !rstd || !dx) return invalid(who, "dy, h, w, rstd and dx must be non-null");
    if (!aligned(dy, 16) || !aligned(h, 16) || !aligned(w, 16) || !aligned(dh, 16) || !aligned(dx, 16) || !aligned(rstd, 4))
        return invalid(who, "dy, h, w, dh and dx must be 16-byte aligned, rstd 4-byte");
    const size_t need = ssba_rms_norm_backward_workspace_bytes(T, D, dtype);
    if (!workspace || ws_bytes < need || !aligned(workspace, 16)) {
        set_error("%s: workspace of %zu bytes (16-byte aligned) required, got %zu", who, need, ws_bytes);
        return SSBA_ERR_WORKSPACE;
    }
    const size_t rows = (size_t)T * D * (dtype == SSBA_BF16 ? 2 : 4);
    const Range DY{dy, rows}, H{h, rows}, DH{dh, rows}, W{w, sizeof(float) * D}, K{rstd, sizeof(float) * T}, DX{dx, rows}, S{workspace, need};
    if (lies_on(DX, {unless_same(DY, dx), H, unless_same(DH, dx), W, K, S}) || lies_on(Range{dw, sizeof(float) * D}, {DY, H, DH, W, K, DX, S}) ||
        lies_on(S, {DY, H, DH, W, K}))
        return invalid(who, "an output or the workspace lies on another tensor of the call (dx may be dy or dh)");
    return launch_rms_norm_backward(dy, h, w, rstd, dh, T, D, dtype, dx, dw, static_cast<float*>(workspace), st);
}

int ssba_linear(const ssba_linear_desc* desc, const void* x, const void* W, const float* x_scale, const float* w_scale,
                const float* bias, const void* r, void* y, void* z, void* stream)
{
    SSBA_NVTX_RANGE("ssba_linear");
    return linear("ssba_linear", desc, x, W, x_scale, w_scale, bias, r, y, z, stream, kWaitBudgetNs, 0);
}

int ssba_test_linear_timeout(const ssba_linear_desc* desc, const void* x, const void* W, void* y, uint64_t budget_ns,
                             void* stream)
{
    SSBA_NVTX_RANGE("ssba_test_linear_timeout");
    if (!desc || desc->T <= 0 || desc->dtype != SSBA_BF16) return invalid("ssba_test_linear_timeout", "needs bf16 and at least one row");
    const uint64_t ns = budget_ns < 1000000ull ? 1000000ull : budget_ns > kWaitBudgetNs ? kWaitBudgetNs : budget_ns;
    return linear("ssba_test_linear_timeout", desc, x, W, nullptr, nullptr, nullptr, nullptr, y, nullptr, stream, ns, 1);
}

size_t ssba_linear_backward_workspace_bytes(const ssba_linear_desc* desc)
{
    if (check_linear("ssba_linear_backward_workspace_bytes", desc) != SSBA_OK) return 0;
    const size_t dz = desc->act == SSBA_ACT_NONE ? 0 : round256((size_t)desc->T * desc->N * (desc->gated ? 4 : 2));
    const size_t part = desc->gated || !desc->T ? 0 : round256(sizeof(float) * desc->N * (size_t)act_backward_parts(desc->T, desc->N));
    const size_t sums = desc->T && desc->dtype == SSBA_BF16 ? round256(gradients_workspace_bytes(desc->T, desc->gated ? 2 * desc->N : desc->N, desc->K)) : 0;
    return dz + part + sums;
}

int ssba_linear_backward(const ssba_linear_desc* desc, const void* dy, const void* x, const void* W, const void* z, void* dx,
                         void* dW, float* db, void* workspace, size_t ws_bytes, void* stream)
{
    static const char who[] = "ssba_linear_backward";
    SSBA_NVTX_RANGE(who);
    int rc = check_linear(who, desc);
    if (rc != SSBA_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool gated = desc->gated != 0, act = desc->act != SSBA_ACT_NONE;
    const int T = desc->T, N = desc->N, K = desc->K, rows = gated ? 2 * N : N;
    if (desc->dtype != SSBA_BF16) return invalid(who, "the gradients are those of bf16 products");
    if (gated && db) return invalid(who, "a gated product has no bias");
    if ((dx && !W) || (dW && !x && T)) return invalid(who, "dx needs W, and dW needs x");
    if (!aligned(dy, 16) || !aligned(x, 16) || !aligned(W, 16) || !aligned(z, 16) || !aligned(dx, 16) || !aligned(dW, 16) || !aligned(db, 4))
        return invalid(who, "dy, x, W, z, dx and dW must be 16-byte aligned, db 4-byte");
    if (T == 0) {
        cudaError_t e = dW ? cudaMemsetAsync(dW, 0, (size_t)rows * K * 2, st) : cudaSuccess;
        if (e == cudaSuccess && db) e = cudaMemsetAsync(db, 0, sizeof(float) * N, st);
        if (e == cudaSuccess) return SSBA_OK;
        cudaGetLastError();
        set_error("%s: %s", who, cudaGetErrorString(e));
        return SSBA_ERR_CUDA;
    }
    if (!dy || (act && !z)) return invalid(who, "dy, and z with an activation, must be non-null");
    const size_t need = ssba_linear_backward_workspace_bytes(desc);
    if (need && (!workspace || ws_bytes < need || !aligned(workspace, 16))) {
        set_error("%s: workspace of %zu bytes (16-byte aligned) required, got %zu", who, need, ws_bytes);
        return SSBA_ERR_WORKSPACE;
    }
    {
        const size_t t = T, n = N, k = K;
        const Range DY{dy, t * n * 2}, X{dW ? x : nullptr, t * k * 2}, M{dx ? W : nullptr, rows * k * 2}, Z{act ? z : nullptr, t * rows * 2};
        const Range DX{dx, t * k * 2}, DW{dW, rows * k * 2}, DB{db, 4 * n}, S{workspace, need};
        if (lies_on(DX, {DY, X, M, Z}) || lies_on(DW, {DY, X, M, Z, DX}) || lies_on(DB, {DY, X, M, Z, DX, DW}) ||
            lies_on(S, {DY, X, M, Z, DX, DW, DB}))
            return invalid(who, "an output or the workspace lies on another tensor of the call");
    }
    const void* dz = dy;
    const size_t dzb = act ? round256((size_t)T * rows * 2) : 0;
    const size_t part = gated ? 0 : round256(sizeof(float) * N * (size_t)act_backward_parts(T, N));
    if (act || db) {
        if (act) dz = workspace;
        rc = launch_act_backward(dy, z, act ? workspace : nullptr, db, db ? reinterpret_cast<float*>(static_cast<char*>(workspace) + dzb) : nullptr,
                                 T, N, desc->act, gated, who, st);
        if (rc != SSBA_OK) return rc;
    }
    if (dx || dW) rc = launch_gradients(dz, x, W, dx, dW, reinterpret_cast<float*>(static_cast<char*>(workspace) + dzb + part), T, rows, K, who, st);
    return rc;
}

int ssba_rope_axes(const ssba_rope_desc* desc, const void* x, const int64_t* x_stride, const int32_t* pos, int64_t pos_batch,
                   void* out, const int64_t* out_stride, void* stream)
{
    static const char who[] = "ssba_rope_axes";
    SSBA_NVTX_RANGE(who);
    if (!desc) return invalid(who, "null descriptor");
    const ssba_rope_desc& d = *desc;
    if (d.B < 0 || d.T < 0 || d.heads <= 0 || d.head_dim <= 0) {
        set_error("%s: B=%d and T=%d must be >= 0, heads=%d and head_dim=%d positive", who, d.B, d.T, d.heads, d.head_dim);
        return SSBA_ERR_INVALID;
    }
    if (d.dtype != SSBA_BF16 && d.dtype != SSBA_FP32) return invalid(who, "dtype must be SSBA_BF16 or SSBA_FP32");
    if (d.axes < 1 || d.axes > SSBA_ROPE_MAX_AXES) {
        set_error("%s: axes=%d must be 1..%d", who, d.axes, SSBA_ROPE_MAX_AXES);
        return SSBA_ERR_INVALID;
    }
    long long P = 0;
    for (int a = 0; a < d.axes; ++a) {
        if (d.sections[a] <= 0) return invalid(who, "every axis has at least one pair");
        P += d.sections[a];
    }
    if (2 * P > d.head_dim) {
        set_error("%s: the sections' %lld pairs do not fit head_dim=%d", who, P, d.head_dim);
        return SSBA_ERR_INVALID;
    }
    if (d.layout != SSBA_ROPE_PAIRS && d.layout != SSBA_ROPE_HALVES) return invalid(who, "unknown layout");
    if (!(d.base > 1.0) || std::isinf(d.base)) return invalid(who, "base must be finite and > 1");
    if (d.head_dim > SSBA_ROPE_MAX_HEAD_DIM || d.head_dim % 2 || (long long)d.B * d.T > (1ll << 30)) {
        set_error("%s: head_dim=%d must be even and at most %d, and B * T at most 2^30", who, d.head_dim, SSBA_ROPE_MAX_HEAD_DIM);
        return SSBA_ERR_UNSUPPORTED;
    }
    if (!x_stride || !out_stride) return invalid(who, "the strides must be non-null");
    const int64_t es = d.dtype == SSBA_BF16 ? 2 : 4;
    int64_t xs[3], os[3];  // a dimension of one has no stride
    const int32_t sizes[3] = {d.B, d.T, d.heads};
    for (int i = 0; i < 3; ++i) {
        xs[i] = sizes[i] > 1 ? x_stride[i] : 0;
        os[i] = sizes[i] > 1 ? out_stride[i] : 0;
        if (xs[i] < 0 || os[i] < 0 || xs[i] > (1ll << 42) || os[i] > (1ll << 42)) return invalid(who, "strides must be >= 0 and at most 2^42 elements");
    }
    if (pos_batch < 0) return invalid(who, "pos_batch must be >= 0");
    if (d.B == 0 || d.T == 0) return SSBA_OK;
    if (!x || !pos || !out) return invalid(who, "x, pos and out must be non-null");
    // adjacent pairs are read together
    const int64_t unit = d.layout == SSBA_ROPE_PAIRS ? 2 * es : es;
    bool fits = aligned(x, unit) && aligned(out, unit) && aligned(pos, 4);
    if (d.layout == SSBA_ROPE_PAIRS)
        for (int i = 0; i < 3; ++i) fits = fits && xs[i] % 2 == 0 && os[i] % 2 == 0;
    if (!fits) return invalid(who, "x and out must be aligned to an element (adjacent pairs: to a pair, strides too), pos to 4 bytes");
    if (rope_overlaps(d, x, xs, out, os, es)) return invalid(who, "out lies on x (it may be x with the same strides)");
    const Range positions{pos, sizeof(int32_t) * ((size_t)(d.B - 1) * (size_t)pos_batch + (size_t)d.T * d.axes)};
    if (rope_extent(d, out, os, es).meets(positions)) return invalid(who, "out lies on pos");
    return launch_rope(d, x, xs, pos, pos_batch, out, os, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
