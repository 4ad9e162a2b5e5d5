// linear_bwd.cu -- what stands between an output's gradient and the products of the backward pass:
//
//   dz = dy act'(z), db = sum_t dz           (ssba_linear_backward)
//   dg = dy u act'(g), du = dy act(g)        (gated: z = [g, u], dz = [dg, du])
//
// dz is rounded to bf16: the products behind it are bf16 ones, and dz in two bf16 parts would double them. dx and dW are then off by 2.3e-3
// of their norm, where their own rounding alone is 1.7e-3.
// Bound by HBM: z and dy are read once, 16 bytes a thread, and dz is written once. The bias's
// gradient sums dz in fp32 before that rounding: a CTA takes 256 columns of a run of rows (a warp a
// row, a lane 8 columns), its warps meet in shared memory, and the runs' sums (if more than one) in a second launch, in
// one order.
#include "layer.cuh"

namespace ssba {
namespace layer {
namespace {

using namespace ptx;

constexpr int kWarps = 8, kCols = 256, kCtas = 3;  // kCtas: of an SM

struct ActArgs {
    const uint4 *dy, *z;
    uint4* dz;    // null: not wanted (no activation)
    float* part;  // null: no sums
    int T, N, rows;  // rows of a CTA
    int act;
};

__device__ __forceinline__ void get8(const uint4& v, float* f)
{
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 p = unpack2(u[i]);
        f[2 * i] = p.x;
        f[2 * i + 1] = p.y;
    }
}

__device__ __forceinline__ uint4 put8(const float* f)
{
    return make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}

template <int kAct, bool kSum>
__global__ void __launch_bounds__(kWarps * 32, kCtas) ssba_act_bwd_kernel(const ActArgs p)
{
    __shared__ float sums[kSum ? kWarps : 1][kCols];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * kCols + lane * 8;
    grid_dep_wait();
    grid_dep_launch();
    const long long t1 = min((long long)p.T, ((long long)blockIdx.y + 1) * p.rows);
    float s[8] = {};
    if (c < p.N) {
        // four rows a round, all loads under way at once
        for (long long t = (long long)blockIdx.y * p.rows + warp; t < t1; t += 4 * kWarps) {
            uint4 dy[4], z[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool in = t + r * kWarps < t1;
                const size_t i = ((size_t)(t + r * kWarps) * p.N + c) / 8;
                dy[r] = in ? p.dy[i] : make_uint4(0, 0, 0, 0);
                if (kAct != SSBA_ACT_NONE) z[r] = in ? p.z[i] : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float d[8];
                get8(dy[r], d);
                if (kAct != SSBA_ACT_NONE) {
                    float f[8];
                    get8(z[r], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float v;
                        d[e] *= act_slope<kAct>(f[e], v);
                    }
                    if (t + r * kWarps < t1) p.dz[((size_t)(t + r * kWarps) * p.N + c) / 8] = put8(d);
                }
                if (kSum) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += d[e];
                }
            }
        }
    }
    if (kSum) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[warp][lane * 8 + e] = s[e];
        __syncthreads();
        const int col = blockIdx.x * kCols + threadIdx.x;
        if (col < p.N) {
            float a = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) a += sums[w][threadIdx.x];
            p.part[(size_t)blockIdx.y * p.N + col] = a;
        }
    }
}

template <int kAct>
__global__ void __launch_bounds__(256) ssba_gated_bwd_kernel(const ActArgs p)
{
    grid_dep_wait();
    grid_dep_launch();
    const int n8 = p.N / 8;
    const long long all = (long long)p.T * n8;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long long)gridDim.x * 256) {
        const long long t = i / n8, c = i - t * n8, at = t * 2 * n8 + c;
        float d[8], g[8], u[8];
        get8(p.dy[i], d);
        get8(p.z[at], g);
        get8(p.z[at + n8], u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v;
            const float k = act_slope<kAct>(g[e], v);
            g[e] = d[e] * u[e] * k;
            u[e] = d[e] * v;
        }
        p.dz[at] = put8(g);
        p.dz[at + n8] = put8(u);
    }
}

int rows_of(int T, int N)
{
    // runs of rows, as many as run at once, of 32 rows at least; up to 128 rows one, whose sums need no join
    if (T <= 128) return T > 0 ? T : 1;
    const long long wide = (N + kCols - 1) / kCols, most = (long long)kCtas * device_sm_count();
    long long runs = most / wide;
    if (runs < 1) runs = 1;
    long long rows = (T + runs - 1) / runs;
    return (int)(rows < 32 ? 32 : rows);
}

int launched(cudaError_t e, const char* who)
{
    if (e == cudaSuccess) return SSBA_OK;
    set_error("%s: launch of the activation's backward: %s", who, cudaGetErrorString(e));
    return SSBA_ERR_CUDA;
}

}  // namespace

int act_backward_parts(int T, int N) { return (T + rows_of(T, N) - 1) / rows_of(T, N); }

int launch_act_backward(const void* dy, const void* z, void* dz, float* db, float* part, int T, int N, int act, bool gated,
                        const char* who, cudaStream_t st)
{
    const int parts = act_backward_parts(T, N);
    const ActArgs p{static_cast<const uint4*>(dy), static_cast<const uint4*>(z), static_cast<uint4*>(dz), parts == 1 ? db : part, T, N, rows_of(T, N), act};
    if (gated) {
        const long long ctas = ((long long)T * (N / 8) + 255) / 256, most = 32ll * device_sm_count();
        const dim3 grid((unsigned)(ctas < most ? ctas : most));
        auto go = [&](auto k) { return launched(launch_early(k, grid, 256, 0, st, 1, p), who); };
        if (act == SSBA_ACT_SILU) return go(ssba_gated_bwd_kernel<SSBA_ACT_SILU>);
        return act == SSBA_ACT_GELU ? go(ssba_gated_bwd_kernel<SSBA_ACT_GELU>) : go(ssba_gated_bwd_kernel<SSBA_ACT_RELU>);
    }
    const dim3 grid((N + kCols - 1) / kCols, parts);
    auto go = [&](auto k) { return launched(launch_early(k, grid, kWarps * 32, 0, st, 1, p), who); };
    int rc;
    if (act == SSBA_ACT_NONE)
        rc = go(ssba_act_bwd_kernel<SSBA_ACT_NONE, true>);
    else if (act == SSBA_ACT_RELU)
        rc = db ? go(ssba_act_bwd_kernel<SSBA_ACT_RELU, true>) : go(ssba_act_bwd_kernel<SSBA_ACT_RELU, false>);
    else if (act == SSBA_ACT_GELU)
        rc = db ? go(ssba_act_bwd_kernel<SSBA_ACT_GELU, true>) : go(ssba_act_bwd_kernel<SSBA_ACT_GELU, false>);
    else
        rc = db ? go(ssba_act_bwd_kernel<SSBA_ACT_SILU, true>) : go(ssba_act_bwd_kernel<SSBA_ACT_SILU, false>);
    return rc == SSBA_OK && db && parts > 1 ? launch_column_sum(part, parts, N, db, who, st) : rc;
}

}  // namespace layer
}  // namespace ssba
