// cache_api.cu -- the entry points of the paged 8-bit cache (include/ssba.h): argument validation on the
// host and kernel launches on the caller's stream.
#include <algorithm>
#include <climits>
#include <cmath>

#include "cache.cuh"

namespace ssba {
namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_cache_desc(const ssba_cache_desc* d, const char* who)
{
    if (!d) {
        set_error("%s: null descriptor", who);
        return SSBA_ERR_INVALID;
    }
    if (d->heads <= 0 || d->kv_heads <= 0 || d->pages <= 0 || d->head_dim <= 0) {
        set_error("%s: sizes must be positive (heads=%d kv_heads=%d head_dim=%d pages=%d)", who, d->heads, d->kv_heads,
                  d->head_dim, d->pages);
        return SSBA_ERR_INVALID;
    }
    if (d->heads % d->kv_heads) {
        set_error("%s: heads=%d must be a multiple of kv_heads=%d", who, d->heads, d->kv_heads);
        return SSBA_ERR_INVALID;
    }
    if (d->dtype != SSBA_BF16 && d->dtype != SSBA_FP32) {
        set_error("%s: unknown dtype %d", who, d->dtype);
        return SSBA_ERR_INVALID;
    }
    if (!(d->softmax_scale >= 0.f) || std::isinf(d->softmax_scale)) {
        set_error("%s: softmax_scale must be finite and >= 0 (0 = 1/sqrt(head_dim))", who);
        return SSBA_ERR_INVALID;
    }
    if (d->head_dim != 64 && d->head_dim != 128) {
        set_error("%s: head_dim=%d: 64 and 128 are supported", who, d->head_dim);
        return SSBA_ERR_UNSUPPORTED;
    }
    if (d->heads > SSBA_CACHE_MAX_HEADS || (long long)d->pages * d->kv_heads > INT_MAX) {
        set_error("%s: at most %d heads and %d pages times kv_heads", who, SSBA_CACHE_MAX_HEADS, INT_MAX);
        return SSBA_ERR_UNSUPPORTED;
    }
    return SSBA_OK;
}

int check_cache(const ssba_cache* c, const char* who)
{
    if (!c || !c->K || !c->V || !c->k_scale || !c->v_scale || !c->k_mean) {
        set_error("%s: the cache and its buffers must be non-null", who);
        return SSBA_ERR_INVALID;
    }
    if (!aligned(c->K, 128) || !aligned(c->V, 128) || !aligned(c->k_mean, 16) || !aligned(c->k_scale, 4) ||
        !aligned(c->v_scale, 4)) {
        set_error("%s: K and V must be 128-byte aligned, k_mean 16-byte, the scales 4-byte", who);
        return SSBA_ERR_INVALID;
    }
    return SSBA_OK;
}

int check_batch(int32_t T, const int32_t* table, int32_t width, const int32_t* lens, const int32_t* cu, int32_t B,
                const char* who)
{
    if (T < 0 || B < 0 || width <= 0) {
        set_error("%s: T=%d and B=%d must be >= 0, width=%d positive", who, T, B, width);
        return SSBA_ERR_INVALID;
    }
    if (T > SSBA_CACHE_MAX_ROWS || B > SSBA_CACHE_MAX_ROWS || width > INT_MAX / 2 / SSBA_CACHE_PAGE) {
        set_error("%s: at most %d rows and sequences and %d pages a sequence", who, SSBA_CACHE_MAX_ROWS,
                  INT_MAX / 2 / SSBA_CACHE_PAGE);
        return SSBA_ERR_UNSUPPORTED;
    }
    if (T > 0 && B > 0 && (!table || !lens || !cu || !aligned(table, 4) || !aligned(lens, 4) || !aligned(cu, 4))) {
        set_error("%s: table, lens and cu must be non-null and 4-byte aligned", who);
        return SSBA_ERR_INVALID;
    }
    return SSBA_OK;
}

bool make_pool(const ssba_cache_desc* d, const ssba_cache* c, const char* who, cache::Pool* p)
{
    p->K = static_cast<uint8_t*>(c->K);
    p->V = static_cast<uint8_t*>(c->V);
    p->k_scale = c->k_scale;
    p->v_scale = c->v_scale;
    p->k_mean = c->k_mean;
    p->pages = d->pages;
    p->heads = d->heads;
    p->kv_heads = d->kv_heads;
    p->status = device_status_word();
    if (!p->status) set_error("%s: the device status word cannot be reached", who);
    return p->status != nullptr;
}

// ssba_cache_attend, and its test hook with a limit of its own and copies that never come.
int attend(const char* who, const ssba_cache_desc* desc, const ssba_cache* cache, const void* q, int32_t T,
           const int32_t* table, int32_t width, const int32_t* lens, const int32_t* cu, int32_t B, const int32_t* idx,
           const int32_t* cnt, int32_t keep, void* O, float* lse, void* workspace, size_t ws_bytes, void* stream,
           uint64_t budget_ns, int withhold)
{
    int rc = check_cache_desc(desc, who);
    if (rc == SSBA_OK) rc = check_cache(cache, who);
    if (rc == SSBA_OK) rc = check_batch(T, table, width, lens, cu, B, who);
    if (rc != SSBA_OK) return rc;
    if ((idx != nullptr) != (cnt != nullptr) || (idx && (keep <= 0 || keep > SSBA_CACHE_MAX_WIDTH)) ||
        !aligned(idx, 4) || !aligned(cnt, 4)) {
        set_error("%s: idx and cnt come together, 4-byte aligned, with 0 < keep <= %d", who, SSBA_CACHE_MAX_WIDTH);
        return SSBA_ERR_INVALID;
    }
    if (T == 0 || B == 0) return SSBA_OK;
    if (!q || !O || !lse || !aligned(q, 16) || !aligned(O, 32) || !aligned(lse, 4)) {
        set_error("%s: q, O and lse must be non-null, q 16-byte and O 32-byte aligned", who);
        return SSBA_ERR_INVALID;
    }
    const size_t need = ssba_cache_attend_workspace_bytes(desc);
    if (!workspace || ws_bytes < need || !aligned(workspace, 16)) {
        set_error("%s: workspace of %zu bytes (16-byte aligned) required, got %zu", who, need, ws_bytes);
        return SSBA_ERR_WORKSPACE;
    }
    cache::Pool p;
    if (!make_pool(desc, cache, who, &p)) return SSBA_ERR_CUDA;
    const float scale = desc->softmax_scale > 0.f ? desc->softmax_scale : 1.0f / std::sqrt((float)desc->head_dim);
    const cache::Batch bt{table, lens, cu, B, width, T};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (desc->dtype == SSBA_BF16) {
        // Rows that share a K/V head's tokens, on average over the batch's sequences: up to 16, which are the columns of one
        // item, as columns of products over the bytes, bound by HBM; more as rows of fp16 products. (16 sequences of
        // up to 8000 tokens, 8 K/V heads of 128: 16 rows 57 us as columns, 72 as rows; 32 rows 86, 73; 64 rows 137, 74;
        // 128 rows 250, 106. One of 30000 tokens: 32 rows 34, 35; 64 rows 46, 39. 24 heads of 64, two of 2000: 32 rows 24, 19.)
        const long long rows = ((long long)T + B - 1) / B * (desc->heads / desc->kv_heads);
        if (!idx && rows > 16)
            return launch_cache_attend_rows(p, bt, desc->head_dim, scale, q, O, lse, workspace, st, budget_ns, withhold);
        return launch_cache_attend_tc(p, bt, desc->head_dim, scale, q, idx, cnt, keep, O, lse, workspace, st, budget_ns, withhold);
    }
    return launch_cache_attend_simt(p, bt, desc->head_dim, scale, q, idx, cnt, keep, O, lse, workspace, st);
}

}  // namespace
}  // namespace ssba

using namespace ssba;

extern "C" {

int ssba_cache_append(const ssba_cache_desc* desc, const ssba_cache* cache, const void* k, const void* v, int32_t T,
                      const int32_t* table, int32_t width, const int32_t* lens, const int32_t* cu, int32_t B,
                      void* stream)
{
    SSBA_NVTX_RANGE("ssba_cache_append");
    const char* who = "ssba_cache_append";
    int rc = check_cache_desc(desc, who);
    if (rc == SSBA_OK) rc = check_cache(cache, who);
    if (rc == SSBA_OK) rc = check_batch(T, table, width, lens, cu, B, who);
    if (rc != SSBA_OK) return rc;
    if (T == 0 || B == 0) return SSBA_OK;
    if (!k || !v || !aligned(k, 16) || !aligned(v, 16)) {
        set_error("%s: k and v must be non-null and 16-byte aligned", who);
        return SSBA_ERR_INVALID;
    }
    cache::Pool p;
    if (!make_pool(desc, cache, who, &p)) return SSBA_ERR_CUDA;
    return launch_cache_append(p, cache::Batch{table, lens, cu, B, width, T}, desc->head_dim, desc->dtype, k, v,
                               static_cast<cudaStream_t>(stream));
}

int ssba_cache_select(const ssba_cache_desc* desc, const ssba_cache* cache, const void* q, int32_t T,
                      const int32_t* table, int32_t width, const int32_t* lens, const int32_t* cu, int32_t B,
                      int32_t keep, int32_t first, int32_t* idx, int32_t* cnt, void* stream)
{
    SSBA_NVTX_RANGE("ssba_cache_select");
    const char* who = "ssba_cache_select";
    int rc = check_cache_desc(desc, who);
    if (rc == SSBA_OK) rc = check_cache(cache, who);
    if (rc == SSBA_OK) rc = check_batch(T, table, width, lens, cu, B, who);
    if (rc != SSBA_OK) return rc;
    if (first < 0 || keep <= first || keep > SSBA_CACHE_MAX_WIDTH) {
        set_error("%s: keep=%d must be more than first=%d (the last page is kept too), first >= 0, keep at most %d", who,
                  keep, first, SSBA_CACHE_MAX_WIDTH);
        return SSBA_ERR_INVALID;
    }
    if (width > SSBA_CACHE_MAX_WIDTH || (long long)(desc->heads / desc->kv_heads) * desc->head_dim > 16384) {
        set_error("%s: at most %d pages a sequence and 16384 channels a group", who, SSBA_CACHE_MAX_WIDTH);
        return SSBA_ERR_UNSUPPORTED;
    }
    if (T == 0 || B == 0) return SSBA_OK;
    if (!q || !idx || !cnt || !aligned(q, 16) || !aligned(idx, 4) || !aligned(cnt, 4)) {
        set_error("%s: q, idx and cnt must be non-null, q 16-byte aligned, the others 4-byte", who);
        return SSBA_ERR_INVALID;
    }
    cache::Pool p;
    if (!make_pool(desc, cache, who, &p)) return SSBA_ERR_CUDA;
    return launch_cache_select(p, cache::Batch{table, lens, cu, B, width, T}, desc->head_dim, desc->dtype, q, keep,
                               first, idx, cnt, static_cast<cudaStream_t>(stream));
}

size_t ssba_cache_attend_workspace_bytes(const ssba_cache_desc* desc)
{
    if (check_cache_desc(desc, "ssba_cache_attend_workspace_bytes") != SSBA_OK) return 0;
    const size_t n = std::max(cache_attend_simt_workspace(), cache_attend_tc_workspace());
    return (std::max(n, cache_attend_rows_workspace()) + 255) & ~(size_t)255;
}

int ssba_cache_attend(const ssba_cache_desc* desc, const ssba_cache* cache, const void* q, int32_t T,
                      const int32_t* table, int32_t width, const int32_t* lens, const int32_t* cu, int32_t B,
                      const int32_t* idx, const int32_t* cnt, int32_t keep, void* O, float* lse, void* workspace,
                      size_t ws_bytes, void* stream)
{
    SSBA_NVTX_RANGE("ssba_cache_attend");
    return attend("ssba_cache_attend", desc, cache, q, T, table, width, lens, cu, B, idx, cnt, keep, O, lse, workspace,
                  ws_bytes, stream, kWaitBudgetNs, 0);
}

int ssba_test_cache_timeout(const ssba_cache_desc* desc, const ssba_cache* cache, const void* q, int32_t T,
                            const int32_t* table, int32_t width, const int32_t* lens, const int32_t* cu, int32_t B,
                            void* O, float* lse, void* workspace, size_t ws_bytes, uint64_t budget_ns, void* stream)
{
    SSBA_NVTX_RANGE("ssba_test_cache_timeout");
    if (desc && desc->dtype != SSBA_BF16) {
        set_error("ssba_test_cache_timeout: bf16 only");
        return SSBA_ERR_UNSUPPORTED;
    }
    const uint64_t limit = std::min<uint64_t>(std::max<uint64_t>(budget_ns, 1000000ull), kWaitBudgetNs);
    return attend("ssba_test_cache_timeout", desc, cache, q, T, table, width, lens, cu, B, nullptr, nullptr, 0, O, lse,
                  workspace, ws_bytes, stream, limit, 1);
}

int ssba_cache_copy(const ssba_cache_desc* desc, const ssba_cache* cache, const int32_t* src, const int32_t* dst,
                    int32_t n, void* stream)
{
    SSBA_NVTX_RANGE("ssba_cache_copy");
    const char* who = "ssba_cache_copy";
    int rc = check_cache_desc(desc, who);
    if (rc == SSBA_OK) rc = check_cache(cache, who);
    if (rc != SSBA_OK) return rc;
    if (n < 0 || (n > 0 && (!src || !dst || !aligned(src, 4) || !aligned(dst, 4)))) {
        set_error("%s: n=%d must be >= 0, src and dst non-null and 4-byte aligned", who, n);
        return SSBA_ERR_INVALID;
    }
    if (n == 0) return SSBA_OK;
    cache::Pool p;
    if (!make_pool(desc, cache, who, &p)) return SSBA_ERR_CUDA;
    return launch_cache_copy(p, desc->head_dim, src, dst, n, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
