// C ABI of the paged cache: argument validation, default resolution, dispatch.
#include <limits.h>
#include <math.h>

#include "hs2_paged.cuh"

namespace hs2 {
namespace {

// Validate the host-visible part of a paged problem and resolve defaults.
hs2_status resolve(const hs2_paged_problem *hp, PagedParams *out)
{
    if (!hp) return HS2_ERR_INVALID_ARG;
    if (hp->batch <= 0 || hp->n_kv_heads <= 0 || hp->n_q_heads <= 0 || hp->n_q_heads % hp->n_kv_heads != 0) return HS2_ERR_INVALID_ARG;
    if (hp->head_dim <= 0 || hp->page_size <= 0 || hp->n_pages <= 0 || hp->max_pages <= 0) return HS2_ERR_INVALID_ARG;
    if ((int64_t)hp->max_pages * hp->page_size > INT_MAX) return HS2_ERR_INVALID_ARG;
    if (hp->window < 0 || hp->n_first < 0) return HS2_ERR_INVALID_ARG;
    if (hp->dtype != HS2_F32 && hp->dtype != HS2_BF16) return HS2_ERR_INVALID_ARG;
    if (!(hp->softmax_scale >= 0.f) || isinf(hp->softmax_scale)) return HS2_ERR_INVALID_ARG;
    if (hp->table_stride < 0 || (hp->table_stride > 0 && hp->table_stride < hp->max_pages)) return HS2_ERR_INVALID_ARG;
    if (!hp->page_table || !hp->kv_lens) return HS2_ERR_INVALID_ARG;
    if ((int64_t)hp->max_pages * hp->page_size > kMaxIndex) return HS2_ERR_UNSUPPORTED;
    if (hp->head_dim > 256 || hp->batch > 65535 || hp->n_q_heads > 65535) return HS2_ERR_UNSUPPORTED;
    PagedParams p{};
    p.B = hp->batch; p.Hq = hp->n_q_heads; p.Hkv = hp->n_kv_heads; p.G = p.Hq / p.Hkv; p.D = hp->head_dim;
    p.ps = hp->page_size; p.n_pages = hp->n_pages; p.max_pages = hp->max_pages;
    p.max_len = hp->max_pages * hp->page_size;
    p.w = hp->window > 0 ? hp->window : INT_MAX;
    p.nf = hp->n_first;
    p.scale = hp->softmax_scale > 0.f ? hp->softmax_scale : 1.0f / sqrtf((float)p.D);
    p.scale_log2 = fmaxf(p.scale * kLog2e, 0x1p-126f);   // normal: -inf times a scale that is flushed to 0 would be NaN
    p.table = hp->page_table;
    p.table_stride = hp->table_stride > 0 ? hp->table_stride : hp->max_pages;
    p.kv_lens = hp->kv_lens;
    auto pair = [&](const int64_t s[2], int64_t &sb, int64_t &sh) {
        if (s[0] == 0 && s[1] == 0) { sh = p.D; sb = (int64_t)p.Hq * p.D; return true; }
        sb = s[0]; sh = s[1];
        return sb >= 0 && (sh >= p.D || p.Hq == 1);
    };
    if (!pair(hp->q_stride, p.qs_b, p.qs_h) || !pair(hp->o_stride, p.os_b, p.os_h)) return HS2_ERR_INVALID_ARG;
    const int64_t *k = hp->kv_stride;
    if (k[0] == 0 && k[1] == 0 && k[2] == 0) { p.ks_h = p.D; p.ks_t = (int64_t)p.Hkv * p.D; p.ks_p = p.ps * p.ks_t; }
    else if (k[0] >= 0 && k[1] >= 0 && (k[2] >= p.D || p.Hkv == 1)) { p.ks_p = k[0]; p.ks_t = k[1]; p.ks_h = k[2]; }
    else return HS2_ERR_INVALID_ARG;
    const int64_t *c = hp->kv_scale_stride;
    if (c[0] == 0 && c[1] == 0 && c[2] == 0) { p.ss_h = 1; p.ss_t = p.Hkv; p.ss_p = (int64_t)p.ps * p.Hkv; }
    else if (c[0] >= 0 && c[1] >= 0 && (c[2] >= 1 || p.Hkv == 1)) { p.ss_p = c[0]; p.ss_t = c[1]; p.ss_h = c[2]; }
    else return HS2_ERR_INVALID_ARG;
    *out = p;
    return HS2_OK;
}

bool ws_ok(const void *ws, size_t ws_bytes, size_t need)
{
    return need == 0 || (ws != nullptr && ws_bytes >= need && reinterpret_cast<uintptr_t>(ws) % 256 == 0);
}

size_t ws_need(PagedParams p)
{
    size_t most = 0;   // the cache may be of either format
    for (int fp8 = 0; fp8 < 2; ++fp8) {
        paged_plan(&p, fp8 != 0);
        if (paged_ws_bytes(p) > most) most = paged_ws_bytes(p);
    }
    return most;
}

hs2_status run(PagedParams &p, hs2_dtype dt, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc,
               const float *sink, const void *gate, void *O, float *LSE, void *ws, size_t ws_bytes, void *cuda_stream)
{
    if (!Q || !K || !V || !O) return HS2_ERR_INVALID_ARG;
    p.sink = sink;
    p.gate = gate;
    if (!ws_ok(ws, ws_bytes, ws_need(p))) return HS2_ERR_WORKSPACE_TOO_SMALL;
    const hs2_status s = check_device();
    if (s != HS2_OK) return s;
    paged_plan(&p, ksc != nullptr);
    const cudaError_t e = launch_paged_decode(p, dt, Q, K, V, ksc, vsc, O, LSE, ws, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? HS2_OK : cuda_fail(e);
}

hs2_status check_pool(const hs2_page_pool *pool, int32_t n = 0)
{
    if (!pool || pool->n_pages <= 0 || pool->page_size <= 0 || pool->max_seqs <= 0 || pool->max_pages <= 0) return HS2_ERR_INVALID_ARG;
    if ((int64_t)pool->max_pages * pool->page_size > INT_MAX) return HS2_ERR_INVALID_ARG;
    if (!pool->ref_counts || !pool->page_table || !pool->lens) return HS2_ERR_INVALID_ARG;
    if ((int64_t)pool->max_pages * pool->page_size > kMaxIndex || pool->n_pages > kMaxIndex || pool->max_seqs > kMaxIndex) return HS2_ERR_UNSUPPORTED;
    if (n > kMaxList) return HS2_ERR_UNSUPPORTED;
    return HS2_OK;
}

hs2_status check_regions(const hs2_page_pool &pool, const hs2_page_region *regions, int32_t n, PageRegions *out)
{
    if (n < 0 || n > HS2_MAX_PAGE_REGIONS || (n > 0 && !regions)) return HS2_ERR_INVALID_ARG;
    out->n = n;
    for (int i = 0; i < n; ++i) {
        const hs2_page_region &g = regions[i];
        if (!g.base || reinterpret_cast<uintptr_t>(g.base) % 4 || g.n_layers < 1 || g.row_bytes <= 0 || g.row_bytes % 4) return HS2_ERR_INVALID_ARG;
        if (g.token_stride < g.row_bytes || g.token_stride % 4 || g.page_stride % 4) return HS2_ERR_INVALID_ARG;
        if (g.page_stride < (pool.page_size - 1) * g.token_stride + g.row_bytes) return HS2_ERR_INVALID_ARG;
        if (g.n_layers > 1 && (g.layer_stride % 4 || g.layer_stride <= 0)) return HS2_ERR_INVALID_ARG;
        out->r[i] = g;
        if (g.n_layers == 1) out->r[i].layer_stride = 0;
    }
    return HS2_OK;
}

}  // namespace
}  // namespace hs2

using namespace hs2;

extern "C" {

size_t hs2_paged_workspace_bytes(const hs2_paged_problem *hp)
{
    PagedParams p;
    if (resolve(hp, &p) != HS2_OK) return 0;
    return ws_need(p);
}

hs2_status hs2_paged_attn_decode(const hs2_paged_problem *hp, const void *Q, const void *K, const void *V, const float *sink,
                                 const void *gate, void *O, float *LSE, void *ws, size_t ws_bytes, void *cuda_stream)
{
    PagedParams p;
    const hs2_status s = resolve(hp, &p);
    if (s != HS2_OK) return s;
    return run(p, hp->dtype, Q, K, V, nullptr, nullptr, sink, gate, O, LSE, ws, ws_bytes, cuda_stream);
}

hs2_status hs2_paged_attn_decode_fp8kv(const hs2_paged_problem *hp, const void *Q, const void *K8, const void *V8,
                                       const float *k_scale, const float *v_scale, const float *sink, const void *gate,
                                       void *O, float *LSE, void *ws, size_t ws_bytes, void *cuda_stream)
{
    PagedParams p;
    const hs2_status s = resolve(hp, &p);
    if (s != HS2_OK) return s;
    if (!k_scale || !v_scale) return HS2_ERR_INVALID_ARG;
    if (hp->dtype != HS2_BF16) return HS2_ERR_UNSUPPORTED;
    return run(p, hp->dtype, Q, K8, V8, k_scale, v_scale, sink, gate, O, LSE, ws, ws_bytes, cuda_stream);
}

size_t hs2_pages_workspace_bytes(const hs2_page_pool *pool, int32_t n)
{
    return check_pool(pool, n) != HS2_OK || n < 0 ? 0 : pages_ws_bytes(*pool, n);
}

hs2_status hs2_pages_reserve(const hs2_page_pool *pool, const hs2_page_region *regions, int32_t n_regions,
                             const int32_t *seqs, const int32_t *n_new, int32_t n, int32_t *start, void *ws,
                             size_t ws_bytes, void *cuda_stream)
{
    hs2_status s = check_pool(pool, n);
    PageRegions rg;
    if (s != HS2_OK || (s = check_regions(*pool, regions, n_regions, &rg)) != HS2_OK) return s;
    if (n < 0 || (n > 0 && (!seqs || !n_new || !start))) return HS2_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, pages_ws_bytes(*pool, n))) return HS2_ERR_WORKSPACE_TOO_SMALL;
    if ((s = check_device()) != HS2_OK) return s;
    const cudaError_t e = launch_pages_reserve(*pool, rg, seqs, n_new, n, start, ws, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? HS2_OK : cuda_fail(e);
}

hs2_status hs2_pages_write(const hs2_page_pool *pool, const hs2_page_region *regions, int32_t n_regions,
                           const void *const *rows, const int64_t *row_strides, const int32_t *seqs, const int32_t *start,
                           const int32_t *n_new, int32_t n, int32_t max_new, void *cuda_stream)
{
    hs2_status s = check_pool(pool, n);
    PageRegions rg;
    if (s != HS2_OK || (s = check_regions(*pool, regions, n_regions, &rg)) != HS2_OK) return s;
    if (n < 0 || max_new < 0 || (n > 0 && (!seqs || !start || !n_new)) || (n_regions > 0 && (!rows || !row_strides))) return HS2_ERR_INVALID_ARG;
    for (int r = 0; r < n_regions; ++r) {
        if (!rows[r] || reinterpret_cast<uintptr_t>(rows[r]) % 4) return HS2_ERR_INVALID_ARG;
        for (int k = 0; k < 3; ++k)
            if (row_strides[3 * r + k] % 4) return HS2_ERR_INVALID_ARG;
    }
    if (max_new > kMaxIndex) return HS2_ERR_UNSUPPORTED;
    if ((s = check_device()) != HS2_OK) return s;
    const cudaError_t e = launch_pages_write(*pool, rg, rows, row_strides, seqs, start, n_new, n, max_new, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? HS2_OK : cuda_fail(e);
}

hs2_status hs2_pages_fork(const hs2_page_pool *pool, const int32_t *src, const int32_t *dst, int32_t n, void *ws,
                          size_t ws_bytes, void *cuda_stream)
{
    hs2_status s = check_pool(pool, n);
    if (s != HS2_OK) return s;
    if (n < 0 || (n > 0 && (!src || !dst))) return HS2_ERR_INVALID_ARG;
    if (!ws_ok(ws, ws_bytes, pages_ws_bytes(*pool, n))) return HS2_ERR_WORKSPACE_TOO_SMALL;
    if ((s = check_device()) != HS2_OK) return s;
    const cudaError_t e = launch_pages_fork(*pool, src, dst, n, ws, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? HS2_OK : cuda_fail(e);
}

hs2_status hs2_pages_free(const hs2_page_pool *pool, const int32_t *seqs, const int32_t *keep, int32_t n, void *cuda_stream)
{
    hs2_status s = check_pool(pool, n);
    if (s != HS2_OK) return s;
    if (n < 0 || (n > 0 && !seqs)) return HS2_ERR_INVALID_ARG;
    if ((s = check_device()) != HS2_OK) return s;
    const cudaError_t e = launch_pages_free(*pool, seqs, keep, n, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? HS2_OK : cuda_fail(e);
}

hs2_status hs2_pages_compact(const hs2_page_pool *pool, const hs2_page_region *regions, int32_t n_regions, int32_t *moved,
                             void *ws, size_t ws_bytes, void *cuda_stream)
{
    hs2_status s = check_pool(pool);
    PageRegions rg;
    if (s != HS2_OK || (s = check_regions(*pool, regions, n_regions, &rg)) != HS2_OK) return s;
    if (!ws_ok(ws, ws_bytes, pages_ws_bytes(*pool, 0))) return HS2_ERR_WORKSPACE_TOO_SMALL;
    if ((s = check_device()) != HS2_OK) return s;
    const cudaError_t e = launch_pages_compact(*pool, rg, moved, ws, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? HS2_OK : cuda_fail(e);
}

hs2_status hs2_pages_copy(const hs2_page_pool *pool, const hs2_page_region *regions, int32_t n_regions, const int32_t *src,
                          const int32_t *dst, int32_t n, void *cuda_stream)
{
    hs2_status s = check_pool(pool, n);
    PageRegions rg;
    if (s != HS2_OK || (s = check_regions(*pool, regions, n_regions, &rg)) != HS2_OK) return s;
    if (n < 0 || (n > 0 && (!src || !dst))) return HS2_ERR_INVALID_ARG;
    if ((s = check_device()) != HS2_OK) return s;
    const cudaError_t e = launch_pages_copy(*pool, rg, src, dst, n, (cudaStream_t)cuda_stream);
    return e == cudaSuccess ? HS2_OK : cuda_fail(e);
}

}  // extern "C"
