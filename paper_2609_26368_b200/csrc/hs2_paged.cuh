// Internal declarations of the paged decode attention: validated parameters, the visible keys of a sequence, the rule
// that splits them, and the launchers.
#pragma once

#include <atomic>

#include "hs2_common.cuh"

namespace hs2 {

// Lengths, capacities and counts of pages and sequences end here: an index in tiles, or one grid further on, then stays in int32.
constexpr int64_t kMaxIndex = (1ll << 31) - (1ll << 22);
constexpr int32_t kMaxList = 1 << 30;   // entries of a list of sequences or pages

// One new token per sequence against a cache in pages.  table == nullptr: page b is sequence b itself (a contiguous
// cache of ps tokens per sequence).
struct PagedParams {
    int B, Hq, Hkv, G, D;
    int ps, n_pages, max_pages;
    int max_len;                // longest context the table can hold
    int w, nf;                  // window (INT_MAX: everything) and first tokens
    float scale, scale_log2;
    const int32_t *table;
    int64_t table_stride;
    const int32_t *kv_lens;     // or nullptr: max_len
    const int32_t *q_start;     // or nullptr: the query is the last token
    int64_t qs_b, qs_h, os_b, os_h;
    int64_t ks_p, ks_t, ks_h;   // elements: page, slot, head
    int64_t ss_p, ss_t, ss_h;   // floats
    const float *sink;
    const void *gate;
    // the split: a CTA takes `chunk` visible keys, the partial results of (b, head, split) are
    // part_ml[..][2] = (running maximum in log2 units, denominator) and part_o[..][D] (not normalised)
    int chunk, n_split;
    float *part_ml, *part_o;
};

// The visible keys of a sequence as a list of slots: nf first tokens, then the keys lo .. lo + n - nf - 1.
struct PagedKeys {
    int nf, lo, n;
    __device__ __forceinline__ int key(int slot) const { return slot < nf ? slot : lo + (slot - nf); }
};

__device__ __forceinline__ PagedKeys paged_keys(const PagedParams &p, int b)
{
    const int given = p.kv_lens ? p.kv_lens[b] : p.max_len;
    const int len = given < 0 ? 0 : (given > p.max_len ? p.max_len : given);
    int pos = p.q_start ? p.q_start[b] : (p.table || given < 0 ? len : given) - 1;   // (the window layer's is not held to the cache)
    if (pos < -1) pos = -1;
    const int end = pos < len ? pos + 1 : len;   // keys 0 .. end - 1
    PagedKeys k;
    k.lo = pos < p.w ? 0 : pos - p.w + 1;        // no overflow: w >= 1, pos >= w here
    if (k.lo > end) k.lo = end;
    k.nf = p.nf < k.lo ? p.nf : k.lo;
    k.n = k.nf + end - k.lo;
    return k;
}

// slot in its page and the page of key j; page < 0: the key is void
__device__ __forceinline__ int2 paged_row(const PagedParams &p, int b, int j)
{
    const int col = j / p.ps;
    int page = p.table ? __ldg(p.table + b * p.table_stride + col) : b;
    if (page >= p.n_pages) page = -1;
    return make_int2(page, j - col * p.ps);
}

// The end of a row whose keys are folded: l is the sum of their weights relative to `top` (log2 units, -inf without a key); the
// sink joins the denominator as a key without a value.
struct RowEnd {
    float at, den;   // the maximum with the sink, and the denominator relative to it
    float factor;    // of the sums of weighted values; 0 without a key
    // natural logarithm of the whole; -inf where there is nothing to sum
    __device__ __forceinline__ float lse() const { return den == 0.f ? -INFINITY : (at + log2f(den)) * kLn2; }
};
__device__ __forceinline__ RowEnd row_end(float top, float l, const float *sink, int h)
{
    RowEnd e{top, l, 0.f};
    if (sink) {
        const float s2 = sink[h] * kLog2e;
        e.at = fmaxf(top, s2);
        if (e.at != -INFINITY || s2 != s2) e.den = l * exp2f(top - e.at) + exp2f(s2 - e.at);
    }
    // a denominator that is NaN (a logit or the sink was) is neither an empty one nor a factor of 0
    if (l != 0.f) e.factor = e.den > 0.f ? exp2f(top - e.at) / e.den : e.den;
    return e;
}

// e4m3: the power of two above the largest V scale, kept where it and its reciprocal are normal numbers
__device__ __forceinline__ float v_unit_of(float top)
{
    return fmaxf(__uint_as_float(__float_as_uint(fminf(top, 0x1p124f)) & 0x7f800000u) * 2.f, 0x1p-126f);
}

// e4m3: what a row of q, largest magnitude `top` (NaN and infinities pass), is divided by to become an f16 operand of magnitudes
// below 2^15, of which those down to 2^-29 of the largest are normal numbers: exact, as bf16 has fewer bits than f16.
__device__ __forceinline__ float q_unit_of(float top)
{
    const float unit = __uint_as_float(__float_as_uint(top) & 0x7f800000u);   // the power of two at or below it
    return fminf(fmaxf(unit, 0x1p-100f), 0x1p126f) * 0x1p-14f;
}

constexpr int kPagedMaxChunk = 2048;   // visible keys of one CTA at most: ragged batches then balance over many CTAs

// Which groups run on the tcgen05 kernel.  Measured there and on mma.sync, us: head_dim 128, 64 x 16K keys: 32 heads 131 and 120
// (e4m3: 116, 108), 64 heads 137 and 185 (126, 186); head_dim 256, 32 x 16K: 8 heads 100 and 111 (86, 64), 16 heads 101 and 128
// (87, 77), 32 heads 105 and 130 (90, 111).  By the shape alone, although one short sequence is faster on mma.sync: bf16, 8 heads at
// head_dim 256, 1 x 100 keys 8.4 and 7.0, 1 x 4K 15.8 and 14.2; but 1 x 32K 35 and 59, 8 x 4K 16.2 and 20.7.
inline bool paged_on_tc5(const PagedParams &p, bool fp8) { return (p.D == 256 && (p.G > 16 || !fp8)) || (p.D == 128 && p.G > 32); }
// Fills chunk and n_split: the split that ends first if all contexts are as long as the table allows.
void paged_plan(PagedParams *p, bool fp8);
size_t paged_ws_bytes(const PagedParams &p);   // of a planned problem
size_t paged_ws_bound(const PagedParams &p);   // of every plan with at most p.max_len visible keys, cache not e4m3

// K, V: elements of dtype `dt`, or e4m3 codes when ksc / vsc are given (dt then describes Q and O)
cudaError_t launch_paged_decode(PagedParams p, hs2_dtype dt, const void *Q, const void *K, const void *V, const float *ksc,
                                const float *vsc, void *O, float *LSE, void *ws, cudaStream_t st);
// the tensor-core kernel (hs2_paged_mma.cu): leaves the partial results, or finishes sequences of one chunk
bool paged_mma_supported(const PagedParams &p, hs2_dtype dt, bool fp8, const void *Q, const void *K, const void *V, const void *O);
cudaError_t launch_paged_mma(const PagedParams &p, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc,
                             void *O, float *LSE, cudaStream_t st);
// the tcgen05 kernel (hs2_paged_tc5.cu)
cudaError_t launch_paged_tc5(const PagedParams &p, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc,
                             void *O, float *LSE, cudaStream_t st);
cudaError_t read_paged_error(unsigned *out);
// sliding window over a contiguous cache: fp32 FMAs, any shape (hs2_window_simt.cu)
cudaError_t launch_window_simt(const Params &p, int nf, hs2_dtype dt, const void *Q, const void *K, const void *V,
                                  const float *sink, void *O, float *LSE, cudaStream_t st);
// heads and queries (gp | G, gp tq <= rows) of a row tile
void window_row_tile(const Params &p, int rows, int key_tile, int *gp, int *tq);

// the same on tcgen05 (hs2_window_tc5.cu)
bool window_tc5_supported(const Params &p, hs2_dtype dt, const void *Q, const void *K, const void *V, const void *O);
cudaError_t launch_window_tc5(const Params &p, int nf, const void *Q, const void *K, const void *V, const float *sink, void *O, float *LSE,
                              cudaStream_t st);
cudaError_t read_window_error(unsigned *out);

// the opt-in to large dynamic shared memory is an attribute of the kernel on each device; `ready` remembers the devices
template <typename Kernel>
cudaError_t opt_in_smem(Kernel kernel, int bytes, std::atomic<unsigned long long> &ready)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (ready.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes)) == cudaSuccess)
        ready.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// page bookkeeping (hs2_pages.cu)
__host__ __device__ __forceinline__ int pages_of(int len, int ps) { return (int)(((int64_t)len + ps - 1) / ps); }
// The table entries of a sequence of `len` tokens that go when it keeps the first `keep` of them: x .. y - 1, and none at x >= y.
// A keep of any size names no entry behind those of the sequence, so that a thread's index added to x stays in int32.
__host__ __device__ __forceinline__ int2 released_entries(int len, int keep, int ps, int max_pages)
{
    const int held = len < 0 ? 0 : len, kept = keep < 0 ? 0 : keep;
    const int have = pages_of(held, ps), end = have < max_pages ? have : max_pages;
    return make_int2(pages_of(kept < held ? kept : held, ps), end);
}

struct PageRegions {
    hs2_page_region r[HS2_MAX_PAGE_REGIONS];
    int n;
};
size_t pages_ws_bytes(const hs2_page_pool &pool, int n);
cudaError_t launch_pages_reserve(const hs2_page_pool &pool, const PageRegions &rg, const int32_t *seqs, const int32_t *n_new,
                                 int n, int32_t *start, void *ws, cudaStream_t st);
cudaError_t launch_pages_write(const hs2_page_pool &pool, const PageRegions &rg, const void *const *rows, const int64_t *row_strides,
                               const int32_t *seqs, const int32_t *start, const int32_t *n_new, int n, int max_new, cudaStream_t st);
cudaError_t launch_pages_fork(const hs2_page_pool &pool, const int32_t *src, const int32_t *dst, int n, void *ws, cudaStream_t st);
cudaError_t launch_pages_free(const hs2_page_pool &pool, const int32_t *seqs, const int32_t *keep, int n, cudaStream_t st);
cudaError_t launch_pages_compact(const hs2_page_pool &pool, const PageRegions &rg, int32_t *moved, void *ws, cudaStream_t st);
cudaError_t launch_pages_copy(const hs2_page_pool &pool, const PageRegions &rg, const int32_t *src, const int32_t *dst, int n,
                              cudaStream_t st);

}  // namespace hs2
