// Bookkeeping of a paged cache on the device: reserve, write, fork, free, compact, copy.
//
// The tables are small (a few bytes per page), the contents are not: what bounds these calls is latency for the plans and
// memory for the copies (2 x the bytes that move).  A plan is one launch of one thread-block cluster, whose CTAs scan the
// counts of a share of the pages each and agree on their offsets through distributed shared memory; it leaves a list of
// (source, destination) pages that the copy kernel works through.  No launch waits for another one.
#include <cooperative_groups.h>
#include <limits.h>

#include "hs2_paged.cuh"

namespace hs2 {

namespace cg = cooperative_groups;

namespace {

constexpr int kPlanCtas = 8, kPlanThreads = 512;
constexpr int kCopyThreads = 256;

// Scratch: int32 arrays, the union of what reserve, fork and compact need.
struct PagesWs {
    int32_t *head;    // [16] totals
    int32_t *claim;   // [max_seqs] first list entry that names a sequence
    int32_t *list_a;  // [n_pages] free pages / pages to move
    int32_t *list_b;  // [n_pages + 2 n] destinations, or (source, destination) pairs of the copies on write
    int32_t *base;    // [n] rank of the first fresh page of a request
    int32_t *flags;   // [n] what a request gets (reserve), new length (fork)
    int32_t *rows;    // [n][max_pages] staged table rows (fork)
};

size_t align64(size_t x) { return (x + 63) / 64 * 64; }

size_t layout(const hs2_page_pool &pool, int n, void *ws, PagesWs *out)
{
    size_t at = 0;
    auto take = [&](size_t count) {
        int32_t *p = reinterpret_cast<int32_t *>(static_cast<char *>(ws) + at);
        at += align64(count * sizeof(int32_t));
        return p;
    };
    PagesWs w;
    w.head = take(16);
    w.claim = take(pool.max_seqs);
    w.list_a = take(pool.n_pages);
    w.list_b = take((size_t)pool.n_pages + 2 * (size_t)n);
    w.base = take(n);
    w.flags = take(n);
    w.rows = take((size_t)n * pool.max_pages);
    if (out) *out = w;
    return at;
}

// exclusive prefix of `v` over the CTA; `total` the sum
template <typename T>
__device__ __forceinline__ T cta_scan(T v, T &total, T *scratch /* [32] */)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    T x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();   // the scratch of the call before has been read
    if (lane == 31) scratch[warp] = x;
    __syncthreads();
    if (warp == 0) {
        T s = lane < warps ? scratch[lane] : T(0);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const T y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        scratch[lane] = s;
    }
    __syncthreads();
    total = scratch[warps - 1];
    return x - v + (warp ? scratch[warp - 1] : T(0));
}

// The pages of this CTA's share of the pool, [p0, p1): shares differ by the cluster rank only.
__device__ __forceinline__ void page_share(int n_pages, int rank, int &p0, int &p1)
{
    const int per = (n_pages + kPlanCtas - 1) / kPlanCtas;
    p0 = min(n_pages, rank * per);
    p1 = min(n_pages, p0 + per);
}

// Number of pages in use below this CTA's share and in all, agreed over the cluster.
__device__ __forceinline__ void count_used(cg::cluster_group &cluster, const int32_t *refs, int p0, int p1, int &below, int &all,
                                           int *counts /* shared [kPlanCtas] */, int *scratch)
{
    int mine = 0, total;
    for (int p = p0 + threadIdx.x; p < p1; p += blockDim.x) mine += __ldcg(refs + p) > 0;
    cta_scan(mine, total, scratch);
    const int rank = (int)cluster.block_rank();
    cluster.sync();   // all CTAs of the cluster have started: their shared memory may be written
    if (threadIdx.x < kPlanCtas) cluster.map_shared_rank(counts, threadIdx.x)[rank] = total;
    cluster.sync();
    below = all = 0;
    for (int i = 0; i < kPlanCtas; ++i) {
        if (i < rank) below += counts[i];
        all += counts[i];
    }
}

// ---------------------------------------------------------------- reserve
// flags: bit 0 accepted, bit 1 the shared last page gets a copy
__global__ void __cluster_dims__(kPlanCtas, 1, 1) __launch_bounds__(kPlanThreads)
k_pages_reserve(const hs2_page_pool pool, const int32_t *__restrict__ seqs, const int32_t *__restrict__ n_new, int n,
                int32_t *__restrict__ start, PagesWs ws)
{
    __shared__ int counts[kPlanCtas], scratch[32];
    __shared__ long long scratch64[32], carry;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank();
    int p0, p1, used_below, used;
    page_share(pool.n_pages, rank, p0, p1);
    count_used(cluster, pool.ref_counts, p0, p1, used_below, used, counts, scratch);
    // the free pages in ascending order
    int at = p0 - used_below;
    for (int c = p0; c < p1; c += blockDim.x) {
        const int p = c + threadIdx.x;
        const int is_free = p < p1 && __ldcg(pool.ref_counts + p) <= 0;
        int total;
        const int r = cta_scan(is_free, total, scratch);
        if (is_free) ws.list_a[at + r] = p;
        at += total;
    }
    const int n_free = pool.n_pages - used, ps = pool.page_size;
    // which request is the first of its sequence
    if (rank == 0) {
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int s = seqs[i];
            if (s >= 0 && s < pool.max_seqs) ws.claim[s] = INT_MAX;
        }
        __threadfence();
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int s = seqs[i];
            if (s >= 0 && s < pool.max_seqs) atomicMin(ws.claim + s, i);
        }
        __threadfence();
    }
    cluster.sync();   // also: the list of free pages is complete, and every count has been read
    if (rank != 0) return;
    // what each request needs, and where its pages begin in the list
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int c = 0; c < n; c += blockDim.x) {
        const int i = c + threadIdx.x;
        int ok = 0, cow = 0, len = 0, last = -1;
        long long need = 0;
        if (i < n) {
            const int s = seqs[i], add = n_new[i];
            if (s >= 0 && s < pool.max_seqs && __ldcg(ws.claim + s) == i && add >= 0) {
                len = max(0, pool.lens[s]);
                const int64_t want = (int64_t)len + add;
                if (want <= (int64_t)pool.max_pages * ps) {
                    ok = 1;
                    const int have = pages_of(len, ps);
                    if (add > 0 && len % ps) {
                        last = pool.page_table[(int64_t)s * pool.max_pages + have - 1];
                        if (last >= pool.n_pages) last = -1;
                        cow = last >= 0 && __ldcg(pool.ref_counts + last) > 1;
                    }
                    need = (long long)pages_of((int)want, ps) - have + cow;
                }
            }
        }
        long long total;
        const long long before = carry;
        const long long base = before + cta_scan(need, total, scratch64);   // (cta_scan synchronises: `before` is read by all)
        if (ok && base + need > n_free) ok = 0;
        if (i < n) {
            ws.base[i] = (int)base;
            ws.flags[i] = ok | (ok && cow ? 2 : 0);
            start[i] = ok ? len : -1;
            // the pages to copy: read by the copy kernel
            ws.list_b[2 * i] = ok && cow ? last : -1;
            ws.list_b[2 * i + 1] = ok && cow ? ws.list_a[base] : -1;
        }
        __syncthreads();
        if (threadIdx.x == 0) carry = before + total;
        __syncthreads();
    }
    // a warp per request enters its pages
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x >> 5; i < n; i += blockDim.x >> 5) {
        const int fl = ws.flags[i];
        if (!(fl & 1)) continue;
        const int s = seqs[i], len = max(0, pool.lens[s]), add = n_new[i], cow = fl >> 1;
        const int have = pages_of(len, ps), want = pages_of(len + add, ps);
        int32_t *row = pool.page_table + (int64_t)s * pool.max_pages;
        const int32_t *fresh = ws.list_a + ws.base[i];
        if (cow && lane == 0) {
            atomicSub(pool.ref_counts + ws.list_b[2 * i], 1);
            row[have - 1] = fresh[0];
            pool.ref_counts[fresh[0]] = 1;
        }
        for (int c = have + lane; c < want; c += 32) {
            const int p = fresh[cow + c - have];
            row[c] = p;
            pool.ref_counts[p] = 1;
        }
        __syncwarp();
        if (lane == 0) pool.lens[s] = len + add;
    }
}

// ---------------------------------------------------------------- compact
// list_a: pages that move, list_b: where to, head[0]: how many; `moved` and the counts are written here, the
// table by k_pages_rename.
__global__ void __cluster_dims__(kPlanCtas, 1, 1) __launch_bounds__(kPlanThreads)
k_pages_compact(const hs2_page_pool pool, int32_t *__restrict__ moved, PagesWs ws)
{
    __shared__ int counts[kPlanCtas], low_counts[kPlanCtas], scratch[32];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank();
    int p0, p1, used_below, used;
    page_share(pool.n_pages, rank, p0, p1);
    count_used(cluster, pool.ref_counts, p0, p1, used_below, used, counts, scratch);
    // pages in use at `used` or above, and free pages below it, each in ascending order.  Below this share:
    //   free pages below min(p0, used):  that many pages less the used ones; known from the counts when p0 <= used
    int n_high = 0, n_low = 0, total;
    for (int p = p0 + threadIdx.x; p < p1; p += blockDim.x) {
        const bool u = __ldcg(pool.ref_counts + p) > 0;
        n_high += u && p >= used;
        n_low += !u && p < used;
    }
    cta_scan(n_high, total, scratch);
    const int high_mine = total;
    cta_scan(n_low, total, scratch);
    const int low_mine = total;
    __syncthreads();
    if (threadIdx.x < kPlanCtas) {
        cluster.map_shared_rank(low_counts, threadIdx.x)[rank] = low_mine;
    }
    cluster.sync();
    if (threadIdx.x < kPlanCtas) cluster.map_shared_rank(counts, threadIdx.x)[rank] = high_mine;
    cluster.sync();
    int high_at = 0, low_at = 0, n_move = 0;
    for (int i = 0; i < kPlanCtas; ++i) {
        if (i < rank) { high_at += counts[i]; low_at += low_counts[i]; }
        n_move += counts[i];
    }
    for (int c = p0; c < p1; c += blockDim.x) {
        const int p = c + threadIdx.x;
        const bool u = p < p1 && __ldcg(pool.ref_counts + p) > 0;
        const int hi = u && p >= used, lo = p < p1 && !u && p < used;
        int th, tl;
        const int rh = cta_scan(hi, th, scratch);
        const int rl = cta_scan(lo, tl, scratch);
        if (hi) ws.list_a[high_at + rh] = p;
        if (lo) ws.list_b[low_at + rl] = p;
        high_at += th;
        low_at += tl;
        if (moved && p < p1 && !hi) moved[p] = u ? p : -1;
    }
    cluster.sync();
    if (rank == 0 && threadIdx.x == 0) ws.head[0] = n_move;
    for (int i = rank * blockDim.x + threadIdx.x; i < n_move; i += kPlanCtas * blockDim.x) {
        const int from = __ldcg(ws.list_a + i), to = __ldcg(ws.list_b + i);
        pool.ref_counts[to] = pool.ref_counts[from];
        pool.ref_counts[from] = 0;
        if (moved) moved[from] = to;
    }
}

// Table entries follow their pages: the pages that moved are sorted, so an entry finds itself by bisection.
__global__ void __launch_bounds__(256) k_pages_rename(const hs2_page_pool pool, PagesWs ws)
{
    const int n = ws.head[0];
    if (n == 0) return;
    const int first = ws.list_a[0];
    const int64_t total = (int64_t)pool.max_seqs * pool.max_pages;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
        const int p = pool.page_table[e];
        if (p < first) continue;
        int lo = 0, hi = n;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (ws.list_a[mid] < p) lo = mid + 1;
            else hi = mid;
        }
        if (lo < n && ws.list_a[lo] == p) pool.page_table[e] = ws.list_b[lo];
    }
}

// ---------------------------------------------------------------- copies of pages
// Entry e of the list: page src[e * step] -> dst[e * step] in every (region, layer).  Work is cut into pieces of up to
// kPiece bytes of one page of one layer; CTAs take pieces in turn, a thread has kFlight 16-byte loads in flight.
constexpr int kFlight = 8;   // 1 GB of pages: 209 us with 4, 194 with 8
constexpr int kPiece = kCopyThreads * 16 * kFlight;

__device__ __forceinline__ void copy_bytes(char *dst, const char *src, int bytes)
{
    if (((reinterpret_cast<uintptr_t>(dst) | reinterpret_cast<uintptr_t>(src) | (uintptr_t)bytes) & 15u) == 0) {
        const uint4 *s = reinterpret_cast<const uint4 *>(src);
        uint4 *d = reinterpret_cast<uint4 *>(dst);
        const int n = bytes >> 4;
        uint4 v[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
            if ((int)threadIdx.x + k * kCopyThreads < n) v[k] = __ldcs(s + threadIdx.x + k * kCopyThreads);
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
            if ((int)threadIdx.x + k * kCopyThreads < n) __stcs(d + threadIdx.x + k * kCopyThreads, v[k]);
    } else {
        const uint32_t *s = reinterpret_cast<const uint32_t *>(src);
        uint32_t *d = reinterpret_cast<uint32_t *>(dst);
        for (int i = threadIdx.x; i < bytes >> 2; i += kCopyThreads) d[i] = s[i];
    }
}

__global__ void __launch_bounds__(kCopyThreads)
k_pages_copy(const __grid_constant__ PageRegions rg, int n_pages, int page_size, const int32_t *__restrict__ src,
             const int32_t *__restrict__ dst, int step, int n_max, const int32_t *__restrict__ n_dev)
{
    const int n = n_dev ? min(*n_dev, n_max) : n_max;
    for (int r = 0; r < rg.n; ++r) {
        const hs2_page_region &g = rg.r[r];
        const bool dense = g.token_stride == g.row_bytes;
        const int64_t run = dense ? (int64_t)page_size * g.row_bytes : g.row_bytes;   // contiguous bytes
        const int64_t runs = dense ? 1 : page_size;
        const int64_t pieces = (run + kPiece - 1) / kPiece;
        const int64_t per_page = (int64_t)g.n_layers * runs * pieces;
        for (int64_t u = blockIdx.x; u < per_page * n; u += gridDim.x) {
            const int64_t e = u / per_page;
            int64_t rest = u - e * per_page;
            const int a = src[e * step], b = dst[e * step];
            if (a < 0 || a >= n_pages || b < 0 || b >= n_pages || a == b) continue;
            const int64_t layer = rest / (runs * pieces);
            rest -= layer * runs * pieces;
            const int64_t row = rest / pieces, piece = rest - row * pieces;
            const int64_t off = layer * g.layer_stride + row * g.token_stride + piece * kPiece;
            const int bytes = (int)min((int64_t)kPiece, run - piece * kPiece);
            char *base = static_cast<char *>(g.base) + off;
            copy_bytes(base + b * g.page_stride, base + a * g.page_stride, bytes);
        }
    }
}

// ---------------------------------------------------------------- write
struct WriteRows {
    const char *rows[HS2_MAX_PAGE_REGIONS];
    int64_t stride[HS2_MAX_PAGE_REGIONS][3];   // layer, request, token
};

// A CTA takes kWriteTokens tokens of one request in one layer of one region, a warp four of its rows at a time: up to eight
// 16-byte loads per thread in flight.
constexpr int kWriteTokens = 32;

__global__ void __launch_bounds__(256)
k_pages_write(const hs2_page_pool pool, const __grid_constant__ PageRegions rg, const __grid_constant__ WriteRows wr,
              const int32_t *__restrict__ seqs, const int32_t *__restrict__ start, const int32_t *__restrict__ n_new, int max_new)
{
    const int i = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int r = 0, layer = blockIdx.z;
    while (layer >= rg.r[r].n_layers) layer -= rg.r[r++].n_layers;
    const hs2_page_region &g = rg.r[r];
    const int s = seqs[i], first = start[i], count = min(n_new[i], max_new);
    if (s < 0 || s >= pool.max_seqs || first < 0) return;
    const int32_t *row = pool.page_table + (int64_t)s * pool.max_pages;
    const char *src0 = wr.rows[r] + layer * wr.stride[r][0] + i * wr.stride[r][1];
    char *dst0 = static_cast<char *>(g.base) + layer * g.layer_stride;
    const bool wide = ((reinterpret_cast<uintptr_t>(src0) | reinterpret_cast<uintptr_t>(dst0) | (uintptr_t)wr.stride[r][2] |
                        (uintptr_t)g.page_stride | (uintptr_t)g.token_stride | (uintptr_t)g.row_bytes) & 15u) == 0;
    for (int t0 = blockIdx.y * kWriteTokens + warp * 4; t0 < count; t0 += gridDim.y * kWriteTokens) {
        const char *src[4];
        char *dst[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {   // where the rows go; null: nowhere
            const int t = t0 + k;
            const int64_t pos = (int64_t)first + t;
            const int64_t col = pos / pool.page_size;
            const int page = t < count && col < pool.max_pages ? row[col] : -1;
            src[k] = src0 + (int64_t)t * wr.stride[r][2];
            dst[k] = page < 0 || page >= pool.n_pages ? nullptr : dst0 + page * g.page_stride + (pos - col * pool.page_size) * g.token_stride;
        }
        if (wide) {
            const int n = g.row_bytes >> 4;
            for (int c = lane; c < n; c += 64) {
                uint4 v[4][2];
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (dst[k] && c + 32 * h < n) v[k][h] = __ldcs(reinterpret_cast<const uint4 *>(src[k]) + c + 32 * h);
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (dst[k] && c + 32 * h < n) reinterpret_cast<uint4 *>(dst[k])[c + 32 * h] = v[k][h];
            }
        } else {
            for (int k = 0; k < 4; ++k)
                for (int c = lane; dst[k] && c < g.row_bytes >> 2; c += 32)
                    reinterpret_cast<uint32_t *>(dst[k])[c] = reinterpret_cast<const uint32_t *>(src[k])[c];
        }
    }
}

// ---------------------------------------------------------------- fork
// First launch: the rows of the sources are staged (a destination may be another entry's source), and an entry looks whether
// it is the first with its destination (a scan of the list: quadratic, but lists are short and the alternative is a launch
// more, to clear claims).  Second launch: the rows change.
__global__ void __launch_bounds__(128)
k_pages_fork_stage(const hs2_page_pool pool, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, PagesWs ws)
{
    const int i = blockIdx.x, s = src[i], d = dst[i];
    bool ok = s >= 0 && s < pool.max_seqs && d >= 0 && d < pool.max_seqs;
    bool beaten = false;
    if (ok)
        for (int j = threadIdx.x; j < i; j += 128) beaten |= dst[j] == d && src[j] >= 0 && src[j] < pool.max_seqs;
    ok = !__syncthreads_or(beaten) && ok;
    const int len = ok ? max(0, pool.lens[s]) : -1;
    if (threadIdx.x == 0) ws.flags[i] = len;
    if (!ok) return;
    const int cols = min(pages_of(len, pool.page_size), pool.max_pages);
    for (int c = threadIdx.x; c < cols; c += 128) ws.rows[(int64_t)i * pool.max_pages + c] = pool.page_table[(int64_t)s * pool.max_pages + c];
}

__global__ void __launch_bounds__(128) k_pages_fork(const hs2_page_pool pool, const int32_t *__restrict__ dst, PagesWs ws)
{
    const int i = blockIdx.x, len = ws.flags[i];
    if (len < 0) return;
    const int d = dst[i];
    const int have = min(pages_of(max(0, pool.lens[d]), pool.page_size), pool.max_pages);
    const int want = min(pages_of(len, pool.page_size), pool.max_pages);
    int32_t *row = pool.page_table + (int64_t)d * pool.max_pages;
    for (int c = threadIdx.x; c < max(have, want); c += 128) {
        const int old = c < have ? row[c] : -1;
        const int now = c < want ? ws.rows[(int64_t)i * pool.max_pages + c] : -1;
        if (old == now) continue;
        if (now >= 0 && now < pool.n_pages) atomicAdd(pool.ref_counts + now, 1);
        if (old >= 0 && old < pool.n_pages) atomicSub(pool.ref_counts + old, 1);
        row[c] = now;
    }
    __syncthreads();   // every thread has read the old length
    if (threadIdx.x == 0) pool.lens[d] = len;
}

// ---------------------------------------------------------------- free
// An entry leaves the table by an exchange, so a sequence that is listed twice gives each page back once.
__global__ void __launch_bounds__(128)
k_pages_free(const hs2_page_pool pool, const int32_t *__restrict__ seqs, const int32_t *__restrict__ keep)
{
    const int i = blockIdx.x, s = seqs[i];
    if (s < 0 || s >= pool.max_seqs) return;
    const int kept = keep ? max(0, keep[i]) : 0;
    const int len = *reinterpret_cast<volatile int32_t *>(pool.lens + s);
    const int2 gone = released_entries(len, kept, pool.page_size, pool.max_pages);
    int32_t *row = pool.page_table + (int64_t)s * pool.max_pages;
    for (int64_t c = (int64_t)gone.x + threadIdx.x; c < gone.y; c += 128) {
        const int p = atomicExch(row + c, -1);
        if (p >= 0 && p < pool.n_pages) atomicSub(pool.ref_counts + p, 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) atomicMin(pool.lens + s, kept);
}

// CTAs of the copy kernel for at most n pages
unsigned copy_grid(const hs2_page_pool &pool, const PageRegions &rg, int64_t n)
{
    int64_t units = 0;
    for (int r = 0; r < rg.n; ++r) {
        const hs2_page_region &g = rg.r[r];
        const bool dense = g.token_stride == g.row_bytes;
        const int64_t run = dense ? (int64_t)pool.page_size * g.row_bytes : g.row_bytes;
        const int64_t u = n * g.n_layers * (dense ? 1 : pool.page_size) * ((run + kPiece - 1) / kPiece);
        if (u > units) units = u;
    }
    return (unsigned)(units < 1 ? 1 : units > 148 * 8 ? 148 * 8 : units);
}

cudaError_t copy_pages(const hs2_page_pool &pool, const PageRegions &rg, const int32_t *src, const int32_t *dst, int step, int n,
                       const int32_t *n_dev, cudaStream_t st)
{
    if (rg.n == 0 || n == 0) return cudaSuccess;
    k_pages_copy<<<copy_grid(pool, rg, n), kCopyThreads, 0, st>>>(rg, pool.n_pages, pool.page_size, src, dst, step, n, n_dev);
    count_launch();
    return cudaGetLastError();
}

}  // namespace

size_t pages_ws_bytes(const hs2_page_pool &pool, int n) { return layout(pool, n, nullptr, nullptr); }

cudaError_t launch_pages_reserve(const hs2_page_pool &pool, const PageRegions &rg, const int32_t *seqs, const int32_t *n_new,
                                 int n, int32_t *start, void *ws, cudaStream_t st)
{
    if (n == 0) return cudaSuccess;
    PagesWs w;
    layout(pool, n, ws, &w);
    k_pages_reserve<<<kPlanCtas, kPlanThreads, 0, st>>>(pool, seqs, n_new, n, start, w);
    count_launch();
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : copy_pages(pool, rg, w.list_b, w.list_b + 1, 2, n, nullptr, st);
}

cudaError_t launch_pages_write(const hs2_page_pool &pool, const PageRegions &rg, const void *const *rows, const int64_t *row_strides,
                               const int32_t *seqs, const int32_t *start, const int32_t *n_new, int n, int max_new, cudaStream_t st)
{
    if (n == 0 || max_new == 0 || rg.n == 0) return cudaSuccess;
    WriteRows wr{};
    for (int r = 0; r < rg.n; ++r) {
        wr.rows[r] = static_cast<const char *>(rows[r]);
        for (int k = 0; k < 3; ++k) wr.stride[r][k] = row_strides[3 * r + k];
    }
    int layers = 0;
    for (int r = 0; r < rg.n; ++r) layers += rg.r[r].n_layers;
    const int64_t blocks = ((int64_t)max_new + kWriteTokens - 1) / kWriteTokens;
    const dim3 grid((unsigned)n, (unsigned)(blocks < 65535 ? blocks : 65535), (unsigned)layers);
    k_pages_write<<<grid, 256, 0, st>>>(pool, rg, wr, seqs, start, n_new, max_new);
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_pages_fork(const hs2_page_pool &pool, const int32_t *src, const int32_t *dst, int n, void *ws, cudaStream_t st)
{
    if (n == 0) return cudaSuccess;
    PagesWs w;
    layout(pool, n, ws, &w);
    k_pages_fork_stage<<<(unsigned)n, 128, 0, st>>>(pool, src, dst, w);
    count_launch();
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    k_pages_fork<<<(unsigned)n, 128, 0, st>>>(pool, dst, w);
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_pages_free(const hs2_page_pool &pool, const int32_t *seqs, const int32_t *keep, int n, cudaStream_t st)
{
    if (n == 0) return cudaSuccess;
    k_pages_free<<<(unsigned)n, 128, 0, st>>>(pool, seqs, keep);
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_pages_compact(const hs2_page_pool &pool, const PageRegions &rg, int32_t *moved, void *ws, cudaStream_t st)
{
    PagesWs w;
    layout(pool, 0, ws, &w);
    k_pages_compact<<<kPlanCtas, kPlanThreads, 0, st>>>(pool, moved, w);
    count_launch();
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int64_t entries = (int64_t)pool.max_seqs * pool.max_pages;
    const int64_t blocks = (entries + 255) / 256;
    k_pages_rename<<<(unsigned)(blocks < 148 * 8 ? blocks : 148 * 8), 256, 0, st>>>(pool, w);
    count_launch();
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    return copy_pages(pool, rg, w.list_a, w.list_b, 1, pool.n_pages / 2 + 1, w.head, st);
}

cudaError_t launch_pages_copy(const hs2_page_pool &pool, const PageRegions &rg, const int32_t *src, const int32_t *dst, int n,
                              cudaStream_t st)
{
    return copy_pages(pool, rg, src, dst, 1, n, nullptr, st);
}

}  // namespace hs2
