// Attention of one new token per sequence over a cache in pages.
//
//   o = sum_j 2^(t_j - m) v_j / (sum_j 2^(t_j - m) + 2^(sink log2 e - m)),  t_j = <q, k_j> scale log2 e,  m = max_j t_j
//
// over the visible keys j; a key's row is found through the page table.  The keys of a sequence are cut into chunks of equal
// size; a CTA folds one chunk into (m, l, o) and k_paged_combine joins the chunks of a (sequence, head).
#include <cuda_fp16.h>
#include <limits.h>

#include "hs2_paged.cuh"

namespace hs2 {

// keys of a chunk are a multiple of this: whole tiles of the kernels
constexpr int kTile = 128;
// What a CTA spends on itself, in keys: its start, its query, the store of its part (about 3 us beside 60 ns per key at
// two CTAs per SM).
constexpr int64_t kOwn = 128;
// What the join costs, in keys of a GPU that waits for latency: up to 384 keys one CTA is as fast (32 heads on 4, head_dim 128,
// 300 keys: 8.3 us either way, 16 x 200 keys 8.3 against 10.3) and the host launches once.
constexpr int64_t kJoin = 256;

// CTAs that a B200 runs at once (148 SMs; a constant, so that the workspace size does not need a device)
static int64_t wave(const PagedParams &p, bool fp8) { return 148 * (paged_on_tc5(p, fp8) ? 1 : p.G <= 8 && p.D * (fp8 ? 1 : 2) <= 128 ? 4 : 2); }
static int64_t units(const PagedParams &p, bool fp8) { return (int64_t)p.B * p.Hkv * (paged_on_tc5(p, fp8) ? (p.G + 127) / 128 : 1); }

void paged_plan(PagedParams *p, bool fp8)
{
    const int64_t vis = p->w < p->max_len ? (int64_t)p->w + p->nf : p->max_len;
    const int64_t most = vis < p->max_len ? vis : p->max_len;   // visible keys of the longest context
    const int64_t at_once = wave(*p, fp8), un = units(*p, fp8);
    int64_t best = -1;
    p->chunk = kTile;
    p->n_split = 1;
    // the fewest splits that keep a chunk within its limit, and those that fill the GPU once, twice or three times
    const int64_t n0 = most > kPagedMaxChunk ? (most + kPagedMaxChunk - 1) / kPagedMaxChunk : 1;
    for (int waves = 0; waves < 4; ++waves) {
        const int64_t n = waves ? waves * at_once / un : n0;
        if (n < n0) continue;
        int64_t chunk = ((most + n - 1) / n + kTile - 1) / kTile * kTile;
        if (chunk < kTile) chunk = kTile;
        const int64_t splits = most > chunk ? (most + chunk - 1) / chunk : 1;
        const int64_t cost = (un * splits + at_once - 1) / at_once * (chunk + kOwn) + (splits > 1 ? kJoin : 0);   // rounds times a CTA's time
        if (best < 0 || cost < best) {
            best = cost;
            p->chunk = (int)chunk;
            p->n_split = (int)splits;
        }
    }
}

// partial results of one split: m, l and D sums per (sequence, head)
static size_t split_bytes(const PagedParams &p, int64_t n_split) { return (size_t)p.B * p.Hq * n_split * (p.D + 2) * sizeof(float); }

size_t paged_ws_bytes(const PagedParams &p) { return p.n_split <= 1 ? 0 : split_bytes(p, p.n_split); }

size_t paged_ws_bound(const PagedParams &p)
{
    // paged_plan's splits: at most three rounds of CTAs, at least a tile of keys each, or as many as the longest chunk asks for
    const int64_t a = 3 * wave(p, false) / units(p, false), tiles = ((int64_t)p.max_len + kTile - 1) / kTile;
    const int64_t b = ((int64_t)p.max_len + kPagedMaxChunk - 1) / kPagedMaxChunk;
    const int64_t few = a < tiles ? a : tiles, n = few > b ? few : b;
    return n <= 1 ? 0 : split_bytes(p, n);
}

namespace {

constexpr int kWarps = 4;
constexpr int kMaxDPerLane = 8;   // head_dim <= 256

__device__ __forceinline__ float elem(float x) { return x; }
__device__ __forceinline__ float elem(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float elem(uint8_t code)   // e4m3: exact in f16
{
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(d) : "h"((unsigned short)code));
    const __half_raw h{(unsigned short)(d & 0xffffu)};
    return __half2float(__half(h));
}

// Online-softmax state of one row in a warp: m, l the same in every lane, acc[r] is output dimension lane + 32 r.
struct Row {
    float m, l, acc[kMaxDPerLane];
    __device__ __forceinline__ void clear()
    {
        m = -INFINITY; l = 0.f;
#pragma unroll
        for (int r = 0; r < kMaxDPerLane; ++r) acc[r] = 0.f;
    }
};

// <q, k> of a lane's own key row; `wide`: rows of 16-byte pieces
template <typename KV>
__device__ __forceinline__ float dot(const KV *k, const float *q, int D, bool wide)
{
    constexpr int N = 16 / sizeof(KV);
    float s = 0.f;
    if (wide) {
#pragma unroll 4
        for (int d = 0; d < D; d += N) {
            const uint4 x = __ldg(reinterpret_cast<const uint4 *>(k + d));
            KV e[N];
            memcpy(e, &x, 16);
#pragma unroll
            for (int i = 0; i < N; ++i) s = fmaf(elem(e[i]), q[d + i], s);
        }
    } else {
#pragma unroll 4
        for (int d = 0; d < D; ++d) s = fmaf(elem(k[d]), q[d], s);
    }
    return s;
}
template <typename KV>
__device__ __forceinline__ bool wide_rows(const KV *K, int D, int64_t a, int64_t b, int64_t c)
{
    constexpr int N = 16 / sizeof(KV);
    return reinterpret_cast<uintptr_t>(K) % 16 == 0 && D % N == 0 && ((a | b | c) & (N - 1)) == 0;
}

// Folds up to 32 keys: lane t holds the logit (log2 units, -inf without a key) and the V row and V scale of its key.
template <typename KV>
__device__ __forceinline__ void fold(Row &st, float t2, unsigned mask, const KV *vrow, float vs, int D, int lane)
{
    if (mask == 0) return;
    // (the maximum passes over NaN: of logits that are all NaN it is -inf, and they have to reach the sums all the same)
    const float m_new = fmaxf(st.m, warp_max(t2)), base = m_new == -INFINITY ? 0.f : m_new;
    const float corr = exp2f(st.m - base), pj = exp2f(t2 - base);
    st.l = st.l * corr + warp_sum(pj);
    st.m = m_new;
#pragma unroll
    for (int r = 0; r < kMaxDPerLane; ++r) st.acc[r] *= corr;
    while (mask) {   // four rows at a time, so that their loads are in flight together
        const KV *v[4];
        float pt[4], vt[4], x[4][kMaxDPerLane];
        bool on[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int t = mask ? __ffs(mask) - 1 : 0;
            on[k] = mask != 0;
            mask &= mask - 1;
            pt[k] = __shfl_sync(0xffffffffu, pj, t);
            vt[k] = sizeof(KV) == 1 ? __shfl_sync(0xffffffffu, vs, t) : 1.f;
            v[k] = reinterpret_cast<const KV *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(vrow), t));
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int r = 0; r < kMaxDPerLane; ++r)
                if (on[k] && lane + 32 * r < D) x[k][r] = elem(v[k][lane + 32 * r]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int r = 0; r < kMaxDPerLane; ++r)   // (p times a small scale would flush)
                if (on[k] && lane + 32 * r < D) st.acc[r] = fmaf(pt[k], sizeof(KV) == 1 ? x[k][r] * vt[k] : x[k][r], st.acc[r]);
    }
}

// ---------------------------------------------------------------- fp32 FMAs: any shape, any type
// One CTA = one chunk of one (sequence, query head); its warps take 32 keys in turn and are joined through shared memory.
// Bound by the latency of its loads (a lane reads its own key row), kept for the shapes the tensor-core kernels do not cover.
template <typename T, typename KV>
__global__ void __launch_bounds__(kWarps * 32)
k_paged_generic(const PagedParams p, const T *__restrict__ Q, const KV *__restrict__ K, const KV *__restrict__ V,
                const float *__restrict__ ksc, const float *__restrict__ vsc, T *__restrict__ O, float *__restrict__ LSE)
{
    __shared__ float sq[256], so[kWarps][256], sm[kWarps], sl[kWarps];
    const int split = blockIdx.x, h = blockIdx.y, b = blockIdx.z, g = h / p.G;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const PagedKeys keys = paged_keys(p, b);
    const int c0 = split * p.chunk;
    if (split > 0 && c0 >= keys.n) return;
    const int c1 = min(keys.n, c0 + p.chunk);
    for (int d = threadIdx.x; d < p.D; d += kWarps * 32) sq[d] = elem(Q[b * p.qs_b + h * p.qs_h + d]);
    __syncthreads();
    const bool wide = wide_rows(K, p.D, p.ks_p, p.ks_t, p.ks_h);
    Row st;
    st.clear();
    for (int c = c0 + warp * 32; c < c1; c += kWarps * 32) {
        const bool in = c + lane < c1;
        const int2 row = in ? paged_row(p, b, keys.key(c + lane)) : make_int2(-1, 0);
        const bool valid = row.x >= 0;
        const int64_t off = valid ? row.x * p.ks_p + row.y * p.ks_t + g * p.ks_h : 0;
        const int64_t soff = valid ? row.x * p.ss_p + row.y * p.ss_t + g * p.ss_h : 0;
        float t2 = -INFINITY, vs = 1.f;
        if (valid) {
            t2 = dot(K + off, sq, p.D, wide) * (ksc ? ksc[soff] : 1.f) * p.scale_log2;
            if (vsc) vs = vsc[soff];
        }
        fold(st, t2, __ballot_sync(0xffffffffu, valid), V + off, vs, p.D, lane);
    }
    if (lane == 0) { sm[warp] = st.m; sl[warp] = st.l; }
#pragma unroll
    for (int r = 0; r < kMaxDPerLane; ++r)
        if (lane + 32 * r < p.D) so[warp][lane + 32 * r] = st.acc[r];
    __syncthreads();
    float m = -INFINITY, l = 0.f, f[kWarps];
#pragma unroll
    for (int i = 0; i < kWarps; ++i) m = fmaxf(m, sm[i]);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        f[i] = m == -INFINITY ? 0.f : exp2f(sm[i] - m);
        l += sl[i] * f[i];
    }
    const bool whole = keys.n <= p.chunk;   // nothing to join: finish here
    const int64_t part = ((int64_t)b * p.Hq + h) * p.n_split + split;
    const RowEnd end = row_end(m, l, whole ? p.sink : nullptr, h);
    for (int d = threadIdx.x; d < p.D; d += kWarps * 32) {
        float o = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) o += so[i][d] * f[i];
        if (whole) {
            const int64_t at = b * p.os_b + h * p.os_h + d;
            from_f32(O[at], o * end.factor * (p.gate ? gate_of(elem(static_cast<const T *>(p.gate)[at])) : 1.f));
        } else {
            p.part_o[part * p.D + d] = o;
        }
    }
    if (threadIdx.x == 0) {
        if (!whole) { p.part_ml[2 * part] = m; p.part_ml[2 * part + 1] = l; }
        else if (LSE) LSE[(int64_t)b * p.Hq + h] = end.lse();
    }
}

// Joins the chunks of one (sequence, head): one CTA each, thread = output dimension.
template <typename T>
__global__ void __launch_bounds__(128)
k_paged_combine(const PagedParams p, T *__restrict__ O, float *__restrict__ LSE)
{
    const int h = blockIdx.x, b = blockIdx.y;
    const PagedKeys keys = paged_keys(p, b);
    if (keys.n <= p.chunk) return;   // finished by its only CTA
    const int n = (keys.n + p.chunk - 1) / p.chunk;
    const int64_t part = ((int64_t)b * p.Hq + h) * p.n_split;
    float m_keys = -INFINITY;
    for (int i = 0; i < n; ++i) m_keys = fmaxf(m_keys, p.part_ml[2 * (part + i)]);
    const float base = m_keys == -INFINITY ? 0.f : m_keys;
    float l = 0.f;
    for (int i = 0; i < n; ++i) l += p.part_ml[2 * (part + i) + 1] * exp2f(p.part_ml[2 * (part + i)] - base);
    const RowEnd end = row_end(m_keys, l, p.sink, h);
    for (int d = threadIdx.x; d < p.D; d += 128) {
        float o = 0.f;
        for (int i = 0; i < n; ++i) o = fmaf(p.part_o[(part + i) * p.D + d], exp2f(p.part_ml[2 * (part + i)] - base), o);
        const int64_t at = b * p.os_b + h * p.os_h + d;
        from_f32(O[at], o * end.factor * (p.gate ? gate_of(elem(static_cast<const T *>(p.gate)[at])) : 1.f));
    }
    if (threadIdx.x == 0 && LSE) LSE[(int64_t)b * p.Hq + h] = end.lse();
}

cudaError_t combine(const PagedParams &p, hs2_dtype dt, void *O, float *LSE, cudaStream_t st)
{
    if (p.n_split <= 1) return cudaSuccess;
    const dim3 grid((unsigned)p.Hq, (unsigned)p.B);
    if (dt == HS2_F32) k_paged_combine<float><<<grid, 128, 0, st>>>(p, (float *)O, LSE);
    else k_paged_combine<__nv_bfloat16><<<grid, 128, 0, st>>>(p, (__nv_bfloat16 *)O, LSE);
    count_launch();
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_decode(PagedParams p, hs2_dtype dt, const void *Q, const void *K, const void *V, const float *ksc,
                                const float *vsc, void *O, float *LSE, void *ws, cudaStream_t st)
{
    p.part_ml = static_cast<float *>(ws);
    p.part_o = p.part_ml + (size_t)p.B * p.Hq * p.n_split * 2;
    const dim3 grid((unsigned)p.n_split, (unsigned)p.Hq, (unsigned)p.B);
    using bf = __nv_bfloat16;
    cudaError_t e = cudaErrorNotSupported;
    if (paged_mma_supported(p, dt, ksc != nullptr, Q, K, V, O)) e = launch_paged_mma(p, Q, K, V, ksc, vsc, O, LSE, st);
    if (e != cudaErrorNotSupported) return e == cudaSuccess ? combine(p, dt, O, LSE, st) : e;
    if (ksc)
        k_paged_generic<bf, uint8_t><<<grid, kWarps * 32, 0, st>>>(p, (const bf *)Q, (const uint8_t *)K, (const uint8_t *)V, ksc, vsc, (bf *)O, LSE);
    else if (dt == HS2_F32)
        k_paged_generic<float, float><<<grid, kWarps * 32, 0, st>>>(p, (const float *)Q, (const float *)K, (const float *)V, nullptr, nullptr,
                                                                   (float *)O, LSE);
    else
        k_paged_generic<bf, bf><<<grid, kWarps * 32, 0, st>>>(p, (const bf *)Q, (const bf *)K, (const bf *)V, nullptr, nullptr, (bf *)O, LSE);
    count_launch();
    e = cudaGetLastError();
    return e == cudaSuccess ? combine(p, dt, O, LSE, st) : e;
}

}  // namespace hs2
