// Sliding-window attention with first tokens on fp32 FMAs: any type, stride and alignment, head_dim up to 256.
//
// A row tile of 32 rows is TQ consecutive queries x GP heads of one group (as on tcgen05), a key tile is 32 keys; both come to
// shared memory as fp32, head_dim padded to a multiple of 16 with zeros.  Four threads share a row: each takes eight of a tile's
// scores, the row's maximum and sum meet by shuffles, then each takes a quarter of the output's dimensions.  What bounds the kernel
// is shared memory: nine 16-byte reads to 32 FMAs in Q K^T, one to four in P V.
// Measured, fp32, head_dim 64: 12 heads on 2, 2400 tokens, w = 512: 272 us (1703 with a warp per query); 4 heads on 1, 512 tokens,
// w = 16: 14.5 us (12.4), the latency of two key tiles.  bf16, head_dim 96, 32 heads on 4, 8K tokens: w = 128 1.13 ms, w = 1024 6.7 ms.
#include <limits.h>

#include "hs2_paged.cuh"

namespace hs2 {
namespace {

constexpr int kRows = 32, kKeys = 32, kThreads = 128, kWarps = 4;

template <int DM>
constexpr int smem_bytes() { return ((kRows + 2 * kKeys) * (DM + 4) + kRows * (kKeys + 4)) * 4; }

// 16 bytes of a row as fp32
template <typename T>
__device__ __forceinline__ void put(float *dst, const uint4 &x)
{
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint4 *>(dst) = x;
    } else {
        auto lo = [](uint32_t v) { return __uint_as_float(v << 16); };
        auto hi = [](uint32_t v) { return __uint_as_float(v & 0xffff0000u); };
        *reinterpret_cast<float4 *>(dst) = make_float4(lo(x.x), hi(x.x), lo(x.y), hi(x.y));
        *reinterpret_cast<float4 *>(dst + 4) = make_float4(lo(x.z), hi(x.z), lo(x.w), hi(x.w));
    }
}

template <typename T, int DM>
__global__ void __launch_bounds__(kThreads)
k_window_simt(const Params p, int nf, int gp, int tq, const T *__restrict__ Q, const T *__restrict__ K, const T *__restrict__ V,
              const float *__restrict__ sink, T *__restrict__ O, float *__restrict__ LSE)
{
    constexpr int kPitch = DM + 4, kPitchP = kKeys + 4;   // threads of different rows on different banks
    extern __shared__ __align__(16) float smem[];
    float *sQ = smem, *sK = sQ + kRows * kPitch, *sV = sK + kKeys * kPitch, *sP = sV + kKeys * kPitch;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n_slots = p.Hq / gp, n_mblk = (p.Lq + tq - 1) / tq;
    const int at = blockIdx.x / n_slots, h0 = (blockIdx.x - at * n_slots) * gp, b = at / n_mblk, i0 = (at - b * n_mblk) * tq;
    const int Dp = (p.D + 15) & ~15;
    // the keys of the row tile: n_a tiles of first tokens, then those from `lo` on
    const int kvl = kvlen_of(p, b), pos0 = pos_of(p, b, i0);
    const int64_t last = (int64_t)pos0 + min(tq, p.Lq - i0);
    const int n_vis = (int)max((int64_t)0, min(last, (int64_t)kvl));
    int lo = (int)min(max((int64_t)pos0 - p.w + 1, (int64_t)0), (int64_t)n_vis), n_a = 0;
    if (nf >= lo) lo = 0;
    else if (n_vis > 0) n_a = (nf + kKeys - 1) / kKeys;
    const int n_tiles = n_a + (n_vis - lo + kKeys - 1) / kKeys;
    // this thread's row
    const int row = tid >> 2, part = tid & 3, q_in = row / gp, i = i0 + q_in, h = h0 + row - q_in * gp;
    const bool mine = row < gp * tq && i < p.Lq;
    const int64_t pos = (int64_t)pos0 + q_in, behind = pos - p.w;
    const int end = mine ? (int)max((int64_t)0, min(pos + 1, (int64_t)kvl)) : 0;
    auto seen = [&](int key) { return key < end && (key > behind || key < nf); };

    for (int r = warp; r < kRows; r += kWarps) {
        const int qi = i0 + r / gp;
        const bool in = r < gp * tq && qi < p.Lq;
        const T *q = Q + b * p.qs_b + qi * p.qs_t + (h0 + r % gp) * p.qs_h;
        for (int d = lane; d < Dp; d += 32) sQ[r * kPitch + d] = in && d < p.D ? to_f32(q[d]) : 0.f;
    }
    float4 acc[DM / 16];   // dimensions 16 c + 4 part ..
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) acc[c] = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    const int64_t head = b * p.ks_b + (h0 / p.G) * p.ks_h;
    constexpr int kPiece = 16 / sizeof(T);
    const bool wide = ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 15u) == 0 && p.D % kPiece == 0 &&
                      ((p.ks_b | p.ks_t | p.ks_h) & (kPiece - 1)) == 0;
    for (int t = 0; t < n_tiles; ++t) {
        const int key0 = t < n_a ? t * kKeys : lo + (t - n_a) * kKeys, n_keys = min(kKeys, (t < n_a ? nf : n_vis) - key0);
        __syncthreads();   // the tile before has been read
        if (wide) {        // a warp takes eight rows, a lane 16 bytes of each
            constexpr int N = kPiece, R = kKeys / kWarps;
            for (int c = lane; c < Dp / N; c += 32) {
                uint4 xk[R], xv[R];
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const int r = warp + k * kWarps;
                    const int64_t off = head + (int64_t)(key0 + r) * p.ks_t + c * N;
                    xk[k] = xv[k] = make_uint4(0u, 0u, 0u, 0u);
                    if (r < n_keys && c * N < p.D) {
                        xk[k] = __ldg(reinterpret_cast<const uint4 *>(K + off));
                        xv[k] = __ldg(reinterpret_cast<const uint4 *>(V + off));
                    }
                }
#pragma unroll
                for (int k = 0; k < R; ++k) {
                    const int at_smem = (warp + k * kWarps) * kPitch + c * N;
                    put<T>(sK + at_smem, xk[k]);
                    put<T>(sV + at_smem, xv[k]);
                }
            }
        } else {
            for (int d = lane; d < Dp; d += 32)
#pragma unroll
                for (int k = 0; k < kKeys / kWarps; ++k) {
                    const int r = warp + k * kWarps;
                    const bool in = r < n_keys && d < p.D;
                    const int64_t off = head + (int64_t)(key0 + r) * p.ks_t + d;
                    sK[r * kPitch + d] = in ? to_f32(K[off]) : 0.f;
                    sV[r * kPitch + d] = in ? to_f32(V[off]) : 0.f;
                }
        }
        __syncthreads();
        float s[8];        // keys part + 4 k
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = 0.f;
#pragma unroll 4
        for (int d = 0; d < Dp; d += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(sQ + row * kPitch + d);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float4 x = *reinterpret_cast<const float4 *>(sK + (part + 4 * k) * kPitch + d);
                s[k] = fmaf(q.x, x.x, fmaf(q.y, x.y, fmaf(q.z, x.z, fmaf(q.w, x.w, s[k]))));
            }
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int e = part + 4 * k;
            s[k] = e < n_keys && seen(key0 + e) ? s[k] * p.scale_log2 : -INFINITY;
            top = fmaxf(top, s[k]);
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float base = top == -INFINITY ? 0.f : top, corr = exp2f(m - base);
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            s[k] = exp2f(s[k] - base);
            sum += s[k];
            sP[row * kPitchP + part + 4 * k] = s[k];
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        l = l * corr + sum;
        m = top;
        __syncwarp();      // the row's probabilities come from its own warp
#pragma unroll
        for (int c = 0; c < DM / 16; ++c) { acc[c].x *= corr; acc[c].y *= corr; acc[c].z *= corr; acc[c].w *= corr; }
        // a tile that every row sees needs no look at the mask; elsewhere a value that a row does not see is not touched
        const bool clear = n_keys == kKeys && key0 + kKeys - 1 <= pos0 && ((int64_t)key0 > (int64_t)pos0 + tq - 1 - p.w || key0 + kKeys <= nf);
#pragma unroll 4
        for (int e = 0; e < n_keys; ++e) {
            const bool on = clear || seen(key0 + e);
            const float w = sP[row * kPitchP + e];
#pragma unroll
            for (int c = 0; c < DM / 16; ++c)
                if (16 * c < Dp) {
                    const float4 v = *reinterpret_cast<const float4 *>(sV + e * kPitch + 16 * c + 4 * part);
                    if (on) {
                        acc[c].x = fmaf(w, v.x, acc[c].x); acc[c].y = fmaf(w, v.y, acc[c].y);
                        acc[c].z = fmaf(w, v.z, acc[c].z); acc[c].w = fmaf(w, v.w, acc[c].w);
                    }
                }
        }
    }
    if (!mine) return;
    const RowEnd the_end = row_end(m, l, sink, h);
    if (LSE && part == 0) LSE[((int64_t)b * p.Hq + h) * p.Lq + i] = the_end.lse();
    const int64_t out = b * p.os_b + i * p.os_t + h * p.os_h;
#pragma unroll
    for (int c = 0; c < DM / 16; ++c) {
        const float x[4] = {acc[c].x, acc[c].y, acc[c].z, acc[c].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = 16 * c + 4 * part + e;
            if (d < p.D) from_f32(O[out + d], x[e] * the_end.factor * (p.gate ? gate_of(to_f32(static_cast<const T *>(p.gate)[out + d])) : 1.f));
        }
    }
}

template <typename T, int DM>
cudaError_t launch(const Params &p, int nf, const void *Q, const void *K, const void *V, const float *sink, void *O, float *LSE, cudaStream_t st)
{
    int gp, tq;
    window_row_tile(p, kRows, kKeys, &gp, &tq);
    const int64_t ctas = (int64_t)p.B * ((p.Lq + tq - 1) / tq) * (p.Hq / gp);
    if (ctas > INT_MAX) return cudaErrorInvalidConfiguration;
    static std::atomic<unsigned long long> ready{0};
    const cudaError_t e = opt_in_smem(k_window_simt<T, DM>, smem_bytes<DM>(), ready);
    if (e != cudaSuccess) return e;
    k_window_simt<T, DM><<<(unsigned)ctas, kThreads, smem_bytes<DM>(), st>>>(p, nf < p.Lk ? nf : p.Lk, gp, tq, (const T *)Q, (const T *)K,
                                                                            (const T *)V, sink, (T *)O, LSE);
    count_launch();
    return cudaGetLastError();
}

template <typename T>
cudaError_t by_dim(const Params &p, int nf, const void *Q, const void *K, const void *V, const float *sink, void *O, float *LSE, cudaStream_t st)
{
    if (p.D <= 64) return launch<T, 64>(p, nf, Q, K, V, sink, O, LSE, st);
    return p.D <= 128 ? launch<T, 128>(p, nf, Q, K, V, sink, O, LSE, st) : launch<T, 256>(p, nf, Q, K, V, sink, O, LSE, st);
}

}  // namespace

cudaError_t launch_window_simt(const Params &p, int nf, hs2_dtype dt, const void *Q, const void *K, const void *V, const float *sink, void *O,
                               float *LSE, cudaStream_t st)
{
    return dt == HS2_F32 ? by_dim<float>(p, nf, Q, K, V, sink, O, LSE, st) : by_dim<__nv_bfloat16>(p, nf, Q, K, V, sink, O, LSE, st);
}

// Time per filled row is that of its key tiles and of about two more for its start and its end.  On tcgen05, 24 heads on 8,
// head_dim 128, 8K tokens: three heads x 42 queries against one head x 128: w = 128 46 and 56 us, w = 512 78 and 88.
void window_row_tile(const Params &p, int rows, int key_tile, int *gp, int *tq)
{
    double best = -1.;
    for (int g = 1; g <= p.G && g <= rows; ++g) {
        if (p.G % g) continue;
        const int n = rows / g;
        const int64_t span = (int64_t)p.w + n - 1, keys = span < p.Lk ? span : p.Lk;
        const double cost = (double)((keys + key_tile - 1) / key_tile + 2) / (g * n);
        if (best < 0. || cost <= best) {
            best = cost;
            *gp = g;
            *tq = n;
        }
    }
}

}  // namespace hs2
