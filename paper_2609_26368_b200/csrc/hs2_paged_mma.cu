// Paged decode attention on the tensor cores (mma.sync), bf16 (head_dim 64, 128) or e4m3 cache (128, 256).
//
// One CTA = one chunk of the keys of one (sequence, KV head) and up to 8 NH WH of its query heads.  The keys are read once
// for all those heads, so the kernel is bound by memory (intensity: 2 G flops per byte on a bf16 cache) and the tensor cores
// only keep the arithmetic out of the way:
//   * S^T = K Q^T with 16 keys on the MMA's M and 8 heads on its N: a head group of 8 wastes nothing.  P^T is re-laid out
//     with movmatrix, O^T = V^T P^T reads V through ldmatrix.trans.
//   * four warps: WH of them share the heads (each takes NH tiles of 8), the other 4 / WH share the keys of a tile.
//   * tiles of TK keys travel through a ring of NS stages with 16-byte cp.async, rows XOR-swizzled so that ldmatrix is free
//     of conflicts.  A row's page comes from the table, two tiles ahead of its copy (the entry's latency is never waited
//     for), so a page may end anywhere in a tile.  Void rows (behind the chunk, bad pages) are zero-filled and masked.
//   * online softmax in the base-2 domain; the key warps are joined through shared memory, the chunks by k_paged_combine.
// e4m3: codes become f16 in registers (exact).  The K scale multiplies the score of its key; the V scale, relative to a
// power of two above the largest one met so far, goes into the probability, an f16 number of at most 1 then; all of them are 2^15
// times that, so that they are normal f16 numbers (off by 2^-11) down to 2^-29 and are lost only below 2^-39.  q becomes f16
// in units of a power of two per head (q_unit_of).
#include <cuda_fp16.h>

#include "hs2_paged.cuh"

namespace hs2 {
namespace {

constexpr int kWarps = 4, kThreads = 128;
constexpr float kUpLog2 = 15.f, kDown = 0x1p-15f;   // of the probabilities on an e4m3 cache

template <int D, bool F8, int NH, int WH>
struct Cfg {
    static constexpr int WK = kWarps / WH;
    static constexpr int kRow = D * (F8 ? 1 : 2);                 // bytes of a row
    // keys of a tile: 32 KB of K and V, or 16 KB where four small CTAs fit an SM (128-byte rows, one tile of heads: 64 x 16K
    // keys, 8 heads, e4m3 at head_dim 128 60 us; 66 with 32 KB and two CTAs)
    static constexpr bool kSmall = kRow == 128 && NH == 1;
    static constexpr int kWant = (kSmall ? 8192 : 16384) / kRow;
    static constexpr int TK = kWant < 16 * WK ? 16 * WK : (kWant > 128 ? 128 : kWant);
    static constexpr int KW = TK / WK;                            // keys of a warp per tile
    static constexpr int MT = KW >= 32 ? 2 : 1;                   // 16-key MMA tiles in hand at a time
    static constexpr int NS = 3;
    static constexpr int kTensor = TK * kRow;
    static constexpr int kStage = 2 * kTensor + (F8 ? 2 * TK * 4 : 0);
    static constexpr int HEADS = 8 * NH;                          // heads of a warp
    static constexpr int kPitch = D + 4;                          // floats; lanes of a store hit different banks
    static constexpr int kJoin = kWarps * HEADS * kPitch * 4;
    static constexpr int kBody = NS * kStage > kJoin ? NS * kStage : kJoin;
    static constexpr int kRing = (NS + 1) * TK * 8;
    static constexpr int kSmem = kBody + kRing + kWarps * HEADS * 4 * 4;
    static constexpr int kMinBlocks = kSmall ? 4 : 2 * (kSmem + 1024) <= 227 * 1024 ? 2 : 1;
    static_assert(kMinBlocks * (kSmem + 1024) <= 228 * 1024, "shared memory of an SM");
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(bytes));
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(bytes));
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(a));
    return d;
}
template <bool F8>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2])
{
    if constexpr (F8)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
// two e4m3 codes (low byte first) -> f16x2, exact
__device__ __forceinline__ uint32_t cvt2(uint32_t codes)
{
    uint32_t d;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(d) : "h"((unsigned short)codes));
    return d;
}
template <bool F8> __device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    if constexpr (F8) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    } else {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
}
__device__ __forceinline__ float lo_bf16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

template <int D, bool F8, int NH, int WH>
__global__ void __launch_bounds__(kThreads, Cfg<D, F8, NH, WH>::kMinBlocks)
k_paged_mma(const PagedParams p, const __nv_bfloat16 *__restrict__ Q, const char *__restrict__ K, const char *__restrict__ V,
            const float *__restrict__ ksc, const float *__restrict__ vsc, __nv_bfloat16 *__restrict__ O, float *__restrict__ LSE,
            int head_blocks)
{
    using F = Cfg<D, F8, NH, WH>;
    constexpr int TK = F::TK, NS = F::NS, MT = F::MT, KS = D / 16, ES = F8 ? 1 : 2;
    extern __shared__ __align__(128) char smem[];
    int2 *ring = reinterpret_cast<int2 *>(smem + F::kBody);                    // (page, slot) of every row of NS + 1 tiles
    const int split = blockIdx.x, kvh = blockIdx.y / head_blocks, hb = blockIdx.y - kvh * head_blocks, b = blockIdx.z;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wh = warp / F::WK, wk = warp % F::WK;
    const int g = lane >> 2, t4 = lane & 3, mi = lane >> 3, rr = lane & 7;
    const PagedKeys keys = paged_keys(p, b);
    const int c0 = split * p.chunk;
    if (split > 0 && c0 >= keys.n) return;
    const int c1 = min(keys.n, c0 + p.chunk);
    const int n_tiles = (c1 - c0 + TK - 1) / TK;
    const int head0 = hb * (WH * F::HEADS) + wh * F::HEADS;                    // of the group
    const char *Kh = K + kvh * p.ks_h * ES, *Vh = V + kvh * p.ks_h * ES;
    const uint32_t body = smem_u32(smem);

    auto row_of = [&](int tile) {   // of this thread's row of the tile
        const int slot = c0 + tile * TK + tid;
        return slot < c1 ? paged_row(p, b, keys.key(slot)) : make_int2(-1, 0);
    };
    auto issue = [&](int tile) {
        constexpr int CPR = F::kRow / 16, RPP = kThreads / CPR;               // 16-byte chunks of a row, rows per pass
        const uint32_t stage = body + (tile % NS) * F::kStage;
        const int2 *rows = ring + (tile % (NS + 1)) * TK;
        const int c = tid % CPR, r0 = tid / CPR;
#pragma unroll
        for (int pass = 0; pass < TK / RPP; ++pass) {
            const int r = pass * RPP + r0;
            const int2 at = rows[r];
            const int64_t off = ((int64_t)max(at.x, 0) * p.ks_p + (int64_t)at.y * p.ks_t) * ES + c * 16;
            const int bytes = at.x < 0 ? 0 : 16;
            const uint32_t dst = stage + r * F::kRow + ((uint32_t)(c ^ (r & 7)) << 4);
            cp_async16(dst, Kh + off, bytes);
            cp_async16(dst + F::kTensor, Vh + off, bytes);
        }
        if constexpr (F8) {
            if (tid < TK) {
                const int2 at = rows[tid];
                const int64_t off = (int64_t)max(at.x, 0) * p.ss_p + (int64_t)at.y * p.ss_t + kvh * p.ss_h;
                const uint32_t dst = stage + 2 * F::kTensor + tid * 4;
                cp_async4(dst, ksc + off, at.x < 0 ? 0 : 4);
                cp_async4(dst + TK * 4, vsc + off, at.x < 0 ? 0 : 4);
            }
        }
    };
    if (tid < TK)
        for (int t = 0; t < NS; ++t) ring[t * TK + tid] = row_of(t);
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NS - 1; ++t) {
        if (t < n_tiles) issue(t);
        cp_async_commit();
    }

    // the query fragments (B operand: column = head g, rows = contraction)
    uint32_t qf[NH][KS][2];
    float qs[NH][2];
#pragma unroll
    for (int n = 0; n < NH; ++n) {
        const int h = head0 + n * 8 + g;
        const __nv_bfloat16 *q = Q + b * p.qs_b + (kvh * p.G + min(h, p.G - 1)) * p.qs_h;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int e = 0; e < 2; ++e)   // e4m3: a lane's four codes are dims 4 t .. 4 t + 3
                qf[n][ks][e] = h < p.G ? *reinterpret_cast<const uint32_t *>(q + 16 * ks + (F8 ? 4 * t4 + 2 * e : 2 * t4 + 8 * e)) : 0u;
        qs[n][0] = qs[n][1] = 1.f;
        if constexpr (F8) {
            float top = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int e = 0; e < 2; ++e) top = fmaxf(top, fmaxf(fabsf(lo_bf16(qf[n][ks][e])), fabsf(hi_bf16(qf[n][ks][e]))));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const float unit = q_unit_of(top), inv = 1.f / unit;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int e = 0; e < 2; ++e) qf[n][ks][e] = pack<true>(lo_bf16(qf[n][ks][e]) * inv, hi_bf16(qf[n][ks][e]) * inv);
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) qs[n][hh] = __shfl_sync(0xffffffffu, unit, (2 * t4 + hh) * 4);
        }
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) qs[n][hh] *= p.scale_log2;
    }

    // This thread: heads 2 t4, 2 t4 + 1 of every tile of 8.  bf16: output dims 16 dt + g (o[0..1]) and + 8 (o[2..3]);
    // e4m3: dims 16 dt + 2 g and 2 g + 1.  m is the same over g, l is partial.
    float o[NH][KS][4], m[NH][2], l[NH][2], v_unit = 0.f, v_inv = 0.f;
#pragma unroll
    for (int n = 0; n < NH; ++n) {
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.f;
#pragma unroll
        for (int dt = 0; dt < KS; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][dt][e] = 0.f;
    }

    for (int tile = 0; tile < n_tiles; ++tile) {
        cp_async_wait<NS - 2>();
        __syncthreads();   // the tile is here, and the stage of the tile before is free
        if (tile + NS - 1 < n_tiles) issue(tile + NS - 1);
        cp_async_commit();
        int2 next = make_int2(-1, 0);
        if (tid < TK && tile + NS < n_tiles) next = row_of(tile + NS);

        const uint32_t kbase = body + (tile % NS) * F::kStage, vbase = kbase + F::kTensor;
        const int2 *rows = ring + (tile % (NS + 1)) * TK;
        const float *sks = reinterpret_cast<const float *>(smem + (tile % NS) * F::kStage + 2 * F::kTensor), *svs = sks + TK;
#pragma unroll
        for (int kb = 0; kb < F::KW; kb += 16 * MT) {
            const int row0 = wk * F::KW + kb;
            float s[MT][NH][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
                for (int n = 0; n < NH; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[mt][n][e] = 0.f;
                const uint32_t rowaddr = kbase + (row0 + mt * 16 + (mi & 1) * 8 + rr) * F::kRow;
                if constexpr (F8) {
#pragma unroll
                    for (int c = 0; c < KS; c += 2) {   // one ldmatrix = 16 keys x 32 dims = two MMA steps
                        uint32_t a[4];
                        ldmatrix_x4(a, rowaddr + ((uint32_t)((c + (mi >> 1)) ^ rr) << 4));
                        const uint32_t a0 = cvt2(a[0]), a1 = cvt2(a[1]), a2 = cvt2(a[0] >> 16), a3 = cvt2(a[1] >> 16);
                        const uint32_t b0 = cvt2(a[2]), b1 = cvt2(a[3]), b2 = cvt2(a[2] >> 16), b3 = cvt2(a[3] >> 16);
#pragma unroll
                        for (int n = 0; n < NH; ++n) {
                            mma<true>(s[mt][n], a0, a1, a2, a3, qf[n][c]);
                            mma<true>(s[mt][n], b0, b1, b2, b3, qf[n][c + 1]);
                        }
                    }
                } else {
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        uint32_t a[4];
                        ldmatrix_x4(a, rowaddr + ((uint32_t)((2 * ks + (mi >> 1)) ^ rr) << 4));
#pragma unroll
                        for (int n = 0; n < NH; ++n) mma<false>(s[mt][n], a[0], a[1], a[2], a[3], qf[n][ks]);
                    }
                }
            }
            // rows of this thread: row0 + 16 mt + g + 8 r
            bool ok[MT][2];
            float kf[MT][2], vf[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int row = row0 + mt * 16 + g + 8 * r;
                    ok[mt][r] = rows[row].x >= 0;
                    kf[mt][r] = F8 ? sks[row] : 1.f;
                    vf[mt][r] = F8 ? svs[row] : 1.f;
                }
            float v_corr = 1.f;
            if constexpr (F8) {
                float top = 0.f;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) top = fmaxf(top, fmaxf(fabsf(vf[mt][0]), fabsf(vf[mt][1])));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                if (top > v_unit) {   // the same for the whole warp
                    const float unit = v_unit_of(top);
                    v_inv = 1.f / unit;
                    v_corr = v_unit * v_inv;
                    v_unit = unit;
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) { vf[mt][0] *= v_inv; vf[mt][1] *= v_inv; }
            }
            uint32_t pb[MT][NH][2];
#pragma unroll
            for (int n = 0; n < NH; ++n) {
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float t2 = ok[mt][e >> 1] ? s[mt][n][e] * (F8 ? kf[mt][e >> 1] * qs[n][e & 1] : qs[n][e & 1]) : -INFINITY;
                        s[mt][n][e] = t2;
                        mx[e & 1] = fmaxf(mx[e & 1], t2);
                    }
                float corr[2], use[2];
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    mx[hh] = fmaxf(mx[hh], __shfl_xor_sync(0xffffffffu, mx[hh], 4));
                    mx[hh] = fmaxf(mx[hh], __shfl_xor_sync(0xffffffffu, mx[hh], 8));
                    mx[hh] = fmaxf(mx[hh], __shfl_xor_sync(0xffffffffu, mx[hh], 16));
                    const float m_new = fmaxf(m[n][hh], mx[hh]);
                    use[hh] = m_new == -INFINITY ? 0.f : m_new;
                    corr[hh] = exp2f(m[n][hh] - use[hh]);
                    m[n][hh] = m_new;
                    l[n][hh] *= corr[hh];
                    corr[hh] *= v_corr;
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    float pv[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        pv[e] = exp2f(s[mt][n][e] - (F8 ? use[e & 1] - kUpLog2 : use[e & 1]));
                        l[n][e & 1] += pv[e];
                        if (F8) pv[e] *= vf[mt][e >> 1];
                    }
                    pb[mt][n][0] = movmatrix_trans(pack<F8>(pv[0], pv[1]));   // keys 0 .. 7
                    pb[mt][n][1] = movmatrix_trans(pack<F8>(pv[2], pv[3]));   // keys 8 .. 15
                }
                if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
                    for (int dt = 0; dt < KS; ++dt) {
                        o[n][dt][0] *= corr[0]; o[n][dt][1] *= corr[1];
                        o[n][dt][2] *= corr[0]; o[n][dt][3] *= corr[1];
                    }
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                if constexpr (F8) {
                    const uint32_t rowaddr = vbase + (row0 + mt * 16 + (mi & 1) * 8 + rr) * F::kRow;
#pragma unroll
                    for (int c = 0; c < KS; c += 2) {
                        uint32_t a[4];
                        ldmatrix_x4_trans(a, rowaddr + ((uint32_t)((c + (mi >> 1)) ^ rr) << 4));
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] = __byte_perm(a[e], 0u, 0x3120);   // (dim 2g: two keys | dim 2g + 1: two keys)
                        const uint32_t a0 = cvt2(a[0]), a1 = cvt2(a[0] >> 16), a2 = cvt2(a[1]), a3 = cvt2(a[1] >> 16);
                        const uint32_t b0 = cvt2(a[2]), b1 = cvt2(a[2] >> 16), b2 = cvt2(a[3]), b3 = cvt2(a[3] >> 16);
#pragma unroll
                        for (int n = 0; n < NH; ++n) {
                            mma<true>(o[n][c], a0, a1, a2, a3, pb[mt][n]);
                            mma<true>(o[n][c + 1], b0, b1, b2, b3, pb[mt][n]);
                        }
                    }
                } else {
                    const uint32_t rowaddr = vbase + (row0 + mt * 16 + (mi >> 1) * 8 + rr) * F::kRow;
#pragma unroll
                    for (int dt = 0; dt < KS; ++dt) {
                        uint32_t a[4];
                        ldmatrix_x4_trans(a, rowaddr + ((uint32_t)((2 * dt + (mi & 1)) ^ rr) << 4));
#pragma unroll
                        for (int n = 0; n < NH; ++n) mma<false>(o[n][dt], a[0], a[1], a[2], a[3], pb[mt][n]);
                    }
                }
            }
        }
        if (tid < TK) ring[((tile + NS) % (NS + 1)) * TK + tid] = next;   // the slots of the tile before: nobody reads them now
    }
    cp_async_wait<0>();
    __syncthreads();   // the stages are free: the warps are joined there

    float *so = reinterpret_cast<float *>(smem);
    float *sm = reinterpret_cast<float *>(smem + F::kBody + F::kRing), *sl = sm + kWarps * F::HEADS, *sf = sl + kWarps * F::HEADS;
    const float unit = F8 ? v_unit : 1.f, down = F8 ? kDown : 1.f;
#pragma unroll
    for (int n = 0; n < NH; ++n)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const int row = warp * F::HEADS + n * 8 + 2 * t4 + hh;
            float sum = l[n][hh];
            sum += __shfl_xor_sync(0xffffffffu, sum, 4);
            sum += __shfl_xor_sync(0xffffffffu, sum, 8);
            sum += __shfl_xor_sync(0xffffffffu, sum, 16);
            if (g == 0) { sm[row] = m[n][hh]; sl[row] = sum * down; }
#pragma unroll
            for (int dt = 0; dt < KS; ++dt) {
                so[row * F::kPitch + 16 * dt + (F8 ? 2 * g : g)] = o[n][dt][hh] * down * unit;
                so[row * F::kPitch + 16 * dt + (F8 ? 2 * g + 1 : g + 8)] = o[n][dt][2 + hh] * down * unit;
            }
        }
    __syncthreads();
    const bool whole = keys.n <= p.chunk;   // nothing to join with: finish here
    const int n_heads = min(p.G - hb * (WH * F::HEADS), WH * F::HEADS);
    // a thread per head: the key warps' factors, the result's maximum and denominator
    if (tid < WH * F::HEADS) {
        const int w0 = tid / F::HEADS * F::WK, in = tid % F::HEADS;   // first key warp of the head
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < F::WK; ++w) top = fmaxf(top, sm[(w0 + w) * F::HEADS + in]);
        const float base = top == -INFINITY ? 0.f : top;
        float f[F::WK];
#pragma unroll
        for (int w = 0; w < F::WK; ++w) {
            f[w] = exp2f(sm[(w0 + w) * F::HEADS + in] - base);
            sum += sl[(w0 + w) * F::HEADS + in] * f[w];
        }
        const int h = kvh * p.G + hb * (WH * F::HEADS) + tid;
        float scale = 1.f;
        if (tid < n_heads) {
            if (whole) {
                const RowEnd end = row_end(top, sum, p.sink, h);
                scale = end.factor;
                if (LSE) LSE[(int64_t)b * p.Hq + h] = end.lse();
            } else {
                const int64_t part = ((int64_t)b * p.Hq + h) * p.n_split + split;
                p.part_ml[2 * part] = top;
                p.part_ml[2 * part + 1] = sum;
            }
        }
#pragma unroll
        for (int w = 0; w < F::WK; ++w) sf[(w0 + w) * F::HEADS + in] = f[w] * scale;
    }
    __syncthreads();
    for (int e = tid; e < n_heads * (D / 2); e += kThreads) {
        const int hl = e / (D / 2), d = (e - hl * (D / 2)) * 2, w0 = hl / F::HEADS * F::WK, in = hl % F::HEADS;
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < F::WK; ++w) {
            const int row = (w0 + w) * F::HEADS + in;
            const float2 v = *reinterpret_cast<const float2 *>(so + row * F::kPitch + d);
            x = fmaf(v.x, sf[row], x);
            y = fmaf(v.y, sf[row], y);
        }
        const int h = kvh * p.G + hb * (WH * F::HEADS) + hl;
        if (whole) {
            const int64_t at = b * p.os_b + h * p.os_h + d;
            if (p.gate) {
                const uint32_t gt = *reinterpret_cast<const uint32_t *>(static_cast<const __nv_bfloat16 *>(p.gate) + at);
                x *= gate_of(lo_bf16(gt));
                y *= gate_of(hi_bf16(gt));
            }
            *reinterpret_cast<uint32_t *>(O + at) = pack<false>(x, y);
        } else {
            *reinterpret_cast<float2 *>(p.part_o + (((int64_t)b * p.Hq + h) * p.n_split + split) * D + d) = make_float2(x, y);
        }
    }
}

template <int D, bool F8, int NH, int WH>
cudaError_t launch(const PagedParams &p, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc, void *O,
                   float *LSE, cudaStream_t st)
{
    using F = Cfg<D, F8, NH, WH>;
    const int blocks = (p.G + WH * F::HEADS - 1) / (WH * F::HEADS);
    if ((int64_t)p.Hkv * blocks > 65535 || p.B > 65535) return cudaErrorNotSupported;
    static std::atomic<unsigned long long> ready{0};
    const cudaError_t e = opt_in_smem(k_paged_mma<D, F8, NH, WH>, F::kSmem, ready);
    if (e != cudaSuccess) return e;
    k_paged_mma<D, F8, NH, WH><<<dim3((unsigned)p.n_split, (unsigned)(p.Hkv * blocks), (unsigned)p.B), kThreads, F::kSmem, st>>>(
        p, (const __nv_bfloat16 *)Q, (const char *)K, (const char *)V, ksc, vsc, (__nv_bfloat16 *)O, LSE, blocks);
    count_launch();
    return cudaGetLastError();
}

// by the size of the head group: tiles of 8 heads per warp, and how many warps share the heads instead of the keys
template <int D, bool F8>
cudaError_t by_group(const PagedParams &p, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc, void *O,
                     float *LSE, cudaStream_t st)
{
    if (paged_on_tc5(p, F8)) return launch_paged_tc5(p, Q, K, V, ksc, vsc, O, LSE, st);
    if constexpr (D <= 128 || F8) {
        if (p.G <= 8) return launch<D, F8, 1, 1>(p, Q, K, V, ksc, vsc, O, LSE, st);
        if (p.G <= 16) return launch<D, F8, 2, 1>(p, Q, K, V, ksc, vsc, O, LSE, st);
    }
    if constexpr (D <= 128) {
        if (p.G <= 32) return launch<D, F8, 2, 2>(p, Q, K, V, ksc, vsc, O, LSE, st);
    }
    if constexpr (D == 64) return launch<D, F8, 2, 4>(p, Q, K, V, ksc, vsc, O, LSE, st);
    return cudaErrorNotSupported;
}

}  // namespace

bool paged_mma_supported(const PagedParams &p, hs2_dtype dt, bool fp8, const void *Q, const void *K, const void *V, const void *O)
{
    auto at = [](const void *x, int a) { return reinterpret_cast<uintptr_t>(x) % a == 0; };
    const int row = fp8 ? 16 : 8;   // 16 bytes of the cache
    const int q = paged_on_tc5(p, fp8) ? 16 : 4;   // bytes of a query load
    return dt == HS2_BF16 && (p.D == 128 || p.D == 256 || (p.D == 64 && !fp8)) && at(K, 16) && at(V, 16) && p.ks_p % row == 0 &&
           p.ks_t % row == 0 && p.ks_h % row == 0 && at(Q, q) && p.qs_b % (q / 2) == 0 && p.qs_h % (q / 2) == 0 && at(O, 4) && at(p.gate, 4) &&
           p.os_b % 2 == 0 && p.os_h % 2 == 0;
}

cudaError_t launch_paged_mma(const PagedParams &p, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc,
                             void *O, float *LSE, cudaStream_t st)
{
    if (ksc) return p.D == 128 ? by_group<128, true>(p, Q, K, V, ksc, vsc, O, LSE, st) : by_group<256, true>(p, Q, K, V, ksc, vsc, O, LSE, st);
    if (p.D == 64) return by_group<64, false>(p, Q, K, V, ksc, vsc, O, LSE, st);
    return p.D == 128 ? by_group<128, false>(p, Q, K, V, ksc, vsc, O, LSE, st) : by_group<256, false>(p, Q, K, V, ksc, vsc, O, LSE, st);
}

}  // namespace hs2
