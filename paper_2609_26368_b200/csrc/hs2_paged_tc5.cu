// Paged decode attention on tcgen05, bf16 or e4m3 cache, where mma.sync falls behind the memory: large head groups and
// head_dim 256 (paged_on_tc5).
//
// With 64 heads on one KV head a key costs 128 flops per byte of an e4m3 cache: more than mma.sync delivers beside the
// memory, and converting codes once per head warp would cost more than the products.  So: the heads are the M of one
// tcgen05.mma (M 128, as COPIES copies of a group of up to 128 / COPIES heads), a key tile of 64 is its N, and the codes
// are converted once, on their way into shared memory.
//   look-ups  2 warps, a thread per key of a tile, up to eight tiles ahead: the row's page from the table, its offset, its
//             scales, and its bias: -inf for bad pages and behind the chunk (such rows are zeros).
//   loaders   8 warps: bf16 rows go to shared memory by cp.async, e4m3 rows through registers, converted to f16 (exact) by two
//             groups of four warps, a tile each in turn, so that one loads while the other converts.  Both tensors land as slices of 64 dims in the 128-byte swizzle of the MMA operands.
//   MMA       S = Q K^T (Q in tensor memory) into one of two score buffers, one tile ahead of O += P V (P over its scores).
//   softmax   4 warps, a row per thread: row r is head r % HR, and of a tile's keys it takes block r / HR; the scores of
//             the other copies are the same numbers and their P is zero here.  So 128 threads share the exponentials of 64
//             heads, and each copy is a split of its own: own maximum, own denominator, own sums, joined at the end.
//             Maximum kept lazily (O is rescaled only when it grows by more than 2^8).  e4m3: the K scale multiplies the
//             score of its key, the V scale, relative to a power of two above the largest one met, the probability, an f16
//             number: 2^10 times its value (and the maximum less lazy, 2^5), so that it is a normal one (off by 2^-11) down to 2^-24
//             of the largest and is lost only below 2^-35.  2^7 and 2^8 would save 3 us of 100, 2^13 and 2^2 cost 26.
// Measured (32 x 16K keys, head_dim 256, 64 heads): e4m3 99 us = 2.8 TB/s, bf16 115 us = 4.7 TB/s.  Bound by the chain of a
// tile, which every tile of a CTA walks through: S 0.4 us, then 0.9 us of softmax, whose look-ups and exponentials wait on the
// shared memory that the loaders' stores and the MMA's operands keep busy; the bf16 tiles are near the memory's rate.  A ring of
// codes in shared memory instead of registers took 122 us where these took 104: a third more shared memory traffic.
#include <cuda_fp16.h>

#include "hs2_paged.cuh"
#include "hs2_tc5.cuh"

namespace hs2 {

__device__ unsigned g_paged_error;   // bit 0: an mbarrier wait ran out; bit 1: shared memory not aligned

namespace {

using namespace tc5;

constexpr int BM = 128, BN = 64;
// log2 units: how far a logit may be above the maximum in use; what the probabilities are multiplied by
template <bool F8> constexpr float kRescale = F8 ? 5.f : 8.f;
template <bool F8> constexpr float kUpLog2 = F8 ? 10.f : 0.f;
template <bool F8> constexpr float kDown = F8 ? 0x1p-10f : 1.f;

template <int D, bool F8>
struct Cfg {
    static constexpr int kLoadWarps = 8, kGroups = F8 ? 2 : 1, kLoaders = kLoadWarps * 32 / kGroups;   // loaders of a tile
    static constexpr int kLoadWarp = 4, kLookWarp = kLoadWarp + kLoadWarps, kMmaWarp = kLookWarp + 2, kThreads = (kMmaWarp + 1) * 32;
    static constexpr int NS = D > 128 ? 3 : 4, NM = 8;            // key tiles in shared memory; tiles looked up ahead
    static constexpr uint32_t kTile = D / 64 * BN * 128;
    static constexpr uint32_t kOffK = 0, kOffV = NS * kTile, kOffMeta = 2 * NS * kTile;
    static constexpr uint32_t kMeta = F8 ? BN * 12 + 32 : BN * 4 + 16;   // per tile: bias, whether one of 32 is not 0; K scales, V scales, the largest of 16
    static constexpr int kAny = F8 ? 3 * BN + 4 : BN;
    static constexpr uint32_t kOffOff = kOffMeta + NM * kMeta;    // byte offsets of the rows
    static constexpr uint32_t kOffRow = kOffOff + NM * BN * 8;    // per row: maximum, denominator, factor
    static constexpr uint32_t kOffBar = kOffRow + 3 * BM * 4;
    static constexpr uint32_t kSmem = kOffBar + 512;
    static constexpr uint32_t kTmem = 512;
    static constexpr int kColQ = 2 * BN, kColO = kColQ + D / 2;   // tensor memory: two score buffers, Q, O
    static constexpr int kPitch = D + 4;                          // floats of a joined row
    static constexpr int NP = BN * (D * (F8 ? 1 : 2) / 16) / kLoaders;   // 16-byte pieces of a tile's tensor per loader
    static_assert(BM * kPitch * 4 <= (int)kOffMeta, "the joined rows fit over the tiles");
    static_assert(kColO + D <= 512 && kSmem <= 227 * 1024, "tensor memory, shared memory");
};

enum Bar {
    FULL = 0, FREE = 4, S_FULL = 8, P_FULL = 10, PV_DONE = 12, O_FULL = 14, M_FULL = 15, M_FREE = 23, Q_FULL = 31, N_BARS = 32
};
static_assert(N_BARS * 8 + 8 <= 512, "barriers fit");

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    return tc5::mbar_wait(bar, parity, abort_flag, &g_paged_error);
}
// One arrival per warp: 32 of them on one word are 32 accesses to shared memory, and those of a tile's eleven warps took longer
// than its loads (64 x 16K keys, 64 heads, e4m3 at head_dim 128: 151 us with an arrival per thread).
__device__ __forceinline__ void arrive(uint32_t bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
// one look at a phase, without waiting
__device__ __forceinline__ bool test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t moved(uint64_t d, uint32_t bytes)   // a descriptor `bytes` further on
{
    uint32_t lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(d));
    lo += bytes >> 4;
    uint64_t out;
    asm("mov.b64 %0, {%1, %2};" : "=l"(out) : "r"(lo), "r"(hi));
    return out;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(bytes));
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 ldg_stream(const void *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};\n" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// four e4m3 codes (low byte first) -> two f16x2, exact
__device__ __forceinline__ uint2 cvt4(uint32_t codes)
{
    uint2 d;
    asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}\n" : "=r"(d.x), "=r"(d.y) : "r"(codes));
    return d;
}
template <bool F8> __device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    if constexpr (F8) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    } else {
        return pack_bf16(lo, hi);
    }
}
__device__ __forceinline__ float lo_bf16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
template <int N>
__device__ __forceinline__ void tmem_ldn(uint32_t taddr, float (&v)[N])
{
    static_assert(N == 16 || N == 32 || N == 64, "columns of a thread");
    if constexpr (N == 16) {
        uint32_t *r = reinterpret_cast<uint32_t *>(v);
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                       "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                     : "r"(taddr) : "memory");
    } else {
#pragma unroll
        for (int c = 0; c < N; c += 32) tmem_ld32(taddr + c, *reinterpret_cast<float (*)[32]>(&v[c]));
    }
}

template <int D, bool F8, int COPIES>
__global__ void __launch_bounds__(Cfg<D, F8>::kThreads, 1)
k_paged_tc5(const PagedParams p, const __nv_bfloat16 *__restrict__ Q, const char *__restrict__ K, const char *__restrict__ V,
            const float *__restrict__ ksc, const float *__restrict__ vsc, __nv_bfloat16 *__restrict__ O, float *__restrict__ LSE,
            int head_blocks)
{
    using F = Cfg<D, F8>;
    constexpr int HR = BM / COPIES, NC = BN / COPIES, ES = F8 ? 1 : 2, NP = F::NP, NS = F::NS, NM = F::NM;
    extern __shared__ __align__(1024) char smem[];
    const uint32_t sbase = smem_u32(smem);
    if (sbase & 1023u) {   // never seen; refuse rather than run on a misaligned tile
        if (threadIdx.x == 0) atomicOr(&g_paged_error, 2u);
        return;
    }
    const int split = blockIdx.x, kvh = blockIdx.y / head_blocks, hb = blockIdx.y - kvh * head_blocks, b = blockIdx.z;
    const PagedKeys keys = paged_keys(p, b);
    const int c0 = split * p.chunk;
    if (split > 0 && c0 >= keys.n) return;
    const int c1 = min(keys.n, c0 + p.chunk), n_tiles = (c1 - c0 + BN - 1) / BN;
    const int n_heads = min(p.G - hb * BM, HR);   // (one block of heads unless COPIES is 1)
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t bars = sbase + F::kOffBar;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + F::kOffBar + N_BARS * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + F::kOffBar + N_BARS * 8 + 4);
    auto bar = [&](int i) { return bars + 8u * i; };
    float *s_m = reinterpret_cast<float *>(smem + F::kOffRow), *s_l = s_m + BM, *s_f = s_l + BM;

    if (tid == 0) {
        *abort_flag = 0;
        for (int i = 0; i < N_BARS; ++i) {
            constexpr int kSoft = BM / 32, kLoad = F::kLoaders / 32;
            mbar_init(bar(i), i < FREE ? kLoad : i == P_FULL || i == P_FULL + 1 || i == Q_FULL ? kSoft : i >= M_FREE ? kSoft + kLoad : i >= M_FULL ? 2 : 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == F::kMmaWarp) {   // tensor memory is allocated by a whole warp
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tmem_slot)), "r"(F::kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    float m_used = -INFINITY, l = 0.f, v_unit = 0.f;   // of a softmax thread's row
    bool ok = true;
    if (warp == F::kMmaWarp) {
        // ------------------------------------------------ MMA
        if (elect_one() && n_tiles > 0) {
            constexpr uint32_t kBf16 = (1u << 7) | (1u << 10);   // operand types of the instruction descriptor; 0: f16
            constexpr uint32_t idS = idesc(BM, BN, 0) & ~(F8 ? kBf16 : 0u), idPV = idesc(BM, D, 1) & ~(F8 ? kBf16 : 0u);
            const uint64_t dk = smem_desc(sbase + F::kOffK, 16, 1024), dv = smem_desc(sbase + F::kOffV, BN * 128, 1024);
            auto issue_s = [&](int t) {
                const int use = t / NS, st = t - use * NS;
                if (!wait(bar(FULL + st), use & 1, abort_flag)) return false;
                tc_fence_after();
                const uint64_t db = moved(dk, st * F::kTile);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)   // 16 dims = 32 bytes inside the swizzled 128-byte row
                    umma_ts(tmem + (t & 1) * BN, tmem + F::kColQ + ks * 8, moved(db, (ks >> 2) * (BN * 128) + (ks & 3) * 32), idS, ks > 0);
                umma_commit(bar(S_FULL + (t & 1)));
                return true;
            };
            bool go = wait(bar(Q_FULL), 0, abort_flag) && issue_s(0);
            for (int t = 0, issued = 1; go && t < n_tiles; ++t) {
                const int st = t % NS, sb = t & 1;
                // S of the next tile goes in front of this tile's P V when its K is there first; when memory is late it must not
                // hold up P V, which frees the buffers
                const int use1 = (t + 1) / NS, st1 = t + 1 - use1 * NS;
                uint32_t it = 0;
                while (go && !test(bar(P_FULL + sb), (t >> 1) & 1)) {
                    if (issued == t + 1 && t + 1 < n_tiles && test(bar(FULL + st1), use1 & 1)) {
                        go = issue_s(t + 1);
                        ++issued;
                    }
                    if ((++it & 255u) == 0 && *abort_flag) go = false;
                    if (it > 16 * kSpinLimit) {
                        atomicOr(&g_paged_error, 1u);
                        *abort_flag = 1;
                        go = false;
                    }
                }
                if (!go) break;
                tc_fence_after();
                const uint64_t db = moved(dv, st * F::kTile);
#pragma unroll
                for (int kk = 0; kk < BN / 16; ++kk)   // 16 keys per instruction: P in tensor memory, V MN-major
                    umma_ts(tmem + F::kColO, tmem + sb * BN + kk * 8, moved(db, kk * 2048), idPV, (t > 0 || kk > 0) ? 1u : 0u);
                umma_commit(bar(PV_DONE + sb));
                umma_commit(bar(FREE + st));
                if (t == n_tiles - 1) umma_commit(bar(O_FULL));
                else if (issued == t + 1) {
                    go = issue_s(t + 1);
                    ++issued;
                }
            }
        }
    } else if (warp >= F::kLookWarp) {
        // ------------------------------------------------ look-ups: a thread per key of a tile, up to NM tiles ahead
        const int r = tid - F::kLookWarp * 32;
        int64_t *s_off = reinterpret_cast<int64_t *>(smem + F::kOffOff) + r;   // byte offset of the row, -1: void
        auto row_of = [&](int t) {
            const int slot = c0 + t * BN + r;
            return slot < c1 ? paged_row(p, b, keys.key(slot)) : make_int2(-1, 0);
        };
        int2 at = row_of(0), next = row_of(1);
        for (int t = 0; ok && t < n_tiles; ++t) {
            const int use = t / NM, st = t - use * NM;
            float ks = 0.f, vs = 0.f;
            if (F8 && at.x >= 0) {
                const int64_t s = (int64_t)at.x * p.ss_p + (int64_t)at.y * p.ss_t + kvh * p.ss_h;
                ks = __ldg(ksc + s);
                vs = __ldg(vsc + s);
            }
            const int2 later = row_of(t + 2);
            ok = __all_sync(0xffffffffu, use == 0 || wait(bar(M_FREE + st), (use - 1) & 1, abort_flag));
            if (!ok) break;
            s_off[st * BN] = at.x < 0 ? -1 : ((int64_t)at.x * p.ks_p + (int64_t)at.y * p.ks_t) * ES;
            float *x = reinterpret_cast<float *>(smem + F::kOffMeta + st * F::kMeta);
            x[r] = at.x < 0 ? -INFINITY : 0.f;
            const bool any = __any_sync(0xffffffffu, at.x < 0);
            if (lane == 0) x[F::kAny + r / 32] = any ? 1.f : 0.f;
            if (F8) {
                x[BN + r] = ks;
                x[2 * BN + r] = vs;
                float top = fabsf(vs);   // the largest V scale of every 16 keys
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                if ((r & 15) == 0) x[3 * BN + r / 16] = top;
            }
            arrive(bar(M_FULL + st));
            at = next;
            next = later;
        }
    } else if (warp >= F::kLoadWarp) {
        // ------------------------------------------------ loaders: 16-byte piece c of the rows r0 + i RPP
        constexpr int CPR = D * ES / 16, RPP = F::kLoaders / CPR;
        const int lt = (tid - F::kLoadWarp * 32) % F::kLoaders, c = lt % CPR, r0 = lt / CPR, group = (tid - F::kLoadWarp * 32) / F::kLoaders;
        const char *Kh = K + kvh * p.ks_h * ES + c * 16, *Vh = V + kvh * p.ks_h * ES + c * 16;
        const int64_t *s_off = reinterpret_cast<const int64_t *>(smem + F::kOffOff) + r0;
        auto all = [&](bool got) -> bool { return __all_sync(0xffffffffu, got); };
        auto looked_up = [&](int t) { return all(wait(bar(M_FULL + t % NM), (t / NM) & 1, abort_flag)); };
        if constexpr (F8) {
            // codes wait in registers, two tiles ahead; piece c of a row is dims 16 c .. 16 c + 15: two 16-byte f16 pieces
            const uint32_t odd = (c >> 2) & 1;   // pieces of odd slices of 64 dims go back half first: no two lanes on a bank
            uint4 kd[NP], vd[NP];
            auto fetch = [&](int t) {
                if (t >= n_tiles || !ok || !(ok = looked_up(t))) return;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const int64_t off = s_off[(t % NM) * BN + i * RPP];
                    kd[i] = vd[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (off >= 0) {
                        kd[i] = ldg_stream(Kh + off);
                        vd[i] = ldg_stream(Vh + off);
                    }
                }
                arrive(bar(M_FREE + t % NM));
            };
            auto put = [&](const uint4 (&x)[NP], uint32_t tile) {
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const int r = r0 + i * RPP;
                    const uint32_t at = tile + (c >> 2) * (BN * 128) + r * 128;
                    const uint2 d0 = cvt4(odd ? x[i].z : x[i].x), d1 = cvt4(odd ? x[i].w : x[i].y), d2 = cvt4(odd ? x[i].x : x[i].z), d3 = cvt4(odd ? x[i].y : x[i].w);
                    const uint32_t col = ((c & 3) * 2 + odd) ^ (r & 7);
                    sts128(at + (col << 4), d0.x, d0.y, d1.x, d1.y);
                    sts128(at + ((col ^ 1) << 4), d2.x, d2.y, d3.x, d3.y);
                }
            };
            fetch(group);
            for (int t = group; ok && t < n_tiles; t += F::kGroups) {
                const int use = t / NS, st = t - use * NS;
                if (use > 0 && !(ok = all(wait(bar(FREE + st), (use - 1) & 1, abort_flag)))) break;
                if (t == NS - 1 && !(ok = all(wait(bar(Q_FULL), 0, abort_flag)))) break;   // Q was turned there
                put(kd, sbase + F::kOffK + st * F::kTile);
                put(vd, sbase + F::kOffV + st * F::kTile);
                fence_proxy_async();
                arrive(bar(FULL + st));
                fetch(t + F::kGroups);
            }
        } else {
            // rows by cp.async, a tile of K and of V per copy group; a tile is announced one tile later, when its copies have
            // landed, and before the wait for a buffer (the MMA warp takes S of a tile before P V of the one before)
            auto copy = [&](const char *src, uint32_t tile, int t) {
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const int r = r0 + i * RPP;
                    const int64_t off = s_off[(t % NM) * BN + i * RPP];
                    cp_async16(tile + (c >> 3) * (BN * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4), src + (off < 0 ? 0 : off), off < 0 ? 0 : 16);
                }
            };
            auto announce = [&](int t) {
                fence_proxy_async();
                arrive(bar(FULL + t % NS));
            };
            for (int t = 0; ok && t < n_tiles; ++t) {
                const int use = t / NS, st = t - use * NS;
                if (t >= 2) {
                    cp_async_wait<1>();
                    announce(t - 2);
                }
                ok = looked_up(t) && (use == 0 || all(wait(bar(FREE + st), (use - 1) & 1, abort_flag)));
                if (ok && t == NS - 1) ok = all(wait(bar(Q_FULL), 0, abort_flag));   // Q was turned there
                if (!ok) break;
                copy(Kh, sbase + F::kOffK + st * F::kTile, t);
                copy(Vh, sbase + F::kOffV + st * F::kTile, t);
                cp_async_commit();
                arrive(bar(M_FREE + t % NM));
            }
            if (ok && n_tiles > 1) {
                cp_async_wait<1>();
                announce(n_tiles - 2);
            }
            cp_async_wait<0>();
            if (ok && n_tiles > 0) announce(n_tiles - 1);
        }
    } else {
        // ------------------------------------------------ softmax
        const int row = tid, copy = row / HR;
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
        // Q into tensor memory first, the A operand of S: lane = row, a column = two dims.  (From shared memory it would be read
        // again for every key tile, three times the bytes of K.)  On an e4m3 cache as f16 in units of a power of two per head.
        // The rows come by cp.async into the last K tile's place, which the loaders leave alone until then; short loops, because
        // code that runs once costs mostly its own fetch.
        float f_row = 0.f;   // the row's logit unit, in log2 units
        {
            constexpr int HT = (int)F::kTile / (D * 2), ROUNDS = HR > HT ? HR / HT : 1, HN = HR / ROUNDS;   // heads of a round
            constexpr int PR = D / 8;                                                                         // 16-byte pieces of a row
            char *turn = smem + F::kOffK + (NS - 1) * F::kTile;
#pragma unroll 1
            for (int round = 0; round < ROUNDS; ++round) {
#pragma unroll 4
                for (int e = row; e < HN * PR; e += BM) {
                    const int i = e / PR, c = e % PR, h = round * HN + i;
                    const __nv_bfloat16 *src = Q + b * p.qs_b + (kvh * p.G + hb * BM + min(h, n_heads - 1)) * p.qs_h + c * 8;
                    cp_async16(smem_u32(turn) + i * (D * 2) + ((c ^ (i & 7)) << 4), src, h < n_heads ? 16 : 0);
                }
                cp_async_commit();
                cp_async_wait<0>();
                group_all(1, BM, true);
                const int i = row % HR - round * HN;
                if (ROUNDS == 1 || (warp * 32 % HR) / HN == round) {   // this warp's rows
                    auto piece = [&](int c) { return *reinterpret_cast<const uint4 *>(turn + i * (D * 2) + ((c ^ (i & 7)) << 4)); };
                    float unit = 1.f, inv = 1.f;
                    if (F8) {
                        uint32_t top = 0u;   // of two dims at a time, as magnitudes: larger bits are larger numbers
#pragma unroll 4
                        for (int c = 0; c < PR; ++c) {
                            const uint4 x = piece(c);
                            top = __vmaxu2(top, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
                        }
                        const uint32_t most = max(top >> 16, top & 0xffffu) << 16;
                        unit = q_unit_of(__uint_as_float(most));
                        inv = 1.f / unit;
                    }
                    f_row = fmaxf(unit * p.scale_log2, 0x1p-126f);   // positive: void keys have logits of -inf
#pragma unroll 1
                    for (int c = 0; c < PR; c += 4) {   // 16 columns
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint4 x = piece(c + e);
                            const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int k = 0; k < 4; ++k) w[4 * e + k] = F8 ? pack<true>(lo_bf16(y[k]) * inv, hi_bf16(y[k]) * inv) : y[k];
                        }
                        tmem_st16u(lanes + F::kColQ + c * 4, w);
                    }
                }
                group_all(1, BM, true);
            }
            tmem_wait_st();
            tc_fence_before();
            arrive(bar(Q_FULL));
        }
        for (int t = 0; t < n_tiles; ++t) {
            const int st = t & 1;
            const uint32_t s_at = lanes + st * BN;
            if (!__all_sync(0xffffffffu, wait(bar(M_FULL + t % NM), (t / NM) & 1, abort_flag))) { ok = false; break; }
            // what the look-up left is fetched before the scores are there
            const float *meta = reinterpret_cast<const float *>(smem + F::kOffMeta + (t % NM) * F::kMeta);
            const float4 *bias = reinterpret_cast<const float4 *>(meta) + copy * (NC / 4);
            const bool voids = COPIES == 1 ? meta[F::kAny] + meta[F::kAny + 1] > 0.f : meta[F::kAny + copy * NC / 32] > 0.f;
            float v_top = 0.f;
            constexpr bool kAhead = F8 && NC <= 32;   // (a whole tile's scales do not fit the registers)
            float4 x[kAhead ? NC / 4 : 1];
            if constexpr (F8) {
#pragma unroll
                for (int e = 0; e < NC / 16; ++e) v_top = fmaxf(v_top, meta[3 * BN + copy * (NC / 16) + e]);
                if constexpr (kAhead) {
#pragma unroll
                    for (int e = 0; e < NC / 4; ++e) x[e] = bias[BN / 4 + e];
                }
            }
            if (!__all_sync(0xffffffffu, wait(bar(S_FULL + st), (t >> 1) & 1, abort_flag))) { ok = false; break; }
            tc_fence_after();
            float s[NC];
            tmem_ldn<NC>(s_at + copy * NC, s);
            tmem_wait_ld();
            // s becomes the logit in the row's unit f_row (log2 units: times f_row)
            if constexpr (F8) {
#pragma unroll
                for (int e = 0; e < NC / 4; ++e) {
                    const float4 kv = kAhead ? x[kAhead ? e : 0] : bias[BN / 4 + e];
                    s[4 * e] *= kv.x;
                    s[4 * e + 1] *= kv.y;
                    s[4 * e + 2] *= kv.z;
                    s[4 * e + 3] *= kv.w;
                }
                if constexpr (kAhead) {   // V scales, for later
#pragma unroll
                    for (int e = 0; e < NC / 4; ++e) x[e] = bias[2 * (BN / 4) + e];
                }
            }
            if (voids) {
#pragma unroll
                for (int e = 0; e < NC / 4; ++e) {
                    const float4 bv = bias[e];
                    s[4 * e] += bv.x;
                    s[4 * e + 1] += bv.y;
                    s[4 * e + 2] += bv.z;
                    s[4 * e + 3] += bv.w;
                }
            }
            float top0 = -INFINITY, top1 = -INFINITY;
#pragma unroll
            for (int e = 0; e < NC; e += 4) {
                top0 = max3(top0, s[e], s[e + 1]);
                top1 = max3(top1, s[e + 2], s[e + 3]);
            }
            const float top = fmaxf(top0, top1) * f_row;   // f_row is positive
            const bool need = top > m_used + kRescale<F8>;   // also for the first visible key
            const bool grow = F8 && v_top > v_unit;
            float m_new = m_used;
            if (__any_sync(0xffffffffu, need || grow)) {
                m_new = fmaxf(m_used, top);   // of every row, while the warp is at it
                const float corr_l = m_new > m_used ? exp2f(m_used - m_new) : 1.f;
                l *= corr_l;
                float corr = corr_l;
                if (grow) {
                    const float unit = v_unit_of(v_top);
                    corr *= v_unit / unit;
                    v_unit = unit;
                }
                if (t > 0) {
                    if (!__all_sync(0xffffffffu, wait(bar(PV_DONE + (st ^ 1)), ((t - 1) >> 1) & 1, abort_flag))) { ok = false; break; }
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        float o[16];
                        tmem_ldn<16>(lanes + F::kColO + c * 16, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] *= corr;
                        tmem_st16u(lanes + F::kColO + c * 16, *reinterpret_cast<uint32_t (*)[16]>(&o));
                    }
                    tmem_wait_st();
                }
            }
            m_used = m_new;
            const float base = (m_used == -INFINITY ? 0.f : m_used) - kUpLog2<F8>, v_inv = F8 && v_unit > 0.f ? 1.f / v_unit : 0.f;
            uint32_t pk[NC / 2];
            float l0 = 0.f, l1 = 0.f;
#pragma unroll
            for (int e = 0; e < NC / 4; ++e) {
                float p0 = exp2f(fmaf(s[4 * e], f_row, -base)), p1 = exp2f(fmaf(s[4 * e + 1], f_row, -base));
                float p2 = exp2f(fmaf(s[4 * e + 2], f_row, -base)), p3 = exp2f(fmaf(s[4 * e + 3], f_row, -base));
                l0 += p0 + p2;
                l1 += p1 + p3;
                if constexpr (F8) {
                    const float4 vv = kAhead ? x[kAhead ? e : 0] : bias[2 * (BN / 4) + e];
                    p0 *= vv.x * v_inv; p1 *= vv.y * v_inv; p2 *= vv.z * v_inv; p3 *= vv.w * v_inv;
                }
                pk[2 * e] = pack<F8>(p0, p1);
                pk[2 * e + 1] = pack<F8>(p2, p3);
            }
            l += l0 + l1;
            arrive(bar(M_FREE + t % NM));
            // P of all 64 keys: this copy's block, zeros elsewhere
            if constexpr (COPIES == 1) {
                tmem_st32u(s_at, pk);
            } else {
                constexpr int W = NC / 2;
                uint32_t all[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) all[e] = e / W == copy ? pk[e % W] : 0u;
                tmem_st32u(s_at, all);
            }
            tmem_wait_st();
            tc_fence_before();
            arrive(bar(P_FULL + st));
        }
        if (ok && n_tiles > 0 && !__all_sync(0xffffffffu, wait(bar(O_FULL), 0, abort_flag))) ok = false;
        tc_fence_after();
    }
    __syncthreads();   // no tile is read any more: the rows are joined in their place
    float *so = reinterpret_cast<float *>(smem);
    if (warp < 4) {
        const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
        const float scale = l == 0.f ? 0.f : F8 ? v_unit : 1.f, down = kDown<F8>;
        s_m[tid] = m_used;
        s_l[tid] = l * down;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
            float o[32];
            if (n_tiles > 0) {
                tmem_ld32(lanes + F::kColO + c * 32, o);
                tmem_wait_ld();
            }
#pragma unroll
            for (int e = 0; e < 32; e += 4)
                *reinterpret_cast<float4 *>(so + tid * F::kPitch + c * 32 + e) = l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) :
                    make_float4(o[e] * down * scale, o[e + 1] * down * scale, o[e + 2] * down * scale, o[e + 3] * down * scale);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == F::kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(F::kTmem) : "memory");
    }
    const bool whole = keys.n <= p.chunk;   // nothing to join with: finish here
    if (tid < HR) {   // a thread per head: the copies' factors, the result's maximum and denominator
        float top = -INFINITY, sum = 0.f, f[COPIES];
#pragma unroll
        for (int c = 0; c < COPIES; ++c) top = fmaxf(top, s_m[c * HR + tid]);
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int c = 0; c < COPIES; ++c) {
            f[c] = exp2f(s_m[c * HR + tid] - base);
            sum += s_l[c * HR + tid] * f[c];
        }
        const int h = kvh * p.G + hb * BM + tid;
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
        for (int c = 0; c < COPIES; ++c) s_f[c * HR + tid] = f[c] * scale;
    }
    __syncthreads();
    for (int e = tid; e < n_heads * (D / 2); e += F::kThreads) {
        const int hl = e / (D / 2), d = (e - hl * (D / 2)) * 2;
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int c = 0; c < COPIES; ++c) {
            const float2 v = *reinterpret_cast<const float2 *>(so + (c * HR + hl) * F::kPitch + d);
            const float f = s_f[c * HR + hl];
            x = fmaf(v.x, f, x);
            y = fmaf(v.y, f, y);
        }
        const int h = kvh * p.G + hb * BM + hl;
        if (whole) {
            const int64_t at = b * p.os_b + h * p.os_h + d;
            if (p.gate) {
                const uint32_t gt = *reinterpret_cast<const uint32_t *>(static_cast<const __nv_bfloat16 *>(p.gate) + at);
                x *= gate_of(lo_bf16(gt));
                y *= gate_of(hi_bf16(gt));
            }
            *reinterpret_cast<uint32_t *>(O + at) = pack_bf16(x, y);
        } else {
            *reinterpret_cast<float2 *>(p.part_o + (((int64_t)b * p.Hq + h) * p.n_split + split) * D + d) = make_float2(x, y);
        }
    }
}

template <int D, bool F8, int COPIES>
cudaError_t launch(const PagedParams &p, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc, void *O,
                   float *LSE, cudaStream_t st)
{
    using F = Cfg<D, F8>;
    const int blocks = (p.G + BM - 1) / BM;
    if ((int64_t)p.Hkv * blocks > 65535 || p.B > 65535) return cudaErrorNotSupported;
    static std::atomic<unsigned long long> ready{0};
    const cudaError_t e = opt_in_smem(k_paged_tc5<D, F8, COPIES>, (int)F::kSmem, ready);
    if (e != cudaSuccess) return e;
    k_paged_tc5<D, F8, COPIES><<<dim3((unsigned)p.n_split, (unsigned)(p.Hkv * blocks), (unsigned)p.B), F::kThreads, F::kSmem, st>>>(
        p, (const __nv_bfloat16 *)Q, (const char *)K, (const char *)V, ksc, vsc, (__nv_bfloat16 *)O, LSE, blocks);
    count_launch();
    return cudaGetLastError();
}

template <int D, bool F8>
cudaError_t by_group(const PagedParams &p, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc, void *O,
                     float *LSE, cudaStream_t st)
{
    if constexpr (D > 128) {
        if (p.G <= 32) return launch<D, F8, 4>(p, Q, K, V, ksc, vsc, O, LSE, st);
    }
    if (p.G <= 64) return launch<D, F8, 2>(p, Q, K, V, ksc, vsc, O, LSE, st);
    return launch<D, F8, 1>(p, Q, K, V, ksc, vsc, O, LSE, st);
}

}  // namespace

cudaError_t launch_paged_tc5(const PagedParams &p, const void *Q, const void *K, const void *V, const float *ksc, const float *vsc,
                             void *O, float *LSE, cudaStream_t st)
{
    if (ksc) return p.D == 128 ? by_group<128, true>(p, Q, K, V, ksc, vsc, O, LSE, st) : by_group<256, true>(p, Q, K, V, ksc, vsc, O, LSE, st);
    return p.D == 128 ? by_group<128, false>(p, Q, K, V, ksc, vsc, O, LSE, st) : by_group<256, false>(p, Q, K, V, ksc, vsc, O, LSE, st);
}

cudaError_t read_paged_error(unsigned *out) { return cudaMemcpyFromSymbol(out, g_paged_error, sizeof(unsigned)); }

}  // namespace hs2
