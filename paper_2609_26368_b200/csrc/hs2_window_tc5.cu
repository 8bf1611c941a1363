// Sliding-window attention with first tokens on tcgen05 (bf16, head_dim 64 / 128 / 256).
//
// A row tile of up to 128 rows (MMA M) is TQ consecutive queries x GP heads of one group (GP divides the group, TQ = 128 / GP;
// window_row_tile weighs empty rows against keys), so the keys that it needs span only w + TQ - 1: for the model's w = 128 a
// tile of 128 queries of one head would compute twice what it keeps.  The keys are cut into tiles of 64: the first
// tokens when they lie before the window of every query of the tile, then the keys from the first query's window to the
// last query's position; only tiles on a border pay for masking, and of a short last tile only what is filled.
//
// A row tile of a narrow window is only a few key tiles long, so everything runs on across row tiles:
//   schedule   CTAs (one per SM at head_dim 256, two below) take row tiles one after the other: the grid has a CTA per
//              row tile, and a running CTA cancels the launch of the next one and does its work
//              (clusterlaunchcontrol.try_cancel), asked for one row tile ahead.
//   TMA warp   Q into one of two buffers, the next row tile's while this one's last key tile is in work (at head_dim 256: as soon as
//              the output of the row tile before has left), a ring of K / V tiles, K ahead of V, and the gate, into the row
//              tile's Q buffer once its last Q K^T has run.
//   MMA warp   S = Q K^T into one of 2 to 4 score buffers, ahead of O += P V (P in tensor memory, over the scores it came
//              from), into the next row tile too: while the epilogue holds O, the next row tile's scores and P are made.
//   softmax    4 warps, a row per thread: mask, base-2 online softmax with a lazily updated maximum (O is rescaled only
//              when a row's maximum grew by more than 2^8), P back to tensor memory as bf16.
//   epilogue   O / l times the gate, through shared memory and a TMA store: by the softmax warps where a second CTA covers
//              them, by 8 warps of its own at head_dim 256.  The output leaves from the row tile's Q buffer, where the gate is.
// Measured, us (and the bytes' or products' time at the device's rates): 64 heads on 1, head_dim 256, 8K tokens, w = 128: 156 (83),
// with a gate 192 (125), w = 512: 300 (159); 32 on 4, head_dim 128: 8K, w = 128: 54 (21), w = 1024: 154 (77); 32K, w = 128: 203 (83).
// A narrow window is bound by the chain of a row tile (scores, softmax, P V, epilogue: some 7 us for its 3 key tiles at head_dim
// 256, of which a CTA keeps two in work).  At head_dim 128 a row tile costs its SM 2.4 us and 0.5 us per key tile: a key tile is what
// it is in the full layer's kernel, the fixed part three fifths of w = 128 and a fifth of w = 1024.  P is bf16, V's type on the tensor
// cores: off by 2^-9 of itself, which over many keys moves an output by less than its own rounding.
// What lies behind a cache's end may be anything: keys are masked by selection, V rows are zeroed in shared memory.  A V
// row that is not finite would reach neighbouring queries of the tile as 0 x inf: a row whose sum is not finite is looked
// at again, over its own keys alone.  Behind the first tokens, which end inside a tile, their V is zeros too: the tensor map
// that reads it ends there.
#include "hs2_paged.cuh"
#include "hs2_tc5.cuh"

namespace hs2 {

__device__ unsigned g_window_error;   // bit 0: an mbarrier wait ran out; bit 1: shared memory not aligned

namespace {

using namespace tc5;

constexpr int BM = 128, BN = 64;
constexpr float kRescale = 8.f;   // log2 units
constexpr float kPairedGate = -41.f;   // above it 1 + e^-x is below 2^60, and the product of two of them a normal number

template <int D>
struct Cfg {
    static constexpr int NQ = D / 64;                             // slices of 64 dims = 128-byte rows, 128-byte swizzle
    static constexpr bool kEpi = D > 128;                         // epilogue warps of its own
    static constexpr int kMinBlocks = D > 128 ? 1 : 2;
    static constexpr int NR = D > 64 ? 3 : 6;                     // slots of the K / V ring
    static constexpr uint32_t kQ = NQ * BM * 128, kSlot = NQ * BN * 128;
    static constexpr uint32_t kOffQ = 0, kOffR = 2 * kQ, kOffC = kOffR + NR * kSlot;   // two Q buffers, the ring
    static constexpr uint32_t kOffStat = kOffC + 4 * 16;          // 4 answers of the scheduler; 1 / l of every row
    static constexpr uint32_t kOffBar = kOffStat + (kEpi ? BM * 4 : 0);
    static constexpr uint32_t kSmem = kOffBar + 384;
    static constexpr uint32_t kTmem = D > 128 ? 512 : 256;        // score buffers of 64 columns, then O
    static constexpr int NSB = (kTmem - D) / BN > 4 ? 4 : (kTmem - D) / BN, kColO = NSB * BN;
    static constexpr int A = NSB > 2 ? 2 : 1;                     // K tiles ahead of V: with room for their scores, the V tiles of a
                                                                  // short row tile can all be there before the first P V
    static constexpr int kEpiWarps = kEpi ? 8 : 4, kEpiWarp = kEpi ? 4 : 0;
    static constexpr int kTmaWarp = kEpi ? 12 : 4, kMmaWarp = kTmaWarp + 1;
    static constexpr int kThreads = (kMmaWarp + 1) * 32;
    static constexpr int kReaders = kMmaWarp + 1;                 // warps that read the scheduler's answers
    static_assert(kMinBlocks * (kSmem + 1024) <= 228 * 1024, "shared memory of an SM");
};

enum Bar {
    Q_FULL = 0, Q_FREE = 2, BUF_FREE = 4, S_FULL = 6, P_FULL = 10, PV_DONE = 14, O_FULL = 18, O_FREE, STAT_FULL, STAT_FREE,
    G_FULL = 22,                   // of the gate in either Q buffer: with one for both, the gate of the next row tile, which needs only
                                   // its own Q K^T, could land before the epilogue has looked for this one's
    C_FULL = 24, C_FREE = C_FULL + 4, R_FULL = C_FREE + 4, R_FREE = R_FULL + 6, N_BARS = R_FREE + 6
};
static_assert(N_BARS * 8 + 8 <= 384, "barriers fit");

struct WindowArgs {
    Params p;
    int nf, gp, tq, rows;                // first tokens; heads, queries and rows (gp tq) of a row tile
    int n_slots, slots_per_kv, n_mblk;   // head slots (Hq / gp), of a KV head (G / gp), row tiles of a sequence
    int n_items;
    const float *sink;
    const __nv_bfloat16 *q, *k, *v;
    float *lse;
    int has_gate;
};

// One row tile: which queries, which keys.  Key tiles: n_a of the first tokens, then those from `lo` on.  A row tile that
// sees no key has one key tile without a visible key.
struct Item {
    int b, i0, h0, kvh, pos0;
    int kvl, n_vis, lo, n_a, n_blk;
};

__device__ __forceinline__ Item item_of(const WindowArgs &a, int at)
{
    Item t;
    const Params &p = a.p;
    const int row = at / a.n_slots, slot = at - row * a.n_slots;
    t.b = row / a.n_mblk;
    t.h0 = slot * a.gp;
    t.i0 = (row - t.b * a.n_mblk) * a.tq;
    t.kvh = slot / a.slots_per_kv;
    t.kvl = kvlen_of(p, t.b);
    t.pos0 = pos_of(p, t.b, t.i0);
    const int64_t last = (int64_t)t.pos0 + min(a.tq, p.Lq - t.i0);   // one behind the last query's position
    t.n_vis = (int)max((int64_t)0, min(last, (int64_t)t.kvl));
    const int64_t lo = (int64_t)t.pos0 - p.w + 1;
    t.lo = (int)min(max(lo, (int64_t)0), (int64_t)t.n_vis);
    t.n_a = 0;
    if (a.nf >= t.lo) t.lo = 0;                                      // the first tokens reach into the window: one range
    else if (t.n_vis > 0) t.n_a = (a.nf + BN - 1) / BN;
    t.n_blk = max(1, t.n_a + (t.n_vis - t.lo + BN - 1) / BN);
    return t;
}
// keys of key tile j that any query of the row tile may see
__device__ __forceinline__ int keys_of(const WindowArgs &a, const Item &t, int j)
{
    return j < t.n_a ? min(BN, a.nf - j * BN) : min(BN, t.n_vis - t.lo - (j - t.n_a) * BN);
}
// The order of a row tile's K and V tiles in the ring: K runs A tiles ahead, K0 .. KA V0 K(A+1) V1 ...
template <int A> __device__ __forceinline__ uint32_t k_at(int j) { return (uint32_t)(j <= A ? j : 2 * j - A); }
template <int A> __device__ __forceinline__ uint32_t v_at(int j, int n) { return (uint32_t)(j + A < n ? A + 1 + 2 * j : n + j); }
__device__ __forceinline__ int key0_of(const Item &t, int j) { return j < t.n_a ? j * BN : t.lo + (j - t.n_a) * BN; }

__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int *abort_flag)
{
    return tc5::mbar_wait(bar, parity, abort_flag, &g_window_error);
}
// one arrival per warp: 32 of them on one word are 32 accesses to shared memory
__device__ __forceinline__ void arrive(uint32_t bar)
{
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
// two floats in one 64-bit register: half the instructions for multiplications and sums
__device__ __forceinline__ unsigned long long both(float a, float b)
{
    unsigned long long d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void halves(unsigned long long d, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(d)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b)
{
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float lo_bf16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
// the smaller ones of two pairs, NaN where either is
__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// one look at a phase: the MMA thread looks instead of sleeping, waking up costs it more than the issue slots that it takes
__device__ __forceinline__ bool test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Asks for the index of a CTA of this grid that has not started, which then never will: 16 bytes at `dst`.
__device__ __forceinline__ void ask_next(uint32_t dst, uint32_t bar)
{
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];\n" ::"r"(dst), "r"(bar) : "memory");
}
// The answer: a CTA index, or -1 when every CTA has started.
__device__ __forceinline__ int answer(uint32_t src)
{
    int x;
    asm volatile("{\n .reg .pred p;\n .reg .b128 r;\n ld.shared.b128 r, [%1];\n"
                 " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n mov.b32 %0, -1;\n"
                 " @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n}\n"
                 : "=r"(x) : "r"(src) : "memory");
    return x;
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
// The MMA thread's own instructions are on the critical path of a narrow window, so a descriptor is an addition: the low
// half of `d` (address field, in 16-byte units) plus a constant.
__device__ __forceinline__ uint64_t moved(uint64_t d, uint32_t bytes)
{
    uint32_t lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(d));
    lo += bytes >> 4;
    uint64_t out;
    asm("mov.b64 %0, {%1, %2};" : "=l"(out) : "r"(lo), "r"(hi));
    return out;
}
__device__ __forceinline__ void tma_store_4d(const CUtensorMap *tm, uint32_t src, int c0, int c1, int c2, int c3)
{
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];\n"
                 ::"l"(tm), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}

// Columns [32 c0, 32 c1) of one query and head again, from its keys alone, by a warp: the way out where the sum over the tile is not
// finite, because of a value that the query may or may not see.  A column in which it does see one is settled by a look at the
// query's V rows, at `hint` first, a key whose values were not finite in the row before (-1: none; the next hint is returned); where
// a value that it does not see is to blame, its columns are computed in fp32, as on FMAs.  A lane has eight columns of every
// kGroups-th key; the scores of 32 keys are a lane's each.  One NaN row of V under 64 heads on 1, head_dim 256, w = 4096, where the
// layer takes 1.4 ms: 47 ms (1375 with a row per thread, a column after the other, while all other warps of the CTA wait).
template <int D>
__device__ __noinline__ int row_alone(const WindowArgs &a, const Item &t, int i, int h, int row, char *buf, int c0, int hint)
{
    constexpr int kCols = D > 128 ? D / 2 : D, kPieces = kCols / 8, kGroups = 32 / kPieces;
    const Params &p = a.p;
    const int lane = threadIdx.x & 31, piece = lane % kPieces, group = lane / kPieces, col = c0 * 32 + piece * 8;
    const int pos = t.pos0 + (i - t.i0), end = max(0, min(pos + 1, t.kvl));
    const int lo = (int)max((int64_t)0, min((int64_t)pos - p.w + 1, (int64_t)end)), nf = min(a.nf, lo), n = nf + end - lo;
    auto key = [&](int slot) { return (int64_t)(slot < nf ? slot : lo + (slot - nf)); };   // visible keys in order
    const __nv_bfloat16 *q = a.q + t.b * p.qs_b + i * p.qs_t + h * p.qs_h;
    const __nv_bfloat16 *kh = a.k + t.b * p.ks_b + t.kvh * p.ks_h, *vh = a.v + t.b * p.ks_b + t.kvh * p.ks_h + col;
    auto words = [](const __nv_bfloat16 *x, uint32_t (&w)[4]) {
        const uint4 v = __ldg(reinterpret_cast<const uint4 *>(x));
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    };
    float odd[8], o[8];                             // sums of the values that are not finite; of the others, weighted
#pragma unroll
    for (int e = 0; e < 8; ++e) odd[e] = o[e] = 0.f;
    // adds what is not finite in 8 values; true once no column of the row can change any more
    auto add = [&](const uint32_t (&v)[4]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = e & 1 ? hi_bf16(v[e >> 1]) : lo_bf16(v[e >> 1]);
            if (!(fabsf(x) < INFINITY)) odd[e] += x;
        }
    };
    auto settled = [&]() {
        bool yes = true;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float x = odd[e];
#pragma unroll
            for (int d = kPieces; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
            yes = yes && x != x;
        }
        return __all_sync(0xffffffffu, yes) != 0;
    };
    bool done = false;
    if (hint >= 0 && hint < end && (hint >= lo || hint < nf)) {
        uint32_t v[4];
        words(vh + hint * p.ks_t, v);
        if (group == 0) add(v);
        done = settled();
    }
    constexpr int kAhead = 4;
    for (int s0 = 0; s0 < n && !done; s0 += kGroups * kAhead) {
        uint32_t v[kAhead][4];
        int hit = -1;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int slot = s0 + u * kGroups + group;
            v[u][0] = v[u][1] = v[u][2] = v[u][3] = 0u;
            if (slot < n) words(vh + key(slot) * p.ks_t, v[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)             // an exponent of ones
                if ((v[u][e] & 0x7f80u) == 0x7f80u || (v[u][e] & 0x7f800000u) == 0x7f800000u) hit = s0 + u * kGroups + group;
        const uint32_t hits = __ballot_sync(0xffffffffu, hit >= 0);
        if (!hits) continue;
        hint = (int)key(__shfl_sync(0xffffffffu, hit, __ffs(hits) - 1));
#pragma unroll
        for (int u = 0; u < kAhead; ++u) add(v[u]);
        done = settled();
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int d = kPieces; d < 32; d <<= 1) odd[e] += __shfl_xor_sync(0xffffffffu, odd[e], d);
    bool open = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) open = open || odd[e] == 0.f;
    if (__any_sync(0xffffffffu, open)) {
        float m = -INFINITY, l = 0.f;
        for (int s0 = 0; s0 < n; s0 += 32) {
            float s = -INFINITY;
            if (s0 + lane < n) {
                const __nv_bfloat16 *k = kh + key(s0 + lane) * p.ks_t;
                s = 0.f;
#pragma unroll 4
                for (int d = 0; d < D; d += 8) {
                    uint32_t x[4], y[4];
                    words(q + d, x);
                    words(k + d, y);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s = fmaf(lo_bf16(x[e]), lo_bf16(y[e]), fmaf(hi_bf16(x[e]), hi_bf16(y[e]), s));
                }
                s *= p.scale_log2;
            }
            const float m_new = fmaxf(m, warp_max(s)), base = m_new == -INFINITY ? 0.f : m_new, corr = exp2f(m - base), w = exp2f(s - base);
            m = m_new;
            l = l * corr + warp_sum(w);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] *= corr;
#pragma unroll 4
            for (int u = 0; u < 32; u += kGroups) {
                const float wu = __shfl_sync(0xffffffffu, w, u + group);
                if (s0 + u + group < n) {
                    uint32_t v[4];
                    words(vh + key(s0 + u + group) * p.ks_t, v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        o[2 * e] = fmaf(wu, lo_bf16(v[e]), o[2 * e]);
                        o[2 * e + 1] = fmaf(wu, hi_bf16(v[e]), o[2 * e + 1]);
                    }
                }
            }
        }
        const float factor = row_end(m, l, a.sink, h).factor;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
#pragma unroll
            for (int d = kPieces; d < 32; d <<= 1) o[e] += __shfl_xor_sync(0xffffffffu, o[e], d);
            o[e] *= factor;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = odd[e] == 0.f ? o[e] : odd[e];   // (a NaN is not 0)
    if (a.has_gate) {
        uint32_t x[4];
        words(static_cast<const __nv_bfloat16 *>(p.gate) + t.b * p.os_b + i * p.os_t + h * p.os_h + col, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            o[2 * e] *= gate_of(lo_bf16(x[e]));
            o[2 * e + 1] *= gate_of(hi_bf16(x[e]));
        }
    }
    const int at = col / 8;
    if (group == 0)
        *reinterpret_cast<uint4 *>(buf + (at >> 3) * (BM * 128) + row * 128 + (((at & 7) ^ (row & 7)) << 4)) =
            make_uint4(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]), pack_bf16(o[4], o[5]), pack_bf16(o[6], o[7]));
    return hint;
}

// What finish_row leaves to be done again, of a warp's rows: gates of which a logit is NaN or too low for the paired form (`low`), and
// rows of which a sum is not finite (`alone`).  Out of the way of all others: in finish_row's loop the two cost every call 2 to 4 %.
template <int D>
__device__ __noinline__ void finish_again(const WindowArgs &a, const Item &t, uint32_t o_at, char *buf, int row, int i, int h, float inv, int c0, int c1,
                                          bool alone, bool low)
{
    if (__any_sync(0xffffffffu, low)) {
        const __nv_bfloat16 *gate = static_cast<const __nv_bfloat16 *>(a.p.gate) + t.b * a.p.os_b + i * a.p.os_t + h * a.p.os_h;
#pragma unroll 1
        for (int c = 2 * c0; c < 2 * c1; ++c) {   // 16 columns
            float o[16];
            tmem_ld16(o_at + c * 16, o);
            tmem_wait_ld();
            if (low) {
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = (inv == 0.f ? 0.f : o[e] * inv) * gate_of(to_f32(gate[c * 16 + e]));
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const float *f = o + 8 * q;
                    const int at = 2 * c + q;
                    *reinterpret_cast<uint4 *>(buf + (at >> 3) * (BM * 128) + row * 128 + (((at & 7) ^ (row & 7)) << 4)) =
                        make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
                }
            }
            __syncwarp();
        }
    }
    __syncwarp();
    int hint = -1;
    for (uint32_t rows = __ballot_sync(0xffffffffu, alone); rows; rows &= rows - 1) {
        const int src = __ffs(rows) - 1;
        hint = row_alone<D>(a, t, __shfl_sync(0xffffffffu, i, src), __shfl_sync(0xffffffffu, h, src), row - (threadIdx.x & 31) + src, buf, c0, hint);
    }
}

// Columns [32 c0, 32 c1) of one row's output: O from tensor memory times 1 / denominator and the gate, as bf16 into the
// row's place in the swizzled buffer `buf` (which holds the gate until then).
template <int D>
__device__ __forceinline__ void finish_row(const WindowArgs &a, const Item &t, uint32_t o_at, char *buf, int row, int i, int h, float inv, int c0,
                                           int c1)
{
    float odd = 0.f;                         // NaN if any is not finite
    uint32_t least = 0u;                     // the least gate logits (or 0), NaN if any is
#pragma unroll 1
    for (int c = c0; c < c1; ++c) {
        float o[32];
        tmem_ld32(o_at + c * 32, o);
        tmem_wait_ld();
        float odd0 = 0.f, odd1 = 0.f, odd2 = 0.f, odd3 = 0.f;
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
            odd0 = fmaf(o[e], 0.f, odd0); odd1 = fmaf(o[e + 1], 0.f, odd1);
            odd2 = fmaf(o[e + 2], 0.f, odd2); odd3 = fmaf(o[e + 3], 0.f, odd3);
        }
        odd += (odd0 + odd1) + (odd2 + odd3);
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] *= inv;
        if (inv == 0.f) {   // no key of its own: whatever 0 x V was
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
        }
        __syncwarp();
        char *dst = buf + (c >> 1) * (BM * 128) + row * 128;
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            uint4 *cell = reinterpret_cast<uint4 *>(dst + ((((c & 1) * 4 + q4) ^ (row & 7)) << 4));
            float *f = o + 8 * q4;
            if (a.has_gate) {
                const uint4 gt = *cell;
                const uint32_t wd[4] = {gt.x, gt.y, gt.z, gt.w};
                least = min_bf16x2(least, min_bf16x2(min_bf16x2(gt.x, gt.y), min_bf16x2(gt.z, gt.w)));
                // 1 / (1 + e^-x) and 1 / (1 + e^-y) with one reciprocal: the exponential unit is the busiest one here
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float u = 1.f + exp2f(lo_bf16(wd[e]) * -kLog2e), v = 1.f + exp2f(hi_bf16(wd[e]) * -kLog2e);
                    const float inv_uv = __fdividef(1.f, u * v);
                    f[2 * e] *= v * inv_uv;
                    f[2 * e + 1] *= u * inv_uv;
                }
            }
            *cell = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        }
    }
    // (a row whose logits are NaN, or one without a key, has its sums)
    const bool mine = i < a.p.Lq && row < a.rows, alone = odd != 0.f && inv == inv && inv != 0.f && mine;
    const bool low = mine && !(lo_bf16(least) > kPairedGate && hi_bf16(least) > kPairedGate);
    if (__any_sync(0xffffffffu, alone || low)) finish_again<D>(a, t, o_at, buf, row, i, h, inv, c0, c1, alone, low);
}

template <int D>
__global__ void __launch_bounds__(Cfg<D>::kThreads, Cfg<D>::kMinBlocks)
k_window_tc5(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
             const __grid_constant__ CUtensorMap tmF, const __grid_constant__ CUtensorMap tmO, const __grid_constant__ CUtensorMap tmG, const __grid_constant__ WindowArgs a)
{
    using F = Cfg<D>;
    constexpr int NQ = F::NQ, NR = F::NR;
    extern __shared__ __align__(1024) char smem[];
    const uint32_t sbase = smem_u32(smem);
    if (sbase & 1023u) {   // never seen; refuse rather than run on a misaligned tile
        if (threadIdx.x == 0) atomicOr(&g_window_error, 2u);
        return;
    }
    const uint32_t bars = sbase + F::kOffBar;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + F::kOffBar + N_BARS * 8);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + F::kOffBar + N_BARS * 8 + 4);
    auto bar = [&](int i) { return bars + 8u * i; };
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Params &p = a.p;

    if (tid == 0) {
        *abort_flag = 0;
        for (int i = 0; i < N_BARS; ++i)
            mbar_init(bar(i), (i >= P_FULL && i < P_FULL + 4) || i == STAT_FULL ? BM / 32 : i == O_FREE || i == STAT_FREE ? F::kEpiWarps :
                              i >= C_FREE && i < C_FREE + 4 ? F::kReaders : 1);
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
    auto buffer = [&](uint32_t k) { return sbase + F::kOffQ + (k & 1) * F::kQ; };   // Q, then gate and output of row tile k

    // The row tile behind the k-th one of this CTA, or -1; every warp asks once per k.  (`one`: a single thread speaks for
    // its warp.)
    auto next_item = [&](uint32_t k, bool one) -> int {
        const uint32_t slot = k & 3;
        bool got = wait(bar(C_FULL + slot), (k >> 2) & 1, abort_flag);
        if (!one) got = __all_sync(0xffffffffu, got);
        if (!got) return -1;
        const int at = answer(sbase + F::kOffC + slot * 16);
        fence_proxy_async();   // the next answer comes through the async proxy
        if (!one) __syncwarp();
        if (one || lane == 0) mbar_arrive(bar(C_FREE + slot));
        return at;
    };

    if (warp == F::kTmaWarp) {
        // ------------------------------------------------ loads, and the questions to the scheduler
        if (elect_one()) {
            uint32_t k = 0, r = 0, n_g = 0;   // row tiles, ring slots and gates so far
            bool ok = true;
            auto load = [&](const CUtensorMap *tm, const Item &t, int j) {
                const uint32_t use = r / NR, slot = r - use * NR;
                if (use > 0 && !wait(bar(R_FREE + slot), (use - 1) & 1, abort_flag)) return false;
                mbar_expect_tx(bar(R_FULL + slot), F::kSlot);
#pragma unroll
                for (int sl = 0; sl < NQ; ++sl)
                    tma_load_4d(sbase + F::kOffR + slot * F::kSlot + sl * BN * 128, tm, bar(R_FULL + slot), 64 * sl, t.kvh, key0_of(t, j), t.b);
                ++r;
                return true;
            };
            int at = blockIdx.x;
            for (; ok && at >= 0; ++k) {
                const Item t = item_of(a, at);
                if (k >= 4 && !wait(bar(C_FREE + (k & 3)), ((k >> 2) - 1) & 1, abort_flag)) break;
                mbar_expect_tx(bar(C_FULL + (k & 3)), 16);
                ask_next(sbase + F::kOffC + (k & 3) * 16, bar(C_FULL + (k & 3)));
                if (k >= 2 && !wait(bar(BUF_FREE + (k & 1)), ((k >> 1) - 1) & 1, abort_flag)) { ++k; break; }
                mbar_expect_tx(bar(Q_FULL + (k & 1)), NQ * a.rows * 128);
#pragma unroll
                for (int sl = 0; sl < NQ; ++sl) tma_load_4d(buffer(k) + sl * BM * 128, &tmQ, bar(Q_FULL + (k & 1)), 64 * sl, t.h0, t.i0, t.b);
                for (int j = 0; ok && j < F::A && j < t.n_blk; ++j) ok = load(&tmK, t, j);
                for (int j = 0; ok && j < t.n_blk; ++j) {
                    if (j + F::A < t.n_blk) ok = load(&tmK, t, j + F::A);
                    ok = ok && load(j < t.n_a ? &tmF : &tmV, t, j);
                }
                if (ok && a.has_gate && (ok = wait(bar(Q_FREE + (k & 1)), (k >> 1) & 1, abort_flag))) {   // into Q's place
                    mbar_expect_tx(bar(G_FULL + (k & 1)), NQ * a.rows * 128);
#pragma unroll
                    for (int sl = 0; sl < NQ; ++sl) tma_load_4d(buffer(k) + sl * BM * 128, &tmG, bar(G_FULL + (k & 1)), 64 * sl, t.h0, t.i0, t.b);
                    ++n_g;
                }
                if (ok) at = next_item(k, true);
            }
            if (*abort_flag) {   // let what is in flight land before the CTA goes away: this thread's last uses of each barrier
                auto land = [&](uint32_t b, uint32_t parity) { for (uint32_t it = 0; it < kSpinLimit && !mbar_try_wait(b, parity); ++it) {} };
                for (uint32_t u = r > NR ? r - NR : 0; u < r; ++u) land(bar(R_FULL + u % NR), (u / NR) & 1);
                for (uint32_t u = k > 4 ? k - 4 : 0; u < k; ++u) land(bar(C_FULL + (u & 3)), (u >> 2) & 1);
                for (uint32_t u = k > 2 ? k - 2 : 0; u < k; ++u) land(bar(Q_FULL + (u & 1)), (u >> 1) & 1);
                for (uint32_t u = n_g > 2 ? n_g - 2 : 0; u < n_g; ++u) land(bar(G_FULL + (u & 1)), (u >> 1) & 1);
            }
        }
    } else if (warp == F::kMmaWarp) {
        // ------------------------------------------------ MMA
        if (elect_one()) {
            constexpr uint32_t idS = idesc(BM, BN, 0), idPV = idesc(BM, D, 1);
            const uint64_t dq = smem_desc(sbase + F::kOffQ, 16, 1024), dk = smem_desc(sbase + F::kOffR, 16, 1024),
                           dv = smem_desc(sbase + F::kOffR, BN * 128, 1024);
            // One thread, two queues: S of the next key tile (of this row tile or, when that has all of its S, of the next one)
            // as soon as its K, its Q and a score buffer are there, and P V of the oldest key tile as soon as P, V and O are.
            uint32_t k = 0, base = 0, Ts = 0, Tp = 0;   // row tile of P V, its place in the ring; S and P V issued so far
            Item t = item_of(a, blockIdx.x), nx = t;
            int js = 0, jn = 0, jp = 0;                 // S issued of this and of the next row tile, P V issued of this one
            int next = 0;                               // the next row tile: 0 not asked yet, 1 known, -1 there is none
            uint32_t idle = 0;
            while (true) {
                bool moved_on = false;
                if (next == 0 && js == t.n_blk && test(bar(C_FULL + (k & 3)), (k >> 2) & 1)) {
                    const int at = next_item(k, true);
                    next = at >= 0 ? 1 : -1;
                    if (next > 0) nx = item_of(a, at);
                    moved_on = true;
                }
                const bool ahead = js == t.n_blk;       // the next S is one of the next row tile
                const int j = ahead ? jn : js, n = ahead ? nx.n_blk : t.n_blk;
                if (Ts - Tp < F::NSB && (!ahead || (next > 0 && jn < n))) {
                    const uint32_t kk = k + ahead, u = base + (ahead ? 2 * t.n_blk : 0) + k_at<F::A>(j), use = u / NR, slot = u - use * NR;
                    if (test(bar(R_FULL + slot), use & 1) && (j > 0 || test(bar(Q_FULL + (kk & 1)), (kk >> 1) & 1))) {
                        const uint64_t da = moved(dq, (kk & 1) * F::kQ), db = moved(dk, slot * F::kSlot);
                        const uint32_t sb = Ts % F::NSB, at = tmem + sb * BN;
                        tc_fence_after();
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)   // 16 dims = 32 bytes inside the swizzled 128-byte row
                            umma(at, moved(da, (ks >> 2) * (BM * 128) + (ks & 3) * 32), moved(db, (ks >> 2) * (BN * 128) + (ks & 3) * 32), idS, ks > 0);
                        umma_commit(bar(S_FULL + sb));
                        umma_commit(bar(R_FREE + slot));
                        if (j == n - 1) umma_commit(bar(Q_FREE + (kk & 1)));
                        ++Ts;
                        ++(ahead ? jn : js);
                        moved_on = true;
                    }
                }
                if (jp < js) {
                    const uint32_t sb = Tp % F::NSB, u = base + v_at<F::A>(jp, t.n_blk), use = u / NR, slot = u - use * NR;
                    if (test(bar(P_FULL + sb), (Tp / F::NSB) & 1) && test(bar(R_FULL + slot), use & 1) &&
                        (jp > 0 || k == 0 || test(bar(O_FREE), (k - 1) & 1))) {
                        tc_fence_after();
                        const int steps = (keys_of(a, t, jp) + 15) / 16;   // 16 keys per instruction: P in tensor memory, V MN-major
                        const uint64_t db = moved(dv, slot * F::kSlot);
                        const uint32_t pa = tmem + sb * BN;
#pragma unroll
                        for (int kk = 0; kk < BN / 16; ++kk)
                            if (kk < steps) umma_ts(tmem + F::kColO, pa + kk * 8, moved(db, kk * 2048), idPV, (jp > 0 || kk > 0) ? 1u : 0u);
                        umma_commit(bar(PV_DONE + sb));
                        umma_commit(bar(R_FREE + slot));
                        ++Tp;
                        if (++jp == t.n_blk) {
                            umma_commit(bar(O_FULL));
                            while (next == 0 && !test(bar(C_FULL + (k & 3)), (k >> 2) & 1)) {   // (asked for long ago)
                                if (++idle > 64 * kSpinLimit || ((idle & 1023u) == 0 && *abort_flag)) break;
                            }
                            if (next == 0) {
                                const int at = next_item(k, true);
                                next = at >= 0 ? 1 : -1;
                                if (next > 0) nx = item_of(a, at);
                            }
                            if (next < 0) break;
                            base += 2 * t.n_blk;
                            t = nx;
                            js = jn;
                            jn = jp = 0;
                            next = 0;
                            ++k;
                        }
                        moved_on = true;
                    }
                }
                idle = moved_on ? 0 : idle + 1;
                if ((idle & 1023u) == 1023u && *abort_flag) break;
                if (idle > 16 * kSpinLimit) {
                    atomicOr(&g_window_error, 1u);
                    *abort_flag = 1;
                    break;
                }
            }
        }
    } else {
        const int quarter = warp & 3, row = quarter * 32 + lane;   // row: tensor memory lane
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
        float *s_inv = reinterpret_cast<float *>(smem + F::kOffStat);
        const int q_in = row / a.gp, h_in = row - q_in * a.gp;     // this row's query and head in the tile
        const bool leader = tid == F::kEpiWarp * 32;
        uint32_t k = 0;                                            // row tiles so far
        bool ok = true;
        int at = blockIdx.x;
        // The leader, once the store of the row tile before has left its buffer: the buffer is free for Q again.
        auto pass_on = [&]() {
            if (k > 0) {
                asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");
                mbar_arrive(bar(BUF_FREE + ((k - 1) & 1)));
            }
        };
        // The output of row tile k; false: somebody gave up, all leave.
        auto epilogue = [&](const Item &t, float inv, int c0, int c1) -> bool {
            if (ok) ok = __all_sync(0xffffffffu, wait(bar(O_FULL), k & 1, abort_flag));
            if (ok && a.has_gate) ok = __all_sync(0xffffffffu, wait(bar(G_FULL + (k & 1)), (k >> 1) & 1, abort_flag));
            if (!group_all(1, F::kEpiWarps * 32, ok)) return ok = false;
            tc_fence_after();
            finish_row<D>(a, t, lanes + F::kColO, smem + F::kOffQ + (k & 1) * F::kQ, row, t.i0 + q_in, t.h0 + h_in, inv, c0, c1);
            tc_fence_before();
            arrive(bar(O_FREE));
            fence_proxy_async();
            group_all(1, F::kEpiWarps * 32, true);
            if (leader) {
#pragma unroll
                for (int sl = 0; sl < NQ; ++sl) tma_store_4d(&tmO, buffer(k) + sl * BM * 128, 64 * sl, t.h0, t.i0, t.b);
                asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
            }
            return true;
        };
        if (warp < 4) {
            // ------------------------------------------------ softmax
            uint32_t T = 0, r = 0;                                 // key tiles, ring position
            for (; at >= 0; ++k) {
                const Item t = item_of(a, at);
                float m_used = -INFINITY, l = 0.f;
                const int64_t pos = (int64_t)t.pos0 + q_in;
                for (int j = 0; j < t.n_blk; ++j, ++T) {
                    const uint32_t sb = T % F::NSB, ph = (T / F::NSB) & 1;
                    const int key0 = key0_of(t, j), n_keys = keys_of(a, t, j);
                    const uint32_t s_at = lanes + sb * BN;
                    if (!__all_sync(0xffffffffu, wait(bar(S_FULL + sb), ph, abort_flag))) { ok = false; break; }
                    if (!F::kEpi && j == t.n_blk - 1) {
                        if (leader) pass_on();
                        __syncwarp();
                    }
                    tc_fence_after();
                    // visible: e < e_end and (e >= e_win or e < e_first), e = key - key0 clamped to the tile; as bits.  Most
                    // tiles are visible as a whole to all queries of the row tile.
                    const bool clear = n_keys == BN && (j < t.n_a || (key0 + BN - 1 <= t.pos0 &&
                                       (key0 + BN <= a.nf || (int64_t)key0 > (int64_t)t.pos0 + a.tq - 1 - p.w)));
                    const bool wide = n_keys > 32;                 // the second half of a short tile is left out
                    float s[BN];
                    tmem_ld32(s_at, *reinterpret_cast<float (*)[32]>(&s[0]));
                    if (wide) tmem_ld32(s_at + 32, *reinterpret_cast<float (*)[32]>(&s[32]));
                    tmem_wait_ld();
                    if (!clear) {
                        const int e_end = (int)max((int64_t)0, min(pos + 1 - key0, (int64_t)n_keys));
                        const int e_win = j < t.n_a ? 0 : (int)max((int64_t)0, min(pos - p.w + 1 - key0, (int64_t)BN));
                        const int e_first = min(max(a.nf - key0, 0), BN);
                        auto below = [](int n) { return n >= 64 ? ~0ull : (1ull << n) - 1; };
                        const unsigned long long bits = below(e_end) & (~below(e_win) | below(e_first));
                        const uint32_t seen0 = (uint32_t)bits, seen1 = (uint32_t)(bits >> 32);
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            if (!(seen0 & (1u << e))) s[e] = -INFINITY;
                            if (!(seen1 & (1u << e))) s[32 + e] = -INFINITY;
                        }
                    }
                    auto top = [&](const float *x) {               // four chains of 3-input maxima over 32 scores
                        float mx0 = x[0], mx1 = x[1], mx2 = x[2], mx3 = x[3];
#pragma unroll
                        for (int e = 4; e + 8 <= 32; e += 8) {
                            mx0 = max3(mx0, x[e], x[e + 4]); mx1 = max3(mx1, x[e + 1], x[e + 5]);
                            mx2 = max3(mx2, x[e + 2], x[e + 6]); mx3 = max3(mx3, x[e + 3], x[e + 7]);
                        }
                        return fmaxf(max3(mx0, mx1, x[28]), fmaxf(max3(mx2, mx3, x[29]), fmaxf(x[30], x[31])));
                    };
                    float m_raw = top(s);
                    if (wide) m_raw = fmaxf(m_raw, top(s + 32));
                    const float m_blk = m_raw * p.scale_log2;      // the scale is positive
                    const bool need = m_blk > m_used + kRescale;   // also for the first finite tile
                    const float m_new = need ? m_blk : m_used;
                    if (__any_sync(0xffffffffu, need)) {
                        const float corr = need ? exp2f(m_used - m_new) : 1.f;
                        l *= corr;
                        if (j > 0) {
                            if (!__all_sync(0xffffffffu, wait(bar(PV_DONE + (T - 1) % F::NSB), ((T - 1) / F::NSB) & 1, abort_flag))) { ok = false; break; }
                            tc_fence_after();
#pragma unroll 1
                            for (int c = 0; c < D / 16; ++c) {
                                float o[16];
                                tmem_ld16(lanes + F::kColO + c * 16, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] *= corr;
                                tmem_st16u(lanes + F::kColO + c * 16, *reinterpret_cast<uint32_t (*)[16]>(&o));
                            }
                            tmem_wait_st();
                        }
                    }
                    m_used = m_new;
                    const float neg_m = m_used == -INFINITY ? 0.f : -m_used;
                    const unsigned long long scale2 = both(p.scale_log2, p.scale_log2), neg_m2 = both(neg_m, neg_m);
                    auto exps = [&](const float *x, int col) {     // 32 scores: P, 16 columns over the scores they came from
                        uint32_t pk[16];
                        unsigned long long sum = 0ull;             // two sums side by side
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float y0, y1;
                            halves(fma2(both(x[e], x[e + 1]), scale2, neg_m2), y0, y1);
                            const float p0 = exp2f(y0), p1 = exp2f(y1);
                            sum = add2(sum, both(p0, p1));
                            pk[e >> 1] = pack_bf16(p0, p1);
                        }
                        float l0, l1;
                        halves(sum, l0, l1);
                        l += l0 + l1;
                        tmem_st16u(s_at + col, pk);
                    };
                    exps(s, 0);
                    if (wide) exps(s + 32, 16);
                    // what lies behind the cache's end is not the caller's data: no 0 x NaN from there
                    if (t.kvl < p.Lk && key0 + BN > t.kvl) {
                        const uint32_t u = r + v_at<F::A>(j, t.n_blk), slot = u % NR;   // where V of this tile is
                        if (!__all_sync(0xffffffffu, wait(bar(R_FULL + slot), (u / NR) & 1, abort_flag))) { ok = false; break; }
                        const int z0 = max(0, t.kvl - key0);
                        char *v = smem + F::kOffR + slot * F::kSlot;
                        for (int e = row; e < (BN - z0) * 8 * NQ; e += BM) {
                            const int sl = e / ((BN - z0) * 8), in = e - sl * ((BN - z0) * 8);
                            *reinterpret_cast<uint4 *>(v + sl * (BN * 128) + (z0 + in / 8) * 128 + (in & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async();
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    arrive(bar(P_FULL + sb));
                }
                r += 2 * t.n_blk;
                const int i = t.i0 + q_in, h = t.h0 + h_in;
                const RowEnd end = row_end(m_used, l, a.sink, h);   // (h_in is below gp in the rows behind the last one too)
                if (a.lse && i < p.Lq && row < a.rows && ok) a.lse[((int64_t)t.b * p.Hq + h) * p.Lq + i] = end.lse();
                const float inv = end.factor;
                if constexpr (F::kEpi) {   // hand it over; the epilogue of the row tile before has read its own by then
                    if (ok && k > 0) ok = __all_sync(0xffffffffu, wait(bar(STAT_FREE), (k - 1) & 1, abort_flag));
                    if (!ok) break;
                    s_inv[row] = inv;
                    arrive(bar(STAT_FULL));
                } else {
                    if (!epilogue(t, inv, 0, D / 32)) break;
                }
                at = next_item(k, false);
            }
        } else {
            // ------------------------------------------------ epilogue warps: half a row per thread
            const int part = (warp - F::kEpiWarp) >> 2;
            for (; at >= 0; ++k) {
                const Item t = item_of(a, at);
                if (leader) pass_on();
                __syncwarp();
                ok = __all_sync(0xffffffffu, wait(bar(STAT_FULL), k & 1, abort_flag));
                const float inv = s_inv[row];
                if (ok) arrive(bar(STAT_FREE));
                if (!epilogue(t, inv, part * (D / 64), (part + 1) * (D / 64))) break;
                at = next_item(k, false);
            }
        }
        if (leader) asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory");
    }
    // ------------------------------------------------ everybody arrives, then tensor memory is returned
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == F::kMmaWarp) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(F::kTmem) : "memory");
    }
}

template <int D>
cudaError_t launch(WindowArgs &a, const Params &p, const void *Q, const void *K, const void *V, const void *O, cudaStream_t st)
{
    using F = Cfg<D>;
    CUtensorMap tmQ, tmK, tmV, tmF, tmO, tmG;
    // the stride of an axis of one element means nothing: a harmless one; the map ends behind `len` tokens
    auto map = [&](CUtensorMap *tm, const void *x, int L, int len, int H, int64_t sb, int64_t stt, int64_t sh, int rows, int heads) {
        if (H == 1) sh = D;
        if (L == 1) stt = (int64_t)H * sh;
        if (p.B == 1) sb = (int64_t)L * stt;
        return make_tile_map(tm, x, p.B, len, H, sb, stt, sh, rows, heads, D);
    };
    auto cache = [&](CUtensorMap *tm, const void *x, int len) { return map(tm, x, p.Lk, len, p.Hkv, p.ks_b, p.ks_t, p.ks_h, BN, 1); };
    auto result = [&](CUtensorMap *tm, const void *x) { return map(tm, x, p.Lq, p.Lq, p.Hq, p.os_b, p.os_t, p.os_h, a.tq, a.gp); };
    if (!map(&tmQ, Q, p.Lq, p.Lq, p.Hq, p.qs_b, p.qs_t, p.qs_h, a.tq, a.gp) || !cache(&tmK, K, p.Lk) || !cache(&tmV, V, p.Lk) ||
        !cache(&tmF, V, a.nf > 0 ? a.nf : p.Lk) || !result(&tmO, O) || !result(&tmG, p.gate ? p.gate : O))
        return cudaErrorNotSupported;
    static std::atomic<unsigned long long> ready{0};
    cudaError_t e = opt_in_smem(k_window_tc5<D>, (int)F::kSmem, ready);
    if (e != cudaSuccess) return e;
    k_window_tc5<D><<<(unsigned)a.n_items, F::kThreads, F::kSmem, st>>>(tmQ, tmK, tmV, tmF, tmO, tmG, a);
    count_launch();
    return cudaGetLastError();
}

}  // namespace

bool window_tc5_supported(const Params &p, hs2_dtype dt, const void *Q, const void *K, const void *V, const void *O)
{
    auto m8 = [](int64_t s, int n) { return n == 1 || (s % 8 == 0 && s > 0); };   // TMA: strides in multiples of 16 bytes
    const uintptr_t all = reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V) |
                          reinterpret_cast<uintptr_t>(O) | reinterpret_cast<uintptr_t>(p.gate);
    return dt == HS2_BF16 && (p.D == 64 || p.D == 128 || p.D == 256) && all % 16 == 0 && m8(p.qs_b, p.B) && m8(p.qs_t, p.Lq) && m8(p.qs_h, p.Hq) &&
           m8(p.ks_b, p.B) && m8(p.ks_t, p.Lk) && m8(p.ks_h, p.Hkv) && m8(p.os_b, p.B) && m8(p.os_t, p.Lq) && m8(p.os_h, p.Hq) && tma_available();
}

cudaError_t launch_window_tc5(const Params &p, int nf, const void *Q, const void *K, const void *V, const float *sink, void *O, float *LSE,
                              cudaStream_t st)
{
    WindowArgs a;
    a.p = p;
    a.nf = nf < p.Lk ? nf : p.Lk;
    window_row_tile(p, BM, BN, &a.gp, &a.tq);
    a.rows = a.gp * a.tq;
    a.n_slots = p.Hq / a.gp;
    a.slots_per_kv = p.G / a.gp;
    a.n_mblk = (p.Lq + a.tq - 1) / a.tq;
    const int64_t n_items = (int64_t)p.B * a.n_mblk * a.n_slots;
    if (n_items >= 1 << 30) return cudaErrorNotSupported;
    a.n_items = (int)n_items;
    a.sink = sink;
    a.q = (const __nv_bfloat16 *)Q; a.k = (const __nv_bfloat16 *)K; a.v = (const __nv_bfloat16 *)V;
    a.lse = LSE;
    a.has_gate = p.gate != nullptr;
    if (p.D == 64) return launch<64>(a, p, Q, K, V, O, st);
    return p.D == 128 ? launch<128>(a, p, Q, K, V, O, st) : launch<256>(a, p, Q, K, V, O, st);
}

cudaError_t read_window_error(unsigned *out) { return cudaMemcpyFromSymbol(out, g_window_error, sizeof(unsigned)); }

}  // namespace hs2
