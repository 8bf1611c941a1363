"""Calls of the sliding-window layer, the paged decode and the page operations at the ends of what their arguments may be."""
import pytest
import torch

import paper_2609_26368_b200 as hs2
import plain_ops

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")
INT_MAX = 2 ** 31 - 1


def rand(g, *shape, dtype=BF16, scale=1.0):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- pages
@pytest.mark.parametrize("ps", [1, 2, 16])
def test_pages_free_keeps_everything_for_a_keep_of_any_size(ps):
    pool, plain = hs2.PagePool.empty(600, ps, 4, 300), plain_ops.Pool(600, ps, 4, 300)
    seqs, n_new = [0, 1, 3], [200, 1, 77]
    assert hs2.hs2_pages_reserve(pool, [], i32(seqs), i32(n_new)).tolist() == plain.reserve(seqs, n_new)
    for keep in ([INT_MAX, INT_MAX - 1, INT_MAX - 127], [200, INT_MAX, 78], [INT_MAX, 0, 30]):
        hs2.hs2_pages_free(pool, i32(seqs), i32(keep))
        plain.free(seqs, keep)
        assert pool.ref_counts.tolist() == plain.refs and pool.lens.tolist() == plain.lens
        assert pool.page_table.tolist() == plain.matrix()


# ---------------------------------------------------------------- sliding window: many row tiles per CTA
MANY = [
    # Hq, Hkv, D, w, first, B, Lq, Lk: with one, two, three and more key tiles per row tile, and thousands of row tiles
    (16, 2, 64, 20, 0, 2, 9001, 9100),
    (16, 2, 64, 49, 3, 2, 9001, 9100),
    (16, 2, 64, 130, 70, 2, 5000, 5007),
    (32, 4, 128, 20, 0, 2, 5000, 5100),
    (32, 4, 128, 49, 4, 2, 5000, 5100),
    (32, 4, 128, 100, 0, 2, 5000, 5000),
    (24, 8, 128, 300, 5, 2, 4001, 4100),
    (64, 1, 256, 20, 0, 2, 3001, 3100),
    (64, 1, 256, 63, 0, 2, 3001, 3100),
    (64, 1, 256, 64, 2, 2, 3001, 3100),
    (64, 1, 256, 128, 0, 2, 3001, 3100),
    (5, 1, 256, 250, 1, 1, 12000, 12001),
]


@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gate"])
@pytest.mark.parametrize("case", MANY, ids=str)
def test_window_of_many_row_tiles(case, gated):
    """Each CTA works through many row tiles, whose loads, products and outputs overlap.  All rows are compared with the fp32
    kernel, which has one row tile per CTA, and sampled ones with the 64-bit form.

    Bounds as in plain_ops; the weights' sum A = sum_j w_j |v_j| comes from the fp32 kernel on |v|.  Both sides have the error of a
    logit, at most (D + 4) 2^-24 scale |q| |k|, so a weight may differ by 4 of them relative to itself."""
    Hq, Hkv, D, w, nf, B, Lq, Lk = case
    g = torch.Generator().manual_seed(sum(case))
    q, k, v = rand(g, B, Lq, Hq, D, scale=1.5), rand(g, B, Lk, Hkv, D), rand(g, B, Lk, Hkv, D)
    sink = torch.randn(Hq, generator=g)
    gate = rand(g, B, Lq, Hq, D, scale=2.0) if gated else None
    lens, starts = [Lk, max(1, Lk - 700)][:B], [Lk - Lq, 11][:B]
    kd, vd = k.cuda(), v.cuda()
    for b in range(B):   # what lies behind a cache's end is never part of an answer
        kd[b, lens[b]:], vd[b, lens[b]:] = NAN, NAN
    prob = hs2.Problem.from_tensors(q, k, 0, w, q_start=i32(starts), kv_lens=i32(lens))
    qd, sd, gd = q.cuda(), sink.cuda(), None if gate is None else gate.cuda()
    out, lse = hs2.hs2_window_attn(prob, qd, kd, vd, nf, sink=sd, gate=gd, want_lse=True)
    assert hs2.hs2_device_error_flags() == 0
    p32 = hs2.Problem.from_tensors(qd.float(), k, 0, w, q_start=i32(starts), kv_lens=i32(lens))
    call32 = lambda x: hs2.hs2_window_attn(p32, qd.float(), kd.float(), x.float(), nf, sink=sd, gate=None if gd is None else gd.float(), want_lse=True)  # noqa: E731
    (o32, l32), (A32, _) = call32(vd), call32(vd.abs())
    logit = (D + 4) * 2.0 ** -24 * D ** -0.5 * float(q.float().norm(dim=-1).max() * k.float().norm(dim=-1).max()) + 2.0 ** -18
    tol = 2.0 ** -8 * o32.abs() + A32 * (2.0 ** -8 + 4 * logit) + 1e-30
    assert torch.isfinite(out).all()
    off = (out.float() - o32).abs() > tol
    assert not off.any(), "%d outputs off, worst %.3g of its bound" % (int(off.sum()), float(((out.float() - o32).abs() / tol).max()))
    assert torch.equal(lse.isinf(), l32.isinf())
    some = ~l32.isinf()
    assert ((lse - l32)[some].abs() <= 2 * logit + 2.0 ** -20 * l32[some].abs()).all()
    again, _ = hs2.hs2_window_attn(prob, qd, kd, vd, nf, sink=sd, gate=gd)
    assert torch.equal(out, again)
    # sampled rows
    for n in range(24):
        b, i = n % B, int(torch.randint(Lq, (), generator=g)) if n > 4 else [0, Lq - 1, Lq // 2, 1, 127][n]
        pos = starts[b] + i
        keys = [j for j in range(min(pos + 1, lens[b])) if j > pos - w or j < nf]
        rows = [x[b, keys].transpose(0, 1).repeat_interleave(Hq // Hkv, 0) for x in (k, v)]
        r = plain_ops.attend(q[b, i], *rows, torch.ones(Hq, len(keys), dtype=torch.bool), D ** -0.5, sink, None if gate is None else gate[b, i])
        ref = r[0][None, None], r[1][None, :, None], r[2][None, None], r[3][None, :, None]
        plain_ops.check(out[b, i][None, None], lse[b, :, i][None, :, None], ref, D, "row %d of %d" % (i, b))


# ---------------------------------------------------------------- gates
@pytest.mark.parametrize("case", [(8, 2, 64, BF16, 300), (8, 1, 128, BF16, 300), (64, 1, 256, BF16, 90), (6, 2, 96, BF16, 90), (4, 2, 64, F32, 90),
                                  (8, 2, 128, BF16, 1), (64, 1, 128, BF16, 1), (4, 2, 64, F32, 1)], ids=str)
def test_gates_of_any_size(case):
    """NaN logits, each of which concerns its own output alone, infinite ones, and ones so low that the factor is tiny or zero: the
    same on every kernel."""
    Hq, Hkv, D, dt, Lq = case
    g = torch.Generator().manual_seed(46)
    Lk, w = 400, 50
    q, k, v = rand(g, 1, Lq, Hq, D, dtype=dt), rand(g, 1, Lk, Hkv, D, dtype=dt), rand(g, 1, Lk, Hkv, D, dtype=dt)
    sink = torch.randn(Hq, generator=g)
    gate = rand(g, 1, Lq, Hq, D, dtype=dt, scale=3.0)
    for d, x in enumerate((NAN, 1.0, -INF, -700.0, INF, 700.0, -50.0, -60.0, -41.0, 3.0, -42.0, -80.0, 2.0, NAN, NAN, -INF)):
        gate[0, :, Hq - 1, d] = x
    gate[0, Lq // 2, 0] = -700.0
    prob = hs2.Problem.from_tensors(q, k, 0, w)
    out, lse = hs2.hs2_window_attn(prob, q.cuda(), k.cuda(), v.cuda(), 2, sink=sink.cuda(), gate=gate.cuda(), want_lse=True)
    nan = gate.isnan().cuda()
    assert out[nan].isnan().all()
    assert (out[0, :, Hq - 1, [2, 3, 15]] == 0).all() and (out[0, Lq // 2, 0] == 0).all()
    ref = plain_ops.window(q, k, v, w, 2, D ** -0.5, [Lk], [Lk - Lq], sink, gate.nan_to_num(0.0, INF, -INF))
    out[nan] = ref[0].cuda()[nan].to(dt)
    plain_ops.check(out, lse, ref, D, "gates")


# ---------------------------------------------------------------- numbers that are not finite
def quantise(x):
    amax = x.float().abs().amax(-1, keepdim=True).clamp(min=1e-20)
    codes = (x.float() / (amax / 448)).to(torch.float8_e4m3fn)
    scale = (amax / 448).squeeze(-1)
    return codes, scale, codes.double() * scale.double()[..., None]


# what runs the call: heads, KV heads, head dim, type, e4m3 cache, bytes that q is shifted by
DECODES = [(8, 2, 128, F32, False, 0), (3, 1, 80, BF16, False, 0), (8, 2, 128, BF16, False, 1), (4, 2, 64, BF16, True, 0),   # FMAs
           (8, 2, 128, BF16, False, 0), (8, 1, 128, BF16, True, 0), (20, 1, 64, BF16, False, 0),                              # mma.sync
           (64, 1, 128, BF16, False, 0), (40, 1, 256, BF16, True, 0), (4, 1, 256, BF16, False, 0)]                            # tcgen05


def decode_setup(g, case, lens, ps=16, table=None, **problem):
    """A cache of the case's kind, its values, and a call of the decode with a query."""
    Hq, Hkv, D, dt, fp8, shift = case
    n_pages = sum(-(-n // ps) for n in lens)
    k, v = rand(g, n_pages, ps, Hkv, D, dtype=F32 if fp8 else dt), rand(g, n_pages, ps, Hkv, D, dtype=F32 if fp8 else dt)
    if table is None:
        cols, at = max(1, max(-(-n // ps) for n in lens)), 0
        table = torch.full((len(lens), cols), -1, dtype=torch.int32)
        for b, n in enumerate(lens):
            m = -(-n // ps)
            table[b, :m] = torch.arange(at, at + m, dtype=torch.int32)
            at += m
    if fp8:
        (k8, ks, kx), (v8, vs, vx) = quantise(k), quantise(v)
        args = [k8.view(torch.uint8).cuda(), v8.view(torch.uint8).cuda(), ks.cuda(), vs.cuda()]
    else:
        kx, vx, args = k, v, [k.cuda(), v.cuda()]

    def call(q, **kw):
        room = torch.zeros(q.numel() + 8, dtype=dt, device="cuda")
        qd = room[shift:shift + q.numel()].view(q.shape)
        qd.copy_(q)
        prob = hs2.PagedProblem.from_tensors(qd, args[0], table.cuda(), i32(lens), **problem)
        return (hs2.hs2_paged_attn_decode_fp8kv if fp8 else hs2.hs2_paged_attn_decode)(prob, qd, *args, want_lse=True, **kw)

    return kx, vx, table, call


@pytest.mark.parametrize("n", [1, 40, 3000])
@pytest.mark.parametrize("case", DECODES, ids=str)
def test_decode_of_a_query_that_is_not_a_number(case, n):
    """One NaN in the query of one head: that head's output is NaN throughout, as the formula has it, and the other heads, and
    the other sequences, know nothing of it."""
    Hq, Hkv, D, dt, fp8, _ = case
    g = torch.Generator().manual_seed(41)
    lens = [n, 70, 0]
    kx, vx, table, call = decode_setup(g, case, lens)
    q = rand(g, 3, 1, Hq, D, dtype=dt)
    ref = plain_ops.paged(q, kx, vx, table, lens, 0, 0, D ** -0.5)
    q[0, 0, Hq - 1, 3] = NAN
    out, lse = call(q)
    assert out[0, 0, Hq - 1].isnan().all()
    out[0, 0, Hq - 1], lse[0, Hq - 1] = ref[0][0, 0, Hq - 1].to(dt).cuda(), ref[1][0, Hq - 1].cuda()
    plain_ops.check(out, lse, ref, D, "beside", p_eps=2.0 ** -8 if dt == BF16 else None)


@pytest.mark.parametrize("n", [1, 40, 3000])
@pytest.mark.parametrize("case", DECODES, ids=str)
def test_decode_lse_of_what_is_not_a_number(case, n):
    """NaN, not the -inf of a sequence without a key; the same for a NaN sink, where the output is NaN too."""
    Hq, Hkv, D, dt, fp8, _ = case
    g = torch.Generator().manual_seed(42)
    lens = [n, 70, 0]
    kx, vx, table, call = decode_setup(g, case, lens)
    q = rand(g, 3, 1, Hq, D, dtype=dt)
    sink = torch.randn(Hq, generator=g)
    sink[1] = NAN
    ref = plain_ops.paged(q, kx, vx, table, lens, 0, 0, D ** -0.5, sink)
    out, lse = call(q, sink=sink.cuda())
    assert out[:2, :, 1].isnan().all() and lse[:, 1].isnan().all()
    keep = [h for h in range(Hq) if h != 1]
    pick = (ref[0][:, :, keep], ref[1][:, keep], ref[2][:, :, keep], ref[3][:, keep])
    plain_ops.check(out[:, :, keep], lse[:, keep], pick, D, "beside", p_eps=2.0 ** -8 if dt == BF16 else None)
    q[0, 0, 0, 1] = NAN
    out, lse = call(q)
    assert lse[0, 0].isnan().all() and out[0, 0, 0].isnan().all() and not lse[1:, 0].isnan().any() and not lse[0, 2:].isnan().any()


# a prompt's kernels: tcgen05 at three head dims, FMAs in bf16 and fp32; one token of the same layer
WINDOWS = [(8, 2, 64, BF16, 90), (8, 1, 128, BF16, 90), (64, 1, 256, BF16, 90), (6, 2, 96, BF16, 90), (4, 2, 64, F32, 90), (8, 2, 128, BF16, 1),
           (4, 2, 64, F32, 1)]


@pytest.mark.parametrize("case", WINDOWS, ids=str)
def test_window_of_queries_and_sinks_that_are_not_numbers(case):
    Hq, Hkv, D, dt, Lq = case
    g = torch.Generator().manual_seed(43)
    Lk, w = 200, 50
    q, k, v = rand(g, 1, Lq, Hq, D, dtype=dt), rand(g, 1, Lk, Hkv, D, dtype=dt), rand(g, 1, Lk, Hkv, D, dtype=dt)
    sink = torch.randn(Hq, generator=g)
    sink[1] = NAN
    ref = plain_ops.window(q, k, v, w, 2, D ** -0.5, [Lk], [Lk - Lq], sink)
    i = Lq // 2
    q[0, i, 0, 5] = NAN
    prob = hs2.Problem.from_tensors(q, k, 0, w)
    out, lse = hs2.hs2_window_attn(prob, q.cuda(), k.cuda(), v.cuda(), 2, sink=sink.cuda(), want_lse=True)
    assert out[:, :, 1].isnan().all() and out[0, i, 0].isnan().all()
    assert lse[:, 1].isnan().all() and lse[0, 0, i].isnan()
    fine = torch.ones(Lq, Hq, dtype=torch.bool)
    fine[:, 1], fine[i, 0] = False, False
    out[0, ~fine], lse[0, ~fine.T] = ref[0][0, ~fine].to(dt).cuda().nan_to_num(0.0), 0.0
    ref = [x.clone() for x in ref]
    ref[0][0, ~fine], ref[1][0, ~fine.T], ref[2][0, ~fine] = 0.0, 0.0, 0.0
    out[0, ~fine] = 0.0
    plain_ops.check(out, lse, ref, D, "beside")
    # no sink: a NaN query's LSE is NaN there too
    out, lse = hs2.hs2_window_attn(prob, q.cuda(), k.cuda(), v.cuda(), 2, want_lse=True)
    assert out[0, i, 0].isnan().all() and lse[0, 0, i].isnan() and int(lse.isnan().sum()) == 1 and int(out.isnan().sum()) == D


# ---------------------------------------------------------------- e4m3 cache: what lies far below the largest probability
@pytest.mark.parametrize("G, D", [(4, 128), (16, 128), (64, 128), (8, 256), (20, 256), (64, 256), (4, 64)])
@pytest.mark.parametrize("below", [8.0, 15.7])
def test_decode_fp8_long_tail_below_one_large_weight(G, D, below):
    """One key holds nearly all of the weight and next to no value (a first token that heads park their attention on); the other
    keys, e^-below of it each, carry the output.  Their weights are far from 2^-24 of the largest: none may be lost, and all are
    rounded by 2^-11 of themselves."""
    g = torch.Generator().manual_seed(44)
    B, n, ps = 300, 1500, 100          # as many sequences as keep all keys of one in one CTA; they share their pages
    q = torch.ones(B, 1, G, D, dtype=BF16)
    c = below / D ** 0.5
    k = -c + 0.1 * torch.randn(15, ps, 1, D, generator=g)
    v = 1 + 0.2 * torch.randn(15, ps, 1, D, generator=g)
    k[3, 7], v[3, 7] = 0.0, 1e-7
    (k8, ks, kx), (v8, vs, vx) = quantise(k), quantise(v)
    table = torch.randperm(15, generator=g).int().expand(B, 15).contiguous()
    ref = plain_ops.paged(q[:1], kx, vx, table[:1], [n], 0, 0, D ** -0.5)
    prob = hs2.PagedProblem.from_tensors(q, k8, table.cuda(), i32([n] * B))
    out, lse = hs2.hs2_paged_attn_decode_fp8kv(prob, q.cuda(), k8.view(torch.uint8).cuda(), v8.view(torch.uint8).cuda(), ks.cuda(), vs.cuda(),
                                               want_lse=True)
    assert torch.equal(out, out[:1].expand_as(out))
    plain_ops.check(out[:1], lse[:1], ref, D, "tail", p_eps=2.0 ** -11)


@pytest.mark.parametrize("G, D", [(4, 128), (16, 128), (64, 128), (8, 256), (20, 256), (64, 256), (4, 64)])
def test_decode_fp8_query_with_one_dimension_far_above_the_others(G, D):
    """One dimension of q is 2^20 times the others, and the keys have next to nothing there: the logits come from the others."""
    g = torch.Generator().manual_seed(47)
    lens, ps = [700, 33], 16
    kx = 300 * torch.randn(60, ps, 1, D, generator=g)
    kx[..., 0] = 0.0
    v = torch.randn(60, ps, 1, D, generator=g)
    (k8, ks, kx), (v8, vs, vx) = quantise(kx), quantise(v)
    q = rand(g, 2, 1, G, D, scale=0.001)
    q[..., 0] = 1000.0
    table = torch.randperm(60, generator=g).int()[:44].expand(2, 44).contiguous()
    ref = plain_ops.paged(q, kx, vx, table, lens, 0, 0, 1.0)
    prob = hs2.PagedProblem.from_tensors(q, k8, table.cuda(), i32(lens), softmax_scale=1.0)
    out, lse = hs2.hs2_paged_attn_decode_fp8kv(prob, q.cuda(), k8.view(torch.uint8).cuda(), v8.view(torch.uint8).cuda(), ks.cuda(), vs.cuda(),
                                               want_lse=True)
    plain_ops.check(out, lse, ref, D, "query", p_eps=2.0 ** -11)


# ---------------------------------------------------------------- softmax scales
@pytest.mark.parametrize("scale", [1e-30, 2e-38, 1e-40, 1e-45])
@pytest.mark.parametrize("case", DECODES, ids=str)
def test_decode_of_softmax_scales_next_to_zero(case, scale):
    """All weights are equal then, and nothing is NaN: tiles with void rows and empty sequences included."""
    Hq, Hkv, D, dt, fp8, _ = case
    g = torch.Generator().manual_seed(48)
    lens = [1, 70, 0]
    kx, vx, table, call = decode_setup(g, case, lens, softmax_scale=scale)
    q = rand(g, 3, 1, Hq, D, dtype=dt, scale=0.01)
    ref = plain_ops.paged(q, kx, vx, table, lens, 0, 0, scale)
    out, lse = call(q)
    plain_ops.check(out, lse, ref, D, "equal weights", p_eps=2.0 ** -8 if dt == BF16 else None)


@pytest.mark.parametrize("scale", [1e-30, 2e-38, 1e-40, 1e-45])
@pytest.mark.parametrize("case", WINDOWS, ids=str)
def test_window_of_softmax_scales_next_to_zero(case, scale):
    Hq, Hkv, D, dt, Lq = case
    g = torch.Generator().manual_seed(49)
    Lk, w = 200, 50
    q, k, v = rand(g, 1, Lq, Hq, D, dtype=dt), rand(g, 1, Lk, Hkv, D, dtype=dt), rand(g, 1, Lk, Hkv, D, dtype=dt)
    start = Lk - Lq - 20 if Lq > 1 else Lk - 1
    ref = plain_ops.window(q, k, v, w, 2, scale, [Lk], [start])
    prob = hs2.Problem.from_tensors(q, k, 0, w, softmax_scale=scale, q_start=i32([start]))
    out, lse = hs2.hs2_window_attn(prob, q.cuda(), k.cuda(), v.cuda(), 2, want_lse=True)
    plain_ops.check(out, lse, ref, D, "equal weights")


# ---------------------------------------------------------------- values that are not finite under wide windows
@pytest.mark.parametrize("case, value, limit", [((32, 4, 128, 1024, 8192, False), NAN, 20), ((64, 1, 256, 4096, 8192, True), NAN, 150),
                                                ((64, 1, 256, 4096, 8192, False), INF, 150), ((16, 2, 64, 2000, 6000, True), INF, 50),
                                                ((8, 1, 128, 300, 3000, True), NAN, 20)], ids=str)
def test_window_one_token_whose_values_are_not_finite(case, value, limit):
    """One V row of NaN or infinities: it reaches the queries that see it, in every column, and no other; and those beside it in a
    tile cost no attention in scalar arithmetic.  Measured in ms: 7, 47, 110, 7 and 2; with a row per thread and one column after
    the other 123 in the first and 1375 in the second, where the layer takes 0.2 and 1.4 on numbers."""
    Hq, Hkv, D, w, L, gated = case
    g = torch.Generator().manual_seed(50)
    q, k, v = rand(g, 1, L, Hq, D).cuda(), rand(g, 1, L, Hkv, D).cuda(), rand(g, 1, L, Hkv, D).cuda()
    gate = rand(g, 1, L, Hq, D).cuda() if gated else None
    at = L // 2 + 37
    prob = hs2.Problem.from_tensors(q, k, 0, w)
    call = lambda x: hs2.hs2_window_attn(prob, q, k, x, 1, gate=gate)[0].float()  # noqa: E731
    clean, A = call(v), call(v.abs())
    bad = v.clone()
    bad[0, at] = value
    call(bad)
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    t0.record()
    out = hs2.hs2_window_attn(prob, q, k, bad, 1, gate=gate)[0]
    t1.record()
    t1.synchronize()
    assert hs2.hs2_device_error_flags() == 0
    sees = torch.zeros(L, dtype=torch.bool, device="cuda")
    sees[at:at + w] = True
    assert out[0, sees].isnan().all() if value != value else (out[0, sees] == value).all()
    # the others: once from tensor cores with weights in bf16, once in fp32 where they share a tile
    assert ((out.float() - clean).abs() <= 2.0 ** -7 * clean.abs() + (2.0 ** -8 + 2.0 ** -14) * A + 1e-30)[0, ~sees].all()
    assert t0.elapsed_time(t1) < limit


# ---------------------------------------------------------------- more sequences or heads than a grid has rows
@pytest.mark.parametrize("B, Hq, Hkv, D, Lk, dt", [(70000, 2, 1, 8, 5, F32), (65536, 1, 1, 64, 3, BF16), (1, 70000, 2, 8, 40, BF16)], ids=str)
def test_window_of_one_token_for_very_many(B, Hq, Hkv, D, Lk, dt):
    g = torch.Generator().manual_seed(51)
    q, k, v = rand(g, B, 1, Hq, D, dtype=dt), rand(g, B, Lk, Hkv, D, dtype=dt), rand(g, B, Lk, Hkv, D, dtype=dt)
    prob = hs2.Problem.from_tensors(q, k, 0, 3)
    out, lse = hs2.hs2_window_attn(prob, q.cuda(), k.cuda(), v.cuda(), 1, want_lse=True)
    o, l, A, S = plain_ops.window(q, k, v, 3, 1, D ** -0.5, [Lk] * B, [Lk - 1] * B)
    plain_ops.check(out, lse, (o, l, A, S), D, "very many")


# ---------------------------------------------------------------- tables wider than the contexts
@pytest.mark.parametrize("case", DECODES, ids=str)
def test_decode_under_a_table_far_wider_than_the_contexts(case):
    """A server's table has room for the longest sequence that it allows, which is what splits are planned for; what stands in it
    behind the contexts is not read."""
    Hq, Hkv, D, dt, fp8, _ = case
    g = torch.Generator().manual_seed(52)
    lens, ps = [4000, 1, 0, 700, 129], 16
    kx, vx, table, _ = decode_setup(g, case, lens)
    g = torch.Generator().manual_seed(52)
    q = rand(g, len(lens), 1, Hq, D, dtype=dt)
    ref = plain_ops.paged(q, kx, vx, table, lens, 0, 0, D ** -0.5)
    for cols in (2048, 70000):
        wide = torch.randint(-2 ** 31, 2 ** 31 - 1, (len(lens), cols), generator=g, dtype=torch.int64).int()
        for b, n in enumerate(lens):
            wide[b, :-(-n // ps)] = table[b, :-(-n // ps)]
        out, lse = decode_setup(torch.Generator().manual_seed(52), case, lens, table=wide)[3](q)
        plain_ops.check(out, lse, ref, D, "%d columns" % cols, p_eps=2.0 ** -8 if dt == BF16 else None)


# ---------------------------------------------------------------- calls at the same time
def test_windows_on_two_streams_at_once():
    """Two layers whose CTAs run side by side, each taking row tiles from its own grid."""
    g = torch.Generator().manual_seed(53)
    jobs = []
    for Hq, Hkv, D, w, gated in ((32, 4, 128, 40, True), (64, 1, 256, 60, True)):
        q, k, v = rand(g, 1, 4000, Hq, D).cuda(), rand(g, 1, 4000, Hkv, D).cuda(), rand(g, 1, 4000, Hkv, D).cuda()
        jobs.append((hs2.Problem.from_tensors(q, k, 0, w), q, k, v, rand(g, 1, 4000, Hq, D).cuda()))
    want = [hs2.hs2_window_attn(p, q, k, v, 2, gate=gt, want_lse=True) for p, q, k, v, gt in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(8):
        for n, (p, q, k, v, gt) in enumerate(jobs):
            got[n].append(hs2.hs2_window_attn(p, q, k, v, 2, gate=gt, want_lse=True, stream=streams[n]))
    torch.cuda.synchronize()
    assert hs2.hs2_device_error_flags() == 0
    for n in range(2):
        for out, lse in got[n]:
            assert torch.equal(out, want[n][0]) and torch.equal(lse, want[n][1])


# ---------------------------------------------------------------- lengths beyond the cache
@pytest.mark.parametrize("Lq", [1, 3])
@pytest.mark.parametrize("D, dt", [(128, BF16), (64, F32), (96, BF16)], ids=str)
def test_window_of_lengths_beyond_the_cache(D, dt, Lq):
    """Without q_start the last query stands at kv_lens[b] - 1, wherever the cache ends: for one token as for a prompt."""
    g = torch.Generator().manual_seed(54)
    B, Lk, w = 4, 60, 20
    q, k, v = rand(g, B, Lq, 8, D, dtype=dt), rand(g, B, Lk, 2, D, dtype=dt), rand(g, B, Lk, 2, D, dtype=dt)
    lens = [Lk, Lk + 7, Lk + 40, 2 ** 31 - 1]
    ref = plain_ops.window(q, k, v, w, 1, D ** -0.5, [min(n, Lk) for n in lens], [n - Lq for n in lens])
    out, lse = hs2.hs2_window_attn(hs2.Problem.from_tensors(q, k, 0, w, kv_lens=i32(lens)), q.cuda(), k.cuda(), v.cuda(), 1, want_lse=True)
    plain_ops.check(out, lse, ref, D, "beyond")
