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
