"""CPU checks of host code and index arithmetic that the sliding-window, paged-decode and page calls share with their kernels."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest
import torch
from torch._subclasses import FakeTensorMode

import paper_2609_26368_b200 as hs2
from paper_2609_26368_b200 import binding
from paper_2609_26368_b200 import build as build_module

INT_MAX = 2 ** 31 - 1


def run_host_code(tmp_path, body, lines):
    """Compiles `body`, a main() that reads numbers and prints answers, with the kernels' own header for the host, and runs it."""
    if shutil.which("nvcc") is None:
        pytest.skip("no nvcc")
    src, exe = tmp_path / "host.cu", tmp_path / "host"
    src.write_text('#include <stdio.h>\n#include "hs2_paged.cuh"\n' + body)
    include = os.path.join(os.path.dirname(os.path.dirname(build_module.CSRC)), "include")
    subprocess.check_call(["nvcc", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I" + include, "-I" + build_module.CSRC,
                           str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, x)) for x in lines), text=True, capture_output=True, check=True)
    return [tuple(map(int, line.split())) for line in out.stdout.splitlines()]


def test_released_entries_stay_in_the_row_for_any_keep(tmp_path):
    """hs2_pages_free: with one token per page a keep near INT_MAX is as many pages, and a thread's index on top of that wraps."""
    rng = random.Random(1)
    cases = []
    for _ in range(400):
        ps = rng.choice([1, 1, 2, 16, 1000])
        max_pages = rng.choice([1, 30, 4096, INT_MAX // ps])
        most = max_pages * ps
        length = rng.choice([-5, 0, 1, most // 2, most, rng.randrange(most + 1)])
        keep = rng.choice([-2 ** 31, -1, 0, 1, length, length + 1 if length < INT_MAX else length, INT_MAX - 126, INT_MAX,
                           rng.randrange(2 ** 31)])
        cases.append((length, keep, ps, max_pages))
    got = run_host_code(tmp_path, """int main()
{
    int len, keep, ps, max_pages;
    while (scanf("%d %d %d %d", &len, &keep, &ps, &max_pages) == 4) {
        const int2 r = hs2::released_entries(len, keep, ps, max_pages);
        printf("%d %d\\n", r.x, r.y);
    }
}
""", cases)
    assert len(got) == len(cases)
    for (length, keep, ps, max_pages), (first, end) in zip(cases, got):
        held, kept = max(0, length), max(0, keep)
        plain = range(-(-kept // ps), min(-(-held // ps), max_pages))   # without a limit on the numbers
        assert 0 <= end <= max_pages and 0 <= first <= max(end, -(-held // ps))
        assert max(0, end - first) == len(plain) and (not plain or first == plain[0])


# ---------------------------------------------------------------- tensors that the library would read past
@pytest.fixture
def cuda():
    """Tensors with shapes, strides and a CUDA device, and no memory."""
    with FakeTensorMode(allow_non_fake_inputs=True):
        yield lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")


def test_page_tables_with_shared_rows_are_refused(cuda):
    """A row stride of 0 would say `packed` to the library, which would then take the rows from behind the one there is."""
    row, lens = cuda(1, 8, dtype=torch.int32), cuda(4, dtype=torch.int32)
    for table in (row.expand(4, 8), cuda(20, dtype=torch.int32).as_strided((4, 8), (4, 1)), cuda(4, 1, dtype=torch.int32)[:1].expand(4, 1)):
        with pytest.raises(AssertionError):
            hs2.PagedProblem(4, 8, 2, 64, 16, 100, table, lens)
    for table in (cuda(4, 8, dtype=torch.int32), cuda(4, 20, dtype=torch.int32)[:, 5:13], cuda(4, 1, dtype=torch.int32)):
        hs2.PagedProblem(4, 8, 2, 64, 16, 100, table, lens)
    hs2.PagedProblem(1, 8, 2, 64, 16, 100, row.expand(1, 8), lens[:1])


def test_tensors_broadcast_along_every_axis_are_refused(cuda):
    """One row, or one scale, expanded to all: strides of 0, which the library takes for packed."""
    B, Hq, Hkv, D, ps, n_pages, L = 3, 4, 2, 64, 16, 10, 20
    table, lens = cuda(B, 4, dtype=torch.int32), cuda(B, dtype=torch.int32)
    prob = hs2.PagedProblem(B, Hq, Hkv, D, ps, n_pages, table, lens)
    one = cuda(1, 1, 1, D)
    q, kv = cuda(B, 1, Hq, D), cuda(n_pages, ps, Hkv, D)
    codes, scales = cuda(n_pages, ps, Hkv, D, dtype=torch.uint8), cuda(n_pages, ps, Hkv, dtype=torch.float32)
    tensor_scale = cuda(1, dtype=torch.float32).expand(n_pages, ps, Hkv)
    refused = "packed|share memory"
    for args in ((one.expand(B, 1, Hq, D), kv, kv), (q, one.expand(n_pages, ps, Hkv, D), one.expand(n_pages, ps, Hkv, D))):
        with pytest.raises(AssertionError, match=refused):
            hs2.hs2_paged_attn_decode(prob, *args)
    for out in (one.expand(B, 1, Hq, D), cuda(1, 1, Hq, D).expand(B, 1, Hq, D)):
        with pytest.raises(AssertionError, match=refused):
            hs2.hs2_paged_attn_decode(prob, q, kv, kv, out=out)
    with pytest.raises(AssertionError, match=refused):
        hs2.hs2_paged_attn_decode_fp8kv(prob, q, codes, codes, tensor_scale, tensor_scale)
    wide = hs2.Problem(B, L, 50, Hq, Hkv, D, 0, 8)
    wq, wkv = cuda(B, L, Hq, D), cuda(B, 50, Hkv, D)
    for args, kw in (((one.expand(B, L, Hq, D), wkv, wkv), {}), ((wq, one.expand(B, 50, Hkv, D), one.expand(B, 50, Hkv, D)), {}),
                     ((wq, wkv, wkv), dict(out=one.expand(B, L, Hq, D)))):
        with pytest.raises(AssertionError, match=refused):
            hs2.hs2_window_attn(wide, *args, **kw)
    sparse = hs2.Problem(B, 1, 50, Hq, Hkv, 128, 0, 8)
    codes, tensor_scale = cuda(B, 50, Hkv, 128, dtype=torch.uint8), cuda(1, dtype=torch.float32).expand(B, 50, Hkv)
    with pytest.raises(AssertionError, match=refused):
        hs2.hs2_sparse_attn_decode_fp8kv(sparse, cuda(B, 1, Hq, 128), codes, codes, tensor_scale, tensor_scale, None)


# ---------------------------------------------------------------- scratch
@pytest.fixture(scope="module")
def lib():
    build_module.build()
    return hs2.load_library()


def window_ws(lib, **kw):
    d = dict(batch=1, q_len=1, kv_len=131072, n_q_heads=64, n_kv_heads=1, head_dim=256, k_sel=0, window=128)
    d.update(kw)
    c = hs2.Problem(**d).c_struct()
    return c, lib.hs2_workspace_bytes(C.byref(c), binding.HS2_OP_WINDOW_ATTN)


def test_scratch_of_one_token_windows_follows_the_keys(lib):
    """The bound was 1777 splits whatever the cache holds: 117 MB for a window of 128 tokens."""
    assert window_ws(lib, kv_len=132)[1] <= 64 * 2 * 258 * 4
    assert window_ws(lib, kv_len=128)[1] <= 64 * 258 * 4
    assert window_ws(lib)[1] <= 64 * 444 * 258 * 4


@pytest.mark.skipif(torch.cuda.is_available(), reason="the pointers are not real")
def test_scratch_of_one_token_windows_is_enough(lib):
    """With the bytes that were named the call comes to look for a device; with what a plan has none of, it says so."""
    rng, small = random.Random(2), 0
    one = C.c_void_p(256)
    for _ in range(3000):
        n_kv, group = rng.choice([1, 2, 8]), rng.choice([1, 4, 8, 9, 16, 33, 64, 130])
        kv_len, w, nf = rng.choice([1, 100, 129, 4000, 40000, 300000]), rng.choice([1, 128, 129, 4096, 100000]), rng.choice([0, 4, 500, 10 ** 6])
        kw = dict(batch=rng.choice([1, 2, 5, 64, 400]), n_q_heads=n_kv * group, n_kv_heads=n_kv, head_dim=rng.choice([64, 80, 128, 256]),
                  window=w, dtype=rng.choice([torch.float32, torch.bfloat16]))
        c, most = window_ws(lib, kv_len=kv_len, **kw)
        need = window_ws(lib, kv_len=min(kv_len, w + nf), **kw)[1]
        assert need <= most
        for n in (need, most):
            st = lib.hs2_window_attn(C.byref(c), nf, one, one, one, None, None, one, None, one if n else None, n, None)
            assert st == binding.HS2_ERR_CUDA, (kv_len, w, nf, kw)
        small += lib.hs2_window_attn(C.byref(c), nf, one, one, one, None, None, one, None, None, 0, None) == binding.HS2_ERR_WORKSPACE_TOO_SMALL
    assert small > 500


# ---------------------------------------------------------------- sizes next to 2^31
def test_sizes_whose_indices_would_wrap_are_refused(lib):
    """Tiles and grids run past an end by up to 2^22: what lies closer to 2^31 than that is not supported."""
    most, one, bad = 2 ** 31 - 2 ** 22, C.c_void_p(256), binding.HS2_ERR_UNSUPPORTED

    def paged(**kw):
        c = binding._CPagedProblem(2, 8, 2, 128, 1, 100, 10, 0, 0, 0.0, binding.HS2_BF16, 256, 0, 256)
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    for c in (paged(max_pages=most + 1), paged(max_pages=INT_MAX), paged(page_size=most + 1, max_pages=1), paged(page_size=INT_MAX // 2, max_pages=2)):
        assert lib.hs2_paged_attn_decode(C.byref(c), one, one, one, None, None, one, None, one, 1 << 62, None) == bad
        assert lib.hs2_paged_workspace_bytes(C.byref(c)) == 0
    assert lib.hs2_paged_workspace_bytes(C.byref(paged(max_pages=most))) > 0
    w = hs2.Problem(1, 2, most + 1, 1, 1, 8, 0, 4).c_struct()
    assert lib.hs2_window_attn(C.byref(w), 0, one, one, one, None, None, one, None, None, 0, None) == bad
    w = hs2.Problem(1, most + 1, 2, 1, 1, 8, 0, 4).c_struct()
    assert lib.hs2_window_attn(C.byref(w), 0, one, one, one, None, None, one, None, None, 0, None) == bad

    def pool(**kw):
        c = binding._CPagePool(100, 1, 8, 10, 256, 256, 256)
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    g = binding._CPageRegion(256, 1, 256, 0, 1 << 50, 256)
    for c, n in ((pool(n_pages=most + 1), 4), (pool(max_pages=most + 1), 4), (pool(max_seqs=INT_MAX), 4), (pool(), (1 << 30) + 1)):
        assert lib.hs2_pages_workspace_bytes(C.byref(c), n) == 0
        assert lib.hs2_pages_reserve(C.byref(c), C.byref(g), 1, one, one, n, one, one, 1 << 62, None) == bad
        assert lib.hs2_pages_fork(C.byref(c), one, one, n, one, 1 << 62, None) == bad
        assert lib.hs2_pages_free(C.byref(c), one, None, n, None) == bad
        assert lib.hs2_pages_copy(C.byref(c), C.byref(g), 1, one, one, n, None) == bad
        rows, strides = (C.c_void_p * 1)(256), (C.c_int64 * 3)(0, 1024, 256)
        assert lib.hs2_pages_write(C.byref(c), C.byref(g), 1, rows, strides, one, one, one, n, 4, None) == bad
        if n == 4:
            assert lib.hs2_pages_compact(C.byref(c), C.byref(g), 1, None, one, 1 << 62, None) == bad
    c = pool()
    assert lib.hs2_pages_write(C.byref(c), C.byref(g), 1, rows, strides, one, one, one, 4, most + 1, None) == bad
    assert lib.hs2_pages_workspace_bytes(C.byref(pool(n_pages=most, max_seqs=most)), 1 << 30) > 0
