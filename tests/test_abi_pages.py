"""Refusals of the entry points for a shared paged cache, on the CPU: every check runs before any HIP call."""
import ctypes
import random

import pytest
import torch

from paper_2607_02980_amd import hils

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first


def params(**kw):
    base = dict(B=2, Hq=8, Hkv=2, N=4, L=256, d=128, topk=8, window=128)
    base.update(kw)
    return hils.Params(**base)


def prefill(p, pages=4, ws=None, nbytes=0, **kw):
    a = dict(q=FAKE, k_pages=FAKE, v_pages=FAKE, lmk_pages=FAKE, block_table=FAKE, out=FAKE, lse=FAKE, idx=FAKE)
    a.update(kw)
    return hils.LIB.hils_prefill_paged_fwd(ctypes.byref(p.c()), a["q"], a["k_pages"], a["v_pages"], a["lmk_pages"], None,
                                           None, a["block_table"], pages, None, None, a["out"], a["lse"], a["idx"], ws,
                                           nbytes, None)


def pool(data=0x1000, nbytes=64):
    return (hils.hils_pool * 1)(hils.hils_pool(data, nbytes))


def reserve(p, pages=4, pools=None, n=0, **kw):
    a = dict(block_table=FAKE, page_refs=FAKE, table_out=FAKE, refs_out=FAKE, copied=FAKE, counts=FAKE)
    a.update(kw)
    return hils.LIB.hils_cache_reserve(ctypes.byref(p.c()), a["block_table"], a["page_refs"], pages, None, None, pools, n,
                                       a["table_out"], a["refs_out"], a["copied"], a["counts"], None)


def fork(p, pages=4, rows=3, seqlens=None, **kw):
    a = dict(parent=FAKE, block_table=ctypes.c_void_p(0x2000), page_refs=FAKE, table_out=FAKE, seqlens_out=FAKE, refs_out=FAKE)
    a.update(kw)
    return hils.LIB.hils_cache_fork(ctypes.byref(p.c()), a["parent"], rows, a["block_table"], a["page_refs"], pages, seqlens,
                                    a["table_out"], a["seqlens_out"], a["refs_out"], None)


def free(p, pages=4, listed=None, nlisted=None, most=0, **kw):
    a = dict(keep=FAKE, block_table=FAKE, page_refs=FAKE, table_out=FAKE, seqlens_out=FAKE, refs_out=FAKE)
    a.update(kw)
    return hils.LIB.hils_cache_free(ctypes.byref(p.c()), a["keep"], listed, nlisted, most, a["block_table"], a["page_refs"],
                                    pages, None, a["table_out"], a["seqlens_out"], a["refs_out"], None)


def compact(p, pages=4, pools=None, n=0, **kw):
    a = dict(block_table=FAKE, page_refs=FAKE, table_out=FAKE, refs_out=FAKE, new_page=FAKE, moved=FAKE, counts=FAKE)
    a.update(kw)
    return hils.LIB.hils_cache_compact(ctypes.byref(p.c()), a["block_table"], a["page_refs"], pages, None, pools, n,
                                       a["table_out"], a["refs_out"], a["new_page"], a["moved"], a["counts"], None)


ALL = [prefill, reserve, fork, free, compact]
NEEDED = {prefill: ["q", "k_pages", "v_pages", "lmk_pages", "block_table", "out", "lse", "idx"],
          reserve: ["block_table", "page_refs", "table_out", "refs_out", "copied", "counts"],
          fork: ["parent", "block_table", "page_refs", "table_out", "seqlens_out", "refs_out"],
          free: ["keep", "block_table", "page_refs", "table_out", "seqlens_out", "refs_out"],
          compact: ["block_table", "page_refs", "table_out", "refs_out", "new_page", "moved", "counts"]}


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("kw,code,msg", [
    (dict(Hq=6, Hkv=4), 1, "multiple of Hkv"), (dict(L=250), 1, "multiple of chunk"), (dict(N=0), 1, "must be >= 1"),
    (dict(N=300), 1, "N"), (dict(d=96), 2, "d=96"), (dict(Hq=6, Hkv=2), 2, "group size"), (dict(topk=65), 2, "topk"),
    (dict(flags=1 << 9), 1, "flags"), (dict(flags=2), 1, "flags|SHARED"), (dict(chunk=32), 2, "chunk"), (dict(B=65536), 1, "B and Hkv"),
])
def test_shapes_are_refused(call, kw, code, msg):
    assert call(params(**kw)) == code
    import re

    assert re.search(msg, hils.hils_last_error())


@pytest.mark.parametrize("call", ALL)
def test_missing_pointers_and_pools(call):
    for name in NEEDED[call]:
        assert call(params(), **{name: None}) == hils.HILS_ERR_INVALID and name in hils.hils_last_error()
    assert call(params(), pages=0) == hils.HILS_ERR_INVALID and "num_pages" in hils.hils_last_error()
    if call is not prefill:
        assert call(params(), pages=(1 << 30) + 1) == hils.HILS_ERR_UNSUPPORTED and "num_pages" in hils.hils_last_error()


def test_prefill_workspace_and_flags():
    p = params()
    n = hils.hils_workspace_size(p, hils.HILS_OP_PREFILL_PAGED)
    assert n > 0
    for ws, nbytes in ((None, 0), (None, n), (FAKE, n - 1)):
        assert prefill(p, ws=ws, nbytes=nbytes) == hils.HILS_ERR_WORKSPACE
    assert prefill(p, ws=ctypes.c_void_p(0x1008), nbytes=n) == hils.HILS_ERR_INVALID and "aligned" in hils.hils_last_error()
    assert prefill(params(flags=hils.HILS_FLAG_HEAD_NORM_SELECT)) == hils.HILS_ERR_UNSUPPORTED
    assert prefill(params(B=60000, N=60000, L=64000), ws=FAKE, nbytes=1 << 62) == hils.HILS_ERR_UNSUPPORTED
    assert "more workgroups" in hils.hils_last_error()


def test_prefill_workspace_grows_with_batch_rows_and_cache():
    size = lambda **kw: hils.hils_workspace_size(params(**kw), hils.HILS_OP_PREFILL_PAGED)  # noqa: E731
    for a, b in ((dict(B=2), dict(B=3)), (dict(N=4), dict(N=200)), (dict(L=256), dict(L=64000))):
        assert size(**a) <= size(**b)
    before = hils.hils_prefill_record_cap(1 << 20)
    try:
        assert size(N=6000, L=64000) < 40 << 20  # (records of 128 rows, and 4 lists of all ranks)
    finally:
        hils.hils_prefill_record_cap(before)


@pytest.mark.parametrize("cap", [0, 1, 1 << 20, 1 << 28])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_prefill_workspace_serves_all_smaller_calls(dtype, cap):
    """The size rises with batch, rows and cache, also where scores or records are cut into blocks of rows and where
    few rows turn into many."""
    r = random.Random(cap)
    size = lambda B, N, L: hils.hils_workspace_size(  # noqa: E731
        params(B=B, N=N, L=L, Hq=32, Hkv=8, topk=16, window=512, dtype=dtype), hils.HILS_OP_PREFILL_PAGED)
    before = hils.hils_prefill_record_cap(cap)
    try:
        for _ in range(3000):
            B, N, L = r.choice([1, 2, 3, 7, 16, 33]), r.randint(1, r.choice([40, 600, 9000])), 64 * r.choice([150, 999, 2100, 16001])
            more = [(B + r.choice([1, 2, 9]), N, L), (B, N + r.choice([1, 60, 128, 2000]), L), (B, N, L + 64 * r.choice([1, 900]))]
            here = size(B, min(N, L), L)
            for b in more:
                assert here <= size(b[0], min(b[1], b[2]), b[2]), ((B, N, L), b)
    finally:
        hils.hils_prefill_record_cap(before)


def test_prefill_segments_keep_a_row_and_a_slot_in_31_bits():
    size = lambda rows: hils.hils_workspace_size(  # noqa: E731
        params(B=1, Hq=1, Hkv=1, N=rows, L=1 << 26, topk=1), hils.HILS_OP_PREFILL_PAGED)
    before = hils.hils_prefill_record_cap(1 << 40)
    try:
        assert size(1 << 23) < size(1 << 24) == size(1 << 25) == size(3 << 24)
    finally:
        hils.hils_prefill_record_cap(before)


def test_workspace_of_the_page_operators_is_none():
    for op in range(hils.HILS_OP_CACHE_RESERVE, hils.HILS_OP_CACHE_COMPACT + 1):
        assert hils.hils_workspace_size(params(flags=hils.HILS_FLAG_GIVEN_IDX), op) == 0
    with pytest.raises(hils.HilsError, match="unknown op"):
        hils.hils_workspace_size(params(), 13)


@pytest.mark.parametrize("call", [reserve, compact])
def test_pools_are_checked(call):
    for pools, n, msg in ((None, 1, "pools must be"), (pool(), -1, "num_pools"), (pool(), 65537, "num_pools"),
                          (pool(data=None), 1, "pool 0 is NULL"), (pool(nbytes=0), 1, "pool 0"), (pool(nbytes=(1 << 32) + 1), 1, "pool 0")):
        assert call(params(), pools=pools, n=n) == hils.HILS_ERR_INVALID and msg in hils.hils_last_error()


def test_fork_and_free_arguments():
    for rows in (0, 65536):
        assert fork(params(), rows=rows) == hils.HILS_ERR_INVALID and "rows" in hils.hils_last_error()
    assert fork(params(), block_table=FAKE) == hils.HILS_ERR_INVALID and "in place" in hils.hils_last_error()
    assert fork(params(), seqlens=FAKE) == hils.HILS_ERR_INVALID and "in place" in hils.hils_last_error()
    for most in (-1, (1 << 30) + 1):
        assert free(params(), most=most, listed=FAKE) == hils.HILS_ERR_INVALID and "max_pages" in hils.hils_last_error()
    assert free(params(), nlisted=FAKE) == hils.HILS_ERR_INVALID and "pages must be" in hils.hils_last_error()


# ---- the binding


@pytest.fixture
def on_gpu(monkeypatch):
    """Tensors pass for GPU tensors, and addresses are not looked at."""
    monkeypatch.setattr(hils, "_gpu", lambda t, name: 0 if isinstance(t, torch.Tensor) else hils._ptr(t, name))
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)


TABLE, REFS = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(9, dtype=torch.int32)


@pytest.mark.parametrize("fn,args", [("hils_cache_reserve", (TABLE, REFS)), ("hils_cache_compact", (TABLE, REFS)),
                                     ("hils_cache_fork", (REFS, TABLE, REFS)), ("hils_cache_free", (REFS, TABLE, REFS))])
def test_cpu_tensors_are_refused(fn, args):
    with pytest.raises(ValueError, match="GPU tensor"):
        getattr(hils, fn)(params(), *args)


@pytest.mark.parametrize("bad", [None, 3, torch.zeros(()), torch.zeros(8, 2), torch.zeros(9, 2, 2).transpose(1, 2)[:, 1]])
@pytest.mark.parametrize("fn", ["hils_cache_reserve", "hils_cache_compact"])
def test_pools_that_do_not_fit(on_gpu, fn, bad):
    with pytest.raises(ValueError, match=r"pools\[1\]"):
        getattr(hils, fn)(params(), TABLE, REFS, [torch.zeros(9, 2), bad])


def test_dimensions_of_the_binding(on_gpu):
    with pytest.raises(ValueError, match="page_refs"):
        hils.hils_cache_free(params(), REFS, TABLE, TABLE)
    with pytest.raises(ValueError, match="parent"):
        hils.hils_cache_fork(params(), TABLE, TABLE, REFS)
    with pytest.raises(ValueError, match="pages"):
        hils.hils_cache_free(params(), REFS, TABLE, REFS, pages=REFS)
    with pytest.raises(ValueError, match="k_pages"):
        hils.hils_prefill_paged_fwd(params(), torch.zeros(1), 7, 7, 7, TABLE)
    with pytest.raises(ValueError, match="needs idx"):
        hils.hils_prefill_paged_fwd(params(flags=1), torch.zeros(1), torch.zeros(4), 7, 7, TABLE, out=REFS, lse=REFS)


@pytest.mark.parametrize("fn", ["hils_cache_reserve", "hils_cache_compact"])
def test_a_pool_without_pages_is_refused(on_gpu, fn):
    with pytest.raises(ValueError, match="page_refs"):
        getattr(hils, fn)(params(), TABLE, REFS[:0], [torch.zeros(0, 2)])
