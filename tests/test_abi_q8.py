"""Refusals of the 8-bit cache's entry points, on the CPU: every check runs before any HIP call."""
import ctypes

import pytest
import torch

from paper_2607_02980_amd import hils

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first


def params(**kw):
    base = dict(B=2, Hq=8, Hkv=2, N=4, L=256, d=128, topk=8, window=128)
    base.update(kw)
    return hils.Params(**base)


def append(p, pages=4, **kw):
    a = dict(k_new=FAKE, v_new=FAKE, k=FAKE, v=FAKE, scale=FAKE, table=FAKE)
    a.update(kw)
    cp = p.c()
    return hils.LIB.hils_q8_append(ctypes.byref(cp), a["k_new"], a["v_new"], a["k"], a["v"], a["scale"], a["table"],
                                   pages, None, None, None)


def landmark(p, pages=4, **kw):
    a = dict(lq=FAKE, k=FAKE, scale=FAKE, table=FAKE, lmk=FAKE, bias=FAKE)
    a.update(kw)
    cp = p.c()
    return hils.LIB.hils_q8_landmark_fwd(ctypes.byref(cp), a["lq"], a["k"], a["scale"], a["table"], pages, None, None,
                                         a["lmk"], a["bias"], None)


def decode(p, pages=4, ws=None, nbytes=0, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, scale=FAKE, lmk=FAKE, table=FAKE, out=FAKE, lse=FAKE, idx=FAKE)
    a.update(kw)
    cp = p.c()
    return hils.LIB.hils_decode_q8_fwd(ctypes.byref(cp), a["q"], a["k"], a["v"], a["scale"], a["lmk"], None, None,
                                       a["table"], pages, None, a["out"], a["lse"], a["idx"], None, ws, nbytes, None)


def evict(p, budget=1, sink=0, most=4, **kw):
    a = dict(acc=FAKE, table=FAKE, weights=None, idx=None, acc_out=FAKE, table_out=FAKE, lens=FAKE, freed=FAKE, n=FAKE)
    a.update(kw)
    cp = p.c()
    return hils.LIB.hils_cache_evict(ctypes.byref(cp), a["acc"], a["table"], None, a["weights"], a["idx"], budget, sink,
                                     most, a["acc_out"], a["table_out"], a["lens"], a["freed"], a["n"], None)


ALL = [append, landmark, decode, evict]


@pytest.mark.parametrize("call", ALL)
@pytest.mark.parametrize("kw,code,msg", [
    (dict(Hq=6, Hkv=4), 1, "multiple of Hkv"), (dict(L=250), 1, "multiple of chunk"), (dict(N=0), 1, "must be >= 1"),
    (dict(N=300), 1, "N"), (dict(d=96), 2, "d=96"), (dict(Hq=6, Hkv=2), 2, "group size"), (dict(topk=65), 2, "topk"),
    (dict(flags=1 << 9), 1, "flags"), (dict(chunk=32), 2, "chunk"),
])
def test_shapes_are_refused(call, kw, code, msg):
    assert call(params(**kw)) == code
    assert msg in hils.hils_last_error()


@pytest.mark.parametrize("call,names", [
    (append, ["k_new", "v_new", "k", "v", "scale", "table"]), (landmark, ["lq", "k", "scale", "table", "lmk", "bias"]),
    (decode, ["q", "k", "v", "scale", "lmk", "table", "out", "lse", "idx"]),
    (evict, ["acc", "table", "acc_out", "table_out", "lens", "n"]),
])
def test_null_pointers_are_refused(call, names):
    for n in names:
        assert call(params(), **{n: None}) == 1, n
        assert "NULL" in hils.hils_last_error()


def test_pages_flags_and_limits():
    for call in (append, landmark, decode):
        assert call(params(), pages=0) == 1 and "num_pages" in hils.hils_last_error()
    for call in (append, evict):
        assert call(params(flags=hils.HILS_FLAG_SHARED_LMK_QUERY)) == 1
    for call in (append, landmark):
        assert call(params(flags=hils.HILS_FLAG_GIVEN_IDX)) == 1
    assert decode(params(flags=hils.HILS_FLAG_HEAD_NORM_SELECT)) == 2 and "8-bit" in hils.hils_last_error()
    assert decode(params(flags=hils.HILS_FLAG_SHARED_LMK_QUERY)) == 1
    assert decode(params(window=4033)) == 2 and evict(params(window=4033)) == 2
    assert decode(params(B=300, N=256)) == 1 and "65535" in hils.hils_last_error()
    assert decode(params()) == 3 and decode(params(), ws=FAKE, nbytes=8) == 3
    for kw in (dict(budget=-1), dict(sink=-1), dict(most=-1)):
        assert evict(params(), **kw) == 1 and ">= 0" in hils.hils_last_error()
    assert evict(params(), freed=None) == 1 and "freed" in hils.hils_last_error()
    assert evict(params(), weights=FAKE) == 1 and "idx" in hils.hils_last_error()
    odd = ctypes.c_void_p(0x1008)
    for call, names in ((append, ["k", "v"]), (landmark, ["k", "lmk"]), (decode, ["k", "v", "lmk"])):
        for n in names:
            assert call(params(), **{n: odd}) == 1 and "16-byte" in hils.hils_last_error()
    for call in (append, landmark, decode):
        assert call(params(), scale=ctypes.c_void_p(0x1004)) == 1 and "8-byte" in hils.hils_last_error()
    # more workgroups than a grid holds, more weights than an int counts
    assert append(params(B=65535, Hkv=64, Hq=64, N=1 << 20, L=1 << 20)) == 2
    assert landmark(params(B=65535, Hkv=64, Hq=64, N=1 << 20, L=1 << 20)) == 2
    assert decode(params(B=65535, Hkv=64, Hq=64, N=1, L=1 << 20)) == 2 and "workgroups" in hils.hils_last_error()
    assert evict(params(Hkv=65535, Hq=65535, N=1 << 20, L=1 << 20), weights=FAKE, idx=FAKE) == 2


def test_workspace_never_falls_as_a_call_grows():
    base = dict(B=3, Hq=32, Hkv=8, N=1, L=64 * 40, d=128, topk=16, window=512)

    def size(**kw):
        return hils.hils_workspace_size(hils.Params(**{**base, **kw}), hils.HILS_OP_DECODE_Q8)

    for key, values in (("B", [1, 2, 3, 7, 8, 40, 130]), ("N", [1, 2, 3, 4, 5, 9]),
                        ("L", [64 * n for n in (10, 63, 64, 65, 128, 300, 2049, 16385)])):
        sizes = [size(**{key: v}) for v in values]
        assert sizes == sorted(sizes), (key, sizes)
    for op in (hils.HILS_OP_Q8_APPEND, hils.HILS_OP_Q8_LANDMARK, hils.HILS_OP_CACHE_EVICT):
        assert hils.hils_workspace_size(hils.Params(**base), op) == 0


def test_every_entry_point_is_exported():
    lib = ctypes.CDLL(hils._LIB_PATH)
    header = open(hils._LIB_PATH.rsplit("/", 2)[0] + "/include/hils.h").read()
    for n in ("hils_q8_append", "hils_q8_landmark_fwd", "hils_decode_q8_fwd", "hils_cache_evict"):
        assert hasattr(lib, n) and hasattr(hils, n) and f"int {n}(" in header


def test_the_binding_refuses_host_tensors():
    p = params()
    x = torch.zeros(p.B, p.Hkv, p.N, p.d, dtype=torch.bfloat16)
    pool = torch.zeros(4, p.Hkv, 64, p.d, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="GPU tensor"):
        hils.hils_q8_append(p, x, x, pool, pool, torch.zeros(4, 2, 2), torch.zeros(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError, match="needs idx"):
        hils.hils_cache_evict(p, torch.zeros(2, 4), torch.zeros(2, 4, dtype=torch.int32), weights=torch.zeros(2, 2, 4, 11))
    assert hils.hils_window_pieces(512) == 9 and hils.hils_window_pieces(1) == 1 and hils.hils_window_pieces(2) == 2
