"""Decode over the 8-bit cache in the forms that large batches and long contexts take, against the float64
oracle with the tolerances of tests/test_gpu_q8.py: more than 128 rows (a workgroup each), slices of 256
candidates, more survivors of them than one wave merges.  (The "many_rows" of tests/test_gpu_q8.py are 96,
which workgroups share.)  Sequences are permutations of one set of pages."""
import numpy as np
import pytest
import torch

from tests import q8_oracle as Q
from tests import test_gpu_q8 as T

pytestmark = pytest.mark.gpu


def world(p, seed):
    r = np.random.default_rng(seed)
    nc, Hl = p.L // 64, p.Hl or p.Hq
    P = nc + 7
    some = Q.encode(r.standard_normal(1 << 16) * 60)

    def codes(*shape):
        return some[r.integers(0, 1 << 16, shape, dtype=np.int32)]

    def grid():
        return np.clip(np.round(r.standard_normal((p.B, p.Hq, p.N, p.d)) * 16) / 16, -4, 4).astype(np.float32)

    return {"k": codes(P, p.Hkv, 64, p.d), "v": codes(P, p.Hkv, p.d, 64),
            "scale": 2.0 ** r.integers(-7, -4, (P, p.Hkv, 2)).astype(np.float32),
            "lmk": Q.encode(8 * np.clip(np.round(r.standard_normal((P, Hl, p.d)) * 4), -15, 15)),
            "bias": np.round(r.standard_normal((P, Hl)) * 1024).astype(np.float32) / 1024,
            "table": np.stack([r.permutation(P)[:nc] for _ in range(p.B)]).astype(np.int32), "q": grid(), "q_route": grid()}


def check(p, seed, bias, route):
    t = world(p, seed)
    q = T.rounded(np.random.default_rng(8).standard_normal(t["q"].shape).astype(np.float32), p.dtype) if route else t["q"]
    r = np.random.default_rng(seed + 1)
    lens = [p.L] + [int(x) for x in r.integers(p.L // 2, p.L, p.B - 1)]
    ref = Q.decode(p, q, t["k"], t["v"], t["scale"], t["lmk"], t["table"], bias=t["bias"] if bias else None,
                   q_route=t["q_route"] if route else None, seqlens=lens)
    got = T.run_decode(p, t, lens, bias, route, q=q)
    torch.cuda.synchronize()
    T.check_decode(p, got, ref)
    return t, q, lens, ref


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("route", [False, True])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_a_workgroup_per_row(d, G, route, dtype):
    """160 rows, one token each: the next part's loads are issued ahead."""
    p = T.hils_().Params(B=20, Hq=8 * G, Hkv=8, N=1, L=2048, d=d, topk=16, window=512, scale=0.125, dtype=dtype)
    check(p, 10 * G + d, bias=G % 4 == 0, route=route)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("route", [False, True])
def test_a_workgroup_per_drafted_row(route, dtype):
    p = T.hils_().Params(B=6, Hq=32, Hkv=8, N=4, L=2048, d=128, topk=16, window=512, scale=0.125, dtype=dtype)
    check(p, 5, bias=False, route=route)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [128, 136])  # the last that share, the first that do not
def test_both_sides_of_the_line_of_sharing(rows, dtype):
    p = T.hils_().Params(B=rows // 8, Hq=32, Hkv=8, N=1, L=1280, d=128, topk=8, window=256, scale=0.125, dtype=dtype)
    check(p, rows, bias=True, route=True)


SCAN = {
    "G4": dict(Hq=8, Hkv=2, B=2), "G8": dict(Hq=16, Hkv=2, B=2), "G1": dict(Hq=2, Hkv=2, B=2), "G2": dict(Hq=4, Hkv=2, B=2),
    "G4_shared": dict(Hq=8, Hkv=2, Hl=2, B=2), "G8_shared": dict(Hq=16, Hkv=2, Hl=2, B=2),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 4, 7])
@pytest.mark.parametrize("name", SCAN)
def test_slices_of_256(name, N, dtype):
    """600 chunks and K = 64 leave slices of 256: four blocks of 64 landmarks, a remainder of 65 to 128 in the last."""
    p = T.hils_().Params(N=N, L=64 * 600, d=128, topk=64, window=512, scale=0.125, dtype=dtype, **SCAN[name])
    check(p, len(name) + N, bias=name.startswith("G8"), route=name == "G4")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,G,N", [(128, 4, 1), (64, 8, 1), (128, 2, 4)])
def test_many_survivors_of_many_rows(d, G, N, dtype):
    """1100 chunks and K = 64: 320 survivors per row, more than 128 rows, narrowed by the whole workgroup."""
    p = T.hils_().Params(B=36 // N, Hq=4 * G, Hkv=4, N=N, L=64 * 1100, d=d, topk=64, window=128, scale=0.125, dtype=dtype)
    check(p, d + G, bias=G == 8, route=G == 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("route", [False, True])
def test_given_selection(route, dtype):
    """A selection that is given: the one that a first call made, with entries taken out."""
    hils = T.hils_()
    kw = dict(B=18, Hq=32, Hkv=8, N=1, L=2048, d=128, topk=16, window=256, scale=0.125, dtype=dtype)
    t, q, lens, ref = check(hils.Params(**kw), 3, bias=True, route=route)
    given = ref[2].copy()
    given[:, :, :, 3::5] = -1
    p = hils.Params(flags=hils.HILS_FLAG_GIVEN_IDX, **kw)
    want = Q.decode(p, q, t["k"], t["v"], t["scale"], t["lmk"], t["table"], bias=t["bias"],
                    q_route=t["q_route"] if route else None, seqlens=lens, given=given)
    T.check_decode(p, T.run_decode(p, t, lens, True, route, q=q, idx=T.dev(given)), want)


def test_a_table_straight_from_eviction():
    """Eviction, then a step on the table as it comes (-1 past what is left): append, landmarks, decode."""
    hils = T.hils_()
    base = dict(B=3, Hq=8, Hkv=2, L=1024, d=64, topk=4, window=64, scale=0.125)
    p = hils.Params(N=2, **base)
    t = world(p, 12)
    P = len(t["k"])
    t["table"] = np.random.default_rng(1).permutation(48).reshape(3, 16).astype(np.int32)  # pages of its own for each
    for n in ("k", "v", "lmk", "scale", "bias"):
        t[n] = np.concatenate([t[n]] * (48 // P + 1))[:48].copy()
    lens = np.int32([1000, 700, 380])
    acc = np.random.default_rng(2).integers(0, 999, (3, 16)).astype(np.float32)
    res = hils.hils_cache_evict(p, T.dev(acc), T.dev(t["table"]), T.dev(lens), budget=6, sink=1)
    want = Q.evict(p, acc, t["table"], lens, 6, 1, 16)
    assert all(np.array_equal(x.cpu().numpy(), y) for x, y in zip(res, want))
    table, lens = want[1], want[2] + 2
    assert (table < 0).any()
    r = np.random.default_rng(3)
    new = [T.rounded(r.standard_normal((3, 2, 2, 64)).astype(np.float32), "bf16") for _ in range(2)]
    lq = T.rounded(r.standard_normal((3, 8, 1, 64)).astype(np.float32), "bf16")
    k, v, s = Q.append(p, *new, t["k"], t["v"], t["scale"], table, lens)
    gk, gv, gs, lm, bias = T.f8(t["k"]), T.f8(t["v"]), T.dev(t["scale"]), T.f8(t["lmk"]), T.dev(t["bias"])
    gl = res[2] + 2
    hils.hils_q8_append(p, *[T.dev(x, torch.bfloat16) for x in new], gk, gv, gs, res[1], gl)
    assert T.same_codes(T.codes(gk), k) and T.same_codes(T.codes(gv), v) and np.array_equal(gs.cpu().numpy(), s)
    hils.hils_q8_landmark_fwd(p, T.dev(lq, torch.bfloat16), gk, gs, res[1], lm, bias, gl)
    got = hils.hils_decode_q8_fwd(p, T.dev(t["q"], torch.bfloat16), gk, gv, gs, lm, res[1], bias, seqlens=gl)
    given = got[2].cpu().numpy()  # (scores off the grid: held to the selection that was made)
    gp = hils.Params(N=2, flags=hils.HILS_FLAG_GIVEN_IDX, **base)
    T.check_decode(p, got, Q.decode(gp, t["q"], k, v, s, T.codes(lm), table, bias=bias.cpu().numpy(), seqlens=lens, given=given))
