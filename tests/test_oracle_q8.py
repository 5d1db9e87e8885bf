"""The float64 oracle of the 8-bit cache's operators, pinned on the CPU: against torch's e4m3
conversions, the library's C oracle of the attention (contiguous caches of the values that the pages
stand for), sorting, and mistakes planted in it."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import oracle
from tests import q8_oracle as Q


def shape(**kw):
    d = dict(B=2, Hq=4, Hkv=2, Hl=0, N=1, L=512, d=64, chunk=64, topk=3, window=100, scale=0.125)
    d.update(kw)
    p = SimpleNamespace(**d)
    p.c = lambda: p
    return p


def pages(p, seed, spread=2):
    """Random pools, every sequence's chunks anywhere among them."""
    r = np.random.default_rng(seed)
    nc, Hl = p.L // 64, p.Hl or p.Hq
    P = p.B * nc + 3
    t = {"k": Q.encode(r.standard_normal((P, p.Hkv, 64, p.d)) * 60), "v": Q.encode(r.standard_normal((P, p.Hkv, p.d, 64)) * 60),
         "scale": 2.0 ** r.integers(-6 - spread, -5, (P, p.Hkv, 2)).astype(np.float32),
         "lmk": Q.encode(r.standard_normal((P, Hl, p.d)) * 20), "bias": r.standard_normal((P, Hl)).astype(np.float32),
         "table": r.permutation(P)[:p.B * nc].reshape(p.B, nc).astype(np.int32)}
    t["q"] = r.standard_normal((p.B, p.Hq, p.N, p.d)).astype(np.float32)
    t["q_route"] = r.standard_normal((p.B, p.Hq, p.N, p.d)).astype(np.float32)
    return t


def test_codes_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(Q.VALUE, want, equal_nan=True)
    x = np.concatenate([np.random.default_rng(1).standard_normal(4000) * s for s in (100, 1, 0.01, 0.002)])
    edges = (Q.VALUE[:126] + Q.VALUE[1:127]) / 2  # halfway: ties to even
    x = np.float32(np.clip(np.concatenate([x, edges, -edges, Q.VALUE[:127]]), -448, 448))
    assert np.array_equal(Q.encode(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("kw,route,bias,lens", [
    (dict(), False, False, [512, 77]),
    (dict(N=3, window=64, Hl=2), True, True, [400, 3]),
    (dict(Hq=8, topk=20, window=1), False, True, [511, 64]),
])
def test_decode_agrees_with_the_c_oracle(kw, route, bias, lens):
    p = shape(**kw)
    t = pages(p, 3)
    nc, Hl = p.L // 64, p.Hl or p.Hq
    out, lse, idx, wt = Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"],
                                 bias=t["bias"] if bias else None, q_route=t["q_route"] if route else None, seqlens=lens)
    sc = t["scale"][t["table"]].astype(np.float64).transpose(0, 2, 1, 3)  # [B, Hkv, nC, 2]
    k = (Q.VALUE[t["k"][t["table"]]].transpose(0, 2, 1, 3, 4) * sc[..., 0, None, None]).reshape(p.B, p.Hkv, p.L, p.d)
    v = (Q.VALUE[t["v"][t["table"]]].transpose(0, 2, 1, 4, 3) * sc[..., 1, None, None]).reshape(p.B, p.Hkv, p.L, p.d)
    lmk = Q.VALUE[t["lmk"][t["table"]]].transpose(0, 2, 1, 3) * np.repeat(sc[..., 0], Hl // p.Hkv, 1)[..., None]
    s = oracle.Shape(B=p.B, Hq=p.Hq, Hkv=p.Hkv, Hl=Hl, N=p.N, L=p.L, d=p.d, chunk=64, topk=p.topk, window=p.window,
                     scale=p.scale)
    ref = oracle.decode(s, t["q"], k.astype(np.float32), v.astype(np.float32), lmk.astype(np.float32), seqlens=lens,
                        bias=t["bias"][t["table"]].transpose(0, 2, 1).copy() if bias else None,
                        q_route=t["q_route"] if route else None)
    assert np.array_equal(idx, ref["idx"])
    np.testing.assert_allclose(out, ref["out"], atol=1e-6)
    np.testing.assert_allclose(lse, ref["lse"], atol=1e-6)
    np.testing.assert_allclose(wt.sum(-1), p.Hq // p.Hkv, atol=1e-9)


def test_landmark_is_prop_3_1():
    p = shape(N=130, B=1, L=256)
    t = pages(p, 5)
    r = np.random.default_rng(6)
    lq = r.standard_normal((1, p.Hq, 3, p.d)).astype(np.float32)
    got = Q.landmark(p, lq, t["k"], t["scale"], t["table"], [200], [130])  # tokens 70 .. 199: chunks 1 and 2
    assert sorted(got) == sorted(int(t["table"][0, c]) for c in (1, 2))
    page = int(t["table"][0, 2])
    x = Q.VALUE[t["k"][page, 1]]
    s = p.scale * float(t["scale"][page, 1, 0]) * x @ lq[0, 3, 1].astype(np.float64)
    w = np.exp(s) / np.exp(s).sum()
    np.testing.assert_allclose(got[page][0][3], w @ x, rtol=1e-9)
    np.testing.assert_allclose(got[page][1][3], -(w * np.log(w)).sum(), rtol=1e-9)


def test_append_by_hand():
    p = shape(B=1, Hq=1, Hkv=1, N=2, L=128, d=64)
    k, v = np.full((3, 1, 64, 64), 0x55, np.uint8), np.full((3, 1, 64, 64), 0x55, np.uint8)
    scale = np.full((3, 1, 2), 2.0 ** -4, np.float32)
    table = np.array([[2, 0]], np.int32)
    new = np.zeros((1, 1, 2, 64), np.float32)
    new[0, 0, 0, 0], new[0, 0, 1, 0] = 448 * 2.0 ** -3, 1.0
    k2, v2, s2 = Q.append(p, new, new, k, v, scale, table, [65], [2])  # positions 63 and 64
    assert s2[2, 0, 0] == 2.0 ** -3 and s2[0, 0, 0] == 2.0 ** -8 and s2[1, 0, 0] == 2.0 ** -4
    assert Q.VALUE[k2[2, 0, 63, 0]] == 448 and Q.VALUE[k2[0, 0, 0, 0]] == 256
    assert Q.VALUE[k2[2, 0, 5, 5]] == Q.VALUE[0x55] / 2 and k2[0, 0, 1, 0] == 0x55 and v2[0, 0, 0, 1] == 0x55
    assert (k2[1] == 0x55).all() and Q.VALUE[v2[2, 0, 0, 63]] == 448


def test_planted_mistakes_show():
    """A mistake in the oracle's scale rule, its mask or its tie rule changes what it returns."""
    p = shape()
    t = pages(p, 9)
    args = (t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"])
    right = Q.decode(p, *args, seqlens=[500, 300])
    wide = Q.decode(p, *args, seqlens=[501, 301])  # a position off
    swapped = Q.decode(p, t["q"], t["k"], t["v"], t["scale"][..., ::-1], t["lmk"], t["table"], seqlens=[500, 300])
    assert np.abs(right[0] - wide[0]).max() > 1e-2 and np.abs(right[0] - swapped[0]).max() > 1e-2
    acc = np.zeros((2, 8))
    a = Q.evict(p, acc, t["table"], [512, 300], 2, 1, 8)
    assert a[4].tolist() == [4, 1] and a[3][0, :4].tolist() == t["table"][0, 1:5].tolist()  # ties: the lowest first
