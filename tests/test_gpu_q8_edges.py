"""The 8-bit cache on the GPU: selections, values and arguments at the edge of what the entry points take,
against the float64 oracle (tests/q8_oracle.py) with the tolerances of tests/test_gpu_q8.py."""
import numpy as np
import pytest
import torch

from tests import q8_oracle as Q
from tests import test_gpu_q8 as T

pytestmark = pytest.mark.gpu


def same(got, ref):
    for x, y in zip(got, ref):
        assert np.array_equal(x.cpu().numpy().astype(np.float64), np.asarray(y, np.float64))


@pytest.mark.parametrize("L", [64 * 40, 64 * 25001])  # totals in LDS, and too many for it
def test_evict_adds_every_slot_of_a_chunk_named_twice(L):
    """Given selections that come back to a chunk: its slots are added one after the other, wherever the rows fall."""
    hils = T.hils_()
    p = hils.Params(B=1, Hq=4, Hkv=4, N=16, L=L, d=64, topk=64, window=64)  # 64 rows of 66 weights: over four rounds
    acc, table, wt, idx = T.evict_inputs(p, 3, None, 3)
    r = np.random.default_rng(5)
    top = min(30, Q.n_candidates(L - 16, 64))
    idx[:] = r.integers(-2, top, idx.shape)  # few chunks, many slots
    idx[0, 0, 0] = -1
    idx[0, 0, 0, :5] = 5, -1, 5, 2, 5
    idx[0, 1, 3, :6] = 1 << 30, 7, 2, 3, 7, -5
    idx[0, 3, 15] = 9
    rows = idx.reshape(-1, 64)
    twice = sum(len(v) > len(set(v)) for v in ([c for t, c in enumerate(x) if c >= 0 and (t == 0 or c > x[t - 1])] for x in rows))
    assert twice > 50
    budget = Q.n_candidates(L - 1, 64) - 12
    ref = Q.evict(p, acc, table, None, budget, 2, L // 64, wt, idx)
    same(hils.hils_cache_evict(p, T.dev(acc), T.dev(table), budget=budget, sink=2, weights=T.dev(wt), idx=T.dev(idx)), ref)


def test_a_given_selection_that_repeats_a_chunk_is_evicted_by_all_its_weight():
    """Decode attends a chunk named twice twice; eviction counts what decode reports, all of it."""
    hils = T.hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, N=2, L=1024, d=64, topk=5, window=128, scale=0.125, flags=hils.HILS_FLAG_GIVEN_IDX)
    t = T.world(p, 6)
    given = np.tile(np.int32([5, -1, 5, 2, 5]), (2, 2, 2, 1))
    got = T.run_decode(p, t, idx=T.dev(given))
    T.check_decode(p, got, Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"], given=given))
    acc = torch.zeros((2, 16), device="cuda")
    res = hils.hils_cache_evict(p, acc, T.dev(t["table"]), budget=100, weights=got[3], idx=got[2])
    w = T.host(got[3])
    assert (w[..., [0, 2, 4]] > 0).all() and (w[..., [1, 3]] == 0).all()
    # (sums of 4 rows of float32 weights of at most 4: roundings of 2^-24 of 16)
    assert np.abs(T.host(res[0])[:, 5] - w[..., [0, 2, 4]].sum((1, 2, 3))).max() <= 12 * 16 * 2.0 ** -24
    assert np.abs(T.host(res[0]).sum(1) - w.sum((1, 2, 3))).max() <= 64 * 16 * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,B", [(64, 2), (128, 70)])  # shared rows, a workgroup each
def test_decode_nan_in_masked_chunks(d, B, dtype):
    """A chunk with a bias of -inf that is chosen because candidates are few weighs nothing, whatever it holds:
    masked for all heads with NaN keys and values, masked for one head with NaN keys."""
    hils = T.hils_()
    p = hils.Params(B=B, Hq=8, Hkv=2, N=1, L=512, d=d, topk=8, window=64, scale=0.125, dtype=dtype)
    t = T.world(p, 17)
    for b in range(B):
        t["bias"][t["table"][b, 1]] = -np.inf
        t["bias"][t["table"][b, 3], 2] = -np.inf  # head 2, of group 0
    clean = T.run_decode(p, t, bias=True)
    T.check_decode(p, clean, Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"], bias=t["bias"]))
    for b in range(B):
        t["k"][t["table"][b, 1], :, 9], t["v"][t["table"][b, 1], :, :, 9] = 0x7f, 0xff
        t["k"][t["table"][b, 3], 0, 5] = 0x7f
    got = T.run_decode(p, t, bias=True)
    keep = [0, 1, 3]  # the heads of group 0 that attend chunk 3
    others = [2, 4, 5, 6, 7]
    assert torch.equal(got[0][:, others], clean[0][:, others])
    assert all(torch.equal(x, y) for x, y in zip(got[1:], clean[1:]))
    assert torch.isnan(got[0][:, keep]).all()


@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("shared", [False, True])
def test_decode_zero_scores_of_either_sign_tie(n, shared):
    """Scores of 0 and -0 (products of -0 with biases of either sign) are equal: the lowest chunks are chosen."""
    hils = T.hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, Hl=2 if shared else 8, N=n, L=64 * 300, d=64, topk=9, window=64, scale=-0.125)
    t = T.world(p, 23)
    t["lmk"][:] = 0
    t["bias"][:] = -0.0
    t["bias"][t["table"][:, 1::2]] = 0.0
    ref = Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"], bias=t["bias"])
    got = T.run_decode(p, t, bias=True)
    assert got[2][0, 0, 0].tolist() == list(range(9))
    T.check_decode(p, got, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_writes_of_chunks_without_a_page(dtype):
    """One table for the kernels and the oracle: chunks whose entry is outside the pool are dropped."""
    hils = T.hils_()
    p = hils.Params(B=3, Hq=4, Hkv=2, N=200, L=256, d=64, topk=1, window=64, dtype=dtype)
    new, pools, scale, table = T.append_inputs(p, 22)
    lens, counts = [256, 201, 64], [200, 200, 64]
    for b, c, bad in ((0, 1, -1), (0, 3, len(pools[0])), (1, 0, -2 ** 31), (1, 3, 2 ** 31 - 1)):
        table[b, c] = bad
    ref = Q.append(p, *new, *pools, scale, table, lens, counts)
    got = T.run_append(p, new, pools, scale, table, lens, counts)
    assert np.array_equal(got[2], ref[2]) and T.same_codes(got[0], ref[0]) and T.same_codes(got[1], ref[1])
    n = len(pools[0])
    lq = rounded_lq(p, 3)
    lm, bias = T.f8(np.full((n, 4, 64), 0x5a, np.uint8)), torch.full((n, 4), 7.0, device="cuda")
    i32 = [T.dev(np.int32(x)) for x in (lens, counts)]
    hils.hils_q8_landmark_fwd(p, T.dev(lq, p.torch_dtype), T.f8(ref[0]), T.dev(ref[2]), T.dev(table), lm, bias, *i32)
    rows = Q.landmark(p, lq, ref[0], ref[2], table, lens, counts)
    assert sorted(rows) == sorted(table[b, c] for b, c in ((0, 0), (0, 2), (1, 1), (1, 2), (2, 0)))
    for page in range(n):
        if page in rows:
            off = np.abs(Q.VALUE[T.codes(lm)[page]] - rows[page][0])
            assert (off <= np.maximum(2.0 ** -4 * np.abs(rows[page][0]), 2.0 ** -10) + 1e-4 * 448).all()
            assert np.abs(bias[page].cpu().numpy() - rows[page][1]).max() <= 1e-4
        else:
            assert (T.codes(lm)[page] == 0x5a).all() and (bias[page] == 7).all()


def rounded_lq(p, seed):
    """Landmark queries of a call's completed chunks, small enough for logits up to 10."""
    x = np.random.default_rng(seed).standard_normal((p.B, p.Hl or p.Hq, (p.N + 63) // 64, p.d)).astype(np.float32)
    return T.rounded(x / 64, p.dtype)


TOTALS = {
    "subnormal": lambda r, n: r.integers(0, 5, n) * 1e-45,
    "one_subnormal_apart": lambda r, n: 1.0 + r.integers(0, 2, n) * 2.0 ** -23,
    "whole_range": lambda r, n: r.choice([-3e38, 3e38, 0.0, -0.0, 1e-40, -1e-40, 5.0], n),
    "infinities": lambda r, n: r.choice([np.inf, -np.inf, 1.0, 2.0, np.nan], n),
    "two_scales": lambda r, n: np.where(r.random(n) < 0.5, r.random(n) * 1e-6, 1e6 * r.random(n)),
    "negative": lambda r, n: -np.exp(r.standard_normal(n) * 10),
    "mostly_equal": lambda r, n: np.where(r.random(n) < 0.99, 7.0, r.standard_normal(n)),
}


@pytest.mark.parametrize("name", TOTALS)
@pytest.mark.parametrize("nC", [70, 1025, 8193, 20481])
def test_evict_totals_of_every_kind(nC, name):
    """Any drop count, over totals whose range, spacing or ties defeat equal steps."""
    hils = T.hils_()
    p = hils.Params(B=3, Hq=1, Hkv=1, N=1, L=64 * nC, d=64, topk=1, window=64)
    r = np.random.default_rng(nC)
    acc = np.stack([TOTALS[name](r, nC) for _ in range(3)]).astype(np.float32)
    table = np.stack([r.permutation(nC) for _ in range(3)]).astype(np.int32)
    lens = [64 * nC, 64 * nC - 900, 64 * (nC // 2)]
    for budget in (0, nC // 3, nC - 3):
        got = hils.hils_cache_evict(p, T.dev(acc), T.dev(table), T.dev(np.int32(lens)), budget=budget, sink=2)
        got = [x.cpu().numpy() for x in got]
        for b, length in enumerate(lens):
            able = np.arange(2, Q.n_candidates(length - 1, 64))
            count = min(max(0, len(able) + 2 - budget), len(able))
            order = np.lexsort((able, np.nan_to_num(acc[b, able], posinf=np.inf, neginf=-np.inf), np.isnan(acc[b, able])))
            gone = np.sort(able[order[:count]])
            kept = np.delete(np.arange(nC), gone)
            assert got[4][b] == count and got[2][b] == length - 64 * count
            assert np.array_equal(got[3][b], np.r_[table[b, gone], np.full(nC - count, -1)])
            assert np.array_equal(got[1][b], np.r_[table[b, kept], np.full(count, -1)])
            assert np.array_equal(got[0][b], np.r_[acc[b, kept], np.zeros(count, np.float32)], equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_streams_at_once(dtype):
    """Calls of two streams over the same pages, each with a workspace of its own: the bits of calls by themselves."""
    hils = T.hils_()
    ps = [hils.Params(B=b, Hq=16, Hkv=4, N=n, L=4096, d=128, topk=16, window=512, scale=0.125, dtype=dtype) for b, n in ((3, 1), (2, 4))]
    t = T.world(ps[0], 51)
    pools = T.f8(t["k"]), T.f8(t["v"]), T.dev(t["scale"]), T.f8(t["lmk"])
    r = np.random.default_rng(1)
    qs = [T.dev(r.standard_normal((p.B, 16, p.N, 128)).astype(np.float32), p.torch_dtype) for p in ps]
    tables = [T.dev(t["table"][:p.B]) for p in ps]
    wss = [torch.empty(hils.hils_workspace_size(p, hils.HILS_OP_DECODE_Q8), dtype=torch.uint8, device="cuda") for p in ps]
    want = [hils.hils_decode_q8_fwd(p, q, *pools, tb, workspace=w) for p, q, tb, w in zip(ps, qs, tables, wss)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in ps], [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(hils.hils_decode_q8_fwd(ps[i], qs[i], *pools, tables[i], workspace=wss[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, y) for g in got[i] for x, y in zip(g, want[i]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,B,n", [(64, 2, 1), (128, 70, 1), (64, 3, 4)])
@pytest.mark.parametrize("shared", [False, True])
def test_decode_nan_landmarks_of_masked_chunks(d, B, n, dtype, shared):
    """A chunk of NaN keys has a NaN landmark; a bias of -inf masks it all the same."""
    hils = T.hils_()
    p = hils.Params(B=B, Hq=8, Hkv=2, Hl=2 if shared else 8, N=n, L=512, d=d, topk=8, window=64, scale=0.125, dtype=dtype)
    t = T.world(p, 18)
    for b in range(B):
        t["bias"][t["table"][b, 2]] = -np.inf
        t["bias"][t["table"][b, 4], 0] = -np.inf
    clean = T.run_decode(p, t, bias=True)
    T.check_decode(p, clean, Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"], bias=t["bias"]))
    for b in range(B):
        t["k"][t["table"][b, 2], :, 9], t["lmk"][t["table"][b, 2]] = 0x7f, 0x7f
        t["lmk"][t["table"][b, 4], 0] = 0xff
    assert all(torch.equal(x, y) for x, y in zip(T.run_decode(p, t, bias=True), clean))
