"""The 8-bit cache on the GPU against the float64 oracle (tests/q8_oracle.py).

Selections are exact: landmarks and routing queries lie on grids on which every score is exact in 32
bits (queries multiples of 1/16 up to 4, landmark codes multiples of 8 up to 120, scale 1/8).
Tolerances, derived beforehand:
  * append and evict: equal codes, scales, ids; totals on a grid, so equal too;
  * landmark rows: half a step of e4m3 (2^-4 of the value, 2^-10 below 2^-6) and 1e-4 of the keys'
    largest code for the float32 sum (64 terms, logits up to about 10 that carry 64 roundings of
    2^-24 each: 64 * 10 * 2^-24 = 4e-5 of a weight); the bias the same 1e-4;
  * out, lse and weights in float32: logits up to about 10 from 128 products carry up to
    128 * 10 * 2^-24 = 8e-5, a weight twice that relative to itself (numerator, denominator), so
    2e-4 of the largest value that takes part; out in bf16: half a step (2^-8 of the value) more."""
import numpy as np
import pytest
import torch

from tests import q8_oracle as Q

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
TOL = 2e-4


def hils_():
    from paper_2607_02980_amd import hils

    return hils


def dev(x, dtype=None):
    t = torch.as_tensor(np.ascontiguousarray(x))
    return (t if dtype is None else t.to(dtype)).cuda()


def f8(x):
    return dev(x).view(F8)


def codes(t):
    return t.view(torch.uint8).cpu().numpy()


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def rounded(x, dtype):
    """x as the storage type holds it, in float32."""
    return torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).float().numpy()


def world(p, seed, poison=True):
    """Pools and queries; whatever lies past a sequence's end, and unused pages, is NaN."""
    r = np.random.default_rng(seed)
    nc, Hl = p.L // 64, p.Hl or p.Hq
    P = p.B * nc + 5
    t = {"k": Q.encode(r.standard_normal((P, p.Hkv, 64, p.d)) * 60), "v": Q.encode(r.standard_normal((P, p.Hkv, p.d, 64)) * 60),
         "scale": 2.0 ** r.integers(-7, -4, (P, p.Hkv, 2)).astype(np.float32),
         "lmk": Q.encode(8 * np.clip(np.round(r.standard_normal((P, Hl, p.d)) * 4), -15, 15)),
         "bias": np.round(r.standard_normal((P, Hl)) * 1024).astype(np.float32) / 1024,
         "table": r.permutation(P)[:p.B * nc].reshape(p.B, nc).astype(np.int32)}

    def grid():
        return np.clip(np.round(r.standard_normal((p.B, p.Hq, p.N, p.d)) * 16) / 16, -4, 4).astype(np.float32)

    t["q"], t["q_route"] = grid(), grid()
    return t


def bury(t, p, lens):
    """NaN in every byte that a call may not use."""
    live = np.zeros(len(t["k"]), bool)
    for b in range(p.B):
        full, part = divmod(int(lens[b]), 64)
        live[t["table"][b, :full]] = True
        if part:
            pg = t["table"][b, full]
            live[pg] = True
            t["k"][pg, :, part:] = 0x7f
            t["v"][pg, :, :, part:] = 0xff
        t["lmk"][t["table"][b, full:]] = 0x7f
    for n in ("k", "v", "lmk"):
        t[n][~live] = 0x7f
    for n in ("scale", "bias"):
        t[n][~live] = np.nan


def run_decode(p, t, lens=None, bias=False, route=False, q=None, **kw):
    hils = hils_()
    dt = p.torch_dtype
    return hils.hils_decode_q8_fwd(
        p, dev(t["q"] if q is None else q, dt), f8(t["k"]), f8(t["v"]), dev(t["scale"]), f8(t["lmk"]), dev(t["table"]),
        bias_pages=dev(t["bias"]) if bias else None, q_route=dev(t["q_route"], dt) if route else None,
        seqlens=None if lens is None else dev(np.int32(lens)), **kw)


def check_decode(p, got, ref, big=4.0 * 448 / 16):
    out, lse, idx, wt = got
    assert np.array_equal(idx.cpu().numpy(), ref[2])
    top = np.abs(ref[0]).max()
    tol = TOL * max(1.0, top) + (2.0 ** -8 * np.abs(ref[0]) if p.dtype == "bf16" else 0.0)
    d = np.abs(host(out) - ref[0])
    print("out", d.max(), "of", top, "lse", np.abs(host(lse) - ref[1]).max(), flush=True)
    assert (d <= tol).all()
    assert np.abs(host(lse) - ref[1]).max() <= TOL
    if wt is not None:
        assert np.abs(host(wt) - ref[3]).max() <= TOL * (p.Hq // p.Hkv)


DECODE = {
    # one token: the whole cache, one token, chunk edges
    "edges_G4": (dict(B=6, Hq=8, Hkv=2, N=1, L=1024, d=128, topk=4, window=128), [1024, 1, 64, 65, 63, 700], True, False),
    "window_1": (dict(B=3, Hq=4, Hkv=4, N=1, L=512, d=64, topk=7, window=1), [512, 2, 129], False, True),
    "window_4032_topk_64": (dict(B=1, Hq=8, Hkv=1, N=1, L=8192, d=64, topk=64, window=4032), [8101], True, True),
    "few_candidates_G2": (dict(B=2, Hq=4, Hkv=2, N=1, L=2048, d=128, topk=33, window=300), [2048, 900], False, False),
    "f32_G4": (dict(B=2, Hq=8, Hkv=2, N=1, L=4096, d=128, topk=16, window=512, dtype="f32"), [4095, 600], True, True),
    "f32_G8_shared": (dict(B=2, Hq=16, Hkv=2, Hl=2, N=1, L=2048, d=64, topk=8, window=256, dtype="f32"), None, True, False),
    "shared_G4": (dict(B=3, Hq=32, Hkv=8, Hl=8, N=1, L=6400, d=128, topk=16, window=512), [6400, 4000, 511], False, False),
    # drafted tokens: fewer and more than a group of queries, crossing a chunk's end
    "drafts_G4": (dict(B=3, Hq=8, Hkv=2, N=4, L=2048, d=128, topk=8, window=512), [2048, 4, 1026], True, False),
    "drafts_7_G4": (dict(B=2, Hq=8, Hkv=2, N=7, L=2048, d=64, topk=6, window=100), [2045, 67], False, True),
    "drafts_G8_shared": (dict(B=2, Hq=16, Hkv=2, Hl=2, N=5, L=1024, d=64, topk=8, window=200), [1000, 322], True, False),
    "drafts_G1": (dict(B=2, Hq=3, Hkv=3, N=11, L=1024, d=128, topk=5, window=64), [1024, 200], False, False),
    "drafts_G2_f32": (dict(B=2, Hq=4, Hkv=2, N=9, L=1024, d=64, topk=5, window=63, dtype="f32"), [1001, 9], True, True),
    "drafts_G4_shared_f32": (dict(B=1, Hq=4, Hkv=1, Hl=1, N=3, L=1024, d=128, topk=5, window=65, dtype="f32"), None, False, True),
    # many rows: the fusion in a launch of its own
    "many_rows": (dict(B=12, Hq=32, Hkv=8, N=1, L=2048, d=64, topk=16, window=512), [2048 - 150 * i for i in range(12)], False, False),
    "many_rows_drafts_f32": (dict(B=4, Hq=16, Hkv=8, N=5, L=1024, d=64, topk=9, window=128, dtype="f32"), [1024, 5, 777, 64], True, False),
    # more survivors than a wave merges alone, and than a workgroup takes in its first round
    "survivors_320": (dict(B=1, Hq=1, Hkv=1, N=1, L=64 * 1200, d=64, topk=64, window=128), [64 * 1200 - 3], False, False),
    "survivors_2112": (dict(B=1, Hq=1, Hkv=1, N=2, L=64 * 8400, d=64, topk=64, window=128), [64 * 8400 - 3], False, False),
}


@pytest.mark.parametrize("name", DECODE)
def test_decode(name):
    hils = hils_()
    kw, lens, bias, route = DECODE[name]
    p = hils.Params(scale=0.125, **kw)
    t = world(p, len(name) * 7 + p.N)
    bury(t, p, lens or [p.L] * p.B)
    q = rounded(np.random.default_rng(8).standard_normal(t["q"].shape).astype(np.float32), p.dtype) if route else t["q"]
    ref = Q.decode(p, q, t["k"], t["v"], t["scale"], t["lmk"], t["table"], bias=t["bias"] if bias else None,
                   q_route=t["q_route"] if route else None, seqlens=lens)
    print(name, flush=True)
    got = run_decode(p, t, lens, bias, route, q=q)
    torch.cuda.synchronize()
    check_decode(p, got, ref)
    assert np.abs(host(got[3]).sum(-1) - p.Hq // p.Hkv).max() <= TOL * (p.Hq // p.Hkv)
    again = run_decode(p, t, lens, bias, route, q=q, want_weights=False)
    assert again[3] is None and all(torch.equal(x, y) for x, y in zip(again[:3], got[:3]))


def test_decode_given_selection():
    """A row's valid entries count, the others not; its own order of slots stays."""
    hils = hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, N=3, L=1024, d=64, topk=6, window=128, scale=0.125, flags=hils.HILS_FLAG_GIVEN_IDX)
    t = world(p, 4)
    given = np.tile(np.int32([0, -1, 3, 3, 2, 9]), (2, 2, 3, 1))
    given[1, 0, 1] = [-1, -1, -1, -1, -1, -1]
    given[0, 1, 2] = [1 << 30, -5, 4, 5, 6, 7]
    lens = [1000, 400]
    ref = Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"], seqlens=lens, given=given)
    got = run_decode(p, t, lens, idx=dev(given))
    check_decode(p, got, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_nan_reaches_only_who_attends_it(dtype):
    hils = hils_()
    p = hils.Params(B=1, Hq=8, Hkv=2, N=4, L=512, d=64, topk=3, window=100, scale=0.125, dtype=dtype)
    t = world(p, 12)
    lens = [451]  # queries at 447 .. 450: a chunk's last position, then the next chunk
    bury(t, p, lens)
    clean = [x.cpu().numpy() if i == 2 else host(x) for i, x in enumerate(run_decode(p, t, lens))]
    t["v"][t["table"][0, 7], 1, 5, 1] = 0x7f  # token 449, head 1, dim 5
    t["k"][t["table"][0, 7], 0, 2, 7] = 0x7f  # token 450, head 0
    out, lse, idx, wt = (host(x) for x in run_decode(p, t, lens))
    keep = np.ones(out.shape, bool)
    keep[:, 4:, 2:, 5] = False
    keep[:, :4, 3] = False
    assert np.isfinite(clean[0]).all() and np.array_equal(out[keep], clean[0][keep])
    assert np.isnan(out[:, 4:, 2:, 5]).all() and np.isnan(out[:, :4, 3]).all()
    assert np.isnan(lse[0, :4, 3]).all() and np.isfinite(lse[0, 4:]).all()


def test_decode_masked_candidates():
    """Biases of -inf: such chunks are chosen last and weigh nothing; with all of them masked the window is all."""
    hils = hils_()
    p = hils.Params(B=2, Hq=4, Hkv=1, N=1, L=1024, d=64, topk=8, window=64, scale=0.125)
    t = world(p, 14)
    t["bias"][t["table"][0, ::2]] = -np.inf
    t["bias"][t["table"][1]] = -np.inf
    lens = [1024, 1020]
    ref = Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"], bias=t["bias"], seqlens=lens)
    out, lse, idx, wt = got = run_decode(p, t, lens, bias=True)
    check_decode(p, got, ref)
    assert (wt[1, 0, 0, :8] == 0).all()


def test_decode_pages_out_of_range_are_clamped():
    hils = hils_()
    p = hils.Params(B=2, Hq=4, Hkv=2, N=1, L=512, d=64, topk=3, window=64, scale=0.125)
    t = world(p, 15)
    ref_t = dict(t, table=t["table"].copy())
    t["table"][0, 2], t["table"][0, 7], t["table"][1, 6:] = 10 ** 9, -4, -1
    ref_t["table"][0, 2], ref_t["table"][0, 7] = len(t["k"]) - 1, 0
    lens = [512, 380]
    ref = Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], ref_t["table"], seqlens=lens)
    check_decode(p, run_decode(p, t, lens), ref)


def test_decode_any_scale():
    """The attention takes any positive scale, not only the powers of two that append writes."""
    hils = hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, N=1, L=640, d=128, topk=20, window=128, dtype="f32")
    t = world(p, 16)
    t["scale"] = (0.01 + 0.02 * np.random.default_rng(1).random(t["scale"].shape)).astype(np.float32)
    ref = Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"])
    check_decode(p, run_decode(p, t), ref)


APPEND = {
    "one_token": (dict(B=4, Hq=2, Hkv=2, N=1, L=256, d=128), [1, 64, 65, 256], None),
    "one_token_d64_f32": (dict(B=3, Hq=2, Hkv=2, N=1, L=256, d=64, dtype="f32"), [100, 128, 2], None),
    "drafts": (dict(B=3, Hq=3, Hkv=3, N=5, L=256, d=64), [5, 66, 133], [5, 3, 0]),
    "prompt": (dict(B=2, Hq=2, Hkv=2, N=256, L=256, d=128), None, None),
    "ragged": (dict(B=5, Hq=1, Hkv=1, N=130, L=384, d=128), [130, 384, 200, 64, 90], [130, 129, 1, 64, 27]),
    "ragged_d64": (dict(B=5, Hq=1, Hkv=1, N=200, L=384, d=64), [200, 384, 200, 64, 301], [200, 129, 61, 63, 140]),
    "ragged_f32": (dict(B=4, Hq=2, Hkv=2, N=131, L=384, d=128, dtype="f32"), [131, 384, 200, 65], [131, 128, 67, 2]),
    # lengths and counts out of range are clamped: more new tokens than tokens, a negative count, a length past L
    "clamped": (dict(B=4, Hq=1, Hkv=1, N=70, L=128, d=64), [40, 128, 1000, -7], [90, -3, 70, 5]),
}


def append_inputs(p, seed):
    r = np.random.default_rng(seed)
    shape = (p.B, p.Hkv, p.N, p.d)
    new = [rounded((r.standard_normal(shape) * 2.0 ** r.uniform(-6, 6, (p.B, p.Hkv, 1, 1))).astype(np.float32), p.dtype)
           for _ in range(2)]
    nc = p.L // 64
    P = p.B * nc + 2
    pools = [r.integers(0, 256, s).astype(np.uint8) for s in ((P, p.Hkv, 64, p.d), (P, p.Hkv, p.d, 64))]
    for x in pools:
        x[(x & 0x7f) == 0x7f] = 0x11  # no NaN in what the pages hold
    scale = 2.0 ** r.integers(-9, -3, (P, p.Hkv, 2)).astype(np.float32)
    return new, pools, scale, r.permutation(P)[:p.B * nc].reshape(p.B, nc).astype(np.int32)


def run_append(p, new, pools, scale, table, lens=None, counts=None):
    hils = hils_()
    k, v, s = f8(pools[0]), f8(pools[1]), dev(scale)
    i32 = [None if x is None else dev(np.int32(x)) for x in (lens, counts)]
    hils.hils_q8_append(p, dev(new[0], p.torch_dtype), dev(new[1], p.torch_dtype), k, v, s, dev(table), *i32)
    torch.cuda.synchronize()
    return codes(k), codes(v), s.cpu().numpy()


def same_codes(a, b):
    nan = ((a & 0x7f) == 0x7f) & ((b & 0x7f) == 0x7f)
    return (nan | (a == b)).all()


@pytest.mark.parametrize("name", APPEND)
def test_append(name):
    hils = hils_()
    kw, lens, counts = APPEND[name]
    p = hils.Params(topk=1, window=64, **kw)
    new, pools, scale, table = append_inputs(p, len(name))
    ref = Q.append(p, *new, *pools, scale, table, lens, counts)
    got = run_append(p, new, pools, scale, table, lens, counts)
    assert np.array_equal(got[2], ref[2])
    assert same_codes(got[0], ref[0]) and same_codes(got[1], ref[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,start", [(64, 0), (3, 0), (3, 30)])
def test_append_extreme_values(dtype, n, start):
    """Zeros, a maximum on a scale's border, the type's largest, subnormal and non-finite values."""
    hils = hils_()
    p = hils.Params(B=7, Hq=1, Hkv=1, N=n, L=64 * (2 if start else 1), d=64, topk=1, window=64, dtype=dtype)
    new, pools, scale, table = append_inputs(p, 3)
    top = float(torch.finfo(p.torch_dtype).max)
    for x in new:
        x[0] = 0
        x[1, 0, 0, 0], x[1, 0, 1, 1] = 448 * 2.0 ** 3, -448 * 2.0 ** 3
        x[1] = np.clip(x[1], -448 * 8, 448 * 8)
        x[2, 0, 1, 5] = rounded(np.float32([448 * 2.0 ** 3 * (1 + 2.0 ** -7)]), dtype)[0]
        x[3, 0, 2, 7] = top
        x[4] = 2.0 ** -126
        x[5, 0, 0, :3] = np.inf, -np.inf, np.nan
        x[6] = np.nan
    lens = [start + n] * 7
    ref = Q.append(p, *new, *pools, scale, table, lens)
    got = run_append(p, new, pools, scale, table, lens)
    assert np.array_equal(got[2], ref[2])
    assert same_codes(got[0], ref[0]) and same_codes(got[1], ref[1])


def test_writes_without_a_page_are_dropped():
    """Table entries outside the pool: nothing is written for those chunks, to no page; the others as ever."""
    hils = hils_()
    p = hils.Params(B=3, Hq=2, Hkv=2, N=200, L=256, d=64, topk=1, window=64, flags=0)
    new, pools, scale, table = append_inputs(p, 21)
    lens, counts = [256, 201, 64], [200, 200, 64]
    lone = table.copy()  # the same call with pages of their own for the chunks without one
    n = len(pools[0])
    for i, (b, c, bad) in enumerate(((0, 1, -1), (0, 3, n), (1, 0, -2 ** 31), (1, 3, 2 ** 31 - 1))):
        table[b, c], lone[b, c] = bad, n + i
    wide = [np.concatenate([x, np.zeros((4,) + x.shape[1:], x.dtype)]) for x in (*pools, scale)]
    ref = Q.append(p, *new, *wide, lone, lens, counts)
    got = run_append(p, new, pools, scale, table, lens, counts)
    assert np.array_equal(got[2], ref[2][:n])
    assert same_codes(got[0], ref[0][:n]) and same_codes(got[1], ref[1][:n])
    lmk, bias = np.full((n, 2, 64), 0x5a, np.uint8), np.full((n, 2), 7, np.float32)
    tl, tb = f8(lmk), dev(bias)
    lq = torch.zeros((3, 2, 4, 64), dtype=torch.bfloat16, device="cuda")
    hils.hils_q8_landmark_fwd(p, lq, f8(got[0]), dev(got[2]), dev(table), tl, tb, dev(np.int32(lens)), dev(np.int32(counts)))
    written = [table[b, c] for b, c in ((0, 0), (0, 2), (1, 1), (1, 2), (2, 0))]
    keep = [i for i in range(n) if i not in written]
    assert (codes(tl)[keep] == 0x5a).all() and (tb.cpu().numpy()[keep] == 7).all()
    assert (np.abs(tb.cpu().numpy()[written] - np.log(64)) < 1e-4).all()


LANDMARK = {
    "step": (dict(B=4, Hq=8, Hkv=2, N=1, L=256, d=128), [64, 63, 256, 129], None, False),
    "prompt": (dict(B=2, Hq=8, Hkv=1, N=300, L=512, d=64), [300, 500], [300, 130], False),
    "shared_query": (dict(B=2, Hq=4, Hkv=2, N=64, L=256, d=128), None, [64, 0], True),
    "f32": (dict(B=2, Hq=2, Hkv=2, N=129, L=256, d=128, dtype="f32"), [256, 192], None, False),
    "f32_shared_heads": (dict(B=1, Hq=8, Hkv=2, Hl=2, N=128, L=256, d=64, dtype="f32"), [200], None, False),
    "shared_heads": (dict(B=2, Hq=8, Hkv=1, Hl=1, N=200, L=256, d=128), [256, 64], [200, 64], True),
}


@pytest.mark.parametrize("name", LANDMARK)
def test_landmark(name):
    hils = hils_()
    kw, lens, counts, shared = LANDMARK[name]
    p = hils.Params(topk=1, window=64, flags=hils.HILS_FLAG_SHARED_LMK_QUERY if shared else 0, **kw)
    t, Hl = world(p, 21), p.Hl or p.Hq
    r = np.random.default_rng(2)
    lq = rounded(r.standard_normal((Hl, p.d) if shared else (p.B, Hl, (p.N + 63) // 64, p.d)).astype(np.float32), p.dtype)
    ref = Q.landmark(p, lq, t["k"], t["scale"], t["table"], lens, counts, shared)
    lm, bias = f8(t["lmk"]), dev(t["bias"])
    i32 = [None if x is None else dev(np.int32(x)) for x in (lens, counts)]
    hils.hils_q8_landmark_fwd(p, dev(lq, p.torch_dtype), f8(t["k"]), dev(t["scale"]), dev(t["table"]), lm, bias, *i32)
    torch.cuda.synchronize()
    lm, bias = codes(lm), bias.cpu().numpy()
    assert ref
    for page, (rows, b) in ref.items():
        d = np.abs(Q.VALUE[lm[page]] - rows)
        assert (d <= np.maximum(2.0 ** -4 * np.abs(rows), 2.0 ** -10) + 1e-4 * 448).all()
        assert np.abs(bias[page] - b).max() <= 1e-4
    others = [i for i in range(len(t["k"])) if i not in ref]
    assert np.array_equal(lm[others], t["lmk"][others]) and np.array_equal(bias[others], t["bias"][others])


def test_landmark_of_equal_keys_at_the_largest_value():
    """A chunk of equal keys is its own landmark; sums of weights may pass 1 by roundings, 448 does not overflow."""
    hils = hils_()
    p = hils.Params(B=1, Hq=4, Hkv=1, N=64, L=64, d=64, topk=1, window=64)
    k = np.full((1, 1, 64, 64), 0x7e, np.uint8)
    k[..., ::2] = 0xfe
    lm, bias = torch.zeros((1, 4, 64), dtype=torch.uint8, device="cuda").view(F8), torch.zeros((1, 4), device="cuda")
    lq = torch.randn((1, 4, 1, 64), generator=torch.Generator().manual_seed(1)).cuda().bfloat16()
    hils.hils_q8_landmark_fwd(p, lq, f8(k), torch.full((1, 1, 2), 2.0 ** -8, device="cuda"),
                              torch.zeros((1, 1), dtype=torch.int32, device="cuda"), lm, bias)
    assert (codes(lm) == k[:, :, 0]).all() and np.abs(host(bias) - np.log(64)).max() <= 1e-5


EVICT = {
    "steps": (dict(B=3, Hq=8, Hkv=4, N=1, L=64 * 40, d=64, topk=6, window=200), [2560, 700, 64], 10, 1, None),
    "drafts": (dict(B=2, Hq=8, Hkv=2, N=5, L=64 * 40, d=64, topk=6, window=64), [2400, 2001], 3, 4, None),
    # sequences that hold nothing, or less than the call's new tokens
    "short_of_drafts": (dict(B=3, Hq=8, Hkv=2, N=200, L=64 * 40, d=64, topk=6, window=64), [0, 150, 2001], 1, 0, None),
    "at_most_7": (dict(B=2, Hq=2, Hkv=1, N=1, L=64 * 50, d=64, topk=4, window=128), [3200, 3000], 0, 2, 7),
    "none": (dict(B=2, Hq=2, Hkv=1, N=1, L=64 * 50, d=64, topk=4, window=128), [3200, 1], 1000, 0, None),
    "zero_most": (dict(B=1, Hq=2, Hkv=1, N=1, L=64 * 50, d=64, topk=4, window=128), None, 1, 0, 0),
    "sinks_past_the_end": (dict(B=1, Hq=2, Hkv=1, N=1, L=64 * 9, d=64, topk=4, window=128), [500], 0, 100, None),
    # more chunks than the totals of which fit in LDS
    "long": (dict(B=1, Hq=4, Hkv=2, N=2, L=64 * 25001, d=64, topk=16, window=512), None, 9000, 3, None),
    "tiles": (dict(B=2, Hq=4, Hkv=2, N=2, L=64 * 5001, d=64, topk=64, window=4032), [64 * 5001 - 5, 64 * 3500], 1800, 3, None),
}


def evict_inputs(p, seed, lens, spread):
    r = np.random.default_rng(seed)
    nc = p.L // 64
    acc = r.integers(0, spread, (p.B, nc)).astype(np.float32) / 16
    table = r.permutation(p.B * nc).reshape(p.B, nc).astype(np.int32)
    wt = r.integers(0, 64, (p.B, p.Hkv, p.N, p.topk + Q.pieces(p.window))).astype(np.float32) / 64
    idx = np.full((p.B, p.Hkv, p.N, p.topk), -1, np.int32)
    for b in range(p.B):
        for n in range(p.N):
            c = Q.n_candidates((p.L if lens is None else min(max(lens[b], p.N), p.L)) - p.N + n, p.window)
            for g in range(p.Hkv):
                m = min(p.topk, c)
                idx[b, g, n, :m] = np.sort(r.choice(c, m, replace=False)) if c else []
    return acc, table, wt, idx


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("name", EVICT)
def test_evict(name, ties):
    hils = hils_()
    kw, lens, budget, sink, most = EVICT[name]
    p = hils.Params(**kw)
    acc, table, wt, idx = evict_inputs(p, len(name), lens, 3 if ties else 1 << 16)
    if ties:
        wt[:] = 0
    idx[0, 0, 0, -1] = -7  # entries that do not count
    idx[0, 0, 0, 0] = 1 << 29 if ties else idx[0, 0, 0, 0]
    cap = p.L // 64 if most is None else most
    ref = Q.evict(p, acc, table, lens, budget, sink, cap, wt, idx)
    args = dict(budget=budget, sink=sink, max_evict=most, weights=dev(wt), idx=dev(idx))
    i32 = None if lens is None else dev(np.int32(lens))
    a, tb = dev(acc), dev(table)
    got = hils.hils_cache_evict(p, a, tb, i32, **args)
    for x, y in zip(got, ref):
        assert np.array_equal(x.cpu().numpy().astype(np.float64), np.asarray(y, np.float64))
    assert np.array_equal(a.cpu().numpy(), acc) and np.array_equal(tb.cpu().numpy(), table)
    # in place, and once more: nothing is left to drop but what max_evict held back
    s = dev(np.int32([p.L] * p.B if lens is None else lens))
    got = hils.hils_cache_evict(p, a, tb, s, acc_out=a, table_out=tb, seqlens_out=s, **args)
    for x, y in zip(got, ref):
        assert np.array_equal(x.cpu().numpy().astype(np.float64), np.asarray(y, np.float64))
    ref2 = Q.evict(p, ref[0], ref[1], ref[2], budget, sink, cap)
    got = hils.hils_cache_evict(p, a, tb, s, budget=budget, sink=sink, max_evict=most)
    for x, y in zip(got, ref2):
        assert np.array_equal(x.cpu().numpy().astype(np.float64), np.asarray(y, np.float64))


def test_evict_special_totals():
    """-0 is 0 (the lower index goes), infinities order as numbers, NaN totals stay."""
    hils = hils_()
    p = hils.Params(B=1, Hq=1, Hkv=1, N=1, L=64 * 9, d=64, topk=1, window=64)
    acc = np.float32([[0.0, -0.0, np.nan, -np.inf, 5, np.inf, 1, 7, 9]])  # candidates 0 .. 7
    table = np.arange(9, dtype=np.int32)[None] + 20
    for budget, gone in ((7, [3]), (6, [0, 3]), (5, [0, 1, 3]), (1, [0, 1, 3, 4, 5, 6, 7])):
        got = hils.hils_cache_evict(p, dev(acc), dev(table), budget=budget)
        assert got[3][0, :len(gone)].tolist() == [20 + c for c in gone] and got[4].tolist() == [len(gone)]


def test_evict_negative_nan():
    """A NaN total stays whatever its sign bit."""
    hils = hils_()
    p = hils.Params(B=1, Hq=1, Hkv=1, N=1, L=64 * 9, d=64, topk=1, window=64)
    acc = np.arange(9, dtype=np.float32)[None]
    acc.view(np.uint32)[0, 4] = 0xffc00000
    got = hils.hils_cache_evict(p, dev(acc), torch.arange(9, dtype=torch.int32, device="cuda")[None], budget=1)
    assert got[3][0, :7].tolist() == [0, 1, 2, 3, 5, 6, 7]


@pytest.mark.parametrize("n", [1, 3])
def test_decode_short_sequences_in_a_large_cache(n):
    """Slices enough for the whole workgroup's selection, but no more than 64 survivors in any row: it
    has nothing to narrow down.  The pages past the sequences' ends are one page of NaN."""
    hils = hils_()
    kw = dict(B=12, Hq=16, Hkv=8, N=n, d=64, topk=64, window=128, scale=0.125)
    lens = [130 + 150 * b for b in range(12)]
    small, p = hils.Params(L=2048, **kw), hils.Params(L=64 * 1500, **kw)
    t = world(small, 91 + n)
    bury(t, small, lens)
    ref = Q.decode(small, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"], seqlens=np.int32(lens))
    unused = (set(range(len(t["k"]))) - set(t["table"].ravel().tolist())).pop()
    table = np.full((p.B, p.L // 64), unused, np.int32)
    table[:, :32] = t["table"]
    t["table"] = table
    check_decode(p, run_decode(p, t, lens), ref)


@pytest.mark.parametrize("n", [1, 3])
def test_decode_ties_everywhere(n):
    """Equal scores of every candidate: the lowest chunks are chosen, however many survivors tie."""
    hils = hils_()
    p = hils.Params(B=1, Hq=2, Hkv=2, N=n, L=64 * 1500, d=64, topk=60, window=128, scale=0.125)
    t = world(p, 31)
    t["lmk"][:] = 0
    ref = Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"])
    got = run_decode(p, t)
    check_decode(p, got, ref)
    assert got[2][0, 0, 0].tolist() == list(range(60))


def odd(t):
    """The same values one element past an allocation's start."""
    return torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].view(t.shape)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 3])
def test_views_at_odd_offsets(dtype, n):
    """Queries, new rows, outputs and small arrays need no more than their elements' alignment."""
    hils = hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, N=n, L=1024, d=64, topk=5, window=100, scale=0.125, dtype=dtype)
    t, dt, i32 = world(p, 41), p.torch_dtype, torch.int32
    lens = odd(dev(np.int32([1024, 600])))
    q, qr = dev(t["q"], dt), dev(t["q_route"], dt)
    pools = lambda: (f8(t["k"]), f8(t["v"]), dev(t["scale"]))  # noqa: E731
    k, v, sc = pools()
    args = (f8(t["lmk"]), odd(dev(t["table"])))
    want = hils.hils_decode_q8_fwd(p, q, k, v, sc, *args, bias_pages=odd(dev(t["bias"])), q_route=qr, seqlens=lens)
    outs = [odd(torch.empty_like(x)) for x in want]
    got = hils.hils_decode_q8_fwd(p, odd(q), k, v, sc, *args, bias_pages=odd(dev(t["bias"])), q_route=odd(qr), seqlens=lens,
                                  out=outs[0], lse=outs[1], idx=outs[2], weights=outs[3])
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    new = dev(rounded(np.random.default_rng(1).standard_normal((2, 2, 70 * n, 64)).astype(np.float32), dtype), dt)
    pa = hils.Params(B=2, Hq=8, Hkv=2, N=70 * n, L=1024, d=64, topk=5, window=100, dtype=dtype)
    a, b = pools(), pools()
    hils.hils_q8_append(pa, new, new, *a, dev(t["table"]), lens)
    hils.hils_q8_append(pa, odd(new), odd(new), *b, odd(dev(t["table"])), lens)
    assert all(np.array_equal(codes(x), codes(y)) for x, y in zip(a[:2], b[:2])) and torch.equal(a[2], b[2])
    lq = dev(rounded(np.random.default_rng(2).standard_normal((2, 8, (70 * n + 63) // 64, 64)).astype(np.float32), dtype), dt)
    la, lb = [(f8(t["lmk"]), dev(t["bias"])) for _ in range(2)]
    hils.hils_q8_landmark_fwd(pa, lq, a[0], a[2], dev(t["table"]), *la, lens)
    hils.hils_q8_landmark_fwd(pa, odd(lq), a[0], a[2], dev(t["table"]), lb[0], lb[1], lens)
    assert np.array_equal(codes(la[0]), codes(lb[0])) and torch.equal(la[1], lb[1])


def test_pools_past_4_gib():
    """Pages whose bytes lie past 2^32: a small cache at the end of large pools."""
    hils = hils_()
    p = hils.Params(B=2, Hq=4, Hkv=1, N=1, L=512, d=128, topk=3, window=64, scale=0.125)
    t = world(p, 43)
    n, P = len(t["k"]), 600000
    k, v = (torch.zeros((P, 1) + s, dtype=torch.uint8, device="cuda").view(F8) for s in ((64, 128), (128, 64)))
    lm, sc, table = torch.zeros((P, 4, 128), dtype=torch.uint8, device="cuda").view(F8), torch.ones((P, 1, 2), device="cuda"), t["table"] + P - n
    for big, small in ((k, t["k"]), (v, t["v"]), (lm, t["lmk"])):
        big.view(torch.uint8)[P - n:] = dev(small)
    sc[P - n:] = dev(t["scale"])
    ref = Q.decode(p, t["q"], t["k"], t["v"], t["scale"], t["lmk"], t["table"])
    check_decode(p, hils.hils_decode_q8_fwd(p, dev(t["q"], p.torch_dtype), k, v, sc, lm, dev(table)), ref)
    new = rounded(np.random.default_rng(1).standard_normal((2, 1, 1, 128)).astype(np.float32), "bf16")
    want = Q.append(p, new, new, t["k"], t["v"], t["scale"], t["table"], [400, 512])
    hils.hils_q8_append(p, dev(new, p.torch_dtype), dev(new, p.torch_dtype), k, v, sc, dev(table), dev(np.int32([400, 512])))
    assert same_codes(codes(k[P - n:]), want[0]) and same_codes(codes(v[P - n:]), want[1])
    assert np.array_equal(sc[P - n:].cpu().numpy(), want[2]) and not codes(k[:P - n]).any()


def test_refusals_of_tensors():
    """What the binding says of tensors that a call cannot take."""
    hils = hils_()
    p = hils.Params(B=2, Hq=4, Hkv=2, N=2, L=256, d=64, topk=2, window=64)
    t = world(p, 5)
    good = dict(q=dev(t["q"], torch.bfloat16), k_pages=f8(t["k"]), v_pages=f8(t["v"]), kv_scale=dev(t["scale"]),
                lmk_pages=f8(t["lmk"]), block_table=dev(t["table"]))
    hils.hils_decode_q8_fwd(p, **good)
    for name, bad, what in (("q", good["q"].float(), "dtype"), ("q", good["q"].transpose(1, 2), "contiguous"),
                            ("k_pages", good["v_pages"][:, :, :32], "contiguous"), ("v_pages", good["k_pages"].view(torch.uint8), "dtype"),
                            ("kv_scale", good["kv_scale"][..., 0].contiguous(), "shape"), ("block_table", good["block_table"].long(), "dtype"),
                            ("lmk_pages", good["lmk_pages"].cpu(), "GPU tensor"), ("q", good["q"].cpu(), "GPU tensor")):
        with pytest.raises(ValueError, match=what):
            hils.hils_decode_q8_fwd(p, **{**good, name: bad})
    with pytest.raises(hils.HilsError, match="workspace"):
        hils.hils_decode_q8_fwd(p, **good, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="needs idx"):
        hils.hils_decode_q8_fwd(hils.Params(B=2, Hq=4, Hkv=2, N=2, L=256, d=64, topk=2, window=64, flags=hils.HILS_FLAG_GIVEN_IDX), **good)
    with pytest.raises(ValueError, match="shape"):
        hils.hils_cache_evict(p, torch.zeros((2, 5), device="cuda"), good["block_table"])
    with pytest.raises(hils.HilsError, match=">= 0"):
        hils.hils_cache_evict(p, torch.zeros((2, 4), device="cuda"), good["block_table"], budget=-1)


def test_a_sequence_lives():
    """A prompt in two pieces, decode steps with drafts, eviction, more steps: every output against the
    oracle's own cache, on another stream, the steps captured into a graph and replayed between eager work."""
    hils = hils_()
    B, Hq, Hkv, d, L = 2, 8, 2, 64, 1024
    base = dict(B=B, Hq=Hq, Hkv=Hkv, L=L, d=d, topk=4, window=64, scale=0.125)
    r = np.random.default_rng(77)
    nc = L // 64
    P = B * nc + 2
    table = r.permutation(P)[:B * nc].reshape(B, nc).astype(np.int32)
    kc, vc = np.full((P, Hkv, 64, d), 0x7f, np.uint8), np.full((P, Hkv, d, 64), 0x7f, np.uint8)
    sc, lmk, bias = np.zeros((P, Hkv, 2), np.float32), np.full((P, Hq, d), 0x7f, np.uint8), np.zeros((P, Hq), np.float32)
    acc, lens = np.zeros((B, nc), np.float32), np.zeros(B, np.int32)
    g = dict(k=f8(kc), v=f8(vc), sc=dev(sc), lmk=f8(lmk), bias=dev(bias), table=dev(table), acc=dev(acc), lens=dev(lens))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    ws = torch.empty(hils.hils_workspace_size(hils.Params(N=3, **base), hils.HILS_OP_DECODE_Q8), dtype=torch.uint8, device="cuda")

    def one(n, counts, decode, graph):
        nonlocal kc, vc, sc
        lens[:] = lens + counts
        p = hils.Params(N=n, **base)
        pl = hils.Params(N=n, flags=hils.HILS_FLAG_SHARED_LMK_QUERY, **base)
        kn, vn = (rounded(r.standard_normal((B, Hkv, n, d)).astype(np.float32) * 2.0 ** r.integers(-1, 2), "bf16") for _ in range(2))
        lq = rounded(r.standard_normal((Hq, d)).astype(np.float32), "bf16")
        q = np.clip(np.round(r.standard_normal((B, Hq, n, d)) * 16) / 16, -4, 4).astype(np.float32)
        kc, vc, sc = Q.append(p, kn, vn, kc, vc, sc, table, lens, counts)
        tk, tv, tq, tl, tc = dev(kn, torch.bfloat16), dev(vn, torch.bfloat16), dev(q, torch.bfloat16), dev(lq, torch.bfloat16), dev(np.int32(counts))
        with torch.cuda.stream(stream):
            g["lens"] += tc
            torch.cuda.current_stream().synchronize()

            def work():
                hils.hils_q8_append(p, tk, tv, g["k"], g["v"], g["sc"], g["table"], g["lens"], tc)
                hils.hils_q8_landmark_fwd(pl, tl, g["k"], g["sc"], g["table"], g["lmk"], g["bias"], g["lens"], tc)
                return hils.hils_decode_q8_fwd(p, tq, g["k"], g["v"], g["sc"], g["lmk"], g["table"], g["bias"],
                                               seqlens=g["lens"], workspace=ws) if decode else None

            got = work()  # (a second pass on the same tokens changes nothing)
            if graph:
                cg = torch.cuda.CUDAGraph()
                with torch.cuda.graph(cg, stream=stream):
                    replayed = work()
                for _ in range(3):
                    for x in replayed:
                        x.zero_()
                    cg.replay()
                    torch.cuda.current_stream().synchronize()
                    eager = work()
                    torch.cuda.current_stream().synchronize()
                    assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(got, replayed, eager))
        stream.synchronize()
        assert same_codes(codes(g["k"]), kc) and same_codes(codes(g["v"]), vc) and np.array_equal(g["sc"].cpu().numpy(), sc)
        for page, (rows, bb) in Q.landmark(pl, lq, kc, sc, table, lens, counts, True).items():
            assert (np.abs(Q.VALUE[codes(g["lmk"])[page]] - rows) <= np.maximum(2.0 ** -4 * np.abs(rows), 2.0 ** -10) + 0.05).all()
            lmk[page], bias[page] = codes(g["lmk"])[page], g["bias"].cpu().numpy()[page]
        if not decode:
            return None
        sel = got[2].cpu().numpy()  # (real landmarks: held to the oracle on the selection that was made)
        ref = Q.decode(hils.Params(N=n, flags=hils.HILS_FLAG_GIVEN_IDX, **base), q, kc, vc, sc, lmk, table, bias=bias, seqlens=lens, given=sel)
        check_decode(p, got, ref)
        assert ((sel >= 0).sum(-1) == np.minimum(4, [[[Q.n_candidates(lens[b] - n + i, 64) for i in range(n)]] * Hkv for b in range(B)])).all()
        return p, got

    one(300, np.int32([300, 171]), False, False)
    one(300, np.int32([299, 300]), False, False)
    for step in range(4):
        p, got = one(3, np.int32([3, 3]), True, step == 1)
        budget = 5 if step == 2 else 100
        want = Q.evict(p, acc, table, lens, budget, 1, nc, host(got[3]), got[2].cpu().numpy())
        with torch.cuda.stream(stream):
            res = hils.hils_cache_evict(p, g["acc"], g["table"], g["lens"], budget=budget, sink=1, weights=got[3], idx=got[2],
                                        acc_out=g["acc"], table_out=g["table"], seqlens_out=g["lens"])
        stream.synchronize()
        assert np.abs(host(res[0]) - want[0]).max() <= 1e-5
        assert all(np.array_equal(x.cpu().numpy(), y) for x, y in zip(res[1:], want[1:]))
        acc[:], table[:], lens[:] = g["acc"].cpu().numpy(), want[1], want[2]
        table[table < 0] = 0
        g["table"].clamp_(min=0)
    assert lens[0] < 620
