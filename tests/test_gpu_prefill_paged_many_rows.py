"""hils_prefill_paged_fwd where a call has many rows: windows by k_pp_local, chunks counted in LDS, rows in segments.

Bounds as in test_gpu_prefill_paged.py.  The records' float16 (half a step: 2^-11 of an element) takes its share of
the 2^-8 of every weight, of which a sum of dozens of weights uses a part only."""
import numpy as np
import pytest
import torch

from tests.gpu_helpers import kernels_of
from tests.test_gpu_prefill_paged import World, hils_

pytestmark = pytest.mark.gpu

# (heads x rows x (K + pieces of a window) above the count that takes the windows as work items)
SHAPES = {
    "g4": dict(B=2, Hq=8, Hkv=2, N=500, L=2560, d=128, topk=32, window=700),
    "g1": dict(B=2, Hq=8, Hkv=8, N=500, L=2560, d=64, topk=32, window=700),
    "g2": dict(B=2, Hq=8, Hkv=4, N=500, L=2560, d=128, topk=32, window=700),
    "g8": dict(B=2, Hq=8, Hkv=1, N=500, L=2560, d=64, topk=32, window=700),
    "g8_d128": dict(B=2, Hq=16, Hkv=2, N=250, L=2560, d=128, topk=32, window=700),
}
SHAPES = {f"{n}_{t}": dict(kw, dtype=t) for n, kw in SHAPES.items() for t in ("bf16", "f32")}


def world(kw, seed, **opt):
    w = World(hils_().Params(**kw), [2533, 777], [kw["N"], 233], seed, **opt)
    return w


def some(w):
    return [(b, n) for b in range(2) for n in sorted({0, 1, 15, 16, 63, 64, 100, 127, 128, w.fresh[b] // 2, w.fresh[b] - 1})]


@pytest.mark.parametrize("name", SHAPES)
def test_parity(name):
    w = world(SHAPES[name], sum(map(ord, name)), bias=True, route=name.startswith("g4"))
    got = []
    assert {"k_pp_local", "k_pp_select"} <= kernels_of(lambda: got.extend(w.run()))
    w.check(got, rows=some(w))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windows_over_everything(dtype):
    """No candidates: rows see all that is before them, some of it through an earlier call's pages."""
    kw = dict(B=2, Hq=8, Hkv=2, N=700, L=2560, d=64, topk=32, window=2 ** 31 - 1, dtype=dtype)
    w = world(kw, 9)
    got = w.run()
    assert (got[2][0] == -1).all() and (got[2][1, :, :233] == -1).all()
    w.check(got, rows=some(w))


# enough workgroups that some of sequence 1's take the records first, the window after them
ORDERS = {t: dict(B=2, Hq=32, Hkv=4, N=1100, L=2560, d=64, topk=4, window=100, dtype=t) for t in ("bf16", "f32")}


def two_orders(dtype, **opt):
    return World(hils_().Params(**ORDERS[dtype]), [2500, 2533], [1100, 1090], 31, **opt)


ORDER_ROWS = [(b, n) for b in range(2) for n in (0, 17, 255, 400, 640, 801, 1000, 1089)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_records_before_and_after_the_window(dtype):
    w = two_orders(dtype, bias=True)
    w.check(w.run(), rows=ORDER_ROWS)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_of_later_tokens_in_either_order(dtype):
    w = two_orders(dtype)
    clean = w.run()
    for row in (101, 700):
        at = 2533 - 1090 + row
        w.v[w.table[1, at // 64], 0, at % 64, 3] = np.inf
    got = w.run()
    bound = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -20  # (as above)
    assert ((got[0][1, :, :101] - clean[0][1, :, :101]).float().abs() <= bound * 4).all()
    assert torch.isfinite(got[0][1, :8, 300:700][..., :3].float()).all()
    assert not torch.isfinite(got[0][1, :8, [101, 700], 3]).any()
    assert torch.equal(got[0][1, 8:], clean[0][1, 8:])


@pytest.mark.parametrize("case", ["few", "few_f32", "bf16", "f32"])
def test_biases_of_the_lowest_value(case):
    """Every chunk hidden from all or half of the heads by a bias of float32's lowest value: no weight, as -inf."""
    if case in ORDERS:
        w, rows = two_orders(case, bias=True), ORDER_ROWS
    else:
        kw = dict(SHAPES["g4_f32" if case == "few_f32" else "g4_bf16"], N=40)
        w, rows = World(hils_().Params(**kw), [2533, 777], [40, 33], 7, bias=True), [(0, 0), (0, 39), (1, 0), (1, 32)]
    w.bias[:, ::2] = -np.inf
    w.bias[w.table[1, 3:w.len[1] // 64]] = -np.inf
    w.check(w.run(), rows=rows)
    w.bias[np.isneginf(w.bias)] = np.finfo(np.float32).min
    got = w.run()
    w.check(got, rows=rows)
    for b in range(2):
        assert all(torch.isfinite(x[b, :, :w.fresh[b]].float()).all() for x in got[:2])


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("name", SHAPES)
def test_later_tokens_do_not_reach_earlier_rows(name, value):
    w = world(SHAPES[name], 5)
    clean = w.run()
    row = 177  # of sequence 0, at position `at`
    at = 2533 - w.fresh[0] + row
    pg, key = w.table[0, at // 64], at % 64
    w.v[pg, 0, key, 3] = value
    if np.isnan(value):
        w.k[pg, 0, key, 5] = value
    got = w.run()
    G = w.p.Hq // w.p.Hkv
    bound = 2.0 ** -7 if w.p.dtype == "bf16" else 2.0 ** -20  # (added in another order: twice the error of a result)
    assert torch.equal(got[2][:, :, :row], clean[2][:, :, :row])
    assert ((got[0][0, :, :row] - clean[0][0, :, :row]).float().abs() <= bound * 4).all()
    assert not torch.isfinite(got[0][0, :G, row, 3]).any()
    if G < w.p.Hq:
        assert torch.equal(got[0][0, G:], clean[0][0, G:])  # the other KV groups
    assert all(torch.equal(x[1], y[1]) for x, y in zip(got, clean))  # the other sequence


@pytest.mark.parametrize("name", SHAPES)
def test_given_selection_and_segments(name):
    """A call's own selection given to it, and its rows cut into segments: the same bits; other entries: the formula's."""
    hils = hils_()
    w = world(SHAPES[name], 6, bias=True)
    own = w.run()
    before = hils.hils_prefill_record_cap(1)  # 128 rows of records
    try:
        cut = w.run()
    finally:
        hils.hils_prefill_record_cap(before)
    assert all(torch.equal(x, y) for x, y in zip(own, cut))
    given = World(hils.Params(**SHAPES[name], flags=hils.HILS_FLAG_GIVEN_IDX), [2533, 777], w.new, 6, bias=True)
    got = given.run(idx=own[2].cpu().numpy())
    assert all(torch.equal(x, y) for x, y in zip(own, got))
    # every third of a row's entries left, at odd rows none
    idx = own[2].cpu().numpy()
    few = np.full_like(idx, -1)
    few[..., ::2, :11] = idx[..., ::2, ::3]
    got = given.run(idx=few)
    given.check(got, rows=some(w), given=few)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replays_of_a_captured_call(dtype):
    hils = hils_()
    kw = SHAPES["g4_" + dtype]
    w, w2 = world(kw, 21), world(kw, 22)
    refs = [w.run(), w2.run()]
    a, b = w.args(), w2.args()
    assert all(a[n].shape == b[n].shape for n in ("k_pages", "v_pages", "lmk_pages"))
    ws = torch.empty(hils.hils_workspace_size(w.p, hils.HILS_OP_PREFILL_PAGED), dtype=torch.uint8, device="cuda").random_(256)
    outs = [torch.empty_like(x) for x in refs[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call = lambda: hils.hils_prefill_paged_fwd(w.p, workspace=ws, **a, **dict(zip(("out", "lse", "idx"), outs)))  # noqa: E731
        call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
    inputs = {k: v.clone() for k, v in a.items() if v is not None}
    for i in (1, 0, 1, 1):
        for name, t in a.items():
            if t is not None:
                t.copy_((inputs, b)[i][name])
        outs[0].fill_(7), outs[1].fill_(7), outs[2].fill_(-77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, refs[i]))
        w.run()  # eager work between replays


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("topk,chunks", [(1, 1100), (7, 1100), (16, 1301), (33, 1100), (64, 2200)])
def test_ties_over_many_candidates(topk, chunks, dtype):
    """Landmarks of six kinds: equal scores by the dozen, of which the lower chunks are chosen, bit for bit."""
    p = hils_().Params(B=1, Hq=2, Hkv=1, N=70, L=64 * chunks, d=64, topk=topk, window=64, dtype=dtype)
    w = World(p, [64 * chunks - 7], [70], 3)
    r = np.random.default_rng(5)
    kinds, kind = w.lmk[w.table[0, :6]].copy(), r.integers(0, 6, chunks)
    kind[r.random(chunks) < 0.6] = 0
    kind[:500] = 5  # (for some rows the best kind begins late, for others at once)
    w.lmk[w.table[0, :chunks - 1]] = kinds[kind[:chunks - 1]]
    got = w.run()[2].cpu().numpy()
    score = np.einsum("hnd,khd->nkh", w.q[0].astype(np.float64), kinds.astype(np.float64)).max(-1)  # [N, kinds]
    for n in range(70):
        have = (w.len[0] - w.fresh[0] + n - 64 + 1) // 64
        order = np.lexsort((np.arange(have), -score[n][kind[:have]]))
        assert (got[0, 0, n] == np.sort(order[:topk])).all(), f"row {n}"
