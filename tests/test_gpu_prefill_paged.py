"""hils_prefill_paged_fwd against the float64 oracle.

Tolerances, element by element.  out = sum_j w_j v_j: the weights carry the float32 logits' error
delta <= (d + 4) 2^-24 scale sum|q k| (below 5e-5 for these inputs: scale sum|q k| < 12, d <= 128),
twice (weight and normaliser), and in bf16 one rounding of 2^-8 each as operands of the product
and the output another 2^-8; a chunk's weight carries its landmark score's delta too.  So
|error| <= (2e-4 + r) sum_j w_j |v_j| + r |out| with r = 2^-8 (bf16) or 2^-24, and |error of lse| <= 1e-4.
Selections may differ by ties (tests/gpu_helpers.py); outputs are then compared on the selection made."""
import numpy as np
import pytest
import torch

import oracle
from tests.gpu_helpers import check_selection, np32, oshape
from paper_2607_02980_amd import synth

pytestmark = pytest.mark.gpu


def hils_():
    from paper_2607_02980_amd import hils

    return hils


class World:
    """Sequences of given lengths over pools of NaN: pages anywhere, the first of the last sequence shared with sequence
    0, entries past a length out of range, tokens past a length NaN."""

    def __init__(self, p, lens, new, seed, bias=False, route=False, spread=1.0):
        self.p, self.lens, self.new = p, lens, new
        r = self.r = np.random.default_rng(seed)
        Hl, C = p.Hl or p.Hq, p.L // 64
        clamp = [min(max(a, 0), p.L) for a in lens]
        self.len = clamp
        self.fresh = [min(max(0, min(m, p.N)), a) for a, m in zip(new, clamp)]

        def values(*shape):
            x = torch.as_tensor(r.standard_normal(shape).astype(np.float32) * np.float32(spread))
            return x.to(p.torch_dtype).float().numpy()

        used = [-(-a // 64) for a in clamp]
        P = sum(used) + 5
        perm = r.permutation(P)
        self.table = np.full((p.B, C), P + 3, np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = perm[at:at + u]
            at += u
        if p.B > 1:
            m = min(self.len[0] // 64, (self.len[-1] - self.fresh[-1]) // 64, 3)
            self.table[-1, :m] = self.table[0, :m]
        self.k, self.v = np.full((P, p.Hkv, 64, p.d), np.nan, np.float32), np.full((P, p.Hkv, 64, p.d), np.nan, np.float32)
        self.lmk, self.bias = np.full((P, Hl, p.d), np.nan, np.float32), np.full((P, Hl), np.nan, np.float32)
        for b, a in enumerate(clamp):
            for c in range(used[b]):
                pg, rows = self.table[b, c], min(64, a - 64 * c)
                if np.isnan(self.k[pg, 0, 0, 0]):
                    self.k[pg, :, :rows], self.v[pg, :, :rows] = values(p.Hkv, rows, p.d), values(p.Hkv, rows, p.d)
                    if rows == 64:
                        self.lmk[pg], self.bias[pg] = values(Hl, p.d), r.standard_normal(Hl) * 0.5
        self.q = values(p.B, p.Hq, p.N, p.d)
        self.q_route = values(p.B, p.Hq, p.N, p.d) if route else None
        self.with_bias = bias

    def dev(self, x, dtype=None):
        return torch.as_tensor(x).to("cuda", dtype or self.p.torch_dtype)

    def args(self):
        q = self.q.copy()
        for b, m in enumerate(self.fresh):
            q[b, :, m:] = np.nan  # rows that are none
        return dict(q=self.dev(q), k_pages=self.dev(self.k), v_pages=self.dev(self.v), lmk_pages=self.dev(self.lmk),
                    block_table=self.dev(self.table, torch.int32),
                    bias_pages=self.dev(self.bias, torch.float32) if self.with_bias else None,
                    q_route=None if self.q_route is None else self.dev(self.q_route),
                    seqlens=self.dev(np.int32(self.lens), torch.int32), newlens=self.dev(np.int32(self.new), torch.int32))

    def run(self, idx=None, **kw):
        p, dt = self.p, self.p.torch_dtype
        a = self.args()
        a.update(out=torch.full((p.B, p.Hq, p.N, p.d), 7.0, dtype=dt, device="cuda"),
                 lse=torch.full((p.B, p.Hq, p.N), 7.0, device="cuda"),
                 idx=torch.full((p.B, p.Hkv, p.N, p.topk), -77, dtype=torch.int32, device="cuda") if idx is None else
                 self.dev(idx, torch.int32))
        a.update(kw)
        return hils_().hils_prefill_paged_fwd(p, **a)

    def contiguous(self):
        """The caches that the pages stand for, zeros where nobody may look."""
        p, C = self.p, self.p.L // 64
        pg = np.minimum(self.table, len(self.k) - 1)
        x = {"q": self.q, "q_route": self.q_route}
        for name, pool in (("k", self.k), ("v", self.v)):
            y = np.nan_to_num(pool[pg].transpose(0, 2, 1, 3, 4).reshape(p.B, p.Hkv, C * 64, p.d), posinf=0.0, neginf=0.0)
            for b, a in enumerate(self.len):
                y[b, :, a:] = 0
            x[name] = np.ascontiguousarray(y)
        x["lmk"] = np.nan_to_num(np.ascontiguousarray(self.lmk[pg].transpose(0, 2, 1, 3)))
        x["bias"] = np.nan_to_num(np.ascontiguousarray(self.bias[pg].transpose(0, 2, 1)), neginf=-1e30) if self.with_bias else None
        return x

    def check(self, got, rows=None, given=None):
        p = self.p
        out, lse, idx = got[0].float().cpu().numpy(), got[1].cpu().numpy(), got[2].cpu().numpy()
        every = [(b, n) for b, m in enumerate(self.fresh) for n in range(m)]
        rows = every if rows is None else rows
        for b, m in enumerate(self.fresh):  # rows that are none stay as they were
            assert (out[b, :, m:] == 7).all() and (lse[b, :, m:] == 7).all()
            if given is None:
                assert (idx[b, :, m:] == -77).all()
        if not rows:
            return
        x = self.contiguous()
        pos = np.int32([[a - m + n if n < m else 0 for n in range(p.N)] for a, m in zip(self.len, self.fresh)])
        s = oshape(p)
        kw = dict(bias=x["bias"], q_route=x["q_route"], qpos=pos, rows=np.int32(rows))
        if given is None:
            ref = oracle.fwd(s, x["q"], x["k"], x["v"], x["lmk"], **kw)
            check_selection(p, {n: v for n, v in x.items() if v is not None}, idx, ref["idx"], qpos=pos, rows=rows)
            sel = np.where(idx == -77, -1, idx)
        else:
            sel = given
        ref = oracle.fwd(s, x["q"], x["k"], x["v"], x["lmk"], idx=sel, **kw)
        size = oracle.fwd(s, x["q"], x["k"], np.abs(x["v"]), x["lmk"], idx=sel, **kw)["out"]
        r = 2.0 ** -8 if p.dtype == "bf16" else 2.0 ** -24
        for b, n in rows:
            o, e = out[b, :, n], ref["out"][b, :, n]
            assert np.isfinite(o).all(), f"row {b, n}"
            worst = (np.abs(o - e) / ((2e-4 + r) * size[b, :, n] + r * np.abs(e) + 1e-30)).max()
            assert worst <= 1, f"row {b, n}: {worst} of the bound"
            assert np.abs(lse[b, :, n] - ref["lse"][b, :, n]).max() <= 1e-4, f"row {b, n}"


CASES = {
    "one_token": (dict(B=1, Hq=4, Hkv=1, N=1, L=64, d=64, topk=4, window=64), [1], [1], {}),
    "nothing_new": (dict(B=2, Hq=4, Hkv=1, N=3, L=128, d=64, topk=4, window=64), [100, 0], [0, 0], {}),
    "whole_prompt_g4": (dict(B=1, Hq=8, Hkv=2, N=777, L=832, d=128, topk=4, window=128), [777], [777], {}),
    "ragged_g4": (dict(B=5, Hq=8, Hkv=2, N=70, L=2048, d=128, topk=8, window=300), [2048, 70, 1111, 3, 500], [70, 70, 33, 1, 0], {}),
    "clamped": (dict(B=3, Hq=4, Hkv=2, N=10, L=640, d=64, topk=3, window=64), [9999, -5, 4], [99, 3, 10], {}),
    "g1_window_1": (dict(B=2, Hq=3, Hkv=3, N=67, L=1024, d=64, topk=5, window=1), [1024, 130], [67, 67], dict(route=True)),
    "g2_wide_window": (dict(B=2, Hq=4, Hkv=2, N=40, L=4096, d=128, topk=16, window=3000), [4000, 3333], [40, 39], dict(bias=True)),
    "g8_bias_route": (dict(B=3, Hq=16, Hkv=2, N=150, L=4096, d=128, topk=16, window=512), [4096, 4001, 640], [150, 149, 20],
                      dict(bias=True, route=True)),
    "shared_landmarks": (dict(B=2, Hq=8, Hkv=2, Hl=2, N=130, L=3008, d=64, topk=7, window=200), [3000, 2990], [130, 100],
                         dict(bias=True)),
    "shared_landmarks_g8_f32": (dict(B=2, Hq=8, Hkv=1, Hl=1, N=20, L=1600, d=128, topk=7, window=64, dtype="f32"), [1600, 1234],
                                [20, 17], dict(route=True)),
    "ragged_f32": (dict(B=4, Hq=8, Hkv=2, N=65, L=2048, d=64, topk=8, window=300, dtype="f32"), [2048, 1999, 65, 1], [65, 1, 65, 1], {}),
    "g8_f32_d128": (dict(B=1, Hq=8, Hkv=1, N=50, L=2048, d=128, topk=8, window=128, dtype="f32"), [2011], [50], dict(bias=True)),
    "g1_f32": (dict(B=2, Hq=2, Hkv=2, N=33, L=1024, d=128, topk=4, window=65, dtype="f32"), [1000, 1024], [33, 30], {}),
    "g2_f32": (dict(B=2, Hq=4, Hkv=2, N=33, L=1024, d=64, topk=4, window=65, dtype="f32"), [1000, 1024], [33, 30], dict(route=True)),
    "top_64_all": (dict(B=1, Hq=4, Hkv=1, N=30, L=4096, d=64, topk=64, window=64), [4090], [30], {}),
    "top_1": (dict(B=1, Hq=4, Hkv=1, N=130, L=8192, d=64, topk=1, window=64), [8191], [130], {}),
    "candidates_1100": (dict(B=1, Hq=4, Hkv=1, N=40, L=64 * 1110, d=64, topk=9, window=64), [71001], [40], {}),
    "candidates_300": (dict(B=2, Hq=2, Hkv=1, N=9, L=64 * 320, d=128, topk=16, window=64), [20480, 17000], [9, 9], {}),
}


@pytest.mark.parametrize("name", CASES)
def test_parity(name):
    kw, lens, new, opt = CASES[name]
    w = World(hils_().Params(**kw), lens, new, sum(map(ord, name)), **opt)
    w.check(w.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_to_decode_and_whole_prefill(dtype):
    """One new token each: the paged decode's result; a whole prompt: the prefill's (to the bounds of two results)."""
    hils = hils_()
    p = hils.Params(B=3, Hq=8, Hkv=2, N=1, L=2048, d=64, topk=8, window=128, dtype=dtype, scale=0.125)
    w = World(p, [2048, 700, 65], [1, 1, 1], 4, bias=True)
    a = w.args()
    got = w.run()
    w.check(got)
    ref = hils.hils_decode_paged_fwd(p, a["q"], *(torch.nan_to_num(a[n]) for n in ("k_pages", "v_pages", "lmk_pages")),
                                     a["block_table"], bias_pages=torch.nan_to_num(a["bias_pages"]), seqlens=a["seqlens"])
    assert torch.equal(got[2], ref[2])
    tol = 2e-4 * 4 if dtype == "f32" else 4 * 2.0 ** -8 * 4  # (values up to 4)
    assert (got[0].float() - ref[0].float()).abs().max() <= tol and (got[1] - ref[1]).abs().max() <= 2e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_given_selection(dtype):
    """Entries that are no candidates, out of order or named again are left out, as in the other forward calls."""
    hils = hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, N=40, L=1280, d=64, topk=6, window=128, dtype=dtype, flags=hils.HILS_FLAG_GIVEN_IDX)
    w = World(p, [1250, 600], [40, 37], 8, bias=True)
    r = np.random.default_rng(2)
    idx = np.sort(r.integers(-3, 18, (2, 2, 40, 6)), -1).astype(np.int32)
    idx[:, :, 3] = [5, 5, -1, 7, 2, 9]
    idx[:, :, 4] = [2 ** 31 - 1, -2 ** 31, 0, 0, 1, 1 << 20]
    idx[:, :, 5] = -1
    got = w.run(idx=idx)
    assert torch.equal(got[2].cpu(), torch.as_tensor(idx))
    pos = [[a - m + n for n in range(40)] for a, m in zip(w.len, w.fresh)]
    legal = np.full_like(idx, -1)
    for at in np.ndindex(2, 2, 40):
        nc, row = oracle.n_candidates(pos[at[0]][at[2]], 64, 128), idx[at]
        keep = [c for t, c in enumerate(row) if 0 <= c < nc and (t == 0 or c > row[t - 1])]
        if len(set(keep)) == len(keep) and keep == sorted(keep):
            legal[at][:len(keep)] = keep
        else:
            legal[at][:] = -2  # (the oracle's own reading of a row out of order is not compared)
    rows = [(b, n) for b in range(2) for n in range(w.fresh[b]) if (legal[b, :, n] != -2).all()]
    assert len(rows) > 60
    w.check(got, rows=rows, given=np.where(legal == -2, -1, legal))
    assert torch.isfinite(got[0].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_nan_in_masked_chunks(d, dtype):
    """A chunk with a bias of -inf weighs nothing, whatever it holds: NaN keys, values and landmark masked for all heads;
    NaN landmark masked for its head."""
    p = hils_().Params(B=1, Hq=8, Hkv=2, N=70, L=640, d=d, topk=8, window=64, scale=0.125, dtype=dtype)
    w = World(p, [630], [70], 17, bias=True)
    w.bias[w.table[0, 1]] = -np.inf
    w.bias[w.table[0, 3], 2] = -np.inf
    clean = w.run()
    w.check(clean)
    for x in (w.k, w.v):
        x[w.table[0, 1], :, 9] = np.nan
    w.lmk[w.table[0, 1]] = np.nan
    w.lmk[w.table[0, 3], 2] = np.inf
    got = w.run()
    assert all(torch.equal(x, y) for x, y in zip(got, clean))


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,G", [(64, 1), (128, 4), (128, 8)])
def test_later_tokens_do_not_reach_earlier_rows(d, G, dtype, value):
    """NaN and infinities in a new token's value (and NaN in its key) show in the rows that see it only."""
    p = hils_().Params(B=1, Hq=2 * G, Hkv=2, N=150, L=640, d=d, topk=4, window=64, dtype=dtype)
    w = World(p, [600], [150], 5)
    clean = w.run()
    w.check(clean)
    at = 450 + 77  # the position of row 77
    pg, row = w.table[0, at // 64], at % 64
    w.v[pg, 0, row, 3] = value
    if np.isnan(value):
        w.k[pg, 0, row, 5] = value
    got = w.run()
    bound = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -20  # (added in another order: twice the error of a result)
    assert torch.equal(got[2][:, :, :77], clean[2][:, :, :77])
    assert torch.equal(got[0][:, :, :64 - 2 - 1], clean[0][:, :, :61])  # (rows of blocks before it)
    assert ((got[0][:, :, :77] - clean[0][:, :, :77]).float().abs() <= bound * 4).all()
    assert not torch.isfinite(got[0][0, :G, 77, 3]).any()
    assert torch.equal(got[0][0, G:], clean[0][0, G:])  # the other KV group


def test_rows_cut_into_segments_have_the_same_bits():
    hils = hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, N=700, L=2048, d=128, topk=8, window=128)
    w = World(p, [2048, 1900], [700, 555], 3)
    whole = w.run()
    w.check(whole, rows=[(b, n) for b in range(2) for n in range(0, w.fresh[b], 37)])
    before = hils.hils_prefill_record_cap(2 * 8 * 8 * 129 * 4 * 130)  # 128 rows of records
    try:
        cut = w.run()
    finally:
        hils.hils_prefill_record_cap(before)
    assert all(torch.equal(x, y) for x, y in zip(whole, cut))
    again = w.run()
    assert all(torch.equal(x, y) for x, y in zip(whole, again))


def test_many_rows_over_a_long_cache():
    """More scores than are held at a time (blocks of rows), 1030 candidates; sampled rows."""
    p = hils_().Params(B=1, Hq=8, Hkv=8, N=4300, L=64 * 1040, d=64, topk=16, window=512)
    w = World(p, [66500], [4300], 12)
    w.check(w.run(), rows=[(0, n) for n in (0, 1, 127, 128, 2500, 4095, 4096, 4097, 4298, 4299)])


def test_views_workspace_streams_and_graphs():
    """Tensors at odd addresses; two calls at once with a workspace each; a captured call replayed on new inputs."""
    hils = hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, N=90, L=1024, d=64, topk=6, window=128)
    w = World(p, [1000, 700], [90, 81], 21)
    ref = w.run()
    w.check(ref)

    def odd(t):
        raw = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        raw[1:].copy_(t.flatten())
        return raw[1:].view(t.shape)

    a = w.args()
    got = w.run(**{n: odd(a[n]) for n in ("q", "k_pages", "v_pages", "lmk_pages")},
                out=odd(torch.full((2, 8, 90, 64), 7.0, dtype=torch.bfloat16, device="cuda")))
    assert all(torch.equal(x, y) for x, y in zip(got, ref))
    n = hils.hils_workspace_size(p, hils.HILS_OP_PREFILL_PAGED)
    with pytest.raises(hils.HilsError, match="workspace"):
        w.run(workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
    w2 = World(p, [600, 1024], [90, 90], 22)
    ref2 = w2.run()
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for s, x in zip(streams * 3, (w, w2) * 3):
        with torch.cuda.stream(s):
            results.append(x.run(workspace=torch.empty(n, dtype=torch.uint8, device="cuda").random_(256)))
    torch.cuda.synchronize()
    for i, r in enumerate(results):
        assert all(torch.equal(x, y) for x, y in zip(r, (ref, ref2)[i % 2]))
    a = w.args()
    b = w2.args()
    P = max(len(w.k), len(w2.k))
    for x in (a, b):
        for name in ("k_pages", "v_pages", "lmk_pages"):
            x[name] = torch.cat([x[name], x[name].new_zeros(P - len(x[name]), *x[name].shape[1:])])
    ws, outs = torch.empty(n, dtype=torch.uint8, device="cuda"), dict(
        out=torch.empty_like(ref[0]), lse=torch.empty_like(ref[1]), idx=torch.empty_like(ref[2]))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        hils.hils_prefill_paged_fwd(p, workspace=ws, **a, **outs)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            hils.hils_prefill_paged_fwd(p, workspace=ws, **a, **outs)
    inputs = {k: v.clone() for k, v in a.items() if v is not None}
    for x, r in ((b, ref2), (inputs, ref), (b, ref2)):
        for name, t in a.items():
            if t is not None:
                t.copy_(x[name])
        outs["out"].fill_(7), outs["lse"].fill_(7), outs["idx"].fill_(-77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(outs[n], y) for n, y in zip(("out", "lse", "idx"), r))
        w.run()  # eager work between replays


def test_pool_past_2_to_31_elements():
    hils = hils_()
    p = hils.Params(B=1, Hq=8, Hkv=8, N=20, L=1024, d=128, topk=4, window=64)
    w = World(p, [1000], [20], 6)
    ref = w.run()
    w.check(ref)
    P, n = 33200, len(w.k)  # 33200 * 65536 elements
    a = w.args()
    big = {}
    for name in ("k_pages", "v_pages", "lmk_pages"):
        big[name] = torch.empty((P, *a[name].shape[1:]), dtype=torch.bfloat16, device="cuda")
        big[name][P - n:] = a[name]
    table = torch.where(a["block_table"] < n, a["block_table"] + P - n, a["block_table"])
    got = w.run(**big, block_table=table)
    assert all(torch.equal(x, y) for x, y in zip(got, ref))
