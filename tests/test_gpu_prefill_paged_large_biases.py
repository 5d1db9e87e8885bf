"""hils_prefill_paged_fwd with biases up to float32's largest value (a chunk that must be attended): in log2 units they
would overflow.

Outputs: the bounds of test_gpu_prefill_paged.py.  Log-sum-exps of this size are the largest s^ itself (a smaller one
that float32 can tell apart from it weighs nothing): a product with a rounded constant there and back, 2^-24 each for
product and constant, or two sums of 2^-24 of a value twice as large at most: below 2^-21 of it."""
import numpy as np
import pytest
import torch

from tests.test_gpu_prefill_paged import World, hils_

pytestmark = pytest.mark.gpu

MOST = np.finfo(np.float32).max
# biases of chunks 3, 7 and 11 of head 0 (the others' are ordinary)
VALUES = {"one": (3e38, 0, 0), "largest": (MOST, 0, 0), "several": (MOST, MOST, 1e38), "near_each_other": (3e38, 2.9e38, 3.1e38),
          "below_and_above": (1.7e38, 1.71e38, 1.6e38), "in_range": (1e38, 1e30, 1.6e38), "masked_too": (-np.inf, MOST, -MOST)}


def row_of(p, x, pos, n, h, idx):
    """out, sum of weights times |v|, and log-sum-exp of one row and head in float64, the weights from differences to the
    largest logit and divided by their sum (a log-sum-exp near 2^128 does not hold the logarithm of the sum)."""
    f64, g, scale = np.float64, h // (p.Hq // p.Hkv), float(np.float32(p.d ** -0.5))
    q, k, v = x["q"][0, h, n].astype(f64), x["k"][0, g].astype(f64), x["v"][0, g].astype(f64)
    logits, values = [], []
    for c in idx[idx >= 0]:
        s = scale * (k[64 * c:64 * c + 64] @ q)
        e = np.exp(s - s.max())
        values.append([e @ v[64 * c:64 * c + 64] / e.sum(), e @ np.abs(v[64 * c:64 * c + 64]) / e.sum()])
        logits.append(scale * (x["lmk"][0, h, c].astype(f64) @ q) + f64(x["bias"][0, h, c]))
    near = np.arange((pos - p.window + 1) // 64 * 64, pos + 1)
    logits += list(scale * (k[near] @ q))
    values += [[v[j], np.abs(v[j])] for j in near]
    logits, values = np.array(logits), np.array(values)
    e = np.exp(logits - logits.max())
    out, size = (e[:, None, None] * values).sum(0) / e.sum()
    return out, size, logits.max() + np.log(e.sum())


@pytest.mark.parametrize("name", VALUES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [40, 2500])  # windows as items of the chunks' pass, and by themselves
def test_biases_up_to_the_largest_value(new, dtype, name):
    biases = VALUES[name]
    p = hils_().Params(B=1, Hq=8, Hkv=2, N=new, L=4096, d=64, topk=8, window=64, dtype=dtype)
    w = World(p, [4001], [new], 3, bias=True)
    w.bias[w.table[0, [3, 7, 11]], 0] = biases
    got = w.run()
    out, lse, idx = got[0].float().cpu().numpy(), got[1].cpu().numpy(), got[2].cpu().numpy()
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    rows = [(0, n) for n in (0, 1, new // 2, new - 1)]
    x = w.contiguous()
    r = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for b, n in rows:
        assert {c for c, v in zip((3, 7, 11), biases) if v > 1e20} <= set(idx[b, 0, n])
        for h in range(p.Hq):
            e, size, want = row_of(p, x, 4001 - new + n, n, h, idx[b, h // 4, n])
            assert (np.abs(out[b, h, n] - e) <= (2e-4 + r) * size + r * np.abs(e) + 1e-30).all(), f"row {n}, head {h}"
            assert abs(lse[b, h, n] - want) <= 1e-4 + 2.0 ** -21 * abs(want), f"row {n}, head {h}"
        assert lse[b, 0, n] >= 1e37
