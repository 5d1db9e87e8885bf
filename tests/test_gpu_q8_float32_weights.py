"""The 8-bit cache's softmax weights keep float32's precision in their products with keys and values.

Rows whose sum cancels: half of a chunk's 64 keys have one logit, the others one that lies delta below it, so
every weight is 1 / l or e / l (e = exp(-delta), l = 32 (1 + e)), and the codes of each dimension, +448 and
smaller at the first half, -384 at the second, cancel but for a remainder v of at most 0.01.  A weight held in
16 significant bits shifts the sum by up to 2^-18 of 192 (7e-4), whatever is left of it.  In float32, in units
of the scale:
  * e is off by 2^-23 (the logits are exact), and its operand by as much: 2 * 192 * 2^-23 = 4.6e-5;
  * 64 additions of partial sums of at most 2300, rounded at 2^-24 and divided by l > 62: 1.4e-4;
  * divisions by l and the fusion's factors: 2^-21 of v, nothing.
  So 2e-4, and half a step of the output: 2^-10 for e4m3 codes below 2^-6, 2^-8 of the value for bf16."""
import numpy as np
import pytest
import torch

from tests import q8_oracle as Q
from tests import test_gpu_q8 as T

pytestmark = pytest.mark.gpu
TOL = 2e-4


def codes_that_cancel(r, delta, d):
    """[64, d] values in e4m3: column 0 of 128 at even keys and 120 at odd ones, the others as above."""
    e = np.exp(-delta)
    left = 384 * 32 * e + r.uniform(-0.01, 0.01, d) * 32 * (1 + e)
    x = np.full((64, d), -384.0)
    for i in range(0, 64, 2):
        top = np.searchsorted(Q.VALUE[:127], np.minimum(left, 448), side="right") - 1
        x[i] = Q.VALUE[np.maximum(top, 0)]
        left = left - x[i]
    x[::2, 0], x[1::2, 0] = 128, 120
    return x


def queries(r, n):
    """q[0] of n heads: bf16 values, so that delta = scale * 2^-7 * 8 q[0] and the logits are exact."""
    return r.integers(128, 256, n) / 128 * 2.0 ** r.integers(-1, 2, n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_landmark_rows(d, dtype):
    hils = T.hils_()
    p = hils.Params(B=2, Hq=8, Hkv=8, N=512, L=512, d=d, topk=1, window=64, scale=0.125, dtype=dtype)
    r = np.random.default_rng(d)
    P, lq = 16, np.zeros((2, 8, 8, d), np.float32)
    table = r.permutation(P).reshape(2, 8).astype(np.int32)
    lq[..., 0] = queries(r, (2, 8, 8))
    k = np.zeros((P, 8, 64, d), np.uint8)
    for b in range(2):
        for h in range(8):
            for c in range(8):
                k[table[b, c], h] = Q.encode(codes_that_cancel(r, 0.125 * 2.0 ** -7 * 8 * lq[b, h, c, 0], d))
    scale = np.full((P, 8, 2), 2.0 ** -7, np.float32)
    ref = Q.landmark(p, lq, k, scale, table)
    lm, bias = T.f8(np.zeros((P, 8, d), np.uint8)), torch.zeros((P, 8), device="cuda")
    hils.hils_q8_landmark_fwd(p, T.dev(lq, p.torch_dtype), T.f8(k), T.dev(scale), T.dev(table), lm, bias)
    torch.cuda.synchronize()
    got = Q.VALUE[T.codes(lm)]
    for page, (rows, _) in ref.items():
        assert np.abs(rows[:, 1:]).max() < 2.0 ** -6
        assert np.abs(got[page] - rows)[:, 1:].max() <= 2.0 ** -10 + TOL


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [8, 24])  # 64 rows, which workgroups share, and 192, a workgroup each
@pytest.mark.parametrize("d", [64, 128])
def test_decode(d, B, dtype):
    hils = T.hils_()
    p = hils.Params(B=B, Hq=8, Hkv=8, N=1, L=1024, d=d, topk=16, window=512, scale=0.125, dtype=dtype)
    r = np.random.default_rng(d + B)
    P, q = B * 16, np.zeros((B, 8, 1, d), np.float32)
    table = r.permutation(P).reshape(B, 16).astype(np.int32)
    q[..., 0] = queries(r, (B, 8, 1))
    k, v = np.zeros((P, 8, 64, d), np.uint8), np.zeros((P, 8, d, 64), np.uint8)
    k[:, :, ::2, 0], k[:, :, 1::2, 0] = Q.encode(128), Q.encode(120)
    for b in range(B):
        for h in range(8):
            for c in range(16):
                x = codes_that_cancel(r, 0.125 * 2.0 ** -7 * 8 * q[b, h, 0, 0], d)
                x[:, 0] = x[:, 1]
                v[table[b, c], h] = Q.encode(x.T)
    scale, lmk = np.full((P, 8, 2), 2.0 ** -7, np.float32), np.zeros((P, 8, d), np.uint8)
    ref = Q.decode(p, q, k, v, scale, lmk, table)
    out, lse, idx, wt = hils.hils_decode_q8_fwd(p, T.dev(q, p.torch_dtype), T.f8(k), T.f8(v), T.dev(scale), T.f8(lmk), T.dev(table))
    torch.cuda.synchronize()
    assert np.array_equal(idx.cpu().numpy(), ref[2]) and np.abs(ref[0]).max() < 0.01 * 2.0 ** -7 * 1.01
    off = np.abs(T.host(out) - ref[0])
    assert (off <= TOL * 2.0 ** -7 + (2.0 ** -8 * np.abs(ref[0]) if dtype == "bf16" else 0)).all()


@pytest.mark.parametrize("B", [2, 24])
@pytest.mark.parametrize("d", [64, 128])
def test_small_weights_beside_a_large_one(d, B):
    """A key of weight near 1 whose values are 0, as a sequence's first token often has, and 63 of 2^-12 to 2^-17.

    Relative to the outputs, which these alone make up: logits (exact) in units of log2, up to 17, rounded at 2^-23
    twice: 2 * 17 * 0.7 * 2^-24 = 1.4e-6; exp 2^-23; operands 2^-23, or 2^-37 of a weight of 2^-17: 1e-6; a sum of 63
    positive terms 63 * 2^-24 = 3.8e-6; factors and the division 2^-21: 7e-6 in all."""
    hils = T.hils_()
    p = hils.Params(B=B, Hq=8, Hkv=8, N=1, L=64, d=d, topk=1, window=64, scale=0.125, dtype="f32")
    r = np.random.default_rng(d)
    q = np.zeros((B, 8, 1, d), np.float32)
    q[..., 0] = r.integers(154, 206, (B, 8, 1)) / 128  # logits 7 q[0] apart: 8.4 to 11.3
    k, v = np.zeros((B, 8, 64, d), np.uint8), Q.encode(r.uniform(100, 448, (B, 8, d, 64)))
    k[:, :, 0, 0], v[..., 0] = Q.encode(448), 0
    scale = np.full((B, 8, 2), 2.0 ** -3, np.float32)
    table, lmk = np.arange(B, dtype=np.int32)[:, None], np.zeros((B, 8, d), np.uint8)
    ref = Q.decode(p, q, k, v, scale, lmk, table)
    out = hils.hils_decode_q8_fwd(p, T.dev(q), T.f8(k), T.f8(v), T.dev(scale), T.f8(lmk), T.dev(table))[0]
    off = np.abs(T.host(out) - ref[0]) / ref[0]
    print("off", off.max(), flush=True)
    assert off.max() <= 1e-5
