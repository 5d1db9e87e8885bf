"""Ties of scores of 0 and -0 in hils_prefill_paged_fwd."""
import numpy as np
import pytest

from tests.test_gpu_prefill_paged import World, hils_

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 4])
@pytest.mark.parametrize("chunks,new", [(50, 3), (50, 140), (1200, 40)])
def test_zero_scores_of_either_sign_tie(chunks, new, G, dtype):
    """Scores of 0 and -0 (a negative scale times 0, with biases of either sign) are equal: the lowest chunks are chosen."""
    p = hils_().Params(B=1, Hq=2 * G, Hkv=2, N=new, L=64 * chunks, d=64, topk=9, window=64, scale=-0.125, dtype=dtype)
    w = World(p, [64 * chunks - 5], [new], 3, bias=True)
    at = w.table[0, :chunks - 1]
    w.lmk[at] = 0
    w.bias[at] = -0.0
    w.bias[at[1::2]] = 0.0
    got = w.run()
    assert (got[2].cpu().numpy() == np.arange(9)).all()
    w.check(got, rows=[(0, 0), (0, new // 2), (0, new - 1)])
