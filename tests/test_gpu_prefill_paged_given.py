"""hils_prefill_paged_fwd on given rows that do not ascend: such a row's own result is nobody's business, but a row
[c, -1, c, -1, ...] uses its chunk several times (an entry is compared with the one before it only), and the other
rows have to stay as they were, bit for bit, however often a chunk is used."""
import numpy as np
import pytest
import torch

from tests.test_gpu_prefill_paged import World, hils_

pytestmark = pytest.mark.gpu

# one workgroup of the selection for all rows and its plan; counts in LDS; counts in memory
SHAPES = {
    "few_rows": dict(N=40, L=1280, topk=6),
    "few_rows_top_64": dict(N=64, L=2048, topk=64),
    "many_rows": dict(N=500, L=1280, topk=6),
    "many_chunks": dict(N=70, L=8192, topk=6),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", SHAPES)
def test_rows_out_of_order_change_no_other(name, dtype):
    hils = hils_()
    p = hils.Params(B=2, Hq=8, Hkv=2, d=64, window=128, dtype=dtype, flags=hils.HILS_FLAG_GIVEN_IDX, **SHAPES[name])
    w = World(p, [p.L, p.L - 77], [p.N, p.N - 3], 8, bias=True)
    K, least = p.topk, (p.L - 77 - p.N - 128 + 1) // 64  # candidates of every row, at least
    r = np.random.default_rng(2)
    fine = np.full((2, 2, p.N, K), -1, np.int32)
    for at in np.ndindex(2, 2, p.N):
        m = min(K, least)
        fine[at][:m] = np.sort(r.choice(least, m, replace=False))
    good = np.arange(p.N) % 8 == 5
    none, bad = fine.copy(), fine.copy()
    none[:, :, ~good] = -1
    bad[:, :, ~good, ::2], bad[:, :, ~good, 1::2] = 4, -1
    bad[:, :, 1::8, 1::2] = 3  # (falls and rises again: as many uses)
    uses = (bad == 4).sum((2, 3))
    assert (uses > 64).all()
    n = hils.hils_workspace_size(p, hils.HILS_OP_PREFILL_PAGED)
    got = [w.run(idx=x, workspace=torch.empty(n, dtype=torch.uint8, device="cuda").random_(256)) for x in (bad, none)]
    keep = torch.as_tensor(good, device="cuda")
    for x, y in zip(*got):
        assert torch.equal(x[:, :, keep], y[:, :, keep])
    w.check(got[1], rows=[(b, n) for b in range(2) for n in range(w.fresh[b]) if good[n]], given=none)
    for b in range(2):
        assert torch.isfinite(got[0][0][b, :, :w.fresh[b]].float()).all()
