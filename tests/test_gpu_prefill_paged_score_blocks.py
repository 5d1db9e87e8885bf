"""hils_prefill_paged_fwd where a call has more scores than are held at a time (512 MB): its rows are scored and selected
a block after the other, and counts and ranks of the chunks add up over the blocks."""
import numpy as np
import pytest
import torch

from tests.test_gpu_prefill_paged import World, hils_

pytestmark = pytest.mark.gpu

# Rows of a block: 512 MB / (4 B Hkv L/64) in whole 128s, as equal as that allows; two blocks each.
CASES = {
    # 31744 at most, so 16512 and 16488; the second sequence ends inside the second block, or before it
    "blocks_of_candidates": (dict(B=2, Hq=1, Hkv=1, L=64 * 2112, topk=8), [135000, 20000], [33000, 17000]),
    "in_the_first_block_only": (dict(B=2, Hq=1, Hkv=1, L=64 * 2112, topk=2), [135168, 9000], [33000, 9000]),
    # 65536 at most, a whole prompt, whose rows have from no candidate to all of them
    "whole_prompt": (dict(B=1, Hq=4, Hkv=2, L=64 * 1025, topk=4), [65600], [65600]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_blocks_of_rows(name, dtype):
    hils = hils_()
    kw, lens, new = CASES[name]
    p = hils.Params(N=max(new), d=64, window=64, dtype=dtype, **kw)
    w = World(p, lens, new, 12)
    hils.hils_timing_enable(True)
    try:
        got = w.run()
        launches = {k: v["launches"] for k, v in hils.hils_timing_read().items()}
    finally:
        hils.hils_timing_enable(False)
    assert launches["k_pp_score"] == launches["k_pp_select"] == 2 and launches["k_pp_chunks"] == 1
    cut = (p.N + 255) // 256 * 128  # the second block's first row
    rows = [(b, n) for b in range(p.B) for n in (0, 1, 5000, cut - 129, cut - 1, cut, cut + 1, cut + 128, w.fresh[b] - 1)
            if n < w.fresh[b]]
    w.check(got, rows=rows)
    # the same rows in segments of 128, each a block of its own: the same bits
    before = hils.hils_prefill_record_cap(1)
    try:
        alone = w.run()
    finally:
        hils.hils_prefill_record_cap(before)
    assert all(torch.equal(x, y) for x, y in zip(got, alone))
