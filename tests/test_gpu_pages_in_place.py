"""The page operators write the same in place as into other buffers, counts below 0 (free pages) among them."""
import numpy as np
import pytest
import torch

from tests import pages_oracle as O
from tests.test_gpu_pages import dev, hils_, params, same

pytestmark = pytest.mark.gpu


def state(P, L, B, seed):
    """Rows of pages anywhere in a pool of which half is free, with counts of 0 and below; lengths."""
    r = np.random.default_rng(seed)
    C = L // O.S
    used = r.permutation(P)[:P // 2]
    lens = r.integers(0, L + 1, B)
    table = np.full((B, C), -1, np.int32)
    refs = r.integers(-5, 1, P).astype(np.int32)
    refs[used] = 0
    for b in range(B):
        n = O.chunks(lens[b])
        table[b, :n] = r.choice(used, n)
        np.add.at(refs, table[b, :n], 1)
    refs[used] += 1  # (another holder)
    return table, refs, lens


@pytest.mark.parametrize("P", [9, 700, 5000, 40000])  # (pages of a thread: few, many; several steps)
def test_compact(P):
    hils = hils_()
    p = params(3, 64 * 20)
    table, refs, lens = state(P, p.L, p.B, P)
    assert (refs < 0).any()
    data = [np.arange(P)[:, None]]
    ref = O.compact(p, table, refs, data, lens)
    for in_place in (False, True):
        t, n, pool = dev(table), dev(refs), torch.arange(P, device="cuda", dtype=torch.int64).view(P, 1)
        got = hils.hils_cache_compact(p, t, n, [pool], dev(lens), **(dict(table_out=t, refs_out=n) if in_place else {}))
        same(got, ref, f"in place: {in_place}")
        assert np.array_equal(pool.cpu().numpy(), data[0])


@pytest.mark.parametrize("P", [9, 700, 40000])
def test_reserve_fork_and_free(P):
    hils = hils_()
    p = params(3, 64 * 20, 5)
    table, refs, lens = state(P, p.L, p.B, P + 1)
    keep, parent = [7, 64, 2000], [2, 2, 0]
    for op, out in (("reserve", "table_out"), ("free", "table_out"), ("fork", None)):
        results = []
        for in_place in (False, True):
            t, n, a = dev(table), dev(refs), dev(lens)
            kw = dict(refs_out=n, **({out: t} if out else {})) if in_place else {}
            if op == "reserve":
                got = hils.hils_cache_reserve(p, t, n, seqlens=a, newlens=dev([5, 0, 3]), **kw)
            elif op == "free":
                got = hils.hils_cache_free(p, dev(keep), t, n, a, **kw, **(dict(seqlens_out=a) if in_place else {}))
            else:
                got = hils.hils_cache_fork(p, dev(parent), t, n, a, **kw)
            results.append([x.cpu().numpy() for x in got])
        for x, y in zip(*results):
            assert np.array_equal(x, y), op
