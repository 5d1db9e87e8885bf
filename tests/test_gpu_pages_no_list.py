"""hils_cache_free takes what hils_cache_evict gives where nothing may be dropped: lists of no entries."""
import numpy as np
import pytest
import torch

from tests import pages_oracle as O
from tests.test_gpu_pages import dev, hils_, params, same

pytestmark = pytest.mark.gpu


def test_lists_of_an_eviction_that_may_drop_nothing():
    hils = hils_()
    p = params(2, 640)
    table, refs, lens = np.arange(20, dtype=np.int32).reshape(2, 10), np.ones(20, np.int32), [640, 333]
    acc = torch.zeros((2, 10), device="cuda")
    _, t, a, freed, nfreed = hils.hils_cache_evict(p, acc, dev(table), dev(lens), max_evict=0)
    assert freed.shape == (2, 0) and nfreed.tolist() == [0, 0]
    same(hils.hils_cache_free(p, dev([600, 64]), t, dev(refs), a, freed, nfreed), O.free(p, [600, 64], table, refs, lens))
    with pytest.raises(ValueError, match="npages"):  # (checked all the same)
        hils.hils_cache_free(p, dev([600, 64]), t, dev(refs), a, freed, nfreed[:1])
    with pytest.raises(hils.HilsError, match="pages must be"):  # counts without lists
        hils.hils_cache_free(p, dev([600, 64]), t, dev(refs), a, npages=nfreed)
