"""What the binding of the 8-bit cache says of arguments that are no tensors or do not fit the C interface
(on the CPU: nothing is launched)."""
import pytest
import torch

from paper_2607_02980_amd import hils

P = hils.Params(B=2, Hq=4, Hkv=2, N=2, L=256, d=64, topk=2, window=64)
ACC, TABLE = torch.zeros(2, 4), torch.zeros(2, 4, dtype=torch.int32)


@pytest.mark.parametrize("bad", [None, 7, [1, 2], torch.zeros(())])
def test_pools_that_are_no_tensors(monkeypatch, bad):
    monkeypatch.setattr(hils, "_gpu", lambda t, name: 0)
    x, q, one = torch.zeros(2, 2, 2, 64, dtype=torch.bfloat16), torch.zeros(2, 4, 2, 64), torch.zeros(1)
    with pytest.raises(ValueError, match="k_pages must be a GPU tensor"):
        hils.hils_q8_append(P, x, x, bad, one, one, TABLE)
    with pytest.raises(ValueError, match="k_pages must be a GPU tensor"):
        hils.hils_q8_landmark_fwd(P, x, bad, one, TABLE, one, one)
    with pytest.raises(ValueError, match="k_pages must be a GPU tensor"):
        hils.hils_decode_q8_fwd(P, q, bad, one, one, one, TABLE)


def only(monkeypatch, checked):
    """Of all tensors only the one of that name is looked at."""
    monkeypatch.setattr(hils, "_gpu", lambda t, name: 0)
    monkeypatch.setattr(hils, "_address", lambda t, name, *a: hils._ptr(t, name) if name == checked else 0)


@pytest.mark.parametrize("bad", [7, [1, 2], torch.zeros(())])
def test_a_workspace_that_is_no_gpu_tensor(monkeypatch, bad):
    only(monkeypatch, "workspace")
    with pytest.raises(ValueError, match="workspace must be a GPU tensor"):
        hils.hils_decode_q8_fwd(P, torch.zeros(2, 4, 2, 64), *[torch.zeros(1)] * 4, TABLE, workspace=bad)


@pytest.mark.parametrize("bad", [None, 7, [1, 2], TABLE])
def test_a_block_table_that_is_no_gpu_tensor(monkeypatch, bad):
    only(monkeypatch, "block_table")
    with pytest.raises(ValueError, match="block_table"):
        hils.hils_cache_evict(P, ACC, bad)


@pytest.mark.parametrize("name", ["budget", "sink", "max_evict"])
@pytest.mark.parametrize("value", [1 << 31, 1 << 32, (1 << 32) + 5, -(1 << 31) - 1])
def test_numbers_past_32_bits_are_refused(name, value):
    """(ctypes drops the higher bits: a budget of 2^32 would be one of 0, and cut every sequence.)"""
    with pytest.raises(ValueError, match=f"{name}=.*32 bits"):
        hils.hils_cache_evict(P, ACC, TABLE, **{name: value})
