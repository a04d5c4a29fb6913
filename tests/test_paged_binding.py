"""What the binding of the paged cache keeps from being misused (no GPU needed)."""
import copy

import pytest
import torch

from paper_2605_19726_amd import binding as bd


def _cache(pages=9):
    return bd.PagedCache(*(torch.zeros(pages, 4, 16, 64, dtype=torch.bfloat16) for _ in range(2)))


@pytest.mark.parametrize("name", ["k", "v", "device", "dtype", "pages", "heads", "page", "d"])
def test_a_cache_cannot_come_apart_from_its_descriptors(name):
    """Another tensor in the place of k or v would leave the kernels with the old one's address."""
    cache, other = _cache(), _cache(12)
    with pytest.raises(AttributeError):
        setattr(cache, name, getattr(other, name))
    assert cache.k.data_ptr() == cache._kd.ptr and cache.v.data_ptr() == cache._vd.ptr and cache.pages == 9


def test_copies_of_a_cache_describe_their_own_tensors():
    cache = _cache()
    near, far = copy.copy(cache), copy.deepcopy(cache)
    assert near.k is cache.k and near._kd.ptr == cache.k.data_ptr()
    assert far.k.data_ptr() != cache.k.data_ptr() and far._kd.ptr == far.k.data_ptr() and far._vd.ptr == far.v.data_ptr()


def test_a_workspace_has_the_memory_that_its_size_says():
    q, ints = torch.zeros(3, 8, 64, dtype=torch.bfloat16), lambda *shape: torch.zeros(shape, dtype=torch.int32)
    for ws in (torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(1 << 21, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="ws must be"):
            bd.basa_decode_attn(q, _cache(), ints(3, 7), ints(3), ws=ws)


def test_prompts_that_the_rows_or_the_table_cannot_hold_are_refused_before_anything_is_written(monkeypatch):
    """Keys for fewer rows than there are queries, or a table row that is too short, would be read back as other tokens or zeros."""
    calls = []
    monkeypatch.setattr(bd, "basa_cache_append", lambda *args: calls.append(args))
    q, kv = torch.zeros(40, 8, 64, dtype=torch.bfloat16), torch.zeros(40, 4, 64, dtype=torch.bfloat16)
    table, slots = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(40, dtype=torch.int64)
    for k, cu, cached in ((kv[:30], [0, 10, 40], [5, 0]), (kv[:30], [0, 10, 40], None), (kv, [0, 10, 40], [39, 0]), (kv, [0, 0, 40], [49, 9])):
        with pytest.raises(ValueError, match="cu_seqlens|room for 48"):
            bd.ba_att_cached(q, k, k, cu, _cache(), table, slots[:k.shape[0]], cached=cached)
    assert not calls
    monkeypatch.setattr(bd, "ba_att_varlen", lambda *args: "prompts")          # what reads nothing back needs no room
    assert bd.ba_att_cached(q, kv, kv, [0, 0, 40], _cache(), table[:, :1], slots) == "prompts" and len(calls) == 1
