"""The binding of the paged cache without a GPU: which pools it takes, and that the allocator hears of the streams."""
from types import SimpleNamespace

import pytest
import torch

from paper_2412_04757_amd import LtriError, LtriPagedCache, paged_config


def config(n_pages, heads, page, dim=64):
    return paged_config(2 * heads, heads, dim, "bf16", page_tokens=page, n_pages=n_pages, table_pages=4, max_seqs=3)


@pytest.mark.parametrize("shape,expanded", [
    ((12, 2, 16, 64), (1, 1, 1, 64)), ((12, 1, 1, 64), (1, 1, 1, 64)), ((1, 2, 1, 64), (1, 1, 1, 64)), ((1, 1, 16, 64), (1, 1, 1, 64)),
    ((12, 2, 16, 64), (12, 1, 16, 64)), ((12, 2, 16, 64), (1, 2, 16, 64)), ((12, 2, 16, 64), (12, 2, 1, 64)), ((12, 2, 16, 64), (64,)),
])
def test_expanded_pools_are_refused(shape, expanded):
    """Their rows are one row: with all three strides 0 the library would take them for a dense pool and go past their memory."""
    pool = torch.zeros(expanded, dtype=torch.bfloat16).expand(shape)
    with pytest.raises(ValueError, match="overlap"):
        LtriPagedCache(config(*shape[:3]), None, dry=True, k_pages=pool, v_pages=pool)


def test_axes_of_one_entry_may_have_any_stride():
    for shape in ((1, 1, 1, 64), (5, 1, 1, 64), (1, 3, 1, 64), (1, 1, 8, 64), (5, 1, 8, 64)):
        whole = torch.zeros((5, 3, 8, 64), dtype=torch.bfloat16)
        for pool in (torch.zeros(shape, dtype=torch.bfloat16), whole[:shape[0], :shape[1], :shape[2]],
                     torch.as_strided(whole, shape, [0 if n == 1 else s for n, s in zip(shape, whole.stride())])):
            LtriPagedCache(config(*shape[:3]), None, dry=True, k_pages=pool, v_pages=pool)


def test_pools_whose_rows_overlap_otherwise_are_refused():
    whole = torch.zeros(5 * 3 * 8 * 64, dtype=torch.bfloat16)
    for strides in ((3 * 8 * 64, 64, 64), (8 * 64, 8 * 64, 64), (3 * 8 * 64, 8 * 64, 56)):
        pool = torch.as_strided(whole, (5, 3, 8, 64), (*strides, 1))
        with pytest.raises(LtriError) as e:
            LtriPagedCache(config(5, 3, 8), None, dry=True, k_pages=pool, v_pages=pool)
        assert e.value.status == -1


def test_the_allocator_is_told_of_every_stream():
    """A buffer that only its stream of creation is known for could be given to others while the work of a later stream still uses it."""
    cache = LtriPagedCache(config(5, 3, 8), None, dry=True)
    names, heard = ("k_pages", "v_pages", "weight", "pos", "state", "scratch"), []
    for name in names:
        setattr(cache, name, SimpleNamespace(record_stream=lambda s, name=name: heard.append((name, s))))
    cache.pos = None                                           # (a cache without positions)
    cache.dry, cache.device = False, "here"
    side = SimpleNamespace(device="here", cuda_stream=16)
    cache.set_stream(side)
    assert sorted(heard, key=lambda x: names.index(x[0])) == [(n, side) for n in names if n != "pos"] and cache.stream is side
    with pytest.raises(ValueError):
        cache.set_stream(SimpleNamespace(device="there", cuda_stream=32))
    assert len(heard) == 5 and cache.stream is side
