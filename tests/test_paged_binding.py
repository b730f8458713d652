"""The binding of the paged cache without a GPU: which pools it takes."""
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
