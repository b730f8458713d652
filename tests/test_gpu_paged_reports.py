"""What the paged cache reports from the device, and what it leaves alone then."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paged_util import Case
from paper_2412_04757_amd import LtriPagedCache, paged_config

pytestmark = pytest.mark.gpu


def report(cache):
    """Status and text of the device's report."""
    status = cache.sync_status()
    return status, cache.lib.ltri_paged_last_error(cache.handle).decode()


def same(x, y):
    return torch.equal(torch.nan_to_num(x.float(), nan=-5.0), torch.nan_to_num(y.float(), nan=-5.0))


def crowded(gpu_device, seqs):
    """A pool of one sequence's pages, and a table that names them for `seqs` sequences."""
    c = Case(gpu_device, [640], page=64, spare=0)
    order = torch.from_numpy(c.table[0]).long().to(gpu_device)
    pools = [x[order].contiguous() for x in (c.cache.k_pages, c.cache.v_pages, c.cache.weight, c.cache.pos)]
    cfg = paged_config(c.hq, c.hkv, c.dim, c.dtype, page_tokens=64, n_pages=10, table_pages=10, max_seqs=seqs, weights=True)
    cache = LtriPagedCache(cfg, gpu_device, k_pages=pools[0], v_pages=pools[1], weight=pools[2], pos=pools[3])
    table = torch.arange(10, dtype=torch.int32, device=gpu_device).repeat(seqs, 1)
    return c, cache, table, torch.full((seqs,), 640, dtype=torch.int32, device=gpu_device)


def test_more_tokens_than_the_pool_holds(gpu_device):
    """Reported as that, not as a length beyond the table; rows and positions stay, results are whole, the next call's as well."""
    c, cache, table, lens = crowded(gpu_device, 12)
    before = [x.clone() for x in (cache.k_pages, cache.v_pages, cache.pos)]
    q = c.on(c.q).repeat(12, 1, 1, 1)
    out = cache.attend(table, lens, q, decay=1.0)
    status, text = report(cache)
    assert status == -3 and "than the pool holds" in text and "page table" not in text
    assert cache.sync_status() == 0
    want, _ = c.oracle_attend()
    for s in range(12):
        c.check_attend(out[s:s + 1], None, want, None)
    assert all(same(x, y) for x, y in zip(before, (cache.k_pages, cache.v_pages, cache.pos)))
    # and the length beyond the table as it was
    lens[3] = 641
    cache.attend(table, lens, q)
    status, text = report(cache)
    assert status == -3 and "a length beyond the page table" in text
    # one sequence alone has room
    cache.weight.copy_(torch.rand_like(cache.weight))
    weight = cache.weight.double().cpu().numpy()
    out = cache.attend(table[:1], lens[:1], q[:1].contiguous(), decay=0.5)
    want, _ = O.attend(cache.k_pages.double().cpu().numpy(), cache.v_pages.double().cpu().numpy(), weight, [list(range(10))], [640], c.q, 0.5)
    c.check_attend(out, None, want, None)
    t = c.tolerances()["weight"] + 4 * 2.0 ** -23                  # (as in Case.check_weight)
    assert (np.abs(cache.weight.double().cpu().numpy() - weight) <= t * np.abs(weight) + 2.0 ** -30).all()
    assert cache.sync_status() == 0


@pytest.mark.parametrize("seqs,status", [(1, 0), (2, -3), (12, -3)])
def test_pages_named_twice_with_weights_touch_nothing_else(gpu_device, seqs, status):
    """Which weights such a call leaves is not defined; rows and positions stay, and nothing is written behind the scratch."""
    c, plain, table, lens = crowded(gpu_device, seqs)
    guard = 1 << 20
    scratch = torch.full((plain.scratch_bytes + guard,), 0xFF, dtype=torch.uint8, device=gpu_device)
    cache = LtriPagedCache(plain.cfg, gpu_device, k_pages=plain.k_pages, v_pages=plain.v_pages, weight=plain.weight, pos=plain.pos, scratch=scratch)
    before = [x.clone() for x in (cache.k_pages, cache.v_pages, cache.pos)]
    cache.attend(table, lens, c.on(c.q).repeat(seqs, 1, 1, 1), decay=1.0)
    assert all(same(x, y) for x, y in zip(before, (cache.k_pages, cache.v_pages, cache.pos)))
    assert bool((scratch[plain.scratch_bytes:] == 0xFF).all()) and cache.sync_status() == status
