"""Every compiled form of the paged cache's attention, limits, wide tables, and pages outside the pool wherever a kernel looks at them."""
import itertools

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paged_util import Case
from paper_2412_04757_amd import LtriPagedCache
from test_gpu_paged import check_evict, evict_case

pytestmark = pytest.mark.gpu

# pairs of query row and head per KV head: one block of 16; two; four; four and one more
PAIRS = {"4": (8, 2, 1), "24": (12, 2, 4), "42": (14, 2, 6), "80": (32, 2, 5)}


# ------------------------------------------------------------------ attention, form by form

@pytest.mark.parametrize("dtype,dim,pairs,page", list(itertools.product(("bf16", "f32"), (64, 128), PAIRS, (8, 16))))
def test_every_form_of_the_attention(gpu_device, dtype, dim, pairs, page):
    """With pages that a group of 16 tokens lies in and smaller ones: attention, its weights, and new rows written by the step itself."""
    hq, hkv, rows = PAIRS[pairs]
    c = Case(gpu_device, [0, 1, 700, 64, 17, 333, 2], dtype=dtype, dim=dim, hq=hq, hkv=hkv, page=page, rows=rows)
    for decay in (None, 0.0, 0.5):
        lse = c.new_lse()
        out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse, decay=decay)
        want, want_lse = c.oracle_attend(decay)
        c.check_attend(out, lse, want, want_lse)
        c.check_weight()
    lse = c.new_lse()
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), lse=lse, decay=0.25)
    c.oracle_append()
    want, want_lse = c.oracle_attend(0.25)
    c.check_attend(out, lse, want, want_lse)
    c.check_weight()
    c.check_pools()
    assert torch.equal(c.cache.attend(*c.args(False), c.on(c.q)), out)
    assert c.cache.sync_status() == 0


@pytest.mark.parametrize("dtype,dim,page,pairs", [("bf16", 128, 16, "80"), ("f32", 128, 16, "80"), ("bf16", 128, 64, "42"), ("f32", 128, 32, "42"),
                                                  ("bf16", 64, 16, "80"), ("f32", 64, 16, "24"), ("bf16", 128, 4, "80"), ("bf16", 128, 16, "24")])
def test_many_pairs_over_pools_in_token_order(gpu_device, dtype, dim, page, pairs):
    """[page][token][KV head][d]: tokens lie further apart than a row is long, also where tiles are brought into LDS."""
    hq, hkv, rows = PAIRS[pairs]
    c = Case(gpu_device, [70, 900, 33, 0, 128], dtype=dtype, dim=dim, hq=hq, hkv=hkv, page=page, rows=rows, token_major=True)
    assert c.cache.cfg.token_stride > c.cache.cfg.head_stride
    lse = c.new_lse()
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), lse=lse, decay=0.5)
    c.oracle_append()
    c.check_attend(out, lse, *c.oracle_attend(0.5))
    c.check_weight()
    c.check_pools()
    assert c.cache.sync_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_and_values_in_one_pool(gpu_device, dtype):
    """[page][keys, values][KV head][token][d], as views: a page's stride is twice its rows."""
    c = Case(gpu_device, [300, 45, 1], dtype=dtype, hq=32, rows=5, weights=False)
    both = torch.stack((c.cache.k_pages, c.cache.v_pages), 1)
    before = c.cache
    c.cache = LtriPagedCache(before.cfg, gpu_device, k_pages=both[:, 0], v_pages=both[:, 1])
    assert c.cache.cfg.page_stride == 2 * before.cfg.page_stride
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q))
    c.oracle_append()
    c.check_attend(out, None, *c.oracle_attend())
    c.check_pools()


@pytest.mark.parametrize("lens,hq,hkv,rows,page", [
    ([70, 3], 128, 1, 64, 16),                     # the most rows of the most heads: 8192 pairs
    ([40], 4096, 32, 1, 8),                        # the most query heads
    ([9, 0, 30], 64, 64, 2, 1),                    # a head of its own for every query, a token a page
])
def test_limits_of_heads_and_rows(gpu_device, lens, hq, hkv, rows, page):
    c = Case(gpu_device, lens, dim=64, hq=hq, hkv=hkv, rows=rows, page=page)
    lse = c.new_lse()
    out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse, decay=0.5)
    c.check_attend(out, lse, *c.oracle_attend(0.5))
    c.check_weight()


def test_the_most_sequences(gpu_device):
    lens = (np.arange(4096) % 7).tolist()
    c = Case(gpu_device, lens, dim=64, hq=1, hkv=1, page=4)
    lse = c.new_lse()
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), lse=lse, decay=0.5)
    c.oracle_append()
    c.check_attend(out, lse, *c.oracle_attend(0.5))
    c.check_weight()
    c.check_pools()
    c.cache.weight.copy_(torch.from_numpy(c.weight).float())       # (both evict by the same numbers)
    c.weight = c.cache.weight.double().cpu().numpy()
    check_evict(c, 3, 1, 1)
    assert c.cache.sync_status() == 0


@pytest.mark.parametrize("dtype,hq,hkv,rows", [("bf16", 32, 8, 16), ("f32", 32, 8, 16), ("bf16", 32, 2, 1), ("f32", 12, 2, 4)])
def test_the_same_bits_whatever_ran_before(gpu_device, dtype, hq, hkv, rows):
    """Partial results of many workgroups, by a merge launch or the one that is done last: the same, with another call's in the scratch before."""
    c = Case(gpu_device, [9000, 5, 0, 2500], dtype=dtype, hq=hq, hkv=hkv, rows=rows)
    q, other, first = c.on(c.q), c.on(c.values(c.q.shape)), None
    for _ in range(3):
        lse = c.new_lse()
        out = c.cache.attend(*c.args(False), q, lse=lse, decay=0.0)
        got = [out, lse, torch.nan_to_num(c.cache.weight, nan=-5.0)]
        first = first or got
        assert all(torch.equal(x, y) for x, y in zip(got, first))
        c.cache.attend(c.d_table[1:], c.d_lens[1:], other[1:].contiguous(), decay=1.0)
    c.check_attend(first[0], first[1], *c.oracle_attend())


# ------------------------------------------------------------------ tables wider than their sequences

def widen(c, pages):
    """The same pools under a table of this many entries a sequence."""
    old = c.cache
    table = np.full((len(c.lens), pages), -1, np.int32)
    table[:, :c.table.shape[1]] = c.table
    cfg = type(old.cfg).from_buffer_copy(old.cfg)
    cfg.table_pages = pages
    c.cache = LtriPagedCache(cfg, c.device, k_pages=old.k_pages, v_pages=old.v_pages, weight=old.weight, pos=old.pos)
    c.cache.scratch.fill_(0xFF)
    c.table = table
    c.push()


@pytest.mark.parametrize("pages", [64, 600, 8192, 1 << 20])
@pytest.mark.parametrize("pairs", PAIRS)
def test_attention_under_a_wide_table(gpu_device, pairs, pages):
    hq, hkv, rows = PAIRS[pairs]
    c = Case(gpu_device, [800, 9, 0], hq=hq, hkv=hkv, rows=rows)
    widen(c, pages)
    lse = c.new_lse()
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), lse=lse, decay=0.5)
    c.oracle_append()
    c.check_attend(out, lse, *c.oracle_attend(0.5))
    c.check_weight()
    c.check_pools()
    assert c.cache.sync_status() == 0


@pytest.mark.parametrize("keep", [20, 490, 700])
@pytest.mark.parametrize("pages", [64, 600, 8192, 1 << 20])
def test_eviction_under_a_wide_table(gpu_device, pages, keep):
    """One, two and five launches, of the same sequences."""
    c = evict_case(gpu_device, [800, 500, 9, 0], "ties", hq=3, hkv=3, dim=64)
    widen(c, pages)
    check_evict(c, keep, 4, 10)
    check_evict(c, keep - 1, 0, 3)
    assert c.cache.sync_status() == 0


# ------------------------------------------------------------------ pages outside the pool

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page", [(128, 16), (64, 16), (128, 8), (128, 64)])
@pytest.mark.parametrize("pairs", PAIRS)
def test_pages_outside_the_pool_in_any_tile(gpu_device, dtype, dim, page, pairs):
    """First, middle and last ones: their tokens have no influence, no weight and no new rows, the others have theirs."""
    hq, hkv, rows = PAIRS[pairs]
    c = Case(gpu_device, [700, 333, 90, 16], dtype=dtype, dim=dim, hq=hq, hkv=hkv, page=page, rows=rows)
    last = [-(-int(n) // page) - 1 for n in c.lens]
    for s, p, bad in ((0, 0, -1), (0, last[0] // 2, 1 << 20), (0, last[0] // 2 + 1, -7), (1, last[1], 1 << 30), (1, last[1] // 3, int(c.cache.cfg.n_pages))):
        c.d_table[s, p], c.table[s, p] = bad, bad
    for p in range(last[3] + 1):                                   # a sequence without a page
        c.d_table[3, p], c.table[3, p] = -1, -1
    for decay in (None, 0.0, 0.5):
        lse = c.new_lse()
        out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse, decay=decay)
        c.check_attend(out, lse, *c.oracle_attend(decay))
        c.check_weight()
        assert c.cache.sync_status() == -1 and c.cache.sync_status() == 0
    lse = c.new_lse()
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), lse=lse, decay=0.5)
    c.oracle_append()
    c.check_attend(out, lse, *c.oracle_attend(0.5))
    c.check_weight()
    c.check_pools()
    assert c.cache.sync_status() == -1
    c.cache.append(*c.args(), c.on(c.k_new), c.on(c.v_new))
    c.check_pools()
    assert c.cache.sync_status() == -1


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("bad", [-1, 1 << 30])
@pytest.mark.parametrize("lens,page,keep", [([300, 320, 310], 16, 200), ([1500, 1600, 900], 16, 700), ([6000, 7000, 5500], 32, 5000), ([17000, 20000, 16500], 128, 9000)])
def test_a_sequence_with_a_page_outside_the_pool_is_not_evicted(gpu_device, lens, page, keep, bad, where):
    """By one launch, two and five; the sequences beside it are, and it is as soon as its table is good."""
    c = evict_case(gpu_device, lens, "any", hq=2, hkv=2, dim=64, page=page)
    last = -(-lens[1] // page) - 1
    p = {"first": 0, "middle": last // 2, "last": last}[where]
    good = int(c.table[1, p])
    c.d_table[1, p], c.table[1, p] = bad, bad
    check_evict(c, keep, 4, 50)
    assert c.d_lens.tolist() == [keep, lens[1], keep]
    assert c.cache.sync_status() == -1 and c.cache.sync_status() == 0
    c.d_table[1, p], c.table[1, p] = good, good
    check_evict(c, keep, 4, 50)
    assert c.d_lens.tolist() == [keep] * 3 and c.cache.sync_status() == 0
    check_evict(c, keep - 100, 4, 50)
    assert c.cache.sync_status() == 0
