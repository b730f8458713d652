"""The paged cache against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paged_util import Case, TYPES
from paper_2412_04757_amd import LtriPagedCache, paged_config

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ attention

# lengths around tiles and pages, empty and single ones, one that dwarfs the others
LENS = ([1], [0], [31, 32, 33], [0, 1, 700, 64, 0, 17], [5000], [2049, 3, 128, 129, 127, 300, 40, 999])


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("dtype,dim,hq,hkv,page,rows", [
    ("bf16", 128, 8, 2, 16, 1), ("bf16", 128, 4, 4, 64, 1), ("bf16", 64, 8, 1, 1, 2), ("bf16", 128, 14, 2, 8, 3), ("bf16", 128, 32, 1, 32, 1),
    ("bf16", 64, 6, 2, 256, 16), ("f32", 64, 4, 1, 32, 1), ("f32", 128, 8, 2, 16, 4), ("f32", 128, 3, 3, 128, 1), ("bf16", 128, 8, 2, 2, 5),
    ("f32", 128, 12, 2, 16, 7), ("f32", 64, 10, 2, 4, 6), ("bf16", 128, 10, 2, 64, 6), ("bf16", 64, 31, 1, 32, 1), ("f32", 64, 31, 1, 16, 1),
    ("bf16", 64, 4, 2, 4096, 2),
])
def test_attend(gpu_device, lens, dtype, dim, hq, hkv, page, rows):
    c = Case(gpu_device, lens, dtype=dtype, dim=dim, hq=hq, hkv=hkv, page=page, rows=rows)
    for decay in (None, 0.0, 0.5):
        lse = c.new_lse()
        out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse, decay=decay)
        want, want_lse = c.oracle_attend(decay)
        c.check_attend(out, lse, want, want_lse)
        c.check_weight()
    c.check_pools()
    assert c.cache.sync_status() == 0


def test_attend_64_rows_of_many_heads(gpu_device):
    c = Case(gpu_device, [400, 63, 64, 10], hq=32, hkv=2, rows=64)
    lse = c.new_lse()
    out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse, decay=1.0)
    c.check_attend(out, lse, *c.oracle_attend(1.0))
    c.check_weight()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_many_sequences(gpu_device, dtype):
    """More sequences than a wavefront has lanes, and than a workgroup has threads."""
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 90, 600).tolist()
    c = Case(gpu_device, lens, dtype=dtype, dim=64, hq=2, hkv=1, page=8)
    lse = c.new_lse()
    out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse, decay=1.0)
    c.check_attend(out, lse, *c.oracle_attend(1.0))
    c.check_weight()
    # a part of the batch, by rows of the same tables
    part = c.cache.attend(c.d_table[100:163], c.d_lens[100:163], c.on(c.q[100:163]))
    want, _ = O.attend(c.k, c.v, None, c.table[100:163], c.lens[100:163], c.q[100:163])
    c.check_attend(part, None, want, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sequences_that_share_pages(gpu_device, dtype):
    """A common beginning, held once: three sequences name its pages, a fourth is one of them again."""
    c = Case(gpu_device, [160, 500, 97, 160], dtype=dtype, rows=2, weights=False)
    c.table[1, :6], c.table[2, :6], c.table[3] = c.table[0, :6], c.table[0, :6], c.table[0]
    c.push()
    lse = c.new_lse()
    q = c.on(c.q)
    q[3], c.q[3] = q[0], c.q[0]
    out = c.cache.attend(*c.args(False), q, lse=lse)
    c.check_attend(out, lse, *c.oracle_attend())
    c.check_pools()
    assert c.cache.sync_status() == 0


def test_weights_of_pages_named_twice_stay_in_bounds(gpu_device):
    """Weights want every page named once: a batch that holds more tokens than the pool is reported, and nothing but weights is touched."""
    c = Case(gpu_device, [640] * 12, page=64, spare=0)
    c.table[1:] = c.table[0]
    c.push()
    n_pages = 10
    cfg = paged_config(c.hq, c.hkv, c.dim, c.dtype, page_tokens=64, n_pages=n_pages, table_pages=10, max_seqs=12, rows_max=1, weights=True)
    small = [x[torch.from_numpy(c.table[0]).long().to(gpu_device)].contiguous() for x in (c.cache.k_pages, c.cache.v_pages, c.cache.weight, c.cache.pos)]
    guard = torch.full((1 << 20,), 0xFF, dtype=torch.uint8, device=gpu_device)
    probe = LtriPagedCache(cfg, gpu_device, k_pages=small[0], v_pages=small[1], weight=small[2], pos=small[3])
    scratch = torch.cat([torch.full((probe.scratch_bytes,), 0xFF, dtype=torch.uint8, device=gpu_device), guard])
    cache = LtriPagedCache(cfg, gpu_device, k_pages=small[0], v_pages=small[1], weight=small[2], pos=small[3], scratch=scratch)
    table = torch.arange(10, dtype=torch.int32, device=gpu_device).repeat(12, 1)
    out = cache.attend(table, c.d_lens, c.on(c.q), decay=1.0)
    want, _ = O.attend(c.k, c.v, None, c.table, c.lens, c.q)
    c.check_attend(out, None, want, None)
    assert bool((scratch[probe.scratch_bytes:] == 0xFF).all())
    assert cache.sync_status() == -3
    cache.evict(table, c.d_lens, c.d_lens.clone(), 100)
    assert bool((scratch[probe.scratch_bytes:] == 0xFF).all())
    cache.sync_status()


def test_attend_gives_the_same_bits_again(gpu_device):
    c = Case(gpu_device, [4000, 17, 900, 0, 2500], rows=2)
    q, runs = c.on(c.q), []
    for _ in range(3):
        lse = c.new_lse()
        out = c.cache.attend(*c.args(False), q, lse=lse, decay=0.0)
        runs.append((out, lse, c.cache.weight.clone()))
    for r in runs[1:]:
        assert all(torch.equal(torch.nan_to_num(x, nan=-5.0), torch.nan_to_num(y, nan=-5.0)) for x, y in zip(r, runs[0]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pools_in_token_order(gpu_device, dtype):
    """[page][token][KV head][d], as views."""
    c = Case(gpu_device, [70, 300], dtype=dtype, rows=2, token_major=True)
    assert c.cache.cfg.token_stride > c.cache.cfg.head_stride
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), decay=0.5)
    c.oracle_append()
    c.check_attend(out, None, *c.oracle_attend(0.5))
    c.check_weight()
    c.check_pools()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_is_not_touched_by_tokens_it_does_not_see(gpu_device, dtype):
    """The last new token holds infinities and NaN: the rows before it do not see it, the last row does."""
    c = Case(gpu_device, [333, 40, 32], dtype=dtype, rows=3)
    for s, n in enumerate(c.lens):
        p, i = c.table[s][(n - 1) // c.page], (n - 1) % c.page
        c.v[p, 0, i, ::3], c.v[p, 1, i, ::5] = np.inf, np.nan
        c.k[p, 1, i, 7] = np.nan
    c.cache.k_pages.copy_(c.on(c.k))
    c.cache.v_pages.copy_(c.on(c.v))
    lse = c.new_lse()
    out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want, want_lse = c.oracle_attend()
    t = c.tolerances()
    assert (np.abs(out[:, :2] - want[:, :2]) <= t["out_abs"] + 1.01 * t["out_rel"] * np.abs(want[:, :2])).all()
    assert (np.abs(lse.cpu().numpy()[:, :2] - want_lse[:, :2]) <= t["lse"]).all()
    assert not np.isfinite(out[:, 2, :4, ::3]).any() and np.isnan(out[:, 2, 4:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_any_size(gpu_device, dtype):
    """Scores far below and above zero, and -infinity for some or for all tokens of a sequence."""
    c = Case(gpu_device, [200, 200, 200, 200], dtype=dtype, hq=2, hkv=1, weights=False)
    c.q[:] = 0.0
    c.q[:, :, :, 0] = 1.0
    scores = np.random.default_rng(0).normal(size=200)
    for s, x in enumerate((scores - 3e4, scores + 3e4, np.where(np.arange(200) < 100, -np.inf, scores), np.full(200, -np.inf))):
        i = np.arange(200)
        c.k[c.table[s][i // c.page], 0, i % c.page, 0] = c.round(x)
    c.cache.k_pages.copy_(c.on(c.k))
    lse = c.new_lse()
    out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse)
    want, want_lse = c.oracle_attend()
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    # a score of 3e4 / sqrt(128), in the log2 domain, is held to 2^-24 of 3.9e3: its probability to 2^-12
    vmax = np.nanmax(np.abs(c.v))
    assert (np.abs(got - want) <= 2.0 ** -10 * vmax + 1.01 * torch.finfo(TYPES[dtype]).eps / 2 * np.abs(want)).all()
    assert (np.abs(got_lse[:3] - want_lse[:3]) <= 2.0 ** -10).all()
    assert (got[3] == 0).all() and np.isneginf(got_lse[3]).all()


# 80 pairs of query row and head: a block of 64, whose wavefronts share tiles, and one of 16, of whose wavefronts one has pairs

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [list(range(0, 330, 11)), [37 * i % 200 for i in range(300)], [5000, 3, 2000, 1]])
def test_many_pairs_over_few_and_many_tiles(gpu_device, dtype, lens):
    c = Case(gpu_device, lens, dtype=dtype, hq=32, rows=5)
    lse = c.new_lse()
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), lse=lse, decay=0.5)
    c.oracle_append()
    c.check_attend(out, lse, *c.oracle_attend(0.5))
    c.check_weight()
    c.check_pools()
    assert c.cache.sync_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_pairs_and_pages_outside_the_pool(gpu_device, dtype):
    c = Case(gpu_device, [700, 401, 90], dtype=dtype, hq=32, rows=5, weights=False)
    for s, p, bad in ((0, 3, -1), (0, 4, 1 << 20), (0, 20, -7), (1, 0, 1 << 30), (1, 11, -1)):
        c.d_table[s, p], c.table[s, p] = bad, bad
    lse = c.new_lse()
    out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse)
    c.check_attend(out, lse, *c.oracle_attend())
    assert c.cache.sync_status() == -1 and c.cache.sync_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_pairs_are_not_touched_by_tokens_they_do_not_see(gpu_device, dtype):
    c = Case(gpu_device, [333, 40, 32, 900], dtype=dtype, hq=32, rows=5)
    for s, n in enumerate(c.lens):
        p, i = c.table[s][(n - 1) // c.page], (n - 1) % c.page
        c.v[p, 0, i, ::3], c.v[p, 1, i, ::5], c.k[p, 1, i, 7] = np.inf, np.nan, np.nan
    c.cache.k_pages.copy_(c.on(c.k))
    c.cache.v_pages.copy_(c.on(c.v))
    lse = c.new_lse()
    out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse).double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want, want_lse = c.oracle_attend()
    t = c.tolerances()
    assert (np.abs(out[:, :4] - want[:, :4]) <= t["out_abs"] + 1.01 * t["out_rel"] * np.abs(want[:, :4])).all()
    assert (np.abs(lse.cpu().numpy()[:, :4] - want_lse[:, :4]) <= t["lse"]).all()
    assert not np.isfinite(out[:, 4, :16, ::3]).any() and np.isnan(out[:, 4, 16:]).all()


def test_pool_beyond_32_bit_offsets(gpu_device):
    """Pages whose rows lie past 2^32 elements."""
    n_pages, page, hkv, d, T = 70000, 64, 8, 128, 5 * 64 + 9
    cfg = paged_config(16, hkv, d, "bf16", page_tokens=page, n_pages=n_pages, table_pages=6, max_seqs=2, rows_max=1)
    k = torch.empty((n_pages, hkv, page, d), dtype=torch.bfloat16, device=gpu_device)
    v = torch.empty_like(k)
    cache = LtriPagedCache(cfg, gpu_device, k_pages=k, v_pages=v)
    table = torch.tensor([[69999, 65537, 3, 65535, 69998, 32769], [65536, 1, 69000, 2, 32768, 0]], dtype=torch.int32, device=gpu_device)
    g = torch.Generator(device=gpu_device).manual_seed(1)
    rows = [torch.randn((2, hkv, T, d), generator=g, device=gpu_device).bfloat16() for _ in range(2)]
    lens = torch.tensor([T, T], dtype=torch.int32, device=gpu_device)
    cache.append(table, lens, None, *rows)
    q = torch.randn((2, 1, 16, d), generator=g, device=gpu_device).bfloat16()
    out = cache.attend(table, lens, q)
    for s in range(2):
        for pool, x in ((k, rows[0]), (v, rows[1])):
            got = pool[table[s].long()].transpose(1, 2).reshape(-1, hkv, d)[:T]
            assert torch.equal(got, x[s].transpose(0, 1))
        kk, vv = (x[s].double().repeat_interleave(2, 0) for x in rows)
        p = torch.softmax((kk * q[s, 0].double()[:, None]).sum(-1) / d ** 0.5, -1)
        want = (p[:, :, None] * vv).sum(1)
        # (scores to 2^-14, probabilities to 2^-16, and the rounding of the result)
        assert bool(((out[s, 0].double() - want).abs() <= 2.0 ** -11 + 1.01 * 2.0 ** -8 * want.abs()).all())
    assert cache.sync_status() == 0


# ------------------------------------------------------------------ new rows

@pytest.mark.parametrize("dtype,dim,page,rows,lens", [
    ("bf16", 128, 16, 1, [1, 16, 17, 0, 300]), ("bf16", 64, 4, 37, [37, 40, 200, 0, 12]), ("f32", 64, 8, 5, [5, 3, 9]), ("f32", 128, 64, 700, [700, 1300, 0, 650]),
])
@pytest.mark.parametrize("given", [False, True])
def test_append(gpu_device, dtype, dim, page, rows, lens, given):
    """Rows to their places, those before the sequence's beginning dropped (a padded batch), everything else as it was."""
    c = Case(gpu_device, lens, dtype=dtype, dim=dim, page=page, rows=rows, max_rows=1, seen=[n + 1000 for n in lens])
    w = torch.rand((len(lens), c.hkv, rows), generator=c.gen) if given else None
    c.cache.append(*c.args(), c.on(c.k_new), c.on(c.v_new), w_new=None if w is None else w.to(gpu_device))
    c.oracle_append(None if w is None else w.numpy())
    c.check_pools()
    assert np.array_equal(c.cache.weight.cpu().numpy(), c.weight.astype(np.float32), equal_nan=True)
    assert c.cache.sync_status() == 0


@pytest.mark.parametrize("dtype,dim,hq,hkv,page,rows", [("bf16", 128, 8, 2, 16, 1), ("bf16", 64, 12, 4, 8, 7), ("f32", 128, 4, 4, 32, 2), ("f32", 64, 4, 1, 1, 4)])
@pytest.mark.parametrize("weights", [False, True])
def test_step(gpu_device, dtype, dim, hq, hkv, page, rows, weights):
    lens = [rows, 100, 0, 1234, 33, rows + 31, 1]
    c = Case(gpu_device, lens, dtype=dtype, dim=dim, hq=hq, hkv=hkv, page=page, rows=rows, weights=weights, seen=[n + 50 for n in lens])
    decay = 0.75 if weights else None
    lse = c.new_lse()
    out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), lse=lse, decay=decay)
    c.oracle_append()
    c.check_attend(out, lse, *c.oracle_attend(decay))
    c.check_pools()
    if weights:
        c.check_weight()
    # the same as the two calls
    again = c.cache.attend(*c.args(False), c.on(c.q), lse=lse)
    assert torch.equal(again, out)
    # weights left alone: those of new tokens are 0
    if weights:
        before = c.cache.weight.clone()
        c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q))
        c.weight = before.double().cpu().numpy()
        c.oracle_append()
        assert np.array_equal(c.cache.weight.cpu().numpy(), c.weight.astype(np.float32), equal_nan=True)
    assert c.cache.sync_status() == 0


def test_pages_outside_the_pool_and_lengths_beyond_the_table_are_reported(gpu_device):
    """Their tokens do not count and are not written; the other sequences are served; the report is given once."""
    for bad, status in ((-1, -1), (1 << 20, -1), (None, -3)):
        c = Case(gpu_device, [100, 64, 90], page=16, rows=2, room=6)
        if bad is None:
            c.d_lens[1] = 200
        else:
            c.d_table[1, 3], c.table[1, 3] = bad, bad
        out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), decay=1.0)
        if bad is None:
            c.lens[1] = 0
        c.oracle_append()
        c.check_attend(out, None, *c.oracle_attend(1.0))
        c.check_pools()
        c.check_weight()
        assert c.cache.sync_status() == status and c.cache.sync_status() == 0
        c.cache.append(*c.args(), c.on(c.k_new), c.on(c.v_new))
        c.check_pools()
        assert c.cache.sync_status() == status
        before = c.cache.weight.clone()
        c.cache.evict(*c.args(), 70)
        c.weight = before.double().cpu().numpy()
        O.evict(c.k, c.v, c.weight, c.pos, c.table, c.lens, c.seen, 70)
        c.check_pools()
        want = c.lens.copy()
        if bad is None:
            want[1] = 200
        assert c.d_lens.tolist() == want.tolist()
        assert c.cache.sync_status() == (status if bad is None else 0)      # (64 tokens of the second sequence: not evicted, not looked at)


# ------------------------------------------------------------------ eviction

def evict_case(gpu_device, lens, kind, **kw):
    """Weights by kind; positions as earlier evictions leave them, in any order."""
    c = Case(gpu_device, lens, seen=[3 * n + 5 for n in lens], rows=1, **kw)
    rng = np.random.default_rng(11)
    for s, T in enumerate(lens):
        if not T:
            continue
        i = np.arange(T)
        pg, sl = c.table[s][i // c.page], i % c.page
        for h in range(c.hkv):
            w = {"any": lambda: rng.gamma(0.3, size=T), "ties": lambda: rng.integers(0, 3, T).astype(float), "zero": lambda: np.zeros(T),
                 "odd": lambda: rng.choice([np.nan, np.inf, -np.inf, 0.0, -0.0, -1.5, 1e-42, 3e38, -3e38], T), "signed": lambda: rng.normal(size=T)}[kind]()
            c.weight[pg, h, sl] = w.astype(np.float32)
            c.pos[pg, h, sl] = rng.permutation(np.sort(rng.choice(3 * T + 5, T, replace=False)))
    c.cache.weight.copy_(torch.from_numpy(c.weight).float())
    c.cache.pos.copy_(torch.from_numpy(c.pos).int())
    return c


def check_evict(c, keep, sink, recent):
    c.cache.evict(*c.args(), keep, n_sink=sink, n_recent=recent)
    O.evict(c.k, c.v, c.weight, c.pos, c.table, c.lens, c.seen, keep, sink, recent)
    assert c.d_lens.tolist() == c.lens.tolist()
    c.check_pools()
    got, want = c.cache.weight.cpu().numpy(), c.weight.astype(np.float32)
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("kind", ["any", "ties", "zero", "odd", "signed"])
@pytest.mark.parametrize("lens,page,keep,sink,recent", [
    ([2], 1, 1, 0, 0), ([9, 10, 11, 0, 1], 4, 10, 2, 3), ([1025, 1024, 1023, 64], 16, 1000, 4, 100), ([5000], 64, 37, 0, 37),
    ([3001, 700, 2500], 32, 2499, 4, 600), ([4097, 40], 8, 4096, 0, 0), ([300], 16, 200, 200, 0), ([17000, 20000], 128, 9000, 4, 1000),
])
def test_evict(gpu_device, kind, lens, page, keep, sink, recent):
    c = evict_case(gpu_device, lens, kind, hq=3, hkv=3, dim=64, page=page)
    check_evict(c, keep, sink, recent)
    check_evict(c, keep, sink, recent)                     # nothing more to do
    if keep > 40:
        check_evict(c, 40, 0, 40)
    assert c.cache.sync_status() == 0


@pytest.mark.parametrize("dtype,dim,token_major", [("f32", 128, False), ("bf16", 128, True), ("f32", 64, True)])
def test_evict_rows_of_every_width(gpu_device, dtype, dim, token_major):
    c = evict_case(gpu_device, [600, 90], "any", hq=4, hkv=2, dtype=dtype, dim=dim, token_major=token_major)
    check_evict(c, 75, 4, 20)


@pytest.mark.parametrize("kind,keep,lens", [
    ("any", 60000, [140000, 3000, 70001]), ("any", 139000, [140000, 139001, 500]), ("any", 500, [90000, 501, 0]), ("ties", 40000, [90000, 40001]),
    ("zero", 8192, [70000, 8193, 16384]), ("odd", 30000, [50000]), ("signed", 32768, [65536, 32769]), ("odd", 33000, [41000, 40900]),
])
def test_evict_long(gpu_device, kind, keep, lens):
    """Tables that several workgroups select from."""
    c = evict_case(gpu_device, lens, kind, hq=2, hkv=2, dim=64, page=64)
    check_evict(c, keep, 4, 300)
    check_evict(c, keep, 4, 300)
    check_evict(c, keep // 2, 0, 7)


def test_positions_that_repeat_keep_the_count(gpu_device):
    """Every token protected: the first ones stay, and still exactly `keep` of them."""
    c = evict_case(gpu_device, [500], "any", hkv=2)
    c.pos[c.pos >= 0] = 0
    c.cache.pos.copy_(torch.from_numpy(c.pos).int())
    check_evict(c, 123, 1, 5)


def test_evict_takes_a_large_keep(gpu_device):
    c = evict_case(gpu_device, [100], "any")
    check_evict(c, 2 ** 31 - 1, 4, 2 ** 31 - 8)
    check_evict(c, 111, 0, 0)


# ------------------------------------------------------------------ together

@pytest.mark.parametrize("dtype,rows", [("bf16", 1), ("f32", 3)])
def test_a_prompt_then_tokens_in_a_bounded_cache(gpu_device, dtype, rows):
    """A prompt goes in in pieces, its last rows weigh its tokens, it is evicted to a budget; then steps of `rows` tokens with an eviction
    whenever the cache has 24 more than the budget. The oracle follows on its own rows; it takes the library's weights before an
    eviction, so that both evict by the same numbers."""
    keep, sink, recent = 150, 4, 32
    lens = [400, 90, 251]
    c = Case(gpu_device, lens, dtype=dtype, hq=8, hkv=2, page=16, rows=rows, room=100, max_rows=8)
    width, hkv = c.table.shape[1], c.hkv
    # the prompt again, through append, in pieces of 64
    full = [c.lens.copy(), c.k.copy(), c.v.copy()]
    for pool in (c.cache.k_pages, c.cache.v_pages, c.cache.weight):
        pool.fill_(float("nan"))
    for base in range(0, 400, 64):
        n = 64
        kn, vn = np.zeros((3, hkv, n, c.dim)), np.zeros((3, hkv, n, c.dim))
        now = np.array([min(x, base + 64) for x in lens], np.int32)
        for s in range(3):                                # the piece ends at now[s]; what was there already is written again
            for i in range(n):
                at = int(now[s]) - n + i
                if at >= 0:
                    p = c.table[s][at // c.page]
                    kn[s, :, i], vn[s, :, i] = full[1][p, :, at % c.page], full[2][p, :, at % c.page]
        d = torch.from_numpy(now).to(gpu_device)
        c.cache.append(c.d_table, d, d, c.on(kn), c.on(vn))
    c.weight[np.isfinite(c.weight)] = 0.0
    c.check_pools()
    c.q = c.values((3, 8, 8, c.dim))
    lse = c.new_lse()
    out = c.cache.attend(*c.args(False), c.on(c.q), lse=lse, decay=0.0)
    c.check_attend(out, lse, *c.oracle_attend(0.0))
    c.check_weight()

    def evict():
        c.weight = c.cache.weight.double().cpu().numpy()
        c.cache.evict(*c.args(), keep, n_sink=sink, n_recent=recent)
        O.evict(c.k, c.v, c.weight, c.pos, c.table, c.lens, c.seen, keep, sink, recent)
        assert c.d_lens.tolist() == c.lens.tolist()
        c.check_pools()
        assert np.array_equal(c.cache.weight.cpu().numpy(), c.weight.astype(np.float32), equal_nan=True)

    evict()
    for t in range(40):
        c.q, c.k_new, c.v_new = c.values((3, rows, 8, c.dim)), c.values((3, hkv, rows, c.dim)), c.values((3, hkv, rows, c.dim))
        c.d_lens += rows
        c.d_seen += rows
        c.lens += rows
        c.seen += rows
        lse = c.new_lse()
        out = c.cache.step(*c.args(), c.on(c.k_new), c.on(c.v_new), c.on(c.q), lse=lse, decay=1.0)
        c.oracle_append()
        c.check_attend(out, lse, *c.oracle_attend(1.0))
        if c.lens.max() >= keep + 24:
            # (weights of up to 24 steps: each adds its own rounding)
            got = c.cache.weight.double().cpu().numpy()
            there = ~np.isnan(c.weight)
            assert np.array_equal(there, ~np.isnan(got))
            assert (np.abs(got - c.weight)[there] <= 2.0 ** -12 * np.abs(c.weight[there]) + 2.0 ** -28).all()
            evict()
    # the latest tokens and the first ones are there, once each
    for s in range(3):
        i = np.arange(int(c.lens[s]))
        got = c.cache.pos.cpu().numpy()[c.table[s][i // c.page], :, i % c.page]
        for h in range(hkv):
            p = set(got[:, h].tolist())
            assert len(p) == len(i) and set(range(sink)) <= p and set(range(int(c.seen[s]) - recent, int(c.seen[s]))) <= p
    assert c.cache.sync_status() == 0


def test_captured_steps_follow_lengths_and_tables(gpu_device):
    """A captured step and eviction, replayed with other lengths, tables and rows, gives what eager calls give; a second graph shares the scratch."""
    a = Case(gpu_device, [50, 300, 0, 700], hq=8, hkv=2, rows=1, room=64, seed=5)
    side = torch.cuda.Stream(gpu_device)
    b_cfg = a.cache.cfg
    twin = LtriPagedCache(b_cfg, gpu_device, k_pages=a.cache.k_pages.clone(), v_pages=a.cache.v_pages.clone(), weight=a.cache.weight.clone(),
                          pos=a.cache.pos.clone(), scratch=a.cache.scratch)
    table, lens, seen = a.d_table.clone(), a.d_lens.clone(), a.d_seen.clone()
    k, v, q = a.on(a.k_new), a.on(a.v_new), a.on(a.q)
    out, lse = torch.empty_like(q), a.new_lse()

    def body(cache, n):
        cache.step(table, n, seen, k, v, q, out=out, lse=lse, decay=0.9)
        cache.evict(table, n, seen, 320, n_sink=4, n_recent=20)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        twin.set_stream(side)
        start = [x.clone() for x in (twin.k_pages, twin.v_pages, twin.weight, twin.pos)]
        body(twin, lens.clone())                          # warm
        for x, y in zip((twin.k_pages, twin.v_pages, twin.weight, twin.pos), start):
            x.copy_(y)
        side.synchronize()
        graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            body(twin, lens)
        probe = torch.empty_like(q)
        with torch.cuda.graph(other, stream=side):
            twin.attend(table, lens, q, out=probe)
    for t in range(6):
        new = [a.values(x.shape) for x in (k, v, q)]
        order = torch.randperm(4, generator=a.gen).to(gpu_device)
        for x, y in zip((k, v, q), new):
            x.copy_(a.on(y))
        # sequences change places, and grow by one unless they are padding
        for x in (table, lens, seen):
            x.copy_(x[order].clone())
        seen += (lens > 0).int()
        lens += (lens > 0).int()
        eager_lens = lens.clone()
        a.cache.step(table, eager_lens, seen, k, v, q, out=out, lse=lse, decay=0.9)
        want = [out.clone(), lse.clone()]
        a.cache.evict(table, eager_lens, seen, 320, n_sink=4, n_recent=20)
        want_probe = a.cache.attend(table, eager_lens, q)
        torch.cuda.synchronize()
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        other.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(lens, eager_lens) and torch.equal(probe, want_probe)
        for x, y in ((twin.k_pages, a.cache.k_pages), (twin.v_pages, a.cache.v_pages), (twin.weight, a.cache.weight), (twin.pos, a.cache.pos)):
            assert torch.equal(torch.nan_to_num(x.float(), nan=-5.0), torch.nan_to_num(y.float(), nan=-5.0))
    assert twin.sync_status() == 0 and a.cache.sync_status() == 0


def test_work_goes_to_the_stream_that_is_set(gpu_device):
    c = Case(gpu_device, [900, 20])
    there, q = c.on(c.q), torch.zeros(c.q.shape, dtype=torch.bfloat16, device=gpu_device)
    out, busy = torch.zeros_like(q), torch.randn((4096, 4096), device=gpu_device)
    side = torch.cuda.Stream(gpu_device)
    c.cache.set_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):                         # the queries come behind other work of that stream
        for _ in range(20):
            busy = busy @ busy
        q.copy_(there)
    c.cache.attend(*c.args(False), q, out=out)
    side.synchronize()
    c.check_attend(out, None, *c.oracle_attend())


def test_a_cache_of_another_stream_than_the_current_one(gpu_device):
    """What it allocates (pools, results) is filled on its own stream, whatever the current one is busy with."""
    c = Case(gpu_device, [900, 20], weights=False)
    k, v = np.zeros((2, c.hkv, 900, c.dim)), np.zeros((2, c.hkv, 900, c.dim))
    for s, n in enumerate(c.lens):
        i = np.arange(n)
        for to, pool in ((k, c.k), (v, c.v)):
            to[s, :, 900 - n:] = pool[c.table[s][i // c.page], :, i % c.page].transpose(1, 0, 2)
    rows = c.on(k), c.on(v)
    args, q, busy = c.args(False), c.on(c.q), torch.randn((4096, 4096), device=gpu_device)
    side = torch.cuda.Stream(gpu_device)
    torch.cuda.synchronize()
    for _ in range(20):
        busy = busy @ busy
    cache = LtriPagedCache(c.cache.cfg, gpu_device, stream=side)
    cache.append(*args, None, *rows)
    out = cache.attend(*args, q)
    for _ in range(4):                                    # (results take memory of that stream: nothing of the current one lands in them)
        torch.empty_like(q).fill_(7.0)
    torch.cuda.synchronize()
    c.check_attend(out, None, *c.oracle_attend())
    assert cache.sync_status() == 0


def test_two_caches_share_a_scratch(gpu_device):
    """Two layers, one after the other on one stream."""
    a = Case(gpu_device, [700, 90], seed=1)
    b = Case(gpu_device, [33, 800], seed=2)
    big = max(a.cache.scratch_bytes, b.cache.scratch_bytes)
    scratch = torch.full((big,), 0xFF, dtype=torch.uint8, device=gpu_device)
    for c in (a, b):
        old = c.cache
        c.cache = LtriPagedCache(old.cfg, gpu_device, k_pages=old.k_pages, v_pages=old.v_pages, weight=old.weight, pos=old.pos, scratch=scratch)
    outs = [(c, c.cache.attend(*c.args(False), c.on(c.q), decay=1.0)) for _ in range(2) for c in (a, b)]
    for c, out in outs[:2]:
        c.check_attend(out, None, *c.oracle_attend(1.0))
    for (c, x), (_, y) in zip(outs[:2], outs[2:]):
        assert torch.equal(x, y)
