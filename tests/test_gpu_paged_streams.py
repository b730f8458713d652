"""The paged cache on other streams than those its buffers were allocated on, and in captured graphs."""
import pytest
import torch

from oracle import paged_oracle as O
from paged_util import Case
from paper_2412_04757_amd import LtriPagedCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("given", ["to set_stream", "at creation"])
def test_a_dropped_cache_keeps_its_memory_until_its_stream_is_done(gpu_device, given):
    """The cache goes while the work of its stream still waits behind other work; what the stream of its buffers allocates then lies elsewhere."""
    c = Case(gpu_device, [900, 20], weights=False)
    old, side = c.cache, torch.cuda.Stream(gpu_device)
    args, q, out = c.args(False), c.on(c.q), torch.empty(c.q.shape, dtype=torch.bfloat16, device=gpu_device)
    busy = first = torch.randn((4096, 4096), device=gpu_device)
    pools, scratch = [x.clone() for x in (old.k_pages, old.v_pages)], torch.empty(old.scratch_bytes, dtype=torch.uint8, device=gpu_device)
    if given == "to set_stream":
        cache = LtriPagedCache(old.cfg, gpu_device, k_pages=pools[0], v_pages=pools[1], scratch=scratch)
    else:
        cache = LtriPagedCache(old.cfg, gpu_device, stream=side, k_pages=pools[0], v_pages=pools[1], scratch=scratch)
    mine = {x.data_ptr(): x.numel() * x.element_size() for x in (*pools, scratch)}
    torch.cuda.synchronize()
    if given == "to set_stream":
        mine[cache.state.data_ptr()] = cache.state.numel()
        cache.set_stream(side)
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ first
    cache.attend(*args, q, out=out)
    del cache, pools, scratch
    done = torch.cuda.Event()
    done.record(side)
    new = [torch.full((n,), 0xFF, dtype=torch.uint8, device=gpu_device) for n in mine.values() for _ in range(3)]
    if not done.query():                                       # (else the memory was free to go)
        for x in new:
            assert all(x.data_ptr() + x.numel() <= p or p + n <= x.data_ptr() for p, n in mine.items())
    torch.cuda.synchronize()
    c.check_attend(out, None, *c.oracle_attend())


def bits(x):
    return torch.nan_to_num(x.float(), nan=-5.0)


@pytest.mark.parametrize("dtype,page,tokens,rows,keep", [
    ("bf16", 16, 700, 5, 320), ("f32", 16, 700, 5, 320),          # tiles through LDS, the keys again for the weights, lists and moves
    ("bf16", 8, 300, 2, 290),                                     # small pages, the eviction in one launch
    ("bf16", 64, 18000, 16, 9000),                                # a merge launch, an eviction by several workgroups
])
def test_captured_calls_of_every_way(gpu_device, dtype, page, tokens, rows, keep):
    """The stream is set inside the capture; every replay, with eager work of another cache in between, is the eager call's to the bit."""
    a = Case(gpu_device, [tokens, 40, 0, tokens // 2], dtype=dtype, hq=32, hkv=2, page=page, rows=rows, room=8 * rows, seed=3)
    twin = LtriPagedCache(a.cache.cfg, gpu_device, k_pages=a.cache.k_pages.clone(), v_pages=a.cache.v_pages.clone(), weight=a.cache.weight.clone(),
                          pos=a.cache.pos.clone())
    table, lens, seen = a.d_table, a.d_lens.clone(), a.d_seen.clone()
    k, v, q = a.on(a.k_new), a.on(a.v_new), a.on(a.q)
    out, lse = torch.empty_like(q), a.new_lse()

    def body(cache, n):
        cache.step(table, n, seen, k, v, q, out=out, lse=lse, decay=0.9)
        cache.evict(table, n, seen, keep, n_sink=4, n_recent=20)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        twin.set_stream(torch.cuda.current_stream())
        body(twin, lens)
    for _ in range(5):
        for x in (k, v, q):
            x.copy_(a.on(a.values(x.shape)))
        seen += rows * (lens > 0).int()
        lens += rows * (lens > 0).int()
        eager = lens.clone()
        body(a.cache, eager)
        want = [out.clone(), lse.clone()]
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(lens, eager)
        for x, y in ((twin.k_pages, a.cache.k_pages), (twin.v_pages, a.cache.v_pages), (twin.weight, a.cache.weight), (twin.pos, a.cache.pos)):
            assert torch.equal(bits(x), bits(y))
    assert int(lens.max()) == keep and a.cache.sync_status() == 0
    twin.set_stream(torch.cuda.current_stream())
    assert twin.sync_status() == 0


@pytest.mark.parametrize("lens,page,keep", [([300, 120, 0], 16, 200), ([1500, 900], 16, 700), ([17000, 12000], 128, 9000)])
def test_lengths_that_are_also_the_tokens_seen(gpu_device, lens, page, keep):
    """One array for both, as before anything was ever evicted; the call writes it."""
    c = Case(gpu_device, lens, hq=2, hkv=2, dim=64, page=page)
    both = c.d_lens
    c.cache.evict(c.d_table, both, both, keep, n_sink=4, n_recent=50)
    O.evict(c.k, c.v, c.weight, c.pos, c.table, c.lens, c.seen, keep, 4, 50)
    assert both.tolist() == c.lens.tolist()
    c.check_pools()
    assert c.cache.sync_status() == 0


def test_two_caches_on_two_streams_at_once(gpu_device):
    """Buffers of their own, the calls of both under way together."""
    cases = [Case(gpu_device, [3000, 41, 0, 800], hq=32, rows=5, seed=7 + i) for i in range(2)]
    streams, got = [torch.cuda.Stream(gpu_device) for _ in cases], []
    inputs = [(c.on(c.k_new), c.on(c.v_new), c.on(c.q), c.new_lse()) for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for c, s, (k, v, q, lse) in zip(cases, streams, inputs):
            c.cache.set_stream(s)
            got.append(c.cache.step(*c.args(), k, v, q, lse=lse, decay=0.0))
    torch.cuda.synchronize()
    for c, out, (_, _, _, lse) in zip(cases, got, inputs):
        c.oracle_append()
        c.check_attend(out, lse, *c.oracle_attend(0.0))
        c.check_weight()
        c.check_pools()
        assert c.cache.sync_status() == 0
