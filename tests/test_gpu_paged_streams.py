"""Buffers of the paged cache on other streams than those they were allocated on."""
import pytest
import torch

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
