"""What the compiler makes of the paged cache's kernels, where correctness or speed hangs on what no result shows reliably."""
import re

import pytest

from test_device_code import resources


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """Instructions, and bytes of private memory and LDS, of every kernel."""
    code, sizes = {}, {}
    for source in ("paged_attend.hip", "paged_cache.hip"):
        where = tmp_path_factory.mktemp("device")
        sizes.update(resources(source, where))
        for line in (where / "device.s").read_text().splitlines():
            line = line.split(";")[0].strip()
            if re.match(r"_Z\w+:$", line):
                body = code.setdefault(line[:-1], [])
            elif line.startswith(".Lfunc_end"):
                body = []
            elif code and line and (not line.startswith(".") or line.startswith(".LBB")):
                body.append(line)
    return code, sizes


def test_no_kernel_spills(compiled):
    """Tiles stay in registers: private memory would go through the caches in every tile."""
    sizes = {k: v for k, v in compiled[1].items() if "paged" in k}
    assert len(sizes) == 24 + 4 + 2 + 4 + 6 + 6 and all(private == 0 for private, _ in sizes.values()), sizes
    # two workgroups of an attention kernel share a compute unit
    assert all(2 * lds <= 160 << 10 for k, (_, lds) in sizes.items() if "attend" in k)


def test_stores_are_complete_before_a_ticket_is_taken(compiled):
    """A barrier alone leaves stores of the other wavefronts in flight, so each has to wait for its own (vmcnt counts stores) right before it."""
    seen = 0
    for name, body in compiled[0].items():
        if not re.search("paged_attend_kernel|paged_long_keys_kernel|paged_long_select_kernel", name):
            continue
        tickets = [i for i, x in enumerate(body) if re.match(r"global_atomic_add v\d+, .* sc0$", x) and "offset" not in x]
        assert len(tickets) == 1, name
        barrier = max(i for i in range(tickets[0]) if body[i].startswith("s_barrier"))
        block = []                                   # the instructions in front of the barrier, back to a label or branch
        for x in reversed(body[:barrier]):
            if x.startswith((".LBB", "s_cbranch", "s_branch")):
                break
            block.append(x)
        assert any(re.match(r"s_waitcnt .*vmcnt\(0\)", x) for x in block), f"{name}: {block[:8]}"
        seen += 1
    assert seen == 24 + 2


def test_the_ring_in_lds_is_fed_without_registers(compiled):
    """Where four wavefronts share tiles: rows go straight into LDS, and a wait for part of them stands in front of a barrier."""
    rings = {k: v for k, v in compiled[0].items() if any(x.startswith("global_load_lds_dwordx4") for x in v)}
    assert sorted(rings) == sorted(k for k in compiled[0] if re.search("paged_attend_kernelILi[01]ELi128ELi4ELb0E", k)) and len(rings) == 2
    for name, body in rings.items():
        meets = [i for i, x in enumerate(body) if re.match(r"s_waitcnt vmcnt\((0|8)\) lgkmcnt\(0\)$", x) and body[i + 1].startswith("s_barrier")]
        assert {re.search(r"vmcnt\((\d)\)", body[i]).group(1) for i in meets} == {"0", "8"}, name
