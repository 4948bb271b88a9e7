"""The Newton-Schulz products in the compiler's assembly (no GPU): what keeps their loads in flight, how many of
their waves a SIMD holds, and the order in which shared tiles' partial sums are released."""
import re

import pytest

from test_kernel_assembly import assembly


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    return assembly("newton_schulz.hip", tmp_path_factory.mktemp("asm"))


def bodies(lines, pattern):
    for at, line in enumerate(lines):
        if re.match(r"_ZN\S*" + pattern + r"\S*:", line):
            end = next(i for i in range(at, len(lines)) if lines[i].strip().startswith(".section"))
            yield line.split(":")[0], [x.split(";")[0].split() for x in lines[at:end] if x.startswith("\t") and x.split(";")[0].split()]


def test_memory_is_addressed_as_global(lines):
    """A flat load shares a counter with LDS and returns in any order: every wait would wait for all of them."""
    assert not [x for x in lines if re.match(r"\s+flat_(load|store)", x)]


def test_registers(lines):
    """No spills; two workgroups of 64 x 64 (4 waves) and of eight waves with 32 x 32 fit a compute unit."""
    text = "\n".join(lines)
    assert set(re.findall(r"\.vgpr_spill_count:\s+(\d+)", text)) == {"0"}
    counts = dict(re.findall(r"\.name:\s+(\S+)(?:(?!\.name:)[\s\S])*?\.vgpr_count:\s+(\d+)", text))
    wide = [int(v) for n, v in counts.items() if "k_ns_directILi64E" in n]
    many = [int(v) for n, v in counts.items() if "k_ns_directILi32ELi8E" in n]
    assert wide and max(wide) <= 256 and many and max(many) <= 128


def test_partial_sums_are_waited_for_before_they_are_released(lines):
    """stores of the partial tile, a wait for them, the barrier, then thread 0's write-back and counter."""
    seen = 0
    for name, body in bodies(lines, "k_ns_tiles"):
        ops = [x[0] for x in body]
        back = ops.index("buffer_wbl2")
        barrier = max(i for i in range(back) if ops[i] == "s_barrier")
        store = max(i for i in range(barrier) if ops[i].startswith("global_store"))
        waits = [body[i] for i in range(store, barrier) if ops[i] == "s_waitcnt"]
        assert any("vmcnt(0)" in x for w in waits for x in w), name
        add = ops.index("global_atomic_add", back)
        assert any(ops[i] == "s_waitcnt" and "vmcnt(0)" in " ".join(body[i]) for i in range(back, add)), name
        assert "buffer_inv" in ops[add:], name
        seen += 1
    assert seen >= 15, seen
