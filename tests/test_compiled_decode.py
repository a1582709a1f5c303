"""What the compiled kernels of attention and eviction must not hold: spilled registers, whose loads stand among those of the tiles under way and are
waited for with them (the blocks of eight waves took twice as long with ten in a step), and packed fp32 arithmetic."""
import re

import pytest

from test_compiled_code import kernels


@pytest.mark.parametrize("source,least", [("attend.hip", 90), ("evict.hip", 7)])
def test_nothing_is_spilled_or_packed(source, least):
    found = kernels(source)
    assert len(found) >= least
    for name, body in found:
        assert not re.search(r"^\s+scratch_", body, re.M), f"{name} uses scratch memory"
        assert not re.search(r"^\s+v_pk_(add|mul|fma)_f32", body, re.M), name


def test_tiles_under_way_are_not_waited_for():
    """Waves that have keys of their own have two stages of loads under way: between a stage's first product and the next stage's loads, no wait is for all
    of them.  (Where the compiler does not know that the queries have landed, it waits for everything in front of every stage's products.)"""
    waves = [(name, body) for name, body in kernels("attend.hip") if "attend_wave_kernelILi128" in name and "ELi1ELi1E" in name]
    assert len(waves) == 2
    for name, body in waves:
        loops = [b for b in re.split(r"^\.LBB", body, flags=re.M) if "Loop" in b.split("\n", 1)[0] and "v_mfma" in b]
        assert loops, name
        for b in loops:
            ops = re.findall(r"^\s+(v_mfma|s_waitcnt[^\n]*)", b, re.M)
            inside = ops[ops.index("v_mfma"):len(ops) - ops[::-1].index("v_mfma")]
            assert not any("vmcnt(0)" in op for op in inside), name
