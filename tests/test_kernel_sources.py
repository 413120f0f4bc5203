"""What the kernels' sources have to say themselves because no run can be made to show its absence."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2505_10806_amd", "csrc")


def _sources():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip"))):
        lines = [re.sub(r"//.*", "", line).strip() for line in open(path)]
        yield os.path.basename(path), [line for line in lines if line]


def test_barriers_without_memory_order_stand_between_fences():
    """wave_barrier and s_barrier only order scheduling and arrival: what is exchanged through LDS around them needs a release before and an acquire after."""
    found = 0
    for name, lines in _sources():
        for i, line in enumerate(lines):
            scope = "wavefront" if "__builtin_amdgcn_wave_barrier()" in line else "workgroup" if "__builtin_amdgcn_s_barrier()" in line else None
            if scope is None:
                continue
            found += 1
            fence = '__builtin_amdgcn_fence(__ATOMIC_{}, "%s", "local");' % scope
            assert lines[i - 1] == fence.format("RELEASE") and lines[i + 1] == fence.format("ACQUIRE"), f"{name}: {lines[i - 1:i + 2]}"
    assert found >= 3
