"""A wave barrier orders instructions and not memory: where lanes of a wave exchange
numbers through shared memory, a fence for the compiler stands before it."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_05033_amd", "csrc")


def test_wave_barriers_stand_behind_fences():
    barriers, bare = 0, []
    for path in sorted(glob.glob(os.path.join(CSRC, "*"))):
        if not path.endswith((".h", ".hip")):
            continue
        with open(path) as f:
            lines = [line.strip() for line in f]
        for i, line in enumerate(lines):
            if "__builtin_amdgcn_wave_barrier" in line and not line.startswith("//"):
                barriers += 1
                if not re.match(r'__builtin_amdgcn_fence\(__ATOMIC_\w+, "wavefront"\);', lines[i - 1]):
                    bare.append(f"{os.path.basename(path)}:{i + 1}")
    assert barriers > 0 and bare == []


def test_bytes_in_shared_memory_are_aligned():
    """They are read as words and more, which a byte's own alignment does not allow."""
    found, bare = 0, []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip"))):
        with open(path) as f:
            for number, line in enumerate(f, 1):
                if re.search(r"__shared__[^;]*\buint8_t\b", line):
                    found += 1
                    if "__align__" not in line:
                        bare.append(f"{os.path.basename(path)}:{number}")
    assert found > 0 and bare == []
