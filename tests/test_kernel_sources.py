"""Properties of the kernel sources that no result shows reliably."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_21817_b200", "csrc")
SOURCES = {os.path.basename(p): open(p).read() for p in sorted(glob.glob(os.path.join(CSRC, "*.cu*")))}


def test_waits_for_tensor_memory_loads_name_the_registers():
    # a wait without them orders memory only: the compiler may use the registers before it
    found = 0
    for name, src in SOURCES.items():
        for m in re.finditer(r'asm volatile\(\s*"tcgen05\.wait::ld[^;]*;"(.*?)\);', src, flags=re.S):
            found += 1
            assert '"+r"' in m.group(1), name
    assert found >= 2


def test_device_functions_of_the_blocks_around_the_sublayer_are_called():
    code = {n: re.sub(r"//[^\n]*|/\*.*?\*/", "", t, flags=re.S) for n, t in SOURCES.items()}
    everything = "\n".join(code.values())
    for name in ("ptx.cuh", "layernorm.cu", "attention.cu", "attention_simt.cu", "attention_tc.cu"):
        for f in re.findall(r"__device__ __forceinline__ [\w:<>\*& ]*?(\w+)\(", code[name]):
            assert len(re.findall(rf"\b{f}\b", everything)) > 1, (name, f)
