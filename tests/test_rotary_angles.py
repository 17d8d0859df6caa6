"""Cosine and sine of a fixed-point angle (rotary.cu), compiled for the host from the kernel's source, against 64 bits."""
import re
import subprocess

import numpy as np

from oracle.cache import TRIG
from test_kernel_sources import SOURCES

MAIN = r"""
#include <cmath>
#include <cstdint>
#include <cstdio>
#define __device__
#define __forceinline__ inline
struct float2 { float x, y; };
static float2 make_float2(float x, float y) { return float2{x, y}; }
using std::fmaf;
%s
int main(int, char **argv)
{
    FILE *in = fopen(argv[1], "rb"), *out = fopen(argv[2], "wb");
    unsigned long long a;
    while (fread(&a, 8, 1, in) == 1) { const float2 r = turn_to_cos_sin(a); fwrite(&r, 8, 1, out); }
    return fclose(out);
}
"""


def test_all_quadrants_without_overflow(tmp_path):
    # signed overflow ends the program: the rest of a quadrant has to be found without it
    f = re.search(r"__device__ __forceinline__ float2 turn_to_cos_sin\(.*?\n}\n", SOURCES["rotary.cu"], flags=re.S).group(0)
    src, exe, angles, res = (str(tmp_path / n) for n in ("a.cpp", "a", "in", "out"))
    open(src, "w").write(MAIN % f)
    subprocess.check_call(["g++", "-O1", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", "-o", exe, src])
    r = np.random.default_rng(0)
    eighths = (np.arange(8, dtype=np.uint64) << np.uint64(61))[:, None] + np.array([0, 1, 2 ** 32 - 1, 2 ** 32, 2 ** 60, 2 ** 61 - 1], dtype=np.uint64)
    a = np.concatenate((eighths.ravel(), r.integers(0, 2 ** 64, 200000, dtype=np.uint64)))
    a.tofile(angles)
    subprocess.check_call([exe, angles, res])
    got = np.fromfile(res, dtype=np.float32).reshape(-1, 2).astype(np.float64)
    t = 2 * np.pi * a.astype(np.longdouble) / 2 ** 64
    assert max(np.abs(got[:, 0] - np.cos(t)).max(), np.abs(got[:, 1] - np.sin(t)).max()) <= TRIG
