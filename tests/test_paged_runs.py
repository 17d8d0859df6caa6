"""Integer arithmetic of the paged cache's kernels, compiled for the host from their source (paged.cuh)."""
import re
import subprocess

import pytest

from test_kernel_sources import SOURCES

HEAD = r"""
#include <cstdint>
#include <cstdio>
#include <random>
#define __host__
#define __device__
#define __forceinline__ inline
static uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)
"""

RUNS = r"""
int main()
{
    std::mt19937_64 rng(1);
    for (int ctas : {1, 2, 7, 148, 160, 296, 148 * 8, 160 * 8})
        for (int k = 0; k < 300; ++k) {
            // a few units, around the number of runs, up to 10^12 (2^31 rows of thousands of heads, 16 to a unit)
            const int64_t units = k < 20 ? 1 + k : k < 60 ? ctas + k - 40 : (int64_t)(rng() % (k < 180 ? 100000ull : 1000000000000ull)) + 1;
            if (units < 1) continue;
            const Runs r(units, ctas);
            CHECK(r.n == (units < ctas ? units : ctas));
            CHECK(r.begin(0) == 0 && r.begin(r.n) == units && r.begin(ctas) == units);
            for (int b = 0; b < r.n; ++b) {
                const int64_t u0 = r.begin(b), u1 = r.begin(b + 1);
                CHECK(u0 < u1 && u1 - u0 <= units / r.n + 1);             // none is empty, all are alike
                for (int64_t u : {u0, u0 + (u1 - u0) / 2, u1 - 1}) CHECK(r.of(u) == b);
            }
        }
    return 0;
}
"""

DIVISOR = r"""
int main()
{
    std::mt19937_64 rng(2);
    for (int k = 0; k < 20000; ++k) {
        // pages of 8 rows and more, pieces of a row (2 and more)
        const uint32_t d = k < 5000 ? 2 + k : (uint32_t)(rng() % (1u << 30)) / 8 * 8 + 8;
        const Divisor v = make_divisor(d);
        const int64_t most = 0x7fffffff;
        for (int64_t x : {(int64_t)0, (int64_t)d - 1, (int64_t)d, most, most / d * d, most / d * d - 1, (int64_t)(rng() % (most + 1)), (int64_t)(rng() % (most + 1)) / d * d})
            if (x >= 0) CHECK(div_by((int)x, v) == (int)(x / d));
    }
    return 0;
}
"""

PARTS = {
    "runs": (r"struct Runs \{.*?\n\};\n", RUNS),
    "divisor": (r"struct Divisor .*?\n\}\n|__device__ __forceinline__ int div_by\([^\n]*\n", DIVISOR),
}


@pytest.mark.parametrize("part", PARTS)
def test_runs_and_divisions(part, tmp_path):
    pattern, main = PARTS[part]
    code = "".join(m.group(0) for m in re.finditer(pattern, SOURCES["paged.cuh"], flags=re.S))
    src, exe = str(tmp_path / "a.cpp"), str(tmp_path / "a")
    with open(src, "w") as f:
        f.write(HEAD + code + main)
    subprocess.check_call(["g++", "-O1", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", "-o", exe, src])
    done = subprocess.run([exe], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
