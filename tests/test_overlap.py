"""Whether two matrices of strided rows share memory (csrc/overlap.h), compiled for the host (no GPU needed)."""

import os
import random
import shutil
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_01408_amd", "csrc")
MAIN = """
#include <cstdio>
#include "overlap.h"
int main() {
    long long v[8];
    while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld", v, v + 1, v + 2, v + 3, v + 4, v + 5, v + 6, v + 7) == 8) {
        const Rows a(reinterpret_cast<const void*>(v[0]), v[1], v[2], v[3], 2), b(reinterpret_cast<const void*>(v[4]), v[5], v[6], v[7], 4);
        std::printf("%d%d\\n", overlap(a, b), overlap(b, a));
    }
}
"""


def touched(first, rows, columns, ld, width):
    return {first + (r * ld + c) * width + i for r in range(rows) for c in range(columns) for i in range(width)}


def test_against_the_bytes(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++") or shutil.which("amdclang++", path="/opt/rocm/bin")
    (tmp_path / "main.cpp").write_text(MAIN)
    subprocess.run([cxx, "-std=c++17", "-Wall", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    rng, cases = random.Random(1), []
    for k in range(20_000):
        one, two = [[rng.randrange(0, 7), rng.randrange(0, 6), 0] for _ in range(2)]
        one[2] = max(1, one[1]) + rng.randrange(12)
        two[2] = max(1, two[1]) + rng.randrange(6)
        if k % 2:  # one pitch in bytes
            one[2] = 2 * two[2]
            one[1] = min(one[1], one[2])
        cases.append([1000 + 2 * rng.randrange(60), *one, 1000 + 2 * rng.randrange(60), *two])
    text = "\n".join(" ".join(map(str, c)) for c in cases)
    got = subprocess.run([str(tmp_path / "main")], input=text, capture_output=True, text=True, check=True).stdout.split()
    assert len(got) == len(cases)
    met = 0
    for c, g in zip(cases, got):
        want = bool(touched(*c[:4], 2) & touched(*c[4:], 4))
        met += want
        assert g == ("11" if want else "00"), c
    assert 5_000 < met < 15_000
