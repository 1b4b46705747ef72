"""The rule that picks a product's tile (csrc/tile_rule.h), compiled for the host (no GPU needed)."""

import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_01408_amd", "csrc")
MAIN = """
#include <cstdio>
#include <cstring>
#include "tile_rule.h"
using namespace spingtp;
int main() {
    char kind[8];
    long long m, n;
    while (std::scanf("%7s %lld %lld", kind, &m, &n) == 3)
        std::printf("%d %d\\n",
                    !std::strcmp(kind, "gated") ? gated_tile(m, n) : product_tile(!std::strcmp(kind, "8") ? kPlain8 : kPlain16, m, n),
                    !std::strcmp(kind, "gated") ? gated_fits(m, n) : product_fits(m, n));
}
"""
MOST = 1 << 22


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++") or shutil.which("amdclang++", path="/opt/rocm/bin")
    at = tmp_path_factory.mktemp("tiles")
    (at / "main.cpp").write_text(MAIN)
    subprocess.run([cxx, "-std=c++17", "-Wall", "-I", CSRC, str(at / "main.cpp"), "-o", str(at / "rule")], check=True)

    def pick(cases):
        """[(tile, whether it fits)] of [(kind, rows, columns)], kind "8", "16" or "gated"."""
        text = "".join(f"{k} {m} {n}\n" for k, m, n in cases)
        out = subprocess.run([str(at / "rule")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]

    return pick


def test_a_tile_that_one_launch_holds(rule):
    """Whatever fits in the largest tiles gets tiles that a launch holds."""
    sizes = [1, 64, 65, 300, 5_000, 1 << 18, 1 << 22, (1 << 28) + 1, 300_000_000, 1 << 30, (1 << 30) + 1, (1 << 31) - 1]
    cases = [(k, m, n) for k in ("8", "16", "gated") for m in sizes for n in sizes]
    fitting = 0
    for (kind, m, n), (tile, fits) in zip(cases, rule(cases)):
        columns = 128 if kind == "gated" else tile
        assert fits == (-(-m // 256) * -(-n // (128 if kind == "gated" else 256)) <= MOST)
        if fits:
            fitting += 1
            assert -(-m // tile) * -(-n // columns) <= MOST, (kind, m, n, tile)
    assert fitting > 100
