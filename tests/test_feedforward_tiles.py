"""The rule that picks a product's tile (csrc/tile_rule.h), compiled for the host (no GPU needed)."""

import os
import shutil
import subprocess

import pytest

from tests import feedforward_shapes as shapes

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


def test_the_shapes_that_run_every_tile(rule):
    """feedforward_shapes.py: each size takes the tile it stands for, with enough steps and ends inside them."""
    gated = list(shapes.GATED)
    assert [t for t, _ in rule([("gated", M, F) for M, K, F in gated])] == list(shapes.GATED.values())
    assert all(-(-K // 128) >= 9 and K % 64 and M % 64 and F % 128 for M, K, F in gated)  # 17 steps in bf16
    up = lambda n: -(-n // 64) * 64  # noqa: E731
    for table in (shapes.BACKWARD, shapes.BACKWARD_LONG):
        assert [t for t, _ in rule([("16", M, K) for M, K, F in table])] == [x for x, _ in table.values()]
        assert [t for t, _ in rule([("16", up(F) + F, K) for M, K, F in table])] == [w for _, w in table.values()]
    assert all(2 * up(F) * M > 1 << 31 for M, K, F in shapes.BACKWARD_LONG)
    back = list(shapes.BACKWARD)
    assert all(2 * up(F) // 64 >= 6 and -(-M // 64) >= 6 and M % 64 and K % 64 and F % 64 for M, K, F in back)
    product = list(shapes.PRODUCT8)
    assert [t for t, _ in rule([("8", M, N) for M, N, K in product])] == list(shapes.PRODUCT8.values())
    assert all(-(-K // 128) >= 9 and K % 128 and M % 64 and N % 64 for M, N, K in product)
    for tiles in (shapes.GATED.values(), [x for x, _ in shapes.BACKWARD.values()], [w for _, w in shapes.BACKWARD.values()],
                  shapes.PRODUCT8.values()):
        assert set(tiles) == {64, 128, 256}
    for sizes in (gated, back):  # K a multiple of 8, and not, with each
        tile = shapes.GATED if sizes is gated else shapes.BACKWARD
        assert {(tile[s], s[1] % 8 == 0) for s in sizes} == {(tile[s], fits) for s in sizes for fits in (True, False)}
