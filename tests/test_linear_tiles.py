"""The rule that picks the linear layer's tiles and slices (csrc/tile_rule.h), compiled for the host (no GPU needed)."""

import os
import shutil
import subprocess

import pytest

from tests import linear_shapes as shapes

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_01408_amd", "csrc")
MAIN = """
#include <cstdio>
#include "tile_rule.h"
using namespace spingtp;
int main() {
    int eight;
    long long m, n, steps;
    while (std::scanf("%d %lld %lld %lld", &eight, &m, &n, &steps) == 4) {
        const SumShape s = sum_shape(eight ? kSlices8 : kSlices16, m, n, steps, eight ? 4 : 1);
        std::printf("%d %d %lld %lld\\n", s.tile, s.parts, (long long)s.slices, (long long)s.per);
    }
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
        """[(tile, parts, slices, steps of a slice)] of [(8 bits, rows, columns, steps)]."""
        text = "".join(f"{int(e)} {m} {n} {s}\n" for e, m, n, s in cases)
        out = subprocess.run([str(at / "rule")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]

    return pick


def test_what_a_launch_and_a_workspace_hold(rule):
    sizes = [1, 64, 65, 300, 1000, 5_000, 1 << 18, 1 << 22, 300_000_000, (1 << 31) - 1]
    steps = [1, 2, 3, 4, 7, 8, 9, 15, 16, 24, 43, 64, 128, 1000, 1563, 65_535, 1 << 25]
    cases = [(e, m, n, s) for e in (False, True) for m in sizes for n in sizes for s in steps
             if -(-m // 256) * -(-n // 256) <= MOST]
    for (eight, m, n, s), (tile, parts, slices, per) in zip(cases, rule(cases)):
        what = (eight, m, n, s, tile, parts, slices, per)
        tiles = -(-m // tile) * -(-n // tile)
        assert tile in (64, 128, 256) and tiles <= MOST, what
        # slices cover the sum, the last one has a part of it, and all leave in a launch and in bounded memory
        assert slices == -(-s // per) and (slices == 1 or (slices * tiles <= 1024 and per >= 4)), what
        if slices == 1:
            assert per == s, what
        last = s - (slices - 1) * per
        assert last >= 1, what
        if eight:  # scales are read by words of four steps
            assert slices == 1 or per % 4 == 0, what
            assert parts == 1 or (per % 8 == 0 and last % 8 == 0), what
        if parts > 1:
            assert parts == 2 and tile < 256 and s >= 8, what


def test_the_shapes_that_run_every_tile(rule):
    """linear_shapes.py: each size takes what it stands for, in each of the products."""
    up = lambda n, m: -(-n // m)  # noqa: E731
    seen = set()
    for eight, table in ((False, shapes.FORWARD16), (True, shapes.FORWARD8)):
        got = rule([(eight, M, N, up(K, 128 if eight else 64)) for M, K, N in table])
        for want, (tile, parts, slices, _) in zip(table.values(), got):
            assert want == (tile, parts, slices > 1)
            seen.add((eight, tile, parts, slices > 1))
    for e in (False, True):
        for tile, parts in ((64, 1), (64, 2), (128, 1), (128, 2), (256, 1)):
            assert any(s[:3] == (e, tile, parts) for s in seen), (e, tile, parts)
        assert any(s[0] == e and s[3] for s in seen)
    dx = rule([(False, M, K, up(N, 64)) for M, K, N in shapes.BACKWARD])
    dw = rule([(False, N, K, up(M, 64)) for M, K, N in shapes.BACKWARD])
    for (x, w), a, b in zip(shapes.BACKWARD.values(), dx, dw):
        assert (x, w) == ((a[0], a[1], a[2] > 1), (b[0], b[1], b[2] > 1))
    for got in (dx, dw):
        assert {(t, p) for t, p, _, _ in got} >= {(64, 1), (64, 2), (128, 1), (128, 2), (256, 1)}
        assert any(s > 1 for _, _, s, _ in got)
