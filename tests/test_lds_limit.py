"""Launches with dynamic LDS, in the kernels' sources (no GPU needed)."""

import glob
import os
import re

import pytest

from paper_2607_01408_amd import build

RAISES = ("raise_lds_limit<", "hipFuncAttributeMaxDynamicSharedMemorySize")


def arguments(text, at):
    """The arguments of the call whose bracket opens before `at`."""
    depth, parts = 1, [""]
    while depth:
        c = text[at]
        depth += (c in "([{") - (c in ")]}")
        if depth == 1 and c == ",":
            parts.append("")
        elif depth:
            parts[-1] += c
        at += 1
    return [p.strip() for p in parts]


def launches(path):
    """(line, function up to the launch, dynamic LDS) of every launch of a source."""
    text = open(path).read()
    for found in re.finditer(r"hipLaunchKernelGGL\(", text):
        kernel, *args = arguments(text, found.end())
        while kernel.count("<") > kernel.count(">"):  # a template's commas
            kernel += "," + args.pop(0)
        start = max(m.start() for m in re.finditer(r"^[^\s/#}].*\{$|^[^\s/#}][^;{}]*\{$", text[: found.start()], re.M))
        yield text.count("\n", 0, found.start()) + 1, text[start : found.start()], args[2]


SOURCES = sorted(glob.glob(os.path.join(build.CSRC, "*.hip")) + glob.glob(os.path.join(build.CSRC, "*.h")))


@pytest.mark.parametrize("path", SOURCES, ids=[os.path.basename(p) for p in SOURCES])
def test_launches_with_dynamic_lds_raise_its_limit(path):
    """A kernel's dynamic LDS may be up to 64 KB unless its limit was raised: a launch that asks for any raises it first
    (once per device)."""
    for line, before, lds in launches(path):
        if lds != "0":
            assert any(r in before for r in RAISES), f"{os.path.basename(path)}:{line}: {lds} bytes"


def test_the_launches_are_found():
    of = {os.path.basename(p): [lds for _, _, lds in launches(p)] for p in SOURCES}
    assert "lds" in of["linear.hip"] and "lds" in of["sort_index.hip"] and "Tile::kLds" in of["matmul8.hip"]
    assert sum(map(len, of.values())) > 50
