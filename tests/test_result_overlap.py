"""Strided results whose heads lie on each other: the library's host-side check, compiled on its own, against counting every byte."""
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
#include <stdio.h>
#include "tbe_overlap.h"
int main() {
    long long row, head, rows, heads, len;
    while (scanf("%lld %lld %lld %lld %lld", &row, &head, &rows, &heads, &len) == 5)
        puts(tbe::runs_apart(tbe::HeadRuns{nullptr, row, head, rows, heads, len}) ? "1" : "0");
}
"""


@pytest.fixture(scope="module")
def apart(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2508_03854_amd", "csrc"), str(d / "p.cpp"), "-o", str(d / "p")], check=True)

    def ask(cases):
        r = subprocess.run([str(d / "p")], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True)
        return [x == "1" for x in r.stdout.split()]

    return ask


def test_against_every_byte(apart):
    cases = list(itertools.product(range(0, 14), range(0, 14), range(1, 5), range(1, 5), (1, 2, 3, 5)))
    for c, got in zip(cases, apart(cases)):
        row, head, rows, heads, n = c
        taken = [r * row + h * head + e for r in range(rows) for h in range(heads) for e in range(n)]
        assert got == (len(set(taken)) == len(taken)), c


def test_layouts_of_full_size(apart):
    big = 2 ** 31 - 1
    cases = {(4096, 128, big, 32, 128): True, (128, big * 128, big, 1024, 128): True, (128, 128, big, 2, 128): False, (128, 128, 1, 1024, 128): True,
             (2 ** 40 - 1, 2 ** 40 - 1, big, 1024, 128): False, (384, 256, 2, 2, 128): True, (384, 256, 3, 4, 128): False,
             (128, (big - 1) * 128, big, 2, 128): False, (2 ** 40 - 1, 2 ** 39, big, 2, 256): True, (2 ** 40 - 2, 2 ** 39 - 1, big, 3, 256): False}
    for (c, want), got in zip(cases.items(), apart(cases)):
        assert got == want, c
