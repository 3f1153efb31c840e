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
    long long other, other_heads;   // where another matrix of the same strides begins, and its heads; 0 of them: none
    while (scanf("%lld %lld %lld %lld %lld %lld %lld", &row, &head, &rows, &heads, &len, &other, &other_heads) == 7) {
        const char* const at = (const char*)((long long)1 << 46);
        const tbe::HeadRuns a{at, row, head, rows, heads, len}, b{at + other, row, head, rows, other_heads, len};
        puts((other_heads ? !tbe::runs_meet(a, b) && !tbe::runs_meet(b, a) : tbe::runs_apart(a)) ? "1" : "0");
    }
}
"""


@pytest.fixture(scope="module")
def apart(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "p.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2508_03854_amd", "csrc"), str(d / "p.cpp"), "-o", str(d / "p")], check=True)

    def ask(cases):
        r = subprocess.run([str(d / "p")], input="\n".join(" ".join(map(str, (*c, 0, 0)[:7])) for c in cases), capture_output=True, text=True, check=True)
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


def test_two_matrices_against_every_byte(apart):
    cases = [(row, head, rows, heads, n, at, others) for row, head, rows, heads, n, others in itertools.product((0, 1, 3, 7, 12, 20), (0, 2, 5, 9, 40), (1, 2, 4), (1, 2, 3), (1, 4), (1, 3))
             for at in (-45, -20, -12, -7, -4, -3, -1, 0, 1, 2, 4, 5, 8, 11, 12, 23, 41)]
    for c, got in zip(cases, apart(cases)):
        row, head, rows, heads, n, at, others = c
        a = {r * row + h * head + e for r in range(rows) for h in range(heads) for e in range(n)}
        b = {at + r * row + h * head + e for r in range(rows) for h in range(others) for e in range(n)}
        assert got == (not a & b), c


def test_two_matrices_of_full_size(apart):
    big = 2 ** 31 - 1
    cases = {(6144, 256, big, 16, 256, 4096, 4): True, (6144, 256, big, 16, 256, 4095, 4): False, (6144, 256, big, 16, 256, 6144 * 2 ** 30, 16): False,
             (6144, 256, big, 16, 256, 6144 * 2 ** 30 + 4096, 8): True, (6144, 256, big, 16, 256, 6144 * 2 ** 30 + 4096, 9): False,
             (2 ** 42, 2 ** 31, big, 1024, 1024, 2 ** 41 + 1024, 1024): True, (2 ** 42, 2 ** 31, big, 1024, 1024, 2 ** 41 + 1023, 1024): True,
             (2 ** 42, 2 ** 31, big, 1024, 1024, 2 ** 40 + 1023, 1024): False, (256, 256 * big, big, 8, 256, 256 * big * 8, 8): True}
    for (c, want), got in zip(cases.items(), apart(cases)):
        assert got == want, c
