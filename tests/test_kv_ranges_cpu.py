"""Whether the arrays of a call's caches overlap, on the host: a small C++ program
with the library's own check, against every pair of ranges."""
import itertools
import os
import subprocess

import numpy as np
import pytest

from test_kv_slots_cpu import PKG

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "ls_kv_ranges.h"

// argv: start and length of each range
int main(int argc, char** a) {
    std::vector<ls::KvRange> r;
    for (int i = 1; i + 1 < argc; i += 2) r.push_back(ls::kv_range((const void*)strtoull(a[i], nullptr, 10), atoll(a[i + 1])));
    printf("%d\n", ls::kv_ranges_meet(r.data(), (int64_t)r.size()));
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    d = tmp_path_factory.mktemp("ranges")
    src, exe = str(d / "ranges.cpp"), str(d / "ranges")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-I", os.path.join(PKG, "csrc"), src, "-o", exe])
    return lambda ranges: bool(int(subprocess.check_output([exe, *(str(x) for r in ranges for x in r)], text=True)))


BASE = 0x7F00_0000_0000


@pytest.mark.parametrize("ranges,want", [
    ([], False), ([(BASE, 64)], False),
    ([(BASE, 64), (BASE + 64, 64)], False),                                         # side by side
    ([(BASE + 64, 64), (BASE, 65)], True),                                          # one byte
    ([(BASE, 64), (BASE + 4096, 64), (BASE, 64)], True),                            # the same one
    ([(BASE, 1 << 40), (BASE + (1 << 39), 1), (BASE + (1 << 41), 1)], True),        # one inside another
    ([(BASE, 1 << 40), (BASE + (1 << 40), 1 << 33), (BASE - 16, 16)], False)])
def test_pairs(meet, ranges, want):
    assert meet(ranges) == want


def test_layers(meet):
    """Four arrays for each of many layers, in any order; then one of them where another lies."""
    r = np.random.RandomState(0)
    for n in (1, 2, 33, 131):
        at = BASE + 1000 * r.permutation(4 * n)
        ranges = [(int(x), 1000 if i % 4 < 2 else 40) for i, x in enumerate(at)]
        assert not meet(ranges)
        for i, j in list(itertools.permutations(range(4), 2)) + [(0, 4 * n - 1), (4 * n - 2, 1)]:
            if i != j:
                assert meet([*ranges[:i], ranges[j], *ranges[i + 1:]])
        assert meet([(ranges[0][0], 1001), (ranges[0][0] + 1000, 40), *ranges[4:]])
