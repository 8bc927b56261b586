"""From work slots to rows in the KV-cache launches, on the host: a small C++
program with the library's own arithmetic prints the rows of every slot of a
launch, sequences being found as the kernels find them."""
import os
import subprocess

import numpy as np
import pytest

PKG = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_00946_amd")

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include "ls_kv_slots.h"

// argv: 'b' shift or 't' G and tile; T, B, B + 1 offsets, B pasts.  A line for each slot: sequence, its first row and
// count, the block or tile's place, its rows' start and end.
int main(int, char** a) {
    const bool blocks = a[1][0] == 'b';
    const int x = atoi(a[2]), tile = atoi(a[3]), T = atoi(a[4]), B = atoi(a[5]);
    auto off = [&](int b) { return std::min(std::max(atoi(a[6 + b]), 0), T); };
    auto first = [&](int b) {
        return blocks ? ls::block_slot(off(b), b, x) : ls::tile_slot(off(b), b, x, tile);
    };
    const long long slots = blocks ? (T >> x) + 2LL * B : (long long)T * x / tile + B;
    for (long long s = 0; s < slots; ++s) {
        int b = 0;                       // the last one that starts at or before the slot, the first where none does
        for (int i = 1; i < B; ++i)
            if (first(i) <= s) b = i;
        const int t0 = off(b), n = std::min(std::max(atoi(a[6 + b + 1]), t0), T) - t0;
        const long long past = std::max(atoll(a[6 + B + 1 + b]), 0LL);
        if (blocks) {
            const ls::BlockRows r = ls::block_rows(s - first(b), n, past, x);
            printf("%d %d %d %lld %d %d\n", b, t0, n, (long long)r.j, r.row0, r.row1);
        } else {
            const ls::TileRows r = ls::tile_rows(s - first(b), n, x, tile);
            printf("%d %d %d %lld %d %d\n", b, t0, n, (long long)r.r0, 0, r.rows);
        }
    }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("slots")
    src, exe = str(d / "slots.cpp"), str(d / "slots")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-I", os.path.join(PKG, "csrc"), src, "-o", exe])

    def run(kind, x, tile, T, off, past):
        out = subprocess.check_output([exe, kind, *map(str, (x, tile, T, len(past), *off, *past))], text=True)
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


# offsets from 0, from past 0 on (slots before the first sequence's), past the call's rows, below 0, not in order
OFFSETS = [[0, 1, 2, 40, 40, 173, 200], [160, 161, 170, 170, 181, 190, 200], [199, 199, 199, 199, 199, 199, 200],
           [40, 300, 400, 500, 600, 700, 800], [-50, -3, 7, 60, 61, 120, 200], [90, 20, 150, 3, 3, 180, 110]]
PASTS = [[0, 15, 300, 17, 2 ** 31 - 1, 5], [0] * 6, [-9, 16, 31, 32, 1000, 2 ** 30]]


@pytest.mark.parametrize("past", PASTS)
@pytest.mark.parametrize("off", OFFSETS)
@pytest.mark.parametrize("shift", [4, 7])
def test_blocks_of_slots(program, shift, off, past):
    """Every slot's rows are rows of its sequence, at places from the sequence's first new one on."""
    T, B, size, seen = 200, len(past), 1 << shift, []
    for b, t0, n, j, row0, row1 in program("b", shift, 0, T, off, past):
        if row0 >= row1:
            continue
        p = max(past[b], 0)
        assert j >= p >> shift and 0 <= row0 and row1 <= size
        assert p <= j * size + row0 and j * size + row1 <= p + n and 0 <= t0 and t0 + n <= T
        seen += [(b, j * size + r - p) for r in range(row0, row1)]
    if list(off) == sorted(off) and off[0] >= 0 and off[-1] <= T:
        want = [(b, i) for b in range(B) for i in range(off[b + 1] - off[b])]
        assert sorted(seen) == want


@pytest.mark.parametrize("off", OFFSETS)
@pytest.mark.parametrize("G", [1, 3, 8, 40])
def test_tiles_of_slots(program, G, off):
    """Every slot's rows are rows of its sequence; rows before the first sequence are no tile's."""
    T, past, seen = 200, PASTS[0], []
    for b, t0, n, r0, _, rows in program("t", G, 128, T, off, past):
        if rows == 0:
            continue
        assert 0 <= r0 and 0 < rows <= 128 and r0 + rows <= n * G and t0 + n <= T
        seen += [(b, r0 + r) for r in range(rows)]
    if list(off) == sorted(off) and off[0] >= 0 and off[-1] <= T:
        assert sorted(seen) == [(b, r) for b in range(len(past)) for r in range((off[b + 1] - off[b]) * G)]


def test_large_offsets(program):
    """Products beyond 32 bits."""
    T, G = 2 ** 30 - 1, 1024
    # the program is asked for few slots: the arithmetic alone
    assert np.int64(T) * G // (2 ** 30) + 1 == len(program("t", G, 2 ** 30, T, [0, T], [0]))
