"""Checks of the KV cache's calls on drafts and pages that need no GPU: null
contexts are refused, the binding's structs have the header's fields, and the
kernels' own arithmetic (a C++ program around ls_kv_slots.h) deals every part of
a tree once and gives the bits that the definition gives."""
import os
import re
import subprocess

import numpy as np
import pytest

import kv_draft_oracle as kd
from paper_2606_00946_amd import lodestar
from test_abi_cpu import HEADER
from test_kv_slots_cpu import PKG

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "ls_kv_slots.h"

// argv: 'p' pairs tiles: pair and tile of each part; or 'b', then any number of (rel, n, gone, sink, lo, hi): the bits
int main(int argc, char** a) {
    if (a[1][0] == 'p') {
        const uint32_t pairs = atoi(a[2]), tiles = atoi(a[3]);
        for (uint32_t i = 0; i < pairs * tiles; ++i) {
            const ls::TreePlace p = ls::tree_place(i, pairs, tiles);
            printf("%u %u\n", p.pair, p.tile);
        }
        return 0;
    }
    for (int i = 2; i + 5 < argc; i += 6)
        printf("%u\n", ls::tree_bits(atoi(a[i]), atoi(a[i + 1]), atoi(a[i + 2]), atoi(a[i + 3]),
                                     strtoull(a[i + 4], nullptr, 10), strtoull(a[i + 5], nullptr, 10)));
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("drafts")
    src, exe = str(d / "drafts.cpp"), str(d / "drafts")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I",
                           os.path.join(PKG, "csrc"), src, "-o", exe])
    return lambda *args: subprocess.check_output([exe, *map(str, args)], text=True).split()


@pytest.mark.parametrize("pairs", [1, 3, 7, 8, 9, 16, 61])
@pytest.mark.parametrize("tiles", [1, 2, 3, 17])
def test_parts_are_dealt_once(program, pairs, tiles):
    got = np.array(program("p", pairs, tiles), int).reshape(-1, 2)
    assert sorted(map(tuple, got)) == [(p, t) for p in range(pairs) for t in range(tiles)]
    # a full group's tiles of one pair lie eight parts apart
    at = {tuple(x): i for i, x in enumerate(got)}
    for p in range(pairs & ~7):
        assert [at[p, t] - at[p, 0] for t in range(tiles)] == [8 * t for t in range(tiles)]


def test_bits_follow_the_definition(program):
    r = np.random.RandomState(0)
    args, want = [], []
    for _ in range(3000):
        past, n = int(r.randint(0, 80)), int(r.randint(1, 150))
        tok = 16 * int(r.randint(0, (past + n) // 16 + 2))
        pos, window, sinks = past + int(r.randint(0, 9)), int(r.choice([0, 1, 5, 16, 40, 1000])), int(r.choice([0, 3, 16, 90]))
        row = r.rand(192) < r.choice([0.0, 0.5, 1.0])                   # bits beyond n do not count
        mask = [int(w) for w in kd.words(row[None], 3)[0]]
        rel = tok - past
        w = rel >> 6
        word = lambda i: mask[i] if 0 <= i < 3 else 0  # noqa: E731
        gone = max(pos - window, -1) + 1 - tok if window else 0
        args += [rel, n, gone, sinks - tok, word(w), word(w + 1)]
        bits = 0
        for i in range(16):
            j = tok + i
            if j < past:
                sees = not window or j > pos - window or j < sinks
            else:
                sees = j - past < n and row[j - past]
            bits |= int(sees) << i
        want.append(bits)
    got = []
    for i in range(0, len(args), 6000):
        got += map(int, program("b", *args[i:i + 6000]))
    assert got == want


def test_null_context_is_refused():
    lib, bad = lodestar.library(), lodestar.LS_ERR_INVALID
    assert lib.ls_kv_append_at(None, None, None, None, None, None, 0, None, 0, None, 0, 1, None, 0, None) == bad
    assert lib.ls_kv_attention_tree(None, None, None, None, None, 0, 1, 1.0, 0, 0, None, 0, None) == bad
    assert lib.ls_kv_keep(None, None, 1, None, None, None, None) == bad
    assert lib.ls_kv_fork(None, None, 1, 1, 1, None, None, 1, None, None, None, None) == bad
    assert lib.ls_kv_compact(None, None, 1, 1, 1, None, None, None, None, None) == bad


@pytest.mark.parametrize("struct", [lodestar.ls_positions, lodestar.ls_tree])
def test_structs_follow_the_header(struct):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + struct.__name__ + ";", text).group(1)
    names = [n.strip(" *\n") for line in body.split(";") for n in re.sub(r"^\s*(const )?\w+\s*", "", line).split(",")]
    assert [n for n in names if n] == [f[0] for f in struct._fields_]


def test_the_oracles_codes_round_to_nearest():
    import kv_oracle as ko
    for fmt in ("fp8", "int8"):
        c = np.array([i for i in range(256) if np.isfinite(ko.code_values(np.uint8([i]), fmt))[0] and (fmt == "fp8" or i != 128)], np.uint8)
        np.testing.assert_array_equal(kd.code_of(ko.code_values(c, fmt), fmt), c)
    assert kd.code_of(np.array([2.5, 3.5, -0.5]), "int8").tolist() == [2, 4, 0]
    # halfway between e4m3's 16 and 18, and 18 and 20: to the even code
    assert ko.E4M3[kd.code_of(np.array([17.0, 19.0, 1000.0]), "fp8")].tolist() == [16.0, 20.0, 448.0]


def test_compaction_of_the_oracle():
    table, where, used, moves = kd.compact(8, np.array([[7, 3, -1], [3, 9, 6]]))
    assert used == 3 and moves == [(3, 0), (6, 1), (7, 2)]
    assert table.tolist() == [[2, 0, -1], [0, 9, 1]] and where.tolist() == [-1, -1, -1, 0, -1, -1, 1, 2]
