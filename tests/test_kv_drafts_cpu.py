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

// argv: 'l' units, heads, wanted stretches: the pieces of every stretch (stretch, head, units, first and last stretch of the
// head, slot); 'p' stretches tiles: stretch and tile of each workgroup; 'b', then any number of (rel, n, gone, sink, lo,
// hi): the bits
int main(int argc, char** a) {
    if (a[1][0] == 'l') {
        const int units = atoi(a[2]), heads = atoi(a[3]);
        const long long part = units + ls::kTreeStart, line = part * heads, per = ls::tree_stretch(units, heads, atoi(a[4]));
        const long long w = (line + per - 1) / per;
        for (long long s = 0; s < w; ++s) {
            const long long lo = s * per, hi = lo + per < line ? lo + per : line;
            for (long long h = lo / part; h * part < hi; ++h) {
                const long long place = h * part;
                const int u0 = ls::tree_cut(lo - place, units), u1 = place + part <= hi ? units : ls::tree_cut(hi - place, units);
                if (u0 >= u1) continue;
                const ls::TreePieces p = ls::tree_pieces(place, units, per);
                const long long slot = u0 > 0 || u1 < units ? (long long)ls::tree_slot(p.first, (int)(s - p.first)) : -1;
                printf("%lld %lld %d %d %lld %lld %lld\n", s, h, u0, u1, (long long)p.first, (long long)p.last, slot);
            }
        }
        return 0;
    }
    if (a[1][0] == 'p') {
        const int w = atoi(a[2]), tiles = atoi(a[3]);
        for (int i = 0; i < w * tiles; ++i) {
            const ls::TreePlace p = ls::tree_place(i, w, tiles);
            printf("%d %d\n", p.stretch, p.tile);
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


@pytest.mark.parametrize("heads", [1, 2, 3, 8])
@pytest.mark.parametrize("units", [1, 2, 7, 8, 9, 14, 40, 333, 5000])
def test_every_unit_is_dealt_once(program, units, heads):
    """A head's pieces follow each other over its units, a stretch each, in slots of their own; none is tiny."""
    for want in (1, 2, 3, 5, 7, 8, 9, 16, 31, 64, 200, 512):
        got = np.array(program("l", units, heads, want), int).reshape(-1, 7)
        assert got[:, 0].max() < want
        slots = got[got[:, 6] >= 0, 6]
        assert len(set(slots)) == len(slots) and (slots < 2 * want).all()
        assert set(got[:, 1]) == set(range(heads))
        for h in range(heads):
            mine = got[got[:, 1] == h]
            assert mine[0, 2] == 0 and mine[-1, 3] == units and (mine[1:, 2] == mine[:-1, 3]).all()
            assert (np.diff(mine[:, 0]) == 1).all()
            if len(mine) > 1:
                assert (mine[:, 4] == mine[0, 0]).all() and (mine[:, 5] == mine[-1, 0]).all()
                assert (mine[:, 3] - mine[:, 2]).min() >= 4 and (mine[:, 6] >= 0).all()
            else:
                assert mine[0, 6] == -1


@pytest.mark.parametrize("units,want,each", [(3, 512, 1), (16, 8, 1), (16, 5, 2), (16, 4, 2), (16, 3, 3), (16, 1, 8)])
def test_short_heads_stay_whole(program, units, want, each):
    got = np.array(program("l", units, 8, want), int).reshape(-1, 7)
    assert got[:, :2].tolist() == [[i // each, i] for i in range(8)]


@pytest.mark.parametrize("stretches", [1, 3, 7, 8, 9, 16, 61])
@pytest.mark.parametrize("tiles", [1, 2, 3, 17])
def test_every_stretch_and_tile_has_a_workgroup(program, stretches, tiles):
    got = np.array(program("p", stretches, tiles), int).reshape(-1, 2)
    assert sorted(map(tuple, got)) == [(s, t) for s in range(stretches) for t in range(tiles)]
    # of a full group, the tiles of one stretch lie eight workgroups apart
    at = {tuple(x): i for i, x in enumerate(got)}
    for s in range(stretches & ~7):
        assert [at[s, t] - at[s, 0] for t in range(tiles)] == [8 * t for t in range(tiles)]


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
