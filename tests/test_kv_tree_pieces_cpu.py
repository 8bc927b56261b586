"""The cases of kv_tree_cases reach what they are there for: the kernel's division of the work
carried out on the host, with stretches and pieces from the library's own arithmetic (the program of
test_kv_drafts_cpu)."""
import math

import numpy as np
import pytest

import kv_tree_cases
from test_kv_drafts_cpu import program  # noqa: F401

START, TRIES, WORKSPACE = 6, 6, 64 << 20
CASES = kv_tree_cases.cases()


def tile_rows(c, n_cu, limit):
    rows = [n * c["G"] for _, n in c["seqs"]]
    tiles = min(sum(rows) // 32 + len(rows) // 2, -(-max(rows) // 32) * len(rows))
    many = max(rows) > 32 and tiles * c["H"] > 2 * n_cu
    return 64 if c["D"] != 256 and (many or (max(rows) >= 256 and sum(rows) * limit >= 1 << 26)) else 32


def units(c, past, n, limit):
    """128-token units of what the sequence's rows see."""
    end = min(past + n, limit)
    lo = min(max(past + 1 - c["window"], 0), end) if c["window"] else 0
    sink, win = (min(c["sinks"], lo) + 15) // 16, lo // 16
    if sink >= win:
        sink = win = 0
    return max(-(-(sink + (end + 15) // 16 - win) // 8), 1)


def divide(program, c):  # noqa: F811
    """(rows of a tile, [(pieces of a head, units of each)] of every sequence)."""
    f32 = np.float32
    n_cu = c["cus"] or 256
    limit = max(c["width"], max(-(-(p + n) // 16) * 16 for p, n in c["seqs"]))
    rows = tile_rows(c, n_cu, limit)
    fit = min(n_cu * 2, (WORKSPACE - 65536 - 512) // (rows * (c["D"] + 2) * 8), 4096)
    seqs = [(units(c, p, n, limit), -(-n * c["G"] // rows)) for p, n in c["seqs"]]
    lines = [(u + START) * c["H"] for u, _ in seqs]
    total, tiles = f32(sum(f32(x) * f32(t) for x, (_, t) in zip(lines, seqs))), sum(t for _, t in seqs)
    for k in range(TRIES + 1):
        share = f32(0.3) + f32(0.7) / f32(TRIES - 1) * f32(k)
        room = max(f32(fit) - f32(tiles) * share, f32(0))
        each = f32(2) * total / f32(fit) if k == TRIES else total / room if room else f32(math.inf)
        dealt = []
        for x, (u, t) in zip(lines, seqs):
            want = max(int(min(math.ceil(f32(x) / each), fit)), 1)
            dealt.append(np.array(program("l", u, c["H"], want), int).reshape(-1, 7))
        ways = [int(d[:, 0].max()) + 1 for d in dealt]
        groups, cut = (sum(w * t for w, (_, t) in zip(ways, seqs) if w > least) for least in (0, 1))
        if (groups if k < TRIES else cut) <= fit:
            return rows, [[d[d[:, 1] == h, 3] - d[d[:, 1] == h, 2] for h in range(c["H"])] for d in dealt]
    raise AssertionError("nothing is cut")


@pytest.mark.parametrize("name", CASES)
def test_cases_reach_what_they_are_for(program, name):  # noqa: F811
    c = CASES[name]
    rows, heads = divide(program, c)
    pieces = max((h for s in heads for h in s), key=len)
    most = max(int(h.max()) for s in heads for h in s)
    print(f"{name}: tiles of {rows} rows, {len(pieces)} pieces of {pieces.min()} to {pieces.max()} steps, {most} at most")
    assert rows == c["reaches"][0] and len(pieces) >= c["reaches"][1] and most >= c["reaches"][2]
    if c["reaches"][1] > 1:                      # in long pieces and several of them: the cut head's own
        assert pieces.max() >= c["reaches"][2]
    assert c["reaches"][1] > 1 or len(pieces) == 1
