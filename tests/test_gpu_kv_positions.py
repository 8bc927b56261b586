"""Appending with positions given row by row on several axes, on the GPU.

Against ls_kv_append with a table whose row for each place holds the angles that the
axes ask for: the same arithmetic, so the same bits.  Against the rotation in 64 bits:
half a step of the 16-bit output (2^-8 of its size in bf16, 2^-11 in half), and three
roundings in fp32 of at most the pair's size each, 2^-22 of it together.
"""
import numpy as np
import pytest

import kv_draft_oracle as kd
from gpu_helpers import note
from paper_2606_00946_amd import lodestar
from test_gpu_kv import Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = lodestar.Context(16, (64, 64))
    yield c
    c.close()


# places in their sequences are all different, so that one table can serve every row
SEQS = [(0, 1), (15, 1), (17, 3), (300, 40), (400, 0), (30, 16), (64, 33), (512, 131), (700, 5)]


def angles(n_pos, half):
    turn = np.arange(n_pos)[:, None] * 100.0 ** (-np.arange(half) / half)[None]
    return np.cos(turn).astype(np.float32), np.sin(turn).astype(np.float32)


def axes_of(kind, half, n_axes):
    i = np.arange(half)
    if kind == "runs":                   # runs that end inside a group of eight pairs, too
        return np.minimum(i * n_axes // max(1, half - 3), n_axes - 1)
    if kind == "groups":                 # whole groups of eight
        return i // 8 % n_axes
    return i % n_axes if kind == "turns" else 0 * i


@pytest.mark.parametrize("fmt,kind", [("fp8", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("D,page,rotary,interleaved,axes,n_axes", [
    (128, 16, 128, False, "one", 1), (128, 16, 128, False, "runs", 3), (128, 32, 128, True, "turns", 3),
    (64, 16, 32, False, "turns", 2), (64, 128, 64, True, "groups", 4), (256, 16, 256, False, "runs", 4),
    (256, 64, 96, False, "groups", 3), (128, 16, 64, True, "one", 2), (256, 16, 128, True, "turns", 4)])
def test_rows_turn_by_their_axes(ctx, D, page, rotary, interleaved, axes, n_axes, fmt, kind):
    import torch
    note(f"kv append at D={D} page={page} rotary={rotary}/{interleaved} {axes} {n_axes} {fmt} {kind}")
    a, b = (Setup(SEQS, D=D, page=page, fmt=fmt, kind=kind, seed=D + n_axes) for _ in "ab")
    half, n_pos = rotary // 2, 500
    cos, sin = angles(n_pos, half)
    axis = axes_of(axes, half, n_axes)
    pos = a.rng.randint(0, n_pos, (n_axes, a.T))
    pos[:, ::7] = a.rng.choice([-1, -2 ** 31, n_pos, n_pos + 5, 2 ** 31 - 1], pos[:, ::7].shape)   # held inside the table
    k, v, q = a.tensor(a.H, 1.3, 24), a.tensor(a.H, 0.7), a.tensor(a.H * 2, 1.0, 8)
    rope = lodestar.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), interleaved)
    at = torch.from_numpy(pos.astype(np.int32)).cuda()
    positions = lodestar.Positions(at[0].contiguous() if n_axes == 1 else at, None if axes == "one" else axis)
    got, same = (torch.empty(a.T, a.H * 2, D, dtype=a.kind, device="cuda") for _ in "ab")
    ctx.ls_kv_append_at(a.cache, a.batch, positions, k, v, rope, q=q, q_out=got)
    torch.cuda.synchronize()

    # the table by place
    row = np.concatenate([p + np.arange(n) for p, n in zip(a.past, a.new)])
    held = np.clip(pos[axis], 0, n_pos - 1)                      # [half, T]
    table = [np.zeros((int(row.max()) + 1, half), np.float32) for _ in range(2)]
    for t, src in zip(table, (cos, sin)):
        t[row] = src[held.T, np.arange(half)]
    by_place = lodestar.Rope(*(torch.from_numpy(t).cuda() for t in table), interleaved)
    ctx.ls_kv_append(b.cache, b.batch, k, v, rope=by_place, q=q, q_out=same)
    torch.cuda.synchronize()
    assert torch.equal(got.view(torch.int16), same.view(torch.int16))
    for x, y in zip(a.bufs, b.bufs):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))

    want = kd.rotate_axes(q.double().cpu().numpy(), pos, axis, cos, sin, interleaved)
    size = np.abs(q.double().cpu().numpy()).max(-1, keepdims=True) * 2
    u = 2.0 ** -8 if a.kind == torch.bfloat16 else 2.0 ** -11
    assert (np.abs(got.double().cpu().numpy() - want) <= u * np.abs(want) + 2.0 ** -22 * size + 2.0 ** -25).all()


def test_in_place_and_without_queries(ctx):
    import torch
    a, b = Setup(SEQS, seed=2), Setup(SEQS, seed=2)
    cos, sin = (torch.from_numpy(x).cuda() for x in angles(900, 64))
    rope = lodestar.Rope(cos, sin)
    k, v, q = a.tensor(a.H), a.tensor(a.H), a.tensor(a.H * 4)
    at = lodestar.Positions(torch.randint(0, 900, (3, a.T), dtype=torch.int32, device="cuda"), np.arange(64) % 3)
    out = torch.empty_like(q)
    note("kv append at in place")
    ctx.ls_kv_append_at(a.cache, a.batch, at, k, v, rope, q=q, q_out=out)
    ctx.ls_kv_append_at(a.cache, a.batch, at, k, v, rope, q=q, q_out=q)
    ctx.ls_kv_append_at(b.cache, b.batch, at, k, v, rope)
    torch.cuda.synchronize()
    assert torch.equal(q, out)
    for x, y in zip(a.bufs, b.bufs):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_padded_batches_and_absent_pages(ctx):
    """Rows of no sequence keep their positions to themselves: values stay out, queries are still rotated."""
    import torch
    s = Setup([(40, 9), (3, 20), (200, 5)], seed=12, absent=[(1, 1)])
    cos, sin = (torch.from_numpy(x).cuda() for x in angles(300, 64))
    k, v = s.tensor(s.H), s.tensor(s.H)
    off = torch.tensor([4, 9, 9, 29], dtype=torch.int32, device="cuda")
    batch = lodestar.KVBatch(off, s.batch.past, s.batch.pages, s.T, 20)
    at = lodestar.Positions(torch.randint(0, 300, (s.T,), dtype=torch.int32, device="cuda"))
    note("kv append at padded")
    before = s.host()
    ctx.ls_kv_append_at(s.cache, batch, at, k, v, lodestar.Rope(cos, sin))
    torch.cuda.synchronize()
    after = s.host()
    assert (before.scale["k"][s.table[1, 0]] == after.scale["k"][s.table[1, 0]]).all()
    assert (before.codes["k"][s.table[0, 2]] != after.codes["k"][s.table[0, 2]]).any()
    for bad in ([0, 2 ** 30, 5, -7], [9, 5, 3, 1]):
        off.copy_(torch.tensor(bad, dtype=torch.int32))
        note(f"kv append at offsets {bad}")
        ctx.ls_kv_append_at(s.cache, batch, at, k, v, lodestar.Rope(cos, sin))
    torch.cuda.synchronize()


def test_graph_replays(ctx):
    """Positions change between replays; the axes are part of the captured call."""
    import torch
    a, b = Setup(SEQS, seed=5), Setup(SEQS, seed=5)
    rope = lodestar.Rope(*(torch.from_numpy(x).cuda() for x in angles(400, 64)))
    k, v = a.tensor(a.H), a.tensor(a.H)
    pos = torch.randint(0, 400, (3, a.T), dtype=torch.int32, device="cuda")
    at = lodestar.Positions(pos, np.arange(64) // 8 % 3)
    note("kv append at graph")
    ctx.ls_kv_append_at(a.cache, a.batch, at, k, v, rope)
    ctx.ls_kv_append_at(b.cache, b.batch, at, k, v, rope)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.ls_kv_append_at(a.cache, a.batch, at, k, v, rope)
    for i in range(3):
        pos.copy_(torch.randint(0, 400, (3, a.T), device="cuda"))
        k.add_(0.5)
        g.replay()
        ctx.ls_kv_append_at(b.cache, b.batch, at, k, v, rope)
        torch.cuda.synchronize()
        for x, y in zip(a.bufs, b.bufs):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i


def test_refusals(ctx):
    import ctypes
    import torch
    s = Setup([(40, 3)], seed=17)
    k, v, q = s.tensor(s.H), s.tensor(s.H), s.tensor(s.H * 2)
    cos, sin = (torch.from_numpy(x).cuda() for x in angles(64, 64))
    rope, pos = lodestar.Rope(cos, sin), torch.zeros(3, s.T, dtype=torch.int32, device="cuda")
    axis = np.zeros(64, np.uint8)
    lib = lodestar.library()

    def refused(word, rope=rope.ref, positions=True, **a):
        p = lodestar.ls_positions(3, pos.data_ptr(), axis.ctypes.data)
        for n, x in a.items():
            setattr(p, n, x)
        s.batch.c.dtype = lodestar.LS_BF16
        rc = lib.ls_kv_append_at(ctx.h, s.cache.ref, s.batch.ref, rope, ctypes.byref(p) if positions else None, k.data_ptr(),
                                 s.H * s.D, v.data_ptr(), s.H * s.D, None, 0, 0, None, 0, None)
        assert rc == lodestar.LS_ERR_INVALID and word in ctx.last_error(), (rc, ctx.last_error())

    note("kv append at refusals")
    before = [t.clone() for t in s.bufs]
    refused("rope and positions", rope=None)
    refused("rope and positions", positions=False)
    refused("n_axes", n_axes=0)
    refused("n_axes", n_axes=5)
    refused("pos must", pos=None)
    axis[17] = 3
    refused("axis[17] is 3")
    torch.cuda.synchronize()
    for x, y in zip(before, s.bufs):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    with pytest.raises(ValueError):
        ctx.ls_kv_append_at(s.cache, s.batch, lodestar.Positions(pos[:, :2].contiguous()), k, v, rope)
    with pytest.raises(ValueError):
        ctx.ls_kv_append_at(s.cache, s.batch, lodestar.Positions(pos, axis[:32]), k, v, rope)
    with pytest.raises(ValueError):
        ctx.ls_kv_append_at(s.cache, s.batch, lodestar.Positions(pos), k, v, rope, q=q)
    for bad in (pos.long(), pos.cpu(), pos[:, ::2], pos[0, 0]):
        with pytest.raises(ValueError):
            lodestar.Positions(bad)
    for bad in (np.full(64, -1), np.full(64, 300), np.zeros((2, 32), int)):
        with pytest.raises((ValueError, OverflowError)):
            lodestar.Positions(pos, bad)
