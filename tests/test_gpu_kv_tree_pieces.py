"""Attention of drafted trees where heads are cut into many pieces and into long ones, in tiles
of 32 and of 64 rows (kv_tree_cases; test_kv_tree_pieces_cpu shows that the cases reach these), against
the definition in 64 bits; and padded batches, row by row.

The bound, narrow enough that a lost block of 16 tokens of 60,000 would be several times it: weights are
rounded to half precision one by one, 2^-11 of each at most and independent, so their sum is off by
6 / sqrt(3) * 2^-11 of sqrt(sum (p v)^2) at six standard deviations; scores, exponentials, sums and the smallest
weights give 2^-16 of sum p |v|; the output's own rounding is 2^-8 (bf16) or 2^-11 (half) of it.
"""
import numpy as np
import pytest

import kv_draft_oracle as kd
import kv_tree_cases
from gpu_helpers import note
from paper_2606_00946_amd import lodestar
from test_gpu_kv import Setup
from test_gpu_kv_tree import grown

pytestmark = pytest.mark.gpu

CASES = kv_tree_cases.cases()


@pytest.fixture(scope="module")
def ctx():
    c = lodestar.Context(16, (64, 64))
    yield c
    c.close()


def worst(s, q, out, window=0, sinks=0):
    """The largest share of the bound that any element is off by."""
    import torch
    host, most, G = s.host(), 0.0, q.shape[1] // s.H
    u = 2.0 ** -8 if s.kind == torch.bfloat16 else 2.0 ** -11
    for b in range(len(s.past)):
        n, p0 = int(s.new[b]), int(s.past[b])
        rows = slice(int(s.off[b]), int(s.off[b + 1]))
        (k, there), (v, _) = (host.tokens(name, s.table[b], p0 + n) for name in "kv")
        k, v, there = (torch.from_numpy(x).cuda() for x in (k, v, there))
        near = torch.ones(n, p0, dtype=torch.bool, device="cuda")
        if window:
            j, at = torch.arange(p0, device="cuda")[None], torch.from_numpy(s.pos[rows]).cuda()[:, None]
            near = (j > at.clamp(min=p0) - window) | (j < sinks)
        hidden = ~(torch.cat([near, torch.from_numpy(s.sees[b]).cuda()], 1) & there)
        for h in range(q.shape[1]):
            kh, vh = k[:, h // G].contiguous(), v[:, h // G].contiguous()
            p = torch.softmax((q[rows, h].double() @ kh.T.contiguous() * s.D ** -0.5).masked_fill(hidden, -np.inf), 1)
            want, mag, rms = p @ vh, p @ vh.abs(), ((p * p) @ (vh * vh)).sqrt()
            bound = u * want.abs() + 6 / 3 ** 0.5 * 2.0 ** -11 * rms + 2.0 ** -16 * mag + 2.0 ** -25
            most = max(most, float(((out[rows, h].double() - want).abs() / bound).max()))
    print(f"  {most:.2f} of the bound", flush=True)
    return most


@pytest.mark.parametrize("fmt,kind", [("fp8", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("name", CASES)
def test_pieces(ctx, name, fmt, kind):
    import torch
    c = CASES[name]
    s = Setup(c["seqs"], H=c["H"], D=c["D"], fmt=fmt, kind=kind, seed=len(name), absent=c["absent"])
    if c["width"] > s.table.shape[1] * s.page:
        s.table = np.pad(s.table, ((0, 0), (0, c["width"] // s.page - s.table.shape[1])), constant_values=-1)
        s.batch = lodestar.KVBatch(s.batch.new_off, s.batch.past, torch.from_numpy(s.table.astype(np.int32)).cuda(), s.T,
                                   int(s.new.max()))
    grown(s)
    q = s.tensor(s.H * c["G"])
    out, again = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    note(f"kv tree pieces: {name} {fmt} {kind}")
    ctx.ls_set_cu_limit(c["cus"])
    try:
        for o in (out, again):
            ctx.ls_kv_attention_tree(s.cache, s.batch, s.tree, q, o, window=c["window"], sinks=c["sinks"])
        torch.cuda.synchronize()
    finally:
        ctx.ls_set_cu_limit(0)
    assert worst(s, q, out, c["window"], c["sinks"]) <= 1
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("off,window,sinks", [([4, 9, 9, 29], 0, 0), ([4, 9, 9, 29], 30, 3), ([0, 0, 7, 31], 0, 0), ([33, 34, 34, 34], 0, 0)])
@pytest.mark.parametrize("G", [1, 8])
def test_rows_of_padded_batches(ctx, G, off, window, sinks):
    """A first sequence that starts behind row 0, sequences without rows, rows behind the last one: the sequences' rows are
    the definition's, the others stay as they were."""
    import torch
    past, rows = np.array([40, 3, 200]), 34
    s = Setup([(int(p), 31) for p in past], seed=12, H=2)
    s.new, s.off, s.T = np.diff(off), np.array(off), rows
    count = 1
    s.sees, s.pos, mask = [], np.zeros(rows, np.int64), np.full((rows, count), -1, np.int64).view(np.uint64)
    for b, n in enumerate(s.new):
        sees, depth = kd.ancestry(kd.tree_parents(int(n), 4, s.rng))
        s.sees.append(sees)
        s.pos[off[b]:off[b + 1]] = past[b] + depth
        mask[off[b]:off[b + 1]] = kd.words(sees, count)
    tree = lodestar.Tree(torch.from_numpy(mask.view(np.int64)).cuda(), torch.from_numpy(s.pos.astype(np.int32)).cuda())
    batch = lodestar.KVBatch(torch.tensor(off, dtype=torch.int32, device="cuda"), s.batch.past, s.batch.pages, rows, 31)
    q = s.tensor(s.H * G)
    out = torch.full_like(q, 3.0)
    note(f"kv tree padded rows {off} G={G} window={window}")
    ctx.ls_kv_attention_tree(s.cache, batch, tree, q, out, window=window, sinks=sinks)
    torch.cuda.synchronize()
    assert (out[:off[0]] == 3).all() and (out[off[-1]:] == 3).all()
    want, mag = kd.attention_tree(s.host(), q.double().cpu().numpy(), s.off, past, s.table, s.sees, s.pos, s.D ** -0.5, window, sinks)
    mine = slice(off[0], off[-1])
    got = out.double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * mag + 1e-7)[mine].all()      # as in test_gpu_kv_tree
