"""ls_kv_append_at for padded batches and absent pages, row by row: every row's queries turn by
its own positions, also those of no sequence; what is stored is what ls_kv_append stores from a table that holds
each place's angles.  Tolerances as in test_gpu_kv_positions."""
import numpy as np
import pytest

import kv_draft_oracle as kd
from gpu_helpers import note
from paper_2606_00946_amd import lodestar
from test_gpu_kv import Setup
from test_gpu_kv_positions import angles, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("off", [[4, 9, 9, 29], [0, 20, 21, 21], [0, 0, 0, 34], [30, 30, 33, 34]])
@pytest.mark.parametrize("n_axes", [1, 3])
@pytest.mark.parametrize("D,page,fmt", [(128, 16, "fp8"), (64, 32, "int8"), (256, 16, "int8")])
def test_padded_rows_and_absent_pages(ctx, D, page, fmt, n_axes, off):  # noqa: F811
    import torch
    rows, past = 34, np.array([40, 500, 205])
    # the second page that the last two sequences write to is not there
    absent = [(b, (int(past[b]) // page) + 1) for b in (1, 2)]
    a, b = (Setup([(int(p), rows) for p in past], D=D, page=page, fmt=fmt, seed=12, absent=absent) for _ in "ab")
    half, n_pos = D // 2, 300
    cos, sin = angles(n_pos, half)
    axis, pos = np.arange(half) % n_axes, a.rng.randint(0, n_pos, (n_axes, rows))
    a.T = rows
    k, v, q = a.tensor(a.H), a.tensor(a.H), a.tensor(a.H * 2)
    offsets = torch.tensor(off, dtype=torch.int32, device="cuda")
    batches = [lodestar.KVBatch(offsets, s.batch.past, s.batch.pages, rows, rows) for s in (a, b)]
    at = torch.from_numpy(pos.astype(np.int32)).cuda()
    rope = lodestar.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda())
    got = torch.full_like(q, 3.0)
    note(f"kv append at padded rows {off} D={D} page={page} {fmt} axes={n_axes}")
    ctx.ls_kv_append_at(a.cache, batches[0], lodestar.Positions(at, axis), k, v, rope, q=q, q_out=got)
    torch.cuda.synchronize()

    table, spots = [np.zeros((600, half), np.float32) for _ in range(2)], set()
    for i, p in enumerate(past):
        for r in range(off[i], off[i + 1]):
            place = int(p) + r - off[i]
            spots.add(place)
            for t, src in zip(table, (cos, sin)):
                t[place] = src[pos[axis, r], np.arange(half)]
    assert len(spots) == off[-1] - off[0]                        # one table serves all sequences
    by_place = lodestar.Rope(*(torch.from_numpy(t).cuda() for t in table))
    before = [t.clone() for t in b.bufs]
    ctx.ls_kv_append(b.cache, batches[1], k, v, rope=by_place)
    torch.cuda.synchronize()
    for x, y in zip(a.bufs, b.bufs):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    written = {int(a.table[i, (int(p) + r - off[i]) // page]) for i, p in enumerate(past) for r in range(off[i], off[i + 1])} - {-1}
    for x, y in zip(before, a.bufs):
        x, y = x.view(torch.uint8).view(a.n_pages, -1), y.view(torch.uint8).view(a.n_pages, -1)
        changed = set((x != y).any(1).nonzero().flatten().tolist())
        assert changed <= written and (x.shape[1] < 1024 or changed == written)

    want = kd.rotate_axes(q.double().cpu().numpy(), pos, axis, cos, sin, False)
    size = np.abs(q.double().cpu().numpy()).max(-1, keepdims=True) * 2
    assert (np.abs(got.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * size + 2.0 ** -25).all()
