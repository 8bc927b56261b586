"""The paged 8-bit KV cache's calls where their bounds are reached: offsets that
leave rows to nobody, a first call inside a capture, against the definitions in 64 bits (kv_oracle) with the
tolerances of test_gpu_kv."""
import numpy as np
import pytest

import kv_oracle as ko
from gpu_helpers import note
from paper_2606_00946_amd import lodestar
from test_gpu_kv import Setup, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G,head,fmt", [(4, 160, "fp8"), (8, 161, "int8"), (1, 7, "fp8"), (40, 33, "int8")])
def test_rows_before_the_first_sequence(ctx, G, head, fmt):  # noqa: F811
    """Offsets that start past 0: the rows before them are no sequence's, and the page table ends where it ends."""
    import torch
    s = Setup([(0, head), (0, 1), (50, 70), (33, 1), (200, 2), (3, 130)], fmt=fmt, seed=head, poison=False)
    B, W = len(s.past) - 1, s.table.shape[1]
    off, past, table = s.off[1:], s.past[1:], s.table[1:]
    # before and after the table: pages that no sequence of the call has
    idle = np.resize(s.table[0][s.table[0] >= 0], (1, W))
    around = torch.from_numpy(np.concatenate([idle, table, idle])).to("cuda", torch.int32)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", torch.int32)  # noqa: E731
    batch = lodestar.KVBatch(i32(off), i32(past), around[1:1 + B], s.T, int(s.new.max()))
    note(f"kv rows before the first sequence G={G} head={head} {fmt}")
    k, v, q = s.tensor(s.H), s.tensor(s.H), s.tensor(s.H * G)
    before = s.host()
    ctx.ls_kv_append(s.cache, batch, k, v)
    ko_, vo = (torch.full((s.T, s.H, s.D), 7.0, dtype=s.kind, device="cuda") for _ in "kv")
    ctx.ls_kv_read(s.cache, batch, ko_, vo)
    out = torch.full((s.T, s.H * G, s.D), 7.0, dtype=s.kind, device="cuda")
    ctx.ls_kv_attention(s.cache, batch, q, out)
    torch.cuda.synchronize()
    after = s.host()
    for name in "kv":
        same = np.setdiff1d(np.arange(s.n_pages), table.ravel())
        np.testing.assert_array_equal(before.codes[name][same], after.codes[name][same])
        np.testing.assert_array_equal(before.scale[name][same], after.scale[name][same])
    for t in (ko_, vo, out):
        assert (t[:head] == 7.0).all()
    for name, back in (("k", ko_), ("v", vo)):
        for b in range(B):
            held, _ = after.tokens(name, table[b], int(past[b] + s.new[b + 1]))
            got = back[off[b]:off[b + 1]].double().cpu().numpy()
            assert (np.abs(got - held[past[b]:]) <= 2.0 ** -8 * np.abs(held[past[b]:])).all()
    want, mag = ko.attention(after, q.double().cpu().numpy(), off, past, table, s.D ** -0.5)
    got = out.double().cpu().numpy()
    assert (np.abs(got - want)[head:] <= (2.0 ** -8 * np.abs(want) + 2.0 ** -9 * mag + 1e-7)[head:]).all()


def test_first_call_inside_a_capture():
    """A context's first attention call is refused on a capturing stream; after one outside, capture and replays work."""
    import torch
    own = lodestar.Context(16, (64, 64))
    s = Setup([(9000, 1), (40, 1), (2000, 1)], seed=31)
    q = s.tensor(s.H * 4)
    out, x = torch.zeros_like(q), torch.zeros(4, device="cuda")
    note("kv first call inside a capture")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x.add_(1.0)
        with pytest.raises(lodestar.LodestarError) as e:
            own.ls_kv_attention(s.cache, s.batch, q, out)
    assert e.value.code == lodestar.LS_ERR_STATE and "capturing" in own.last_error()
    g.replay()
    torch.cuda.synchronize()
    assert (x == 1.0).all() and (out == 0).all()
    note("kv first call outside")
    own.ls_kv_attention(s.cache, s.batch, q, out)
    torch.cuda.synchronize()
    want = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        own.ls_kv_attention(s.cache, s.batch, q, out)
    for i in range(3):
        note(f"kv replay {i}")
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    own.close()
