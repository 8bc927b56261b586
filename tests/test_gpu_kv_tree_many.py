"""Attention of drafted trees for batches of many sequences, whose work one workgroup divides for all
the others, and around the number from which on it does; tolerances of test_gpu_kv_tree."""
import numpy as np
import pytest

import kv_draft_oracle as kd
import kv_oracle as ko
from gpu_helpers import note
from paper_2606_00946_amd import lodestar
from test_gpu_kv import Setup
from test_gpu_kv_tree import check, ctx, grown  # noqa: F401

pytestmark = pytest.mark.gpu


def ragged(B, seed, longest=90):
    """Short sequences of every kind; long runs of them, whole chunks among them, have no rows."""
    r = np.random.RandomState(seed)
    seqs = [(int(r.randint(0, longest)), int(r.choice([0, 1, 1, 2, 5]))) for _ in range(B)]
    for b0 in range(70, B - 250, 400):
        seqs[b0:b0 + 150] = [(p, 0) for p, _ in seqs[b0:b0 + 150]]
    return seqs


@pytest.mark.parametrize("B", [127, 129, 191, 192, 193, 1000, 4097])
@pytest.mark.parametrize("D,G,fmt,kind", [(64, 2, "fp8", "bf16"), (128, 16, "int8", "f16")])
def test_many_sequences(ctx, B, D, G, fmt, kind):  # noqa: F811
    note(f"kv tree many sequences B={B} D={D} G={G} {fmt} {kind}")
    check(ctx, grown(Setup(ragged(B, B + G), H=1, D=D, fmt=fmt, kind=kind, seed=B)), G)


@pytest.mark.parametrize("B", [130, 200, 700])
@pytest.mark.parametrize("D,H,G", [(64, 4, 4), (128, 2, 8), (256, 2, 2)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 20)])
def test_long_ones_among_them(ctx, B, D, H, G, window, sinks):  # noqa: F811
    """Heads of the long ones are cut, on either side of what fits the device; twice, with the same bits."""
    import torch
    seqs = ragged(B, B + D, longest=40)
    seqs[0], seqs[B // 2], seqs[-1] = (3000, 9), (6000, 1), (4001, 33)
    s = grown(Setup(seqs, H=H, D=D, seed=B + D))
    q = s.tensor(H * G)
    note(f"kv tree long among B={B} D={D} window={window}")
    a = check(ctx, s, G, window, sinks, q=q)
    b = torch.empty_like(a)
    ctx.ls_kv_attention_tree(s.cache, s.batch, s.tree, q, b, window=window, sinks=sinks)
    assert torch.equal(a, b)


def test_graph_replays(ctx):  # noqa: F811
    """Captured, with other lengths at every replay, beside eager calls on the same workspace."""
    import torch
    seqs = ragged(300, 5, longest=2000)
    s = grown(Setup(seqs, H=1, D=64, seed=15))
    q = s.tensor(4)
    out = torch.empty_like(q)
    call = lambda: ctx.ls_kv_attention_tree(s.cache, s.batch, s.tree, q, out)  # noqa: E731
    note("kv tree many, graph: warm call")
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    past = s.batch.past.clone()
    for i in range(4):
        note(f"kv tree many, graph: replay {i}")
        s.batch.past.copy_(past * (i + 1) // 5)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and (got != 0).any(-1).all()


def test_time_grows_with_the_batch(ctx):  # noqa: F811
    """16 times as many sequences take no more than four times 16 times as long; what they get is the definition's."""
    import torch
    D, most = 64, 65536
    cache = lodestar.KVCache(most, 1, D, dtype="int8")
    g = torch.Generator(device="cuda").manual_seed(1)
    for t in (cache.k, cache.v):
        t.random_(0, 100, generator=g)
    cache.k_scale.fill_(0.02)
    cache.v_scale.uniform_(0.01, 0.02, generator=g)
    pages = torch.randperm(most, device="cuda", generator=g).to(torch.int32)[:, None].contiguous()
    past = torch.randint(0, 15, (most,), device="cuda", generator=g).to(torch.int32)
    times = []
    for B in (4096, most):
        batch = lodestar.KVBatch(torch.arange(B + 1, dtype=torch.int32, device="cuda"), past[:B], pages[:B], B, 1)
        tree = lodestar.Tree(torch.ones(B, 1, dtype=torch.int64, device="cuda"))
        q = torch.randn(B, 2, D, device="cuda", generator=g).bfloat16()
        out = torch.empty_like(q)
        note(f"kv tree batch of {B}")
        ms = []
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            ctx.ls_kv_attention_tree(cache, batch, tree, q, out)
            b.record()
            torch.cuda.synchronize()
            ms.append(a.elapsed_time(b))
        times.append(min(ms))
        host = ko.Cache(*(t.cpu().numpy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)), most, 1, D, 16, "int8")
        pick = np.unique(np.concatenate([np.random.RandomState(B).randint(0, B, 300), [0, 63, 64, B - 1]]))
        p = past.cpu().numpy()[pick]
        want, mag = kd.attention_tree(host, q.double().cpu().numpy()[pick], np.arange(len(pick) + 1), p, pages.cpu().numpy()[pick],
                                      [np.ones((1, 1), bool)] * len(pick), p, D ** -0.5)
        assert (np.abs(out.double().cpu().numpy()[pick] - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * mag + 1e-7).all()
    print(f"  {times[0] * 1e3:.0f} and {times[1] * 1e3:.0f} us", flush=True)
    assert times[1] <= 64 * times[0]
