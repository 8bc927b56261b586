"""Attention of drafted trees over the paged 8-bit KV cache on the GPU, against
the definition in 64 bits (kv_draft_oracle).

Tolerance.  The output's own rounding is half a step: 2^-8 of its size in bf16,
2^-11 in half.  A weight is rounded to half precision: 2^-11 of itself, or, where it
is small, 2^-16 of the sum of the 16 that it goes with, which is at most 2^-12 of
that sum over all of them.  Scores in fp32: sums of up to 256 products of 16-bit
queries and codes, within 2^-24 (256 / 2) of the logits' magnitudes at the worst,
2^-14 for those here.  Together below 2^-10 of sum_j p_j |v_j|; twice that is allowed,
for values that are larger in the small weights' tokens than in the others.
"""
import numpy as np
import pytest

import kv_draft_oracle as kd
import kv_oracle as ko
from gpu_helpers import note
from paper_2606_00946_amd import lodestar
from test_gpu_kv import Setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = lodestar.Context(16, (64, 64))
    yield c
    c.close()


def grown(s, reach=4, extra_words=0, edit=None):
    """Trees for a Setup's new tokens: s.sees[b], s.pos, s.tree; edit(b, sees) may change what is seen."""
    import torch
    s.sees, pos = [], []
    count = max(1, -(-int(s.new.max()) // 64)) + extra_words
    mask = np.zeros((s.T, count), np.uint64)
    for b, n in enumerate(s.new):
        sees, depth = kd.ancestry(kd.tree_parents(int(n), reach, s.rng))
        if edit:
            edit(b, sees)
        s.sees.append(sees)
        pos.append(s.past[b] + depth)
        mask[s.off[b]:s.off[b + 1]] = kd.words(sees, count)
    # bits that no new token has do not count
    for b, n in enumerate(s.new):
        for j in range(int(n), 64 * count, 3):
            mask[s.off[b]:s.off[b + 1], j // 64] |= np.uint64(1 << (j % 64))
    s.pos = np.concatenate(pos) if pos else np.zeros(0, np.int64)
    s.tree = lodestar.Tree(torch.from_numpy(mask.view(np.int64)).cuda(), torch.from_numpy(s.pos.astype(np.int32)).cuda())
    return s


def check(ctx, s, G, window=0, sinks=0, sigma=1.0, extra=0, scale=None, stream=None, q=None):
    import torch
    q = s.tensor(s.H * G, sigma, extra) if q is None else q
    out = torch.full((s.T, s.H * G, s.D), 7.0, dtype=s.kind, device="cuda")
    ctx.ls_kv_attention_tree(s.cache, s.batch, s.tree, q, out, scale=scale, window=window, sinks=sinks, stream=stream)
    torch.cuda.synchronize()
    want, mag = kd.attention_tree(s.host(), q.double().cpu().numpy(), s.off, s.past, s.table, s.sees, s.pos,
                                  s.D ** -0.5 if scale is None else scale, window, sinks)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    u = 2.0 ** -8 if s.kind == torch.bfloat16 else 2.0 ** -11
    off = np.abs(got - want) - (u * np.abs(want) + 2.0 ** -9 * mag + 1e-7)
    assert off.max() <= 0, f"off by {np.abs(got - want).max()} at {np.unravel_index(off.argmax(), off.shape)}"
    return out


SEQS = [(0, 1), (0, 9), (300, 8), (15, 17), (16, 64), (0, 0), (523, 33), (640, 0), (63, 2), (250, 65)]


@pytest.mark.parametrize("fmt,kind", [("fp8", "bf16"), ("int8", "f16"), ("fp8", "f16"), ("int8", "bf16")])
@pytest.mark.parametrize("D,page,G", [(64, 16, 1), (128, 16, 4), (256, 32, 3), (128, 64, 7), (64, 128, 16), (256, 16, 1)])
def test_trees(ctx, D, page, G, fmt, kind):
    note(f"kv tree D={D} page={page} G={G} {fmt} {kind}")
    check(ctx, grown(Setup(SEQS, D=D, page=page, fmt=fmt, kind=kind, seed=D + G)), G)


@pytest.mark.parametrize("n", [1, 2, 7, 8, 15, 16, 17, 63, 64, 65, 129])
@pytest.mark.parametrize("G", [1, 4])
def test_rows_and_words(ctx, n, G):
    """Row counts around the tiles', drafts around the mask's words, from places all over a block."""
    note(f"kv tree rows n={n} G={G}")
    check(ctx, grown(Setup([(past, n) for past in (0, 1, 15, 16, 40, 64)], H=1, seed=n + G), extra_words=n % 2), G)


@pytest.mark.parametrize("D,fmt,kind", [(128, "fp8", "bf16"), (128, "int8", "f16"), (64, "int8", "bf16"), (64, "fp8", "f16"),
                                        (256, "fp8", "bf16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 5)])
def test_many_tiles(ctx, D, fmt, kind, window, sinks):
    """More row tiles of heads than workgroups that fit the device, with pages that are not there."""
    note(f"kv tree many tiles D={D} {fmt} {kind} window={window}")
    check(ctx, grown(Setup(SEQS, H=8, D=D, fmt=fmt, kind=kind, seed=23, absent=((2, 3), (6, 0))), extra_words=1), 16, window, sinks)


@pytest.mark.parametrize("n", [8, 9, 16, 17])
@pytest.mark.parametrize("B", [15, 16, 17, 70])
def test_tiles_around_what_fits(ctx, B, n):
    note(f"kv tree {B} sequences of {n}")
    check(ctx, grown(Setup([(50 * b % 130, n) for b in range(B)], H=16, D=64, seed=B + n)), 4)


def test_chain_is_causal_attention(ctx):
    """A chain of drafts sees what causal attention shows it: the two calls agree."""
    import torch
    s = grown(Setup([(300, 6), (0, 40), (77, 1)], seed=1), reach=1)
    q = s.tensor(s.H * 4)
    note("kv tree chain")
    out = check(ctx, s, 4, q=q)
    same = torch.empty_like(out)
    ctx.ls_kv_attention(s.cache, s.batch, q, same)
    torch.cuda.synchronize()
    assert (out.float() - same.float()).abs().max() <= 2.0 ** -6 * same.float().abs().max()


def test_any_mask(ctx):
    """Masks that are no trees: nothing, everything, later tokens, not itself; rows that see nothing at all."""
    def edit(b, sees):
        sees[:] = np.random.RandomState(b).rand(*sees.shape) < 0.5
        sees[0] = False
        if len(sees) > 3:
            sees[3] = True
    s = grown(Setup([(0, 20), (100, 70), (33, 4), (0, 1)], seed=2), edit=edit)
    note("kv tree any mask")
    out = check(ctx, s, 4)
    assert (out[s.off[0]] == 0).all() and (out[s.off[3]] == 0).all() and (out[1] != 0).any()


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (17, 3), (100, 16), (250, 33), (5000, 0), (64, 1000),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("D,G,fmt", [(128, 4, "fp8"), (64, 8, "int8")])
def test_window_and_sinks(ctx, D, G, fmt, window, sinks):
    seqs = [(0, 5), (900, 9), (300, 30), (1000, 3), (0, 70), (17, 1), (700, 40)]
    note(f"kv tree window={window} sinks={sinks} D={D} G={G} {fmt}")
    check(ctx, grown(Setup(seqs, D=D, fmt=fmt, seed=window % 1000)), G, window, sinks)


def test_positions_of_any_value(ctx):
    """Positions before the cached tokens, far behind them and at the ends of 32 bits; a row may see no cached token."""
    s = grown(Setup([(200, 6), (100, 6), (300, 6)], seed=3))
    s.pos[:] = [200, 0, -5, 260, 2 ** 31 - 1, -2 ** 31, 100, 131, 132, 164, 2 ** 30, 2 ** 30 + 1, 300, 301, 350, 364, 365, 9999]
    import torch
    s.tree.pos.copy_(torch.from_numpy(s.pos.astype(np.int32)))
    note("kv tree positions")
    check(ctx, s, 4, window=64, sinks=0)
    check(ctx, s, 4, window=32, sinks=20)


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 4)])
def test_absent_pages(ctx, window, sinks):
    import torch
    seqs = [(40, 3), (100, 40), (3, 1), (200, 9), (0, 16), (48, 20)]
    absent = [(0, 0), (0, 2), (1, 1), (2, 0), (4, 0), (5, 3), (5, 4)] + [(1, j) for j in range(6, 9)]
    s = Setup(seqs, seed=5, absent=absent)
    s.table[3, 4], s.table[3, 5] = s.n_pages, -7
    s.batch.pages.copy_(torch.from_numpy(s.table).to("cuda", torch.int32))
    note(f"kv tree absent pages window={window}")
    out = check(ctx, grown(s), 4, window, sinks)
    assert (out[s.off[2]] == 0).all() and (out[s.off[4]:s.off[5]] == 0).all()


def test_lengths_past_the_table(ctx):
    import torch
    s = Setup([(100, 5), (30, 2)], seed=9, poison=False)         # whole pages become visible
    s.batch.past.copy_(torch.tensor([2 ** 31 - 20, 30], dtype=torch.int32))
    s.past = np.array([s.table.shape[1] * s.page + 50, 30])      # the same tokens are visible from there
    note("kv tree past the table")
    check(ctx, grown(s), 4)


@pytest.mark.parametrize("window", [0, 20])
def test_nan_where_no_row_sees(ctx, window):
    """NaN codes in new tokens that no row sees, beside others that some see, and in tokens behind the window."""
    hidden = {}

    def edit(b, sees):
        hidden[b] = [j for j in range(len(sees)) if j % 5 == 2]
        sees[:, hidden[b]] = False
    s = grown(Setup([(30, 40), (100, 9), (0, 20), (61, 70)], H=1, seed=6), edit=edit)
    for b, past in enumerate(s.past):
        gone = [int(past) + j for j in hidden[b]] + ([] if not window else list(range(3, int(past) + 1 - window)))
        for name, buf in zip("kv", s.bufs):
            codes, o = buf.view(s.n_pages, -1), ko.offsets(s.page, s.D, name == "v")
            for t in gone:
                codes[int(s.table[b, t // s.page]), o[t % s.page].tolist()] = 0x7F
    note(f"kv tree nan window={window}")
    check(ctx, s, 4, window=window, sinks=3 if window else 0)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [None, 0.0, 1e-38, -0.1])
def test_zero_queries_and_keys(ctx, kind, scale):
    import torch
    s = grown(Setup([(0, 40), (40, 1), (70, 20)], kind=kind, seed=21))
    keys, scales = s.bufs[0].view(s.n_pages, -1), s.bufs[2].view(s.n_pages, -1)
    for b in range(3):
        pages = torch.from_numpy(s.table[b, ::2].copy()).cuda()
        keys[pages[pages >= 0]], scales[pages[pages >= 0]] = 0, 2.0 ** -64
    q = s.tensor(s.H * 4)
    q[::3] = 0
    q[1::3, 0] *= 2.0 ** -60
    note(f"kv tree zero queries and keys {kind} scale={scale}")
    check(ctx, s, 4, scale=scale, q=q)


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_scales_of_zero(ctx, fmt):
    """Pages as a new cache holds them, codes and scales zero."""
    s = Setup([(0, 50), (40, 1), (70, 20), (33, 3)], fmt=fmt, seed=22)
    for t in s.bufs:
        t.view(s.n_pages, -1)[s.table[3, :3].tolist()] = 0
        for b in range(3):
            for j in range(0, s.table.shape[1], 2):
                if s.table[b, j] >= 0:
                    t.view(s.n_pages, -1)[int(s.table[b, j])] = 0
    note(f"kv tree scales of zero {fmt}")
    out = check(ctx, grown(s), 4)
    assert (out[s.off[3]:] == 0).all()


def test_large_logits_and_values(ctx):
    import torch
    s = grown(Setup([(333, 9), (50, 40)], seed=3))
    note("kv tree large logits")
    check(ctx, s, 4, sigma=60.0, scale=1.0)
    s.bufs[3].copy_(torch.where(torch.rand_like(s.bufs[3]) < 0.5, 2.0 ** -60, 2.0 ** -20))
    note("kv tree tiny values")
    check(ctx, s, 4, scale=0.02)
    s.bufs[3].fill_(2.0 ** 40)
    note("kv tree huge values")
    check(ctx, s, 4, scale=0.02)


@pytest.mark.parametrize("D", [64, 128, 256])
def test_first_token_takes_the_weight(ctx, D):
    """One key takes nearly all weight and its value is zero: the others' small weights keep their bits, the drafts' too."""
    import torch
    s = grown(Setup([(700, 20)], H=1, D=D, fmt="int8", kind="f16", seed=31, poison=False))
    q = torch.ones(s.T, 2, D, dtype=torch.float16, device="cuda")
    codes = [b.view(s.n_pages, -1) for b in s.bufs[:2]]
    first = int(s.table[0, 0])
    ok, ov = ko.offsets(s.page, D, False), ko.offsets(s.page, D, True)
    codes[0][first, ok[0].tolist()] = 127
    codes[1][first, ov[0].tolist()] = 0
    s.bufs[2].fill_(0.004)
    note(f"kv tree first token D={D}")
    for scale in (8 / D, 24 / D):
        check(ctx, s, 2, scale=scale, q=q)


def test_strides_and_shared_pages(ctx):
    import torch
    s = Setup([(100, 4), (100, 33), (100, 1)], seed=4)
    s.table[1, :6] = s.table[0, :6]
    s.table[2, :6] = s.table[0, :6]
    s.batch.pages.copy_(torch.from_numpy(s.table).to("cuda", torch.int32))
    note("kv tree strides")
    check(ctx, grown(s), 4, extra=24)


@pytest.mark.parametrize("D,G", [(64, 4), (128, 2), (256, 1)])
def test_long_caches_are_split(ctx, D, G):
    """Long sequences beside short ones: parts of a segment, and groups of parts, are joined; twice, with the same bits."""
    import torch
    s = grown(Setup([(20000, 5), (1, 1), (0, 40), (7001, 40), (333, 3)], H=1, D=D, seed=8))
    q = s.tensor(s.H * G)
    note(f"kv tree long D={D}")
    a = check(ctx, s, G, q=q)
    b = torch.empty_like(a)
    ctx.ls_kv_attention_tree(s.cache, s.batch, s.tree, q, b)
    assert torch.equal(a, b)


def test_many_sequences_stay_whole(ctx):
    """More segments than the workspace has room for: none is cut."""
    note("kv tree many sequences")
    check(ctx, grown(Setup([(37 * b % 90, 3) for b in range(520)] + [(3000, 20)], H=4, D=64, seed=10)), 2)


def test_padded_batches(ctx):
    """Rows behind the last sequence and in front of the first stay as they were; sequences without rows do nothing."""
    import torch
    s = grown(Setup([(40, 9), (3, 20), (200, 5)], seed=12))
    q = s.tensor(s.H * 4)
    off = torch.tensor([4, 9, 9, 29], dtype=torch.int32, device="cuda")
    batch = lodestar.KVBatch(off, s.batch.past, s.batch.pages, s.T, 20)
    out = torch.full_like(q, 3.0)
    note("kv tree padded")
    ctx.ls_kv_attention_tree(s.cache, batch, s.tree, q, out)
    torch.cuda.synchronize()
    assert (out[:4] == 3).all() and (out[29:] == 3).all() and (out[4:29] != 3).any(-1).all()
    for bad in ([0, 2 ** 30, 5, -7], [9, 5, 3, 1], [-5, 40, 60, 90]):
        off.copy_(torch.tensor(bad, dtype=torch.int32))
        note(f"kv tree offsets {bad}")
        ctx.ls_kv_attention_tree(s.cache, batch, s.tree, q, out)
    torch.cuda.synchronize()


def test_overlapping_sequences_leave_nothing_behind(ctx):
    """Offsets that overlap name far more rows than the call has: what a launch has no workgroups for must not stay half done
    in the workspace."""
    import torch
    s = grown(Setup([(20000, 64)], H=1, D=64, seed=13))
    q, past = s.tensor(4), s.batch.past.clone()
    out = torch.empty_like(q)

    def lengths():
        outs = []
        for k in range(40, 157, 2):
            s.batch.past.fill_(128 * k)
            ctx.ls_kv_attention_tree(s.cache, s.batch, s.tree, q, out)
            outs.append(out.clone())
        return torch.stack(outs)

    note("kv tree before overlapping offsets")
    before = lengths()
    for pairs in (70, 80, 81, 82, 83, 84, 85, 90):
        off = torch.tensor([0, s.T] * pairs + [0, 0, s.T], dtype=torch.int32, device="cuda")
        long = torch.zeros(len(off) - 1, dtype=torch.int32, device="cuda")
        long[-1] = 20000
        batch = lodestar.KVBatch(off, long, s.batch.pages.repeat(len(long), 1), s.T, s.T)
        note(f"kv tree {pairs} overlapping sequences")
        ctx.ls_kv_attention_tree(s.cache, batch, s.tree, q, out)
        torch.cuda.synchronize()
    assert torch.equal(before, lengths())
    s.batch.past.copy_(past)
    check(ctx, s, 4, q=q)


def test_offsets_past_32_bits(ctx):
    """Pages beyond 4 GiB of the pool."""
    import torch
    H, D, page, n_pages = 8, 128, 128, 40000
    cache = lodestar.KVCache(n_pages, H, D, dtype="int8", page_tokens=page)
    table = torch.tensor([[39999, 35000, 3]], dtype=torch.int32, device="cuda")
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    T, n = 300, 10
    k, v = (torch.randn(T, H, D, device="cuda").half() for _ in "kv")
    note("kv tree past 32 bits")
    ctx.ls_kv_append(cache, lodestar.KVBatch(i32(0, T), i32(0), table, T), k, v)
    batch = lodestar.KVBatch(i32(0, n), i32(T - n), table, n)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    ctx.ls_kv_read(cache, lodestar.KVBatch(i32(0, T), i32(0), table, T), k2, v2)
    q = torch.randn(n, H * 2, D, device="cuda").half()
    out = torch.empty_like(q)
    tree = lodestar.Tree(torch.tensor([[1 << j] for j in range(n)], device="cuda"))
    ctx.ls_kv_attention_tree(cache, batch, tree, q, out)
    kd_, vd = k2.double(), v2.double()
    seen = torch.cat([torch.ones(n, T - n), torch.eye(n)], 1).cuda().bool()
    for h in range(H * 2):
        p = torch.softmax((q[:, h].double() @ kd_[:, h // 2].T * D ** -0.5).masked_fill(~seen, -torch.inf), 1)
        want, mag = p @ vd[:, h // 2], p @ vd[:, h // 2].abs()
        assert ((out[:, h].double() - want).abs() <= 2.0 ** -9 * (want.abs() + mag)).all()


def test_graph_replays(ctx):
    """Captured, with other lengths, masks and queries at every replay, beside eager calls on the same workspace."""
    import torch
    s = grown(Setup([(40, 9), (900, 17), (15, 1), (6000, 30)], seed=15))
    q = s.tensor(s.H * 4)
    out = torch.empty_like(q)
    call = lambda: ctx.ls_kv_attention_tree(s.cache, s.batch, s.tree, q, out, window=3000, sinks=2)  # noqa: E731
    note("kv tree graph: warm call")
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        note(f"kv tree graph: replay {i}")
        s.batch.past.sub_(torch.tensor([3, 17, 1, 900], dtype=torch.int32, device="cuda"))
        s.tree.mask.bitwise_xor_(1 << i)
        q.mul_(1.1)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out)


def test_first_call_on_a_capturing_stream(ctx):
    import torch
    s = grown(Setup([(40, 3)], seed=16))
    q = s.tensor(s.H * 2)
    fresh = lodestar.Context(16, (64, 64))
    note("kv tree first call captured")
    g = torch.cuda.CUDAGraph()
    x = torch.zeros(1, device="cuda")
    with torch.cuda.graph(g):
        x.add_(1)
        with pytest.raises(lodestar.LodestarError, match="before capturing"):
            fresh.ls_kv_attention_tree(s.cache, s.batch, s.tree, q, torch.empty_like(q))
    fresh.close()


def test_on_another_stream(ctx):
    import torch
    s = grown(Setup([(33, 5), (100, 30)], seed=14))
    side = torch.cuda.Stream()
    q = s.tensor(s.H * 4)
    side.wait_stream(torch.cuda.current_stream())
    note("kv tree on a side stream")
    with torch.cuda.stream(side):
        check(ctx, s, 4, q=q)
    check(ctx, s, 4, q=q, stream=side)


def test_refusals(ctx):
    import ctypes
    import torch
    s = grown(Setup([(40, 3), (3, 66)], seed=17))
    q = s.tensor(s.H * 2)
    out = torch.full_like(q, 5.0)
    lib = lodestar.library()

    def refused(word, tree=None, batch=None, code=lodestar.LS_ERR_INVALID, **a):
        t, b = type(s.tree.c).from_buffer_copy(s.tree.c), type(s.batch.c).from_buffer_copy(s.batch.c)
        b.dtype = lodestar.LS_BF16
        for n, x in (tree or {}).items():
            setattr(t, n, x)
        for n, x in (batch or {}).items():
            setattr(b, n, x)
        g = dict(q=q.data_ptr(), qs=2 * s.H * s.D, hq=2 * s.H, o=out.data_ptr(), os=2 * s.H * s.D, scale=1.0, window=0, sinks=0)
        g.update(a)
        rc = lib.ls_kv_attention_tree(ctx.h, s.cache.ref, ctypes.byref(b), None if tree == {} else ctypes.byref(t), g["q"],
                                      g["qs"], g["hq"], g["scale"], g["window"], g["sinks"], g["o"], g["os"], None)
        assert rc == code and word in ctx.last_error(), (rc, ctx.last_error())

    note("kv tree refusals")
    refused("too large", batch=dict(n_tokens=2 ** 29), code=lodestar.LS_ERR_UNSUPPORTED)
    refused("tree must", tree={})
    refused("mask must", tree=dict(mask=None))
    refused("mask_words", tree=dict(mask_words=1))
    refused("mask_words", tree=dict(mask_words=-1))
    refused("positions", tree=dict(pos=None), window=5)
    refused("batch dtype", batch=dict(dtype=0))
    refused("max_new", batch=dict(max_new=0))
    refused("n_q_heads", hq=3)
    refused("scale", scale=float("inf"))
    refused("window", window=-1)
    refused("sinks", sinks=-1)
    refused("out", o=None)
    refused("q_stride", qs=8)
    torch.cuda.synchronize()
    assert (out == 5).all()
    with pytest.raises(ValueError):
        ctx.ls_kv_attention_tree(s.cache, s.batch, lodestar.Tree(s.tree.mask[:5]), q, out)
    for mask in (s.tree.mask[0], s.tree.mask.int(), s.tree.mask.cpu(), s.tree.mask[:, :1]):
        with pytest.raises(ValueError):
            lodestar.Tree(mask)
    with pytest.raises(ValueError):
        lodestar.Tree(s.tree.mask, s.tree.pos[:3])
