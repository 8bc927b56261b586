"""Keeping drafts, forking and compaction of the paged 8-bit KV cache on the GPU,
against the definitions (kv_draft_oracle).

Tables, ids and copied codes have to be equal.  A kept token's code is the nearest
to code times old / new scale with the factor rounded to 32 bits, as the oracle has it, so
codes are equal too; so are scales.
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


def i32(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


class Layers:
    """`layers` caches of one shape with random codes and scales, and their host copies."""

    def __init__(self, n_pages, layers=2, H=2, D=128, page=16, fmt="fp8", seed=0, spread=2.0):
        import torch
        r = np.random.RandomState(seed)
        self.rng, self.n_pages, self.H, self.D, self.page, self.fmt = r, n_pages, H, D, page, fmt
        self.host, self.bufs, caches = [], [], []
        for _ in range(layers):
            shape = (n_pages, H, page * D)
            if fmt == "fp8":
                codes = [r.choice(np.where(np.isfinite(ko.E4M3))[0], shape).astype(np.uint8) for _ in "kv"]
                scale = 2.0 ** np.round(r.normal(-7, spread, (2, n_pages, H)))
            else:
                codes = [r.randint(-127, 128, shape).astype(np.int8).view(np.uint8) for _ in "kv"]
                scale = np.exp(r.normal(-4.5, spread, (2, n_pages, H)))
            scale = scale.astype(np.float32)
            self.host.append(ko.Cache(codes[0].copy(), codes[1].copy(), scale[0], scale[1], n_pages, H, D, page, fmt))
            bufs = tuple(torch.from_numpy(x).cuda() for x in (*codes, *scale))
            self.bufs.append(bufs)
            caches.append(lodestar.KVCache(n_pages, H, D, dtype=fmt, page_tokens=page, buffers=bufs))
        self.caches = lodestar.KVLayers(caches)

    def same(self):
        """The device's caches are what the oracle made of the host's."""
        for i, (host, bufs) in enumerate(zip(self.host, self.bufs)):
            k, v, ks, vs = (t.cpu().numpy() for t in bufs)
            for name, codes, scale in (("k", k, ks), ("v", v, vs)):
                np.testing.assert_array_equal(scale.reshape(self.n_pages, self.H),
                                              host.scale[name].astype(np.float32), err_msg=f"layer {i} {name} scales")
                got = codes.reshape(self.n_pages, self.H, -1)
                bad = np.argwhere(got != host.codes[name])
                assert not len(bad), f"layer {i} {name}: {len(bad)} codes, the first at {bad[0]}"


# -- keeping drafts --------------------------------------------------------------

def check_keep(ctx, lay, seqs, paths, absent=(), lists=None, count=None, off=None):
    """seqs: (past, new); paths: what each keeps (or `lists` and `count` as the call has them)."""
    past, new = np.array([s[0] for s in seqs]), np.array([s[1] for s in seqs])
    need = -(-(past + new) // lay.page)
    table = np.full((len(seqs), max(1, int(need.max()))), -1)
    ids, at = lay.rng.permutation(lay.n_pages), 0
    assert need.sum() <= lay.n_pages
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    for b, j, p in absent:
        table[b, j] = p
    off = np.concatenate([[0], np.cumsum(new)]) if off is None else np.array(off)
    T = int(new.sum()) if lists is None else len(lists)
    if lists is None:
        lists, count = np.full(T, -9), np.zeros(len(seqs), int)
        for b, p in enumerate(paths):
            lists[off[b]:off[b] + len(p)], count[b] = p, len(p)
    batch = lodestar.KVBatch(i32(off), i32(past), i32(table), T, max(1, int(new.max())))
    for host in lay.host:
        kd.keep(host, off, past, table, np.asarray(lists), np.asarray(count))
    import torch
    ctx.ls_kv_keep(lay.caches, batch, i32(lists), i32(count))
    torch.cuda.synchronize()
    lay.same()
    return batch


SEQS = [(0, 8), (15, 9), (16, 64), (300, 8), (47, 33), (0, 1), (100, 0), (61, 40), (31, 17)]


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 16), (256, 32), (128, 64), (64, 128)])
def test_paths(ctx, D, page, fmt):
    lay = Layers(100, D=D, page=page, fmt=fmt, seed=D + page)
    r = lay.rng
    paths = [sorted(r.choice(n, r.randint(1, min(n, 9) + 1), replace=False).tolist()) if n else [] for _, n in SEQS]
    note(f"kv keep D={D} page={page} {fmt}")
    check_keep(ctx, lay, SEQS, paths)


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_nothing_everything_and_the_last(ctx, page, fmt):
    """Lists that keep no draft, all of them (nothing moves), all but the first (everything moves by one), the last one."""
    seqs = [(20, 30), (20, 30), (20, 130), (5, 77), (0, 16), (16, 16)]
    paths = [[], list(range(30)), list(range(1, 130)), [76], list(range(1, 16)), [0, 1, 15]]
    note(f"kv keep all and none page={page} {fmt}")
    check_keep(ctx, Layers(60, H=3, page=page, fmt=fmt, seed=page), seqs, paths)


def test_even_scales_move_codes_unchanged(ctx):
    """Pages of one scale: a kept token's codes are what they were."""
    import torch
    lay = Layers(8, layers=1, H=1, seed=3, spread=0.0)
    note("kv keep even scales")
    host = ko.Cache(*(t.cpu().numpy().copy() for t in lay.bufs[0]), 8, 1, 128, 16, "fp8")
    batch = check_keep(ctx, lay, [(10, 40)], [[2, 9, 33]])
    table = batch.pages.cpu().numpy()[0]
    now = ko.Cache(*(t.cpu().numpy() for t in lay.bufs[0]), 8, 1, 128, 16, "fp8")
    assert torch.equal(lay.bufs[0][2], torch.from_numpy(host.scale["k"]).float().cuda())
    for name in "kv":
        a, _ = host.tokens(name, table, 50)
        b, _ = now.tokens(name, table, 50)
        np.testing.assert_array_equal(b[10:13], a[[12, 19, 43]])
        np.testing.assert_array_equal(b[:10], a[:10])


def test_absent_pages(ctx):
    """Tokens whose old or new page is absent stay; ids outside the pool count as absent."""
    lay = Layers(60, seed=4)
    note("kv keep absent pages")
    check_keep(ctx, lay, [(14, 60), (40, 20), (0, 40), (33, 33)],
               [[3, 20, 30, 45], [5, 19], [18, 20, 39], [1, 2, 30]],
               absent=[(0, 2, -1), (1, 2, 60), (2, 0, -5), (2, 1, 2 ** 31 - 1), (3, 3, -1)])


def test_lists_that_break_the_rules(ctx):
    """A list ends before the first entry that does not ascend or is no new token; counts are held to the drafts."""
    lay = Layers(80, seed=5)
    seqs = [(14, 8), (30, 8), (50, 8), (3, 8), (17, 8), (70, 8), (9, 70)]
    lists = np.concatenate([[2, 5, 5, 7, 0, 0, 0, 0], [4, 3, 6, 7, 0, 0, 0, 0], [1, 8, 2, 3, 4, 5, 6, 7], [-1, 3, 4, 5, 6, 7, 0, 0],
                            [1, 3, 5, 7, 9, 11, 13, 15], [0, 1, 2, 3, 4, 5, 6, 7], np.arange(70) + 1])
    lists[-4] = 2
    note("kv keep broken lists")
    check_keep(ctx, lay, seqs, None, lists=lists, count=np.array([8, 5, 8, 3, 2 ** 31 - 1, -4, 69]))


def test_padded_batches(ctx):
    lay = Layers(80, seed=6)
    lists = lay.rng.permutation(60)
    note("kv keep padded")
    check_keep(ctx, lay, [(20, 9), (3, 0), (40, 20)], None, lists=np.sort(lists % 20), count=[3, 5, 9], off=[4, 13, 13, 33])
    for bad in ([0, 2 ** 30, 5, -7], [9, 5, 3, 1]):
        batch = lodestar.KVBatch(i32(bad), i32([2 ** 31 - 1, -3, 30]), i32(lay.rng.randint(-2, 90, (3, 5))), 60, 20)
        note(f"kv keep offsets {bad}")
        ctx.ls_kv_keep(lay.caches, batch, i32(lists), i32([60, 60, 60]))
    import torch
    torch.cuda.synchronize()


def test_many_layers(ctx):
    """More layers than a launch takes."""
    lay = Layers(12, layers=131, H=1, D=64, seed=7)
    note("kv keep 131 layers")
    check_keep(ctx, lay, [(10, 20), (3, 40)], [[4, 7, 19], [39]])


# -- forking ---------------------------------------------------------------------

def check_fork(ctx, lay, pages, pages_out, src, dst, tokens, in_place=False):
    import torch
    want = pages_out.copy()
    for host in lay.host:
        out = pages_out.copy()
        kd.fork(host, pages, out, src, dst, tokens)
        want = out
    p = i32(pages)
    o = p if in_place else i32(pages_out)
    ctx.ls_kv_fork(lay.caches, p, o, i32(src), i32(dst), i32(tokens))
    torch.cuda.synchronize()
    np.testing.assert_array_equal(o.cpu().numpy(), want)
    if not in_place:
        np.testing.assert_array_equal(p.cpu().numpy(), pages)
    lay.same()


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("D,page,W", [(64, 16, 5), (128, 16, 300), (256, 32, 4), (128, 128, 3), (64, 64, 257)])
def test_forks(ctx, D, page, W, fmt):
    lay = Layers(64, D=D, page=page, fmt=fmt, seed=D + W)
    r = lay.rng
    pages, out = r.randint(0, 32, (9, W)), r.randint(0, 32, (9, W))
    # all lengths' last pages: fresh ones of their own
    tokens = np.array([0, 1, 15, page - 1, page, page + 1, W * page - 1, W * page, 2 * page + page // 2])
    dst = r.permutation(9)
    for i, d in enumerate(dst):
        if tokens[i] % page:
            out[d, tokens[i] // page] = 40 + i
    note(f"kv fork D={D} page={page} W={W} {fmt}")
    check_fork(ctx, lay, pages, out, r.randint(0, 9, 9), dst, tokens)


def test_in_one_table(ctx):
    """pages_out may be pages where no row is both taken from and written."""
    lay = Layers(40, H=3, seed=1)
    pages = lay.rng.permutation(40).reshape(8, 5)
    note("kv fork in place")
    check_fork(ctx, lay, pages, pages.copy(), [0, 0, 0, 1], [4, 5, 6, 7], [40, 33, 0, 79], in_place=True)


def test_same_and_absent_pages(ctx):
    """A row that goes on by itself; pages that are absent on either side; rows and lengths outside the table."""
    lay = Layers(30, seed=2)
    pages = np.array([[0, 1, 2], [3, -1, 4], [5, 6, 30], [7, 8, 9]])
    out = np.array([[20, 21, 2], [22, 23, 24], [25, -1, 26], [27, 28, 29]])
    note("kv fork same and absent")
    check_fork(ctx, lay, pages, out, [0, 1, 2, 3], [0, 1, 2, 3], [40, 20, 33, 2 ** 31 - 1])
    lay = Layers(30, seed=3)
    check_fork(ctx, lay, pages, out, [-1, 4, 0, 2 ** 31 - 1, 3], [0, 1, -1, 2, 3], [20, 20, 20, 20, -7])
    lay = Layers(30, seed=3)
    check_fork(ctx, lay, pages, out, [0, 3], [2, 1], [17, 18])


def test_beams_change_places(ctx):
    """Two tables in turn: every row takes over another one, or goes on by itself on its own last page."""
    lay = Layers(40, seed=5)
    pages = np.concatenate([np.tile(np.arange(3), (4, 1)), np.arange(3, 7)[:, None]], 1)
    out = np.concatenate([np.tile([30, 31, 32], (4, 1)), np.arange(7, 11)[:, None]], 1)
    out[2, 3] = pages[2, 3]
    note("kv fork beams")
    check_fork(ctx, lay, pages, out, [1, 0, 2, 0], [0, 1, 2, 3], [55] * 4)


def test_fork_of_many_layers_and_none(ctx):
    lay = Layers(9, layers=65, H=1, D=64, seed=6)
    note("kv fork 65 layers")
    check_fork(ctx, lay, np.arange(4).reshape(2, 2), np.arange(4, 8).reshape(2, 2), [0, 1], [1, 0], [17, 31])
    check_fork(ctx, lay, np.arange(4).reshape(2, 2), np.arange(4, 8).reshape(2, 2), [], [], [])


# -- compaction ------------------------------------------------------------------

def check_compact(ctx, lay, pages, in_place=False):
    import torch
    want, where, used, moves = kd.compact(lay.n_pages, pages)
    p = i32(pages)
    o = p if in_place else torch.full_like(p, 77)
    w, n = torch.full((lay.n_pages,), -9, dtype=torch.int32, device="cuda"), i32([-9])
    ctx.ls_kv_compact(lay.caches, p, o, w, n)
    torch.cuda.synchronize()
    assert int(n) == used
    np.testing.assert_array_equal(w.cpu().numpy(), where)
    np.testing.assert_array_equal(o.cpu().numpy(), want)
    for host in lay.host:
        for name in "kv":
            for a, b in moves:
                host.codes[name][b], host.scale[name][b] = host.codes[name][a], host.scale[name][a]
    lay.same()


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("D,page,H,n_pages,named", [(64, 16, 1, 50, 20), (128, 16, 2, 300, 290), (256, 32, 3, 70, 5), (128, 128, 1, 33, 33),
                                                    (64, 16, 5, 1, 1), (64, 64, 2, 64, 32)])
def test_compaction(ctx, D, page, H, n_pages, named, fmt):
    lay = Layers(n_pages, H=H, D=D, page=page, fmt=fmt, seed=n_pages)
    ids = lay.rng.permutation(n_pages)[:named]
    table = np.full((3, named + 4), -1)
    table[0, :named] = ids
    table[1, 2:2 + named // 2] = ids[:named // 2]                 # shared pages stay shared
    table[2, :3] = [n_pages, 2 ** 31 - 1, -2 ** 31]               # absent entries stay as they are
    note(f"kv compact D={D} page={page} H={H} {named} of {n_pages} {fmt}")
    check_compact(ctx, lay, table)


@pytest.mark.parametrize("n_pages", [4095, 4096, 4097, 9000, 40000])
@pytest.mark.parametrize("share", [0.02, 0.5, 0.97])
def test_pools_of_many_chunks(ctx, n_pages, share):
    lay = Layers(n_pages, layers=1, H=1, D=64, seed=n_pages)
    r = lay.rng
    ids = np.where(r.rand(n_pages) < share)[0]
    table = np.resize(r.permutation(ids), (7, len(ids) // 5 + 3))
    note(f"kv compact {n_pages} pages {share}")
    check_compact(ctx, lay, table, in_place=True)


@pytest.mark.parametrize("n_pages,rows,width,share", [
    (65535, 3, 20000, 0.6), (65536, 1, 65536, 0.5), (65537, 7, 9000, 0.5), (70001, 2, 10, 0.9),    # either side of one workgroup's plan
    (5000, 2, 65536, 0.4), (5000, 1, 131073, 0.4), (12289, 64, 2049, 0.97)])                       # and of its table
def test_large_pools_and_tables(ctx, n_pages, rows, width, share):
    lay = Layers(n_pages, layers=1, H=1, D=64, seed=n_pages)
    ids = np.where(lay.rng.rand(n_pages) < share)[0]
    table = lay.rng.choice(ids, (rows, width))
    table[lay.rng.rand(rows, width) < 0.1] = -1
    note(f"kv compact {n_pages} pages, table {rows} x {width}")
    check_compact(ctx, lay, table)


def test_nothing_and_all_named(ctx):
    note("kv compact nothing, all, above, below")
    check_compact(ctx, Layers(20, seed=1), np.full((2, 3), -1))
    check_compact(ctx, Layers(20, seed=1), np.zeros((0, 3), int))
    check_compact(ctx, Layers(20, seed=1), np.arange(20)[None])
    check_compact(ctx, Layers(20, seed=1), np.arange(10, 20)[None])          # all move
    check_compact(ctx, Layers(20, seed=1), np.arange(10)[None], in_place=True)


def test_many_layers_move(ctx):
    note("kv compact 70 layers")
    check_compact(ctx, Layers(24, layers=70, H=1, D=64, seed=2), np.array([[23, 1, 20, -1, 9]]))


# -- together ----------------------------------------------------------------------

def test_graph_replays(ctx):
    """Keep, fork and compaction in one graph, replayed with other lists and tables, beside the oracle."""
    import torch
    lay = Layers(60, seed=8)
    past, off = np.array([20, 37]), np.array([0, 16, 40])
    table = lay.rng.permutation(60)[:16].reshape(4, 4)
    tables, out, comp = i32(table), i32(table), torch.empty(4, 4, dtype=torch.int32, device="cuda")
    batch = lodestar.KVBatch(i32(off), i32(past), i32(table[:2]), 40, 24)
    kept, count = i32(np.zeros(40)), i32([0, 0])
    src, dst, tokens = i32([0, 1]), i32([2, 3]), i32([0, 0])
    where, used = torch.empty(60, dtype=torch.int32, device="cuda"), i32([0])

    def step():
        ctx.ls_kv_keep(lay.caches, batch, kept, count)
        ctx.ls_kv_fork(lay.caches, tables, out, src, dst, tokens)
        ctx.ls_kv_compact(lay.caches, out, comp, where, used)

    def host(lists, n, t):
        o = table.copy()
        for h in lay.host:
            kd.keep(h, off, past, table, lists, n)
            o = table.copy()
            kd.fork(h, table, o, [0, 1], [2, 3], t)
            for a, b in kd.compact(60, o)[3]:
                for name in "kv":
                    h.codes[name][b], h.scale[name][b] = h.codes[name][a], h.scale[name][a]
        return kd.compact(60, o)

    note("kv pages graph: warm call")
    step()
    host(np.zeros(40, int), [0, 0], [0, 0])
    torch.cuda.synchronize()
    lay.same()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        note(f"kv pages graph: replay {i}")
        lists = np.concatenate([np.sort(lay.rng.permutation(16)), np.sort(lay.rng.permutation(24))])
        lists[:5], lists[16:19] = np.sort(lay.rng.choice(16, 5, False)), np.sort(lay.rng.choice(24, 3, False))
        n, t = np.array([5, 3]), np.array([20 + 5, 37 + 3])
        kept.copy_(torch.from_numpy(lists))
        count.copy_(torch.from_numpy(n))
        tokens.copy_(torch.from_numpy(t))
        out.copy_(tables)
        g.replay()
        torch.cuda.synchronize()
        want = host(lists, n, t)
        np.testing.assert_array_equal(comp.cpu().numpy(), want[0])
        assert int(used) == want[2]
        lay.same()


@pytest.mark.parametrize("fmt,D,window", [("fp8", 128, 0), ("int8", 64, 40)])
def test_a_drafting_loop(ctx, fmt, D, window):
    """Prompt, fork, drafts, attention, keep, compaction: what the cache gives at the end is what appending the kept tokens
    one after the other gives, to the codes' steps, and attention at each stage is the definition's on what it holds."""
    import torch
    from test_gpu_kv_tree import check, grown
    H, G, page, n_pages = 2, 4, 16, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()  # noqa: E731
    half = D // 2
    turn = torch.arange(400, device="cuda").double()[:, None] * 100.0 ** (-torch.arange(half, device="cuda").double() / half)
    rope = lodestar.Rope(turn.cos().float(), turn.sin().float())
    caches = [lodestar.KVCache(n_pages, H, D, dtype=fmt, page_tokens=page) for _ in range(2)]
    plain = [lodestar.KVCache(n_pages, H, D, dtype=fmt, page_tokens=page) for _ in range(2)]
    layers = lodestar.KVLayers(caches)
    r = np.random.RandomState(4)
    ids = r.permutation(n_pages)[:24]
    table = np.full((2, 12), -1)
    table[0], table[1] = ids[:12], ids[12:]
    pages = i32(table)
    P = 75
    prompt = lodestar.KVBatch(i32([0, P]), i32([0]), pages[:1].contiguous(), P)
    keys = [rand(P, H, D) for _ in range(4)]
    for c, p, k, v in zip(caches, plain, keys[::2], keys[1::2]):
        ctx.ls_kv_append(c, prompt, k, v, rope=rope)
        ctx.ls_kv_append(p, prompt, k, v, rope=rope)
    note("kv loop: fork")
    ctx.ls_kv_fork(layers, pages, pages, i32([0]), i32([1]), i32([P]))
    for p in plain:
        ctx.ls_kv_fork(p, pages, pages, i32([0]), i32([1]), i32([P]))
    past = np.array([P, P])
    for turn_ in range(3):
        n = np.array([9, 20])
        trees = [kd.ancestry(kd.tree_parents(int(x), 4, r)) for x in n]
        off = np.concatenate([[0], np.cumsum(n)])
        T = int(n.sum())
        batch = lodestar.KVBatch(i32(off), i32(past), pages, T, 20)
        depth = np.concatenate([d + p for (_, d), p in zip(trees, past)])
        at = lodestar.Positions(i32(depth))
        tree = lodestar.Tree(torch.from_numpy(np.concatenate([kd.words(s, 1) for s, _ in trees]).view(np.int64)).cuda(), at.pos)
        new = [rand(T, H, D) for _ in range(4)]
        paths = []
        for s, _ in trees:
            leaf = r.randint(0, len(s))
            paths.append(np.where(s[leaf])[0].tolist())
        kept, count = np.zeros(T, int), np.array([len(p) for p in paths])
        for b, p in enumerate(paths):
            kept[off[b]:off[b] + len(p)] = p
        q = rand(T, H * G, D)
        for c, k, v in zip(caches, new[::2], new[1::2]):
            turned, out = torch.empty_like(q), torch.empty_like(q)
            ctx.ls_kv_append_at(c, batch, at, k, v, rope, q=q, q_out=turned)
            ctx.ls_kv_attention_tree(c, batch, tree, turned, out, window=window, sinks=2)
            torch.cuda.synchronize()
            host = ko.Cache(*(t.cpu().numpy() for t in (c.k, c.v, c.k_scale, c.v_scale)), n_pages, H, D, page, fmt)
            want, mag = kd.attention_tree(host, turned.double().cpu().numpy(), off, past, pages.cpu().numpy(),
                                          [s for s, _ in trees], depth, D ** -0.5, window, 2)
            assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -9 * mag).all()
        note(f"kv loop: keep, turn {turn_}")
        ctx.ls_kv_keep(layers, batch, i32(kept), i32(count))
        # the kept tokens alone, at their positions
        rows = np.concatenate([off[b] + np.array(p) for b, p in enumerate(paths)])
        o2 = np.concatenate([[0], np.cumsum(count)])
        lean = lodestar.KVBatch(i32(o2), i32(past), pages, len(rows))
        for p, k, v in zip(plain, new[::2], new[1::2]):
            ctx.ls_kv_append(p, lean, k[rows].contiguous(), v[rows].contiguous(), rope=rope)
        past = past + count
    moved = torch.empty_like(pages)
    where, used = torch.empty(n_pages, dtype=torch.int32, device="cuda"), i32([0])
    note("kv loop: compaction")
    ctx.ls_kv_compact(layers, pages, moved, where, used)
    torch.cuda.synchronize()
    assert int(used) == len(set(pages.cpu().numpy().ravel().tolist())) and int(moved.max()) == int(used) - 1
    for c, p in zip(caches, plain):
        for b in range(2):
            one = lambda t: lodestar.KVBatch(i32([0, past[b]]), i32([0]), t[b:b + 1].contiguous(), int(past[b]))  # noqa: E731
            got, want = ([torch.empty(int(past[b]), H, D, dtype=torch.float16, device="cuda") for _ in "kv"] for _ in "ab")
            ctx.ls_kv_read(c, one(moved), *got)
            ctx.ls_kv_read(p, one(pages), *want)
            for x, y, scales in zip(got, want, (c.k_scale, c.v_scale)):
                # a code's step at most 1/8 (fp8) or 1/127 of what the page's scale covers; a token was rounded up to five times
                top = y.float().abs().amax()
                assert ((x - y).float().abs() <= (0.16 * y.float().abs() + 2.0 ** -8 * top if fmt == "fp8" else 0.05 * top)).all()


def test_refusals(ctx):
    import ctypes
    import torch
    lay = Layers(20, seed=9)
    other = lodestar.KVCache(21, 2, 128)
    lib = lodestar.library()
    t, z = i32(np.arange(12).reshape(3, 4)), i32([0, 1, 2])
    where, used = torch.zeros(20, dtype=torch.int32, device="cuda"), i32([0])
    batch = lodestar.KVBatch(i32([0, 1, 2, 3]), z, t, 3)

    def refused(word, rc, code=lodestar.LS_ERR_INVALID):
        assert rc == code and word in ctx.last_error(), (rc, ctx.last_error())

    def keep(c=lay.caches.ref, n=2, b=batch.ref, k=z.data_ptr(), m=z.data_ptr()):
        return lib.ls_kv_keep(ctx.h, c, n, b, k, m, None)

    def fork(c=lay.caches.ref, n=2, rows=3, W=4, p=t.data_ptr(), o=t.data_ptr(), m=1, s=z.data_ptr(), d=z.data_ptr(), k=z.data_ptr()):
        return lib.ls_kv_fork(ctx.h, c, n, rows, W, p, o, m, s, d, k, None)

    def compact(c=lay.caches.ref, n=2, rows=3, W=4, p=t.data_ptr(), o=t.data_ptr(), w=where.data_ptr(), u=used.data_ptr()):
        return lib.ls_kv_compact(ctx.h, c, n, rows, W, p, o, w, u, None)

    note("kv pages refusals")
    for call in (keep, fork, compact):
        refused("caches must", call(c=None))
        refused("n_caches", call(n=0))
        for field, value, word in (("dtype", 1 - lay.caches.c[1].dtype, "same"), ("n_pages", 21, "same"), ("head_dim", 64, "same"),
                                   ("page_tokens", 32, "same"), ("n_kv_heads", 1, "same"), ("dtype", 9, "cache dtype"),
                                   ("v", None, "arrays"), ("k", lay.caches.c[1].k + 8, "aligned"), ("head_dim", 96, "head_dim")):
            bad = (lodestar.ls_kv_cache * 2).from_buffer_copy(lay.caches.c)
            setattr(bad[1], field, value)
            refused(word, call(c=bad))
        for name in "kv":
            bad = (lodestar.ls_kv_cache * 2).from_buffer_copy(lay.caches.c)
            setattr(bad[1], name, getattr(bad[0], name))
            refused("twice", call(c=bad))
    many = type(batch.c).from_buffer_copy(batch.c)
    many.n_seqs = 2 ** 24
    refused("too large", keep(b=ctypes.byref(many)), lodestar.LS_ERR_UNSUPPORTED)
    refused("too large", fork(m=2 ** 24), lodestar.LS_ERR_UNSUPPORTED)
    refused("batch must", keep(b=None))
    refused("kept", keep(k=None))
    refused("n_kept", keep(m=None))
    for name in "posdk":
        refused("non-NULL", fork(**{name: None}))
    refused("n_rows", fork(rows=-1))
    refused("n_forks", fork(m=-1))
    refused("pages_stride", fork(W=0))
    refused("at most 2^30", fork(W=2 ** 27))
    for name in "powu":
        refused("non-NULL", compact(**{name: None}))
    refused("n_rows", compact(rows=-1))
    refused("pages_stride", compact(W=0))
    huge = (lodestar.ls_kv_cache * 1).from_buffer_copy(bytes(lay.caches.c)[:ctypes.sizeof(lodestar.ls_kv_cache)])
    huge[0].n_pages = 20_000_000
    refused("16 million", compact(c=huge, n=1), lodestar.LS_ERR_UNSUPPORTED)
    torch.cuda.synchronize()
    lay.same()
    assert t.cpu().numpy().ravel().tolist() == list(range(12)) and int(used) == 0
    with pytest.raises(lodestar.LodestarError, match="same"):
        ctx.ls_kv_keep(lodestar.KVLayers([*lay.caches.caches, other]), batch, z, z)
    with pytest.raises(ValueError):
        lodestar.KVLayers([])
    with pytest.raises(ValueError):
        ctx.ls_kv_keep(lay.caches, batch, z[:2], z)
    with pytest.raises(ValueError):
        ctx.ls_kv_fork(lay.caches, t, t[:2], z, z, z)
    with pytest.raises(ValueError):
        ctx.ls_kv_fork(lay.caches, t, t, z, z[:2], z)
    with pytest.raises(ValueError):
        ctx.ls_kv_compact(lay.caches, t, t, where[:5], used)


def test_first_compaction_on_a_capturing_stream(ctx):
    import torch
    lay = Layers(20, seed=9)
    t = i32(np.arange(12).reshape(3, 4))
    where, used = torch.zeros(20, dtype=torch.int32, device="cuda"), i32([0])
    fresh = lodestar.Context(16, (64, 64))
    x = torch.zeros(1, device="cuda")
    note("kv compact first call captured")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x.add_(1)
        with pytest.raises(lodestar.LodestarError, match="before capturing"):
            fresh.ls_kv_compact(lay.caches, t, t, where, used)
    fresh.close()
