"""The paged 8-bit KV cache on the GPU: appending, attention and reading back,
against the definitions in 64 bits (kv_oracle).

Tolerances.  Attention: the output's own rounding, 2^-8 (bf16) or 2^-10 (half)
of its size -- twice the unit roundoff -- and 2^-9 of sum_j p_j |v_j| for the
probabilities, which enter the product rounded to half precision (2^-11), and
the fp32 scores and sums.  Stored values: half a step of the code, and 2^-20 of
the rotated pair's size for the fp32 rotation and scaling; scales exactly (fp8)
or to 2^-22 (int8).
"""
import numpy as np
import pytest

import kv_oracle as ko
from gpu_helpers import note
from paper_2606_00946_amd import lodestar

pytestmark = pytest.mark.gpu

KINDS = {"bf16": "bfloat16", "f16": "float16"}


@pytest.fixture(scope="module")
def ctx():
    c = lodestar.Context(16, (64, 64))
    yield c
    c.close()


class Setup:
    """Sequences of (past, new) tokens on pages scattered over a pool, the whole cache held by random codes."""

    def __init__(self, seqs, H=2, D=128, page=16, fmt="fp8", kind="bf16", seed=0, poison=True, absent=(), spare=2):
        import torch
        r = np.random.RandomState(seed)
        self.rng, self.H, self.D, self.page, self.fmt = r, H, D, page, fmt
        self.kind = getattr(torch, KINDS[kind])
        past, new = np.array([s[0] for s in seqs]), np.array([s[1] for s in seqs])
        need = -(-(past + new) // page)
        W = max(1, int(need.max()))
        self.n_pages = int(need.sum()) + spare
        ids = r.permutation(self.n_pages)
        table, at = np.full((len(seqs), W), -1), 0
        for b, n in enumerate(need):
            table[b, :n] = ids[at:at + n]
            at += n
        for b, j in absent:
            table[b, j] = -1
        shape = (self.n_pages, H, page * D)
        if fmt == "fp8":
            codes = [r.choice(np.where(np.isfinite(ko.E4M3))[0], shape).astype(np.uint8) for _ in "kv"]
            scale = 2.0 ** r.randint(-9, -6, (2, self.n_pages, H))
        else:
            codes = [r.randint(-127, 128, shape).astype(np.int8).view(np.uint8) for _ in "kv"]
            scale = np.exp(r.normal(-4.5, 0.3, (2, self.n_pages, H)))
        if poison and fmt == "fp8":
            # what no token holds is NaN: rows past a sequence's end, and whole pages of nobody
            for c, name in zip(codes, "kv"):
                o = ko.offsets(page, D, name == "v")
                for p in set(range(self.n_pages)) - set(table.ravel().tolist()):
                    c[p] = 0x7F
                for b in range(len(seqs)):
                    end = int(past[b] + new[b])
                    if end % page and table[b, end // page] >= 0:
                        c[table[b, end // page]][:, o[end % page:].ravel()] = 0xFF
        dev = lambda a, t=None: torch.from_numpy(np.ascontiguousarray(a)).to("cuda", t)  # noqa: E731
        self.past, self.new, self.table = past, new, table
        self.off = np.concatenate([[0], np.cumsum(new)])
        self.T = int(new.sum())
        self.bufs = (dev(codes[0]), dev(codes[1]), dev(scale[0].astype(np.float32)), dev(scale[1].astype(np.float32)))
        self.cache = lodestar.KVCache(self.n_pages, H, D, dtype=fmt, page_tokens=page, buffers=self.bufs)
        self.batch = lodestar.KVBatch(dev(self.off, torch.int32), dev(past, torch.int32), dev(table, torch.int32), self.T,
                                      max(1, int(new.max())))

    def host(self):
        k, v, ks, vs = (t.cpu().numpy().copy() for t in self.bufs)
        return ko.Cache(k, v, ks, vs, self.n_pages, self.H, self.D, self.page, self.fmt)

    def tensor(self, heads, sigma=1.0, extra=0):
        """A random [T x heads x D] tensor; extra > 0: rows that far apart in a wider one."""
        import torch
        x = torch.from_numpy(self.rng.normal(0, sigma, (self.T, heads * self.D + extra)).astype(np.float32))
        x = x.to("cuda", self.kind)[:, :heads * self.D]
        return x.unflatten(1, (heads, self.D))


def check_attention(ctx, s, G, window=0, sinks=0, sigma=1.0, extra=0, scale=None):
    import torch
    q = s.tensor(s.H * G, sigma, extra)
    out = torch.full((s.T, s.H * G, s.D), 7.0, dtype=s.kind, device="cuda")
    ctx.ls_kv_attention(s.cache, s.batch, q, out, scale=scale, window=window, sinks=sinks)
    torch.cuda.synchronize()
    want, mag = ko.attention(s.host(), q.double().cpu().numpy(), s.off, s.past, s.table,
                             s.D ** -0.5 if scale is None else scale, window, sinks)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    u = 2.0 ** -8 if s.kind == torch.bfloat16 else 2.0 ** -10
    off = np.abs(got - want) - (u * np.abs(want) + 2.0 ** -9 * mag + 1e-7)
    assert off.max() <= 0, f"off by {np.abs(got - want).max()} at {np.unravel_index(off.argmax(), off.shape)}"
    return out


DECODE = [(0, 1), (1, 1), (15, 1), (16, 1), (300, 1), (63, 1), (64, 1), (1023, 1)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("D,page,G", [(64, 16, 1), (128, 16, 4), (256, 32, 8), (128, 64, 7), (64, 128, 16), (128, 16, 17)])
def test_decode(ctx, D, page, G, fmt, kind):
    note(f"kv decode D={D} page={page} G={G} {fmt} {kind}")
    check_attention(ctx, Setup(DECODE, D=D, page=page, fmt=fmt, kind=kind, seed=D + G), G)


@pytest.mark.parametrize("fmt,kind", [("fp8", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("D,page,G", [(64, 16, 2), (128, 16, 4), (128, 32, 3), (256, 16, 2), (128, 128, 8)])
def test_prompts(ctx, D, page, G, fmt, kind):
    """Chunks of prompts beside single tokens and sequences without new tokens."""
    seqs = [(0, 1), (0, 200), (37, 70), (500, 0), (129, 1), (640, 33), (0, 0), (5, 131)]
    note(f"kv prompts D={D} page={page} G={G} {fmt} {kind}")
    check_attention(ctx, Setup(seqs, D=D, page=page, fmt=fmt, kind=kind, seed=D + G), G)


@pytest.mark.parametrize("G,new", [(1, 1), (1, 2), (8, 2), (8, 3), (4, 16), (5, 13), (16, 9), (2, 65)])
def test_few_rows(ctx, G, new):
    """Around the row counts where the kernels change: several new tokens over a long past, one kv head."""
    note(f"kv few rows G={G} new={new}")
    check_attention(ctx, Setup([(2000, new), (3, 1), (900, max(1, new // 2))], H=1, seed=G + new), G)


@pytest.mark.parametrize("window,sinks", [(1, 0), (16, 0), (17, 3), (100, 16), (250, 33), (5000, 0), (64, 1000)])
@pytest.mark.parametrize("D,G,fmt", [(128, 4, "fp8"), (64, 8, "int8")])
def test_window_and_sinks(ctx, D, G, fmt, window, sinks):
    seqs = [(0, 1), (900, 1), (300, 130), (1000, 3), (0, 260), (17, 1), (700, 40)]
    note(f"kv window={window} sinks={sinks} D={D} G={G} {fmt}")
    check_attention(ctx, Setup(seqs, D=D, fmt=fmt, seed=window), G, window, sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 4)])
def test_absent_pages(ctx, window, sinks):
    """Pages given back: hidden tokens, rows that see nothing (0), and ids outside the pool."""
    seqs = [(40, 1), (100, 40), (3, 1), (200, 1), (0, 16), (48, 20)]
    absent = [(0, 0), (0, 2), (1, 1), (2, 0), (4, 0), (5, 3), (5, 4)] + [(1, j) for j in range(6, 9)]
    s = Setup(seqs, seed=5, absent=absent)
    import torch
    s.table[3, 4], s.table[3, 5] = s.n_pages, -7
    s.batch.pages.copy_(torch.from_numpy(s.table).to("cuda", torch.int32))
    note(f"kv absent pages window={window}")
    out = check_attention(ctx, s, 4, window, sinks)
    assert (out[s.off[2]] == 0).all() and (out[s.off[4]:s.off[5]] == 0).all()


def test_lengths_past_the_table(ctx):
    """A position past the page table: its tokens are absent, nothing is read beyond the table."""
    import torch
    s = Setup([(100, 5), (30, 2)], seed=9, poison=False)         # whole pages become visible
    s.batch.past.copy_(torch.tensor([2 ** 31 - 20, 30], dtype=torch.int32))
    s.past = np.array([s.table.shape[1] * s.page + 50, 30])      # the same tokens are visible from there
    note("kv past the table")
    check_attention(ctx, s, 4)


def test_large_logits_and_values(ctx):
    """Logits far apart (one key takes all) and scales at both ends of their range."""
    import torch
    s = Setup([(333, 1), (50, 40)], seed=3)
    note("kv large logits")
    check_attention(ctx, s, 4, sigma=60.0, scale=1.0)
    s.bufs[3].copy_(torch.where(torch.rand_like(s.bufs[3]) < 0.5, 2.0 ** -60, 2.0 ** -20))
    note("kv tiny values")
    check_attention(ctx, s, 4, scale=0.02)
    s.bufs[3].fill_(2.0 ** 40)
    s.kind = torch.bfloat16
    note("kv huge values")
    check_attention(ctx, s, 4, scale=0.02)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [None, 0.0, 1e-38, -0.1])
def test_zero_queries_and_keys(ctx, kind, scale):
    """Padding rows: queries and whole blocks of keys of zeros (whose scale is the least) weigh all tokens alike."""
    import torch
    s = Setup([(0, 200), (40, 1), (70, 90), (0, 1)], kind=kind, seed=21)
    keys, scales = s.bufs[0].view(s.n_pages, -1), s.bufs[2].view(s.n_pages, -1)
    for b in range(3):
        pages = torch.from_numpy(s.table[b, :5:2].copy()).cuda()
        keys[pages[pages >= 0]], scales[pages[pages >= 0]] = 0, 2.0 ** -64
    tensor = s.tensor

    def some_zero(heads, *a):
        q = tensor(heads, *a)
        q[::3] = 0
        q[1::3, 0] *= 2.0 ** -60
        return q
    s.tensor = some_zero
    note(f"kv zero queries and keys {kind} scale={scale}")
    check_attention(ctx, s, 4, scale=scale)
    check_attention(ctx, s, 4, window=50, sinks=3, scale=scale)


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_scales_of_zero(ctx, fmt):
    """Pages as a new cache holds them, codes and scales zero: tokens whose score and value are 0."""
    s = Setup([(0, 200), (40, 1), (70, 90), (33, 1)], fmt=fmt, seed=22)
    for b in range(3):
        for j in range(0, 5, 2):
            if 0 <= s.table[b, j] < s.n_pages:
                for t in s.bufs:
                    t.view(s.n_pages, -1)[int(s.table[b, j])] = 0
    for t in s.bufs:
        t.view(s.n_pages, -1)[s.table[3, :3].tolist()] = 0
    note(f"kv scales of zero {fmt}")
    out = check_attention(ctx, s, 4)
    assert (out[s.off[3]] == 0).all()
    check_attention(ctx, s, 4, window=30, sinks=5)


@pytest.mark.parametrize("window,sinks", [(20, 0), (37, 5), (100, 18), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_nan_behind_the_window(ctx, window, sinks):
    """NaN codes in tokens that the window hides from every row, beside visible ones of the same block."""
    s = Setup([(300, 1), (900, 1), (333, 40), (261, 2), (500, 70)], H=1, seed=23)
    for b, past in enumerate(s.past):
        for name, buf in zip("kv", s.bufs):
            codes, o = buf.view(s.n_pages, -1), ko.offsets(s.page, s.D, name == "v")
            for t in range(sinks, past + 1 - window):
                codes[int(s.table[b, t // s.page]), o[t % s.page].tolist()] = 0x7F
    note(f"kv nan behind window={window} sinks={sinks}")
    check_attention(ctx, s, 8, window, sinks)


def test_strides_and_shared_pages(ctx):
    import torch
    s = Setup([(100, 1), (100, 60), (100, 1)], seed=4)
    s.table[1, :5] = s.table[0, :5]
    s.table[2, :6] = s.table[0, :6]
    s.batch.pages.copy_(torch.from_numpy(s.table).to("cuda", torch.int32))
    note("kv strides")
    check_attention(ctx, s, 4, extra=24)


def test_long_cache_splits(ctx):
    """Long sequences beside short ones: the work of one row is split and joined."""
    seqs = [(20000, 1), (1, 1), (0, 1), (7001, 1), (333, 1)]
    note("kv long splits")
    check_attention(ctx, Setup(seqs, H=1, D=64, seed=8), 4)
    note("kv long chunk")
    check_attention(ctx, Setup([(9000, 20), (0, 1), (30, 300)], H=1, D=64, seed=8), 8)


def test_offsets_past_32_bits(ctx):
    """Pages beyond 4 GiB of the pool: append there, read back, attend."""
    import torch
    H, D, page = 8, 128, 128
    n_pages = 40000                                  # 5.2 GB of codes for each of keys and values
    note("kv offsets past 32 bits")
    cache = lodestar.KVCache(n_pages, H, D, dtype="int8", page_tokens=page)
    table = torch.tensor([[39999, 35000, 3]], dtype=torch.int32, device="cuda")
    T = 300
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = lodestar.KVBatch(i32(0, T), i32(0), table, T)
    k, v = (torch.randn(T, H, D, device="cuda").half() for _ in "kv")
    ctx.ls_kv_append(cache, batch, k, v)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    ctx.ls_kv_read(cache, batch, k2, v2)
    torch.cuda.synchronize()
    for x, y in ((k, k2), (v, v2)):
        step = x.float().abs().amax() / 127
        assert ((x.float() - y.float()).abs() <= step * 0.51 + 2.0 ** -10 * x.float().abs()).all()
    one = lodestar.KVBatch(i32(0, 1), i32(T - 1), table, 1)
    q = torch.randn(1, H * 2, D, device="cuda").half()
    out = torch.empty_like(q)
    ctx.ls_kv_attention(cache, one, q, out)
    kd, vd = k2.double(), v2.double()
    for h in range(H * 2):
        p = torch.softmax(kd[:, h // 2] @ q[0, h].double() * D ** -0.5, 0)
        want, mag = p @ vd[:, h // 2], p @ vd[:, h // 2].abs()
        assert ((out[0, h].double() - want).abs() <= 2.0 ** -8 * (want.abs() + mag)).all()


# -- append and read -----------------------------------------------------------

def appended(ctx, s, k, v, rope, q=None, q_out=None):
    ctx.ls_kv_append(s.cache, s.batch, k, v, rope=rope, q=q, q_out=q_out)


def check_append(ctx, s, G=2, rotary=None, interleaved=False, extra=0, edit=None, in_place=False):
    import torch
    rotary = s.D if rotary is None else rotary
    n_pos = int((s.past + s.new).max()) + 1
    turn = np.arange(n_pos)[:, None] * 100.0 ** (-np.arange(max(1, rotary // 2)) / max(1, rotary // 2))[None]
    cos, sin = np.cos(turn).astype(np.float32), np.sin(turn).astype(np.float32)
    rope = lodestar.Rope(torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), interleaved) if rotary else None
    k, v, q = s.tensor(s.H, 1.3, extra), s.tensor(s.H, 0.7, extra), s.tensor(s.H * G, 1.0, extra)
    if edit:
        edit(k, v)
    qd = q.double().cpu().numpy()
    q_out = q if in_place else torch.empty(s.T, s.H * G, s.D, dtype=s.kind, device="cuda")
    before = s.host()
    ctx.ls_kv_append(s.cache, s.batch, k, v, rope=rope, q=q, q_out=q_out)
    ko_, vo = (torch.full((s.T, s.H, s.D), 9.0, dtype=s.kind, device="cuda") for _ in "kv")
    ctx.ls_kv_read(s.cache, s.batch, ko_, vo)
    torch.cuda.synchronize()
    after = s.host()
    u = 2.0 ** -8 if s.kind == torch.bfloat16 else 2.0 ** -10
    touched = np.zeros((s.n_pages, s.page), bool)
    for b in range(len(s.past)):
        n, p0 = int(s.new[b]), int(s.past[b])
        if n == 0:
            continue
        rows, pos = slice(s.off[b], s.off[b + 1]), p0 + np.arange(n)
        kd, vd = k[rows].double().cpu().numpy(), v[rows].double().cpu().numpy()
        pair = np.abs(kd).max(-1, keepdims=True)
        new = {"k": ko.rotate(kd, pos, cos, sin, interleaved) if rotary else kd, "v": vd}
        if rotary:
            want = ko.rotate(qd[rows], pos, cos, sin, interleaved)
            got = q_out[rows].double().cpu().numpy()
            assert (np.abs(got - want) <= u * np.abs(want) + 2.0 ** -20 * np.abs(qd[rows]).max()).all()
        for name, back in (("k", ko_), ("v", vo)):
            x = new[name]
            finite = np.where(np.isfinite(x), np.abs(x), 0.0)
            vals, there = after.tokens(name, s.table[b], p0 + n)
            old, _ = before.tokens(name, s.table[b], p0 + n)
            got = back[rows].double().cpu().numpy()
            assert (np.abs(got - vals[p0:]) <= u * np.abs(vals[p0:])).all()
            for j in range(p0 // s.page, (p0 + n - 1) // s.page + 1):
                p = int(s.table[b, j])
                lo, hi = max(p0, j * s.page), min(p0 + n, (j + 1) * s.page)
                if not 0 <= p < s.n_pages:
                    assert (got[lo - p0:hi - p0] == 0).all()
                    continue
                touched[p, lo - j * s.page:hi - j * s.page] = True
                want = ko.scale_of(finite[lo - p0:hi - p0].max((0, 2)), s.fmt)
                if lo > j * s.page:
                    want = np.maximum(want, before.scale[name][p])
                    touched[p, :lo - j * s.page] = True
                sc = after.scale[name][p]
                assert (np.abs(sc - want) <= (2.0 ** -22 if s.fmt == "int8" else 0.0) * want).all(), (b, j, name)
                step = sc[None, :, None]
                y = np.nan_to_num(x[lo - p0:hi - p0], nan=0.0, posinf=np.inf, neginf=-np.inf)
                top = (127.0 if s.fmt == "int8" else 448.0) * step
                y = np.clip(y, -top, top)
                slack = 2.0 ** -20 * (pair[lo - p0:hi - p0] if np.isfinite(pair).all() else 1.0)
                assert (np.abs(vals[lo:hi] - y) <= ko.half_step(y, step, s.fmt) * (1 + 2.0 ** -18) + slack).all()
                # what the page held: unchanged under the old scale, else within half a step of the new one
                o, m = old[j * s.page:lo], vals[j * s.page:lo]
                grew = (sc > before.scale[name][p])[None, :, None]
                least = step * 2.0 ** -10 if s.fmt == "fp8" else step / 2 * (1 + 2.0 ** -18)
                assert (np.abs(m - o) <= np.where(grew, least, 0.0)).all()
    # nothing else is written
    for name in "kv":
        at = ko.offsets(s.page, s.D, name == "v")
        same = before.codes[name][:, :, at] == after.codes[name][:, :, at]         # [pages, H, token, D]
        assert (same | touched[:, None, :, None]).all()
        idle = ~touched.any(1)
        assert (before.scale[name][idle] == after.scale[name][idle]).all()
    return before, after


APPEND = [(0, 1), (15, 1), (16, 1), (17, 1), (300, 1), (0, 40), (30, 40), (31, 1), (7, 5), (0, 16), (64, 0), (9, 7), (5, 131)]


@pytest.mark.parametrize("fmt,kind", [("fp8", "bf16"), ("int8", "f16"), ("fp8", "f16"), ("int8", "bf16")])
@pytest.mark.parametrize("D,page,rotary,interleaved", [(128, 16, 128, False), (128, 16, 64, True), (64, 32, 32, False),
                                                       (256, 128, 256, True), (64, 64, 0, False), (256, 16, 96, False)])
def test_append_and_read(ctx, D, page, rotary, interleaved, fmt, kind):
    note(f"kv append D={D} page={page} rotary={rotary}/{interleaved} {fmt} {kind}")
    check_append(ctx, Setup(APPEND, D=D, page=page, fmt=fmt, kind=kind, seed=D + page), rotary=rotary,
                 interleaved=interleaved)


def test_append_strided_and_in_place(ctx):
    note("kv append strided, queries in place")
    check_append(ctx, Setup(APPEND, seed=2), extra=40, in_place=True)
    check_append(ctx, Setup(APPEND, seed=2, D=64), extra=8, rotary=32, in_place=True)


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_append_infinities_and_nan(ctx, fmt):
    """Neither reaches the cache, the scales or other rows."""
    def edit(k, v):
        v[3, 0, 5] = float("inf")
        v[10, 1, 7] = float("-inf")
        v[11, 0, 8] = float("nan")
        v[12] = float("nan")
        k[20, 0, 0] = float("nan")
    s = Setup(APPEND, fmt=fmt, seed=6)
    note(f"kv append inf and nan {fmt}")
    _, after = check_append(ctx, s, rotary=0, edit=edit)
    for b in range(len(s.past)):
        for name in "kv":
            x, _ = after.tokens(name, s.table[b], int(s.past[b] + s.new[b]))
            assert np.isfinite(x).all()


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_append_extremes(ctx, fmt):
    """Blocks of zeros, of tiny and of huge values, and scales that grow a lot."""
    def edit(k, v):
        k[s.off[5]:s.off[5] + 16] = 0
        v[s.off[5]:s.off[5] + 16] = 2.0 ** -100
        k[s.off[6]:] *= 1000.0
        v[s.off[8]:] = 1e35
    s = Setup(APPEND, fmt=fmt, seed=7)
    note(f"kv append extremes {fmt}")
    check_append(ctx, s, rotary=0, edit=edit)


def test_append_to_absent_pages(ctx):
    s = Setup(APPEND, seed=11, absent=[(0, 0), (5, 1), (12, 3), (12, 8)])
    note("kv append to absent pages")
    check_append(ctx, s)


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_append_again_is_the_same(ctx, fmt):
    """The same call twice leaves the cache as the first left it."""
    import torch
    s = Setup(APPEND, fmt=fmt, seed=12)
    k, v = s.tensor(s.H, 3.0), s.tensor(s.H, 3.0)
    note(f"kv append twice {fmt}")
    ctx.ls_kv_append(s.cache, s.batch, k, v)
    first = [t.clone() for t in s.bufs]
    ctx.ls_kv_append(s.cache, s.batch, k, v)
    for a, b in zip(first, s.bufs):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_token_by_token_fp8_matches_at_once(ctx):
    """Powers of two as scales: appending one token at a time gives the codes of appending all, subnormals aside."""
    import torch
    a, b = Setup([(0, 48)], seed=13), Setup([(0, 48)], seed=13)
    k, v = a.tensor(a.H), a.tensor(a.H)
    note("kv append token by token")
    ctx.ls_kv_append(a.cache, a.batch, k, v)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for t in range(48):
        one = lodestar.KVBatch(i32(0, 1), i32(t), b.batch.pages, 1)
        ctx.ls_kv_append(b.cache, one, k[t:t + 1], v[t:t + 1])
    ha, hb = a.host(), b.host()
    for name in "kv":
        x, _ = ha.tokens(name, a.table[0], 48)
        y, _ = hb.tokens(name, b.table[0], 48)
        np.testing.assert_array_equal(ha.scale[name][a.table[0]], hb.scale[name][b.table[0]])
        step = np.repeat(ha.scale[name][a.table[0]], 16, 0)[:, :, None] * 2.0 ** -9
        assert (np.abs(x - y) <= step).all() and np.mean(x == y) > 0.98


def test_append_then_attend_on_another_stream(ctx):
    """Work on a side stream, ordered by events, as a serving loop has it."""
    import torch
    s = Setup([(0, 70), (33, 1), (100, 30)], seed=14)
    k, v = s.tensor(s.H), s.tensor(s.H)
    side = torch.cuda.Stream()
    note("kv on a side stream")
    side.wait_stream(torch.cuda.current_stream())
    ctx.ls_kv_append(s.cache, s.batch, k, v, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    check_attention(ctx, s, 4)


def test_graph_replays(ctx):
    """Append and attention captured into a graph: lengths change between replays, every replay matches eager calls."""
    import torch
    s = Setup([(40, 1), (900, 1), (15, 1), (2000, 1)], seed=15)
    k, v, q = s.tensor(s.H), s.tensor(s.H), s.tensor(s.H * 4)
    out = torch.empty_like(q)

    def step():
        ctx.ls_kv_append(s.cache, s.batch, k, v)
        ctx.ls_kv_attention(s.cache, s.batch, q, out)

    note("kv graph: warm call")
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    note("kv graph: capture")
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        note(f"kv graph: replay {i}")
        s.batch.past.sub_(torch.tensor([3, 17, 1, 300], dtype=torch.int32, device="cuda"))
        k.add_(0.25)
        q.mul_(1.1)
        start = [t.clone() for t in s.bufs]
        g.replay()
        torch.cuda.synchronize()
        got, after = out.clone(), [t.clone() for t in s.bufs]
        for t, o in zip(s.bufs, start):
            t.copy_(o)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
        for a, b in zip(after, s.bufs):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_empty_calls(ctx):
    import torch
    s = Setup([(40, 1)], seed=16)
    z = torch.zeros(1, dtype=torch.int32, device="cuda")
    none = lodestar.KVBatch(torch.zeros(2, dtype=torch.int32, device="cuda"), z, s.batch.pages, 0)
    k = torch.empty(0, s.H, s.D, dtype=torch.bfloat16, device="cuda")
    note("kv empty batch")
    ctx.ls_kv_append(s.cache, none, k, k)
    ctx.ls_kv_attention(s.cache, none, k, k)
    ctx.ls_kv_read(s.cache, none, k, k)


def test_refusals(ctx):
    """Bad arguments are turned down on the host; nothing is enqueued and the message names what is wrong."""
    import ctypes
    import torch
    s = Setup([(40, 1), (3, 2)], seed=17)
    k, v, q = s.tensor(s.H), s.tensor(s.H), s.tensor(s.H * 2)
    lib = lodestar.library()

    def refused(word, call=None, code=lodestar.LS_ERR_INVALID, cache=None, batch=None, rope=None, **a):
        """One raw call with its good arguments except what is given."""
        kv, b = type(s.cache.c).from_buffer_copy(s.cache.c), type(s.batch.c).from_buffer_copy(s.batch.c)
        b.dtype = lodestar.LS_BF16
        for n, x in (cache or {}).items():
            setattr(kv, n, x)
        for n, x in (batch or {}).items():
            setattr(b, n, x)
        g = dict(k=k.data_ptr(), ks=s.H * s.D, v=v.data_ptr(), vs=s.H * s.D, q=q.data_ptr(), qs=2 * s.H * s.D, hq=2 * s.H,
                 o=q.data_ptr(), os=2 * s.H * s.D, scale=1.0, window=0, sinks=0)
        g.update(a)
        r = None if rope is None else ctypes.byref(rope)
        if call in (None, "append"):
            rc = lib.ls_kv_append(ctx.h, ctypes.byref(kv), ctypes.byref(b), r, g["k"], g["ks"], g["v"], g["vs"], g["q"],
                                  g["qs"], g["hq"], g["o"], g["os"], None)
            assert rc == code and word in ctx.last_error(), (rc, ctx.last_error())
        if call in (None, "attend"):
            rc = lib.ls_kv_attention(ctx.h, ctypes.byref(kv), ctypes.byref(b), g["q"], g["qs"], g["hq"], g["scale"],
                                     g["window"], g["sinks"], g["o"], g["os"], None)
            assert rc == code and word in ctx.last_error(), (rc, ctx.last_error())

    note("kv refusals")
    before = [t.clone() for t in s.bufs]
    for word, c in (("cache dtype", dict(dtype=7)), ("n_kv_heads", dict(n_kv_heads=0)), ("head_dim", dict(head_dim=96)),
                    ("page_tokens", dict(page_tokens=24)), ("n_pages", dict(n_pages=0)), ("arrays", dict(k=None)),
                    ("arrays", dict(v_scale=None)), ("aligned", dict(v=s.cache.c.v + 8))):
        refused(word, cache=c)
    for word, b in (("batch dtype", dict(dtype=lodestar.LS_FP32)), ("n_seqs", dict(n_seqs=-1)), ("n_tokens", dict(n_tokens=-1)),
                    ("pages_stride", dict(pages_stride=0)), ("max_new", dict(max_new=0)), ("new_off", dict(past=None))):
        refused(word, batch=b)
    refused("n_q_heads", hq=3)
    refused("n_q_heads", hq=0)
    refused("q must be non-NULL", "attend", q=None)
    refused("go together", "append", q=None)
    refused("k must be non-NULL", "append", k=None)
    refused("v_stride", "append", vs=s.H * s.D - 8)
    refused("k_stride", "append", ks=s.H * s.D + 4)
    refused("aligned", "append", k=k.data_ptr() + 2)
    refused("q_stride", qs=8)
    refused("out", "attend", o=None)
    refused("out_stride", "attend", os=2 * s.H * s.D + 2)
    refused("scale", "attend", scale=float("nan"))
    refused("window", "attend", window=-1)
    refused("sinks", "attend", sinks=-1)
    tab = torch.zeros(64, 64, device="cuda")
    for word, f in (("rotary", dict(rotary=48)), ("rotary", dict(rotary=256)), ("n_positions", dict(n_positions=0)),
                    ("cos_tab", dict(cos_tab=None)), ("aligned", dict(sin_tab=tab.data_ptr() + 4))):
        r = lodestar.ls_rope(tab.data_ptr(), tab.data_ptr(), 64, 128, 0)
        for n, x in f.items():
            setattr(r, n, x)
        refused(word, "append", rope=r)
    torch.cuda.synchronize()
    for a, b in zip(before, s.bufs):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # the binding's own checks
    out = torch.empty_like(q)
    for bad in (q.float(), q[:, :, :64], q[:1], q.transpose(0, 1), q.cpu(), q[:, :3]):
        with pytest.raises((ValueError, lodestar.LodestarError)):
            ctx.ls_kv_attention(s.cache, s.batch, bad, out)
    with pytest.raises(ValueError):
        ctx.ls_kv_append(s.cache, s.batch, k, v.half())
    with pytest.raises(ValueError):
        ctx.ls_kv_append(s.cache, s.batch, k, v, q=q)
    with pytest.raises(ValueError):
        lodestar.KVCache(4, 2, 128, dtype="int4")
    with pytest.raises(ValueError):
        lodestar.KVBatch(s.batch.new_off, s.batch.past, s.batch.pages[0], 3)


def test_serving_example():
    """The example's loop: pages taken over give what computing the prompts gave, answers go on from there."""
    import torch
    from examples import serve_kv
    note("kv serving example")
    (cold, warm), (k, v) = serve_kv.main(requests=5, steps=6, system=70, longest=100)
    assert warm[1] <= 5 * serve_kv.BLOCK < cold[1] and k.shape[0] == 64
    assert torch.isfinite(k.float()).all() and (v != 0).any()
    # the same cached codes; the order of sums and their roundings to bf16 differ
    a, b = cold[2].float(), warm[2].float()
    assert (a - b).abs().max() <= 2.0 ** -5 * a.abs().max()
    assert cold[0].shape == warm[0].shape == (5, 6)
