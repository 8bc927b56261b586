"""The paged 8-bit KV cache's calls over large batches and long sequences: the
search of a sequence in more than 64, sequences cut into parts and left whole,
parts joined in groups, at every head dimension; against the definitions in 64
bits (kv_oracle) with the tolerances of test_gpu_kv, and with a narrower one
where a cache is long.

The narrower one: weights are rounded to half precision one by one, 2^-12 of
each at most and independent, so their sum is off by 6 / sqrt(3) * 2^-12 of
sqrt(sum (p v)^2) at six standard deviations; scores, exponentials and sums in
fp32 give 2^-16 of sum p |v|; the output's own rounding is 2^-8 (bf16) or 2^-11
(half) of it.  A lost block of 16 tokens is several times that.
"""
import numpy as np
import pytest

from gpu_helpers import note
from test_gpu_kv import Setup, check_append, check_attention, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


def ragged(B, seed, longest=90, new=(1, 1, 1, 1, 2, 0, 0, 5)):
    """B short sequences of every kind, empty ones among them; the first and the last have tokens."""
    r = np.random.RandomState(seed)
    seqs = [(int(r.randint(0, longest)), int(r.choice(new))) for _ in range(B)]
    seqs[0], seqs[-1] = (3, 1), (longest, 2)
    return seqs


@pytest.mark.parametrize("B", [63, 64, 65, 130, 4097])
@pytest.mark.parametrize("G,fmt,kind", [(2, "fp8", "bf16"), (16, "int8", "f16")])
def test_many_sequences(ctx, B, G, fmt, kind):  # noqa: F811
    """Append with a rotation, read and attention; with G = 16 some sequences are tiles of many rows."""
    s = Setup(ragged(B, B + G), H=1, D=64, fmt=fmt, kind=kind, seed=B)
    note(f"kv many sequences B={B} G={G} {fmt} {kind}")
    check_append(ctx, s, G=1, rotary=32)
    check_attention(ctx, s, G)
    check_attention(ctx, s, G, window=40, sinks=5)


# the most segments (sequence and kv head) that are cut, and one sequence more
@pytest.mark.parametrize("D,H,B", [(64, 8, 661), (64, 8, 662), (128, 8, 336), (128, 8, 337), (256, 2, 677), (256, 2, 678)])
@pytest.mark.parametrize("new", [(1,), (1, 1, 1, 1, 1, 0, 30)])
def test_segments_cut_and_whole(ctx, D, H, B, new):  # noqa: F811
    """Single tokens beside a long sequence, alone and beside tiles of many rows."""
    seqs = ragged(B, B, longest=40, new=new)
    seqs[B // 2], seqs[-1] = (5000, 1), (2600, 1)
    note(f"kv segments D={D} H={H} B={B} new={new}")
    check_attention(ctx, Setup(seqs, H=H, D=D, seed=B), 1 if len(new) == 1 else 2)


def check_long(ctx, s, G, window=0, sinks=0):  # noqa: F811
    import torch
    q = s.tensor(s.H * G)
    out = torch.empty_like(q)
    ctx.ls_kv_attention(s.cache, s.batch, q, out, window=window, sinks=sinks)
    host, worst = s.host(), 0.0
    u = 2.0 ** -8 if s.kind == torch.bfloat16 else 2.0 ** -11
    for b in range(len(s.past)):
        n, p0 = int(s.new[b]), int(s.past[b])
        rows = slice(int(s.off[b]), int(s.off[b + 1]))
        k, v = (torch.from_numpy(host.tokens(name, s.table[b], p0 + n)[0]).cuda() for name in "kv")
        j, i = torch.arange(p0 + n, device="cuda")[None], p0 + torch.arange(n, device="cuda")[:, None]
        hidden = j > i
        if window:
            hidden = hidden | ((j <= i - window) & (j >= sinks))
        for h in range(q.shape[1]):
            kh, vh = k[:, h // G].contiguous(), v[:, h // G].contiguous()
            p = torch.softmax((q[rows, h].double() @ kh.T.contiguous() * s.D ** -0.5).masked_fill(hidden, -np.inf), 1)
            want, mag, rms = p @ vh, p @ vh.abs(), ((p * p) @ (vh * vh)).sqrt()
            off = (out[rows, h].double() - want).abs()
            bound = u * want.abs() + 6 / 3 ** 0.5 * 2.0 ** -12 * rms + 2.0 ** -16 * mag + 2.0 ** -25
            worst = max(worst, float((off / bound).max()))
    print(f"  {worst:.2f} of the bound", flush=True)
    assert worst <= 1


@pytest.mark.parametrize("fmt,kind", [("fp8", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_long_decode(ctx, D, fmt, kind):  # noqa: F811
    """More parts than one workgroup adds: groups of parts, then the groups."""
    note(f"kv long decode D={D} {fmt} {kind}")
    check_long(ctx, Setup([(30000, 1), (1, 1), (20001, 2), (17, 1)], H=1, D=D, fmt=fmt, kind=kind, seed=D), 4)
    note(f"kv long decode under a window D={D} {fmt} {kind}")
    check_long(ctx, Setup([(40000, 1), (25000, 1)], H=2, D=D, fmt=fmt, kind=kind, seed=D + 1), 8, 20000, 40)


@pytest.mark.parametrize("fmt,kind", [("fp8", "bf16"), ("int8", "f16")])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_long_prompts(ctx, D, fmt, kind):  # noqa: F811
    """Tiles over a long cache: a few, whose tokens many workgroups share, and many."""
    note(f"kv long prompt, shared tiles D={D} {fmt} {kind}")
    check_long(ctx, Setup([(20000, 40), (6000, 9)], H=1, D=D, fmt=fmt, kind=kind, seed=D), 4)
    note(f"kv long prompt D={D} {fmt} {kind}")
    check_long(ctx, Setup([(8000, 600)], H=4, D=D, fmt=fmt, kind=kind, seed=D), 32, *((4000, 20) if D == 64 else ()))


@pytest.mark.parametrize("G,seqs", [(4, [(300, 1), (40, 2), (0, 1)]), (8, [(300, 90), (5, 40)])])
def test_small_half_queries(ctx, G, seqs):  # noqa: F811
    """Queries below a half's least normal number count as what they are."""
    note(f"kv small half queries G={G}")
    check_attention(ctx, Setup(seqs, kind="f16", seed=41), G, sigma=2.0 ** -18, scale=2.0 ** 18 * 128 ** -0.5)
