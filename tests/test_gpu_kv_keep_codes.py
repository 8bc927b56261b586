"""Keeping drafts changes nothing that does not move while the page's scale stays: codes
that ls_kv_append never writes, but that a cache may hold (int8 -128, NaN in tokens that no
row sees), among the neighbours of tokens that do."""
import numpy as np
import pytest

import kv_oracle as ko
from gpu_helpers import note
from paper_2606_00946_amd import lodestar
from test_gpu_kv_pages import Layers, ctx, i32  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,odd", [("int8", (0x80,)), ("fp8", (0x7F, 0xFF))])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 32), (256, 16), (128, 128)])
@pytest.mark.parametrize("past,path", [(10, [2]), (13, [1, 5, 20]), (16, [0, 1, 3]), (3, [0, 30]), (30, [4]), (0, [0, 1, 2, 9])])
def test_tokens_that_stay_keep_their_codes(ctx, past, path, D, page, fmt, odd):  # noqa: F811
    import torch
    lay = Layers(12, layers=1, H=3, D=D, page=page, fmt=fmt, seed=past + D, spread=0.0)      # one scale for all pages
    n, ids = 40, lay.rng.permutation(12)
    table = ids[:-(-(past + n) // page)]
    stay = list(range(past)) + [past + i for i, k in enumerate(path) if i == k]
    before = {}
    for c, name in enumerate("kv"):
        codes, at = lay.host[0].codes[name], ko.offsets(page, D, name == "v")
        if fmt == "int8":                        # no page is asked for a larger scale
            codes = np.clip(codes.view(np.int8), -100, 100).view(np.uint8)
        for t in stay:
            codes[table[t // page]][:, at[t % page]] = odd[t % len(odd)]
        lay.bufs[0][c].view(torch.uint8).copy_(torch.from_numpy(codes))
        before[name] = codes
    kept = np.full(n, -1)
    kept[:len(path)] = path
    note(f"kv keep odd codes past={past} {path} D={D} page={page} {fmt}")
    ctx.ls_kv_keep(lay.caches, lodestar.KVBatch(i32([0, n]), i32([past]), i32(table[None]), n), i32(kept), i32([len(path)]))
    torch.cuda.synchronize()
    for c, name in enumerate("kv"):
        codes, at = lay.bufs[0][c].cpu().numpy().view(np.uint8).reshape(before[name].shape), ko.offsets(page, D, name == "v")
        np.testing.assert_array_equal(lay.bufs[0][2 + c].cpu().numpy().reshape(12, 3), lay.host[0].scale[name].astype(np.float32))
        row = lambda x, t: x[table[t // page]][:, at[t % page]]  # noqa: E731
        for t in stay:
            np.testing.assert_array_equal(row(codes, t), row(before[name], t), err_msg=f"{name}: token {t} stays")
        for i, k in enumerate(path):
            np.testing.assert_array_equal(row(codes, past + i), row(before[name], past + k), err_msg=f"{name}: token {past + k} moves")


@pytest.mark.parametrize("fmt", ["int8", "fp8"])
@pytest.mark.parametrize("D,page", [(64, 16), (128, 32), (256, 16)])
def test_zeros_between_the_ends_of_the_scales(ctx, D, page, fmt):  # noqa: F811
    """A token of zeros on a page of the largest scale moves onto one of the smallest, a page of zeros: it stays zero."""
    import torch
    lay = Layers(8, layers=1, H=2, D=D, page=page, fmt=fmt, seed=D, spread=0.0)
    past, n, path = page - 4, page + 4, [0, 1, 9, 12]            # kept tokens 9 and 12 lie on the second page
    table = lay.rng.permutation(8)[:2]
    codes, scales = ([lay.bufs[0][i + c].view(torch.uint8 if i == 0 else torch.float32).view(8, 2, -1) for c in range(2)] for i in (0, 2))
    for c, s in zip(codes, scales):
        c[table[0]] = 0
        s[table[0]], s[table[1]] = 2.0 ** -64, 2.0 ** 64
    for c, name in zip(codes, "kv"):
        at = ko.offsets(page, D, name == "v")
        for k in path:
            c[table[(past + k) // page]][:, torch.from_numpy(at[(past + k) % page]).cuda()] = 0
    want = [x.clone() for x in (*codes, *scales)]
    kept = np.full(n, -1)
    kept[:4] = path
    note(f"kv keep zeros D={D} page={page} {fmt}")
    ctx.ls_kv_keep(lay.caches, lodestar.KVBatch(i32([0, n]), i32([past]), i32(table[None]), n), i32(kept), i32([4]))
    torch.cuda.synchronize()
    for x, y in zip(want, (*codes, *scales)):
        assert torch.equal(x, y)
