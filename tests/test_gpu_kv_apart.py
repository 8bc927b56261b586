"""Calls on all layers' caches refuse arrays that lie where others do: keys, values
and scales of every layer are rewritten each by waves of their own.  The check
itself is tested on the CPU (test_kv_ranges_cpu)."""
import numpy as np
import pytest

from gpu_helpers import note
from paper_2606_00946_amd import lodestar
from test_gpu_kv_pages import Layers, ctx, i32  # noqa: F401

pytestmark = pytest.mark.gpu

FIELDS = ("k", "v", "k_scale", "v_scale")


def test_arrays_that_overlap(ctx):  # noqa: F811
    import torch
    lay = Layers(20, layers=3, seed=9)
    lib, t, z = lodestar.library(), i32(np.arange(12).reshape(3, 4)), i32([0, 1, 2])
    where, used = torch.zeros(20, dtype=torch.int32, device="cuda"), i32([0])
    batch = lodestar.KVBatch(i32([0, 1, 2, 3]), z, t, 3)
    T, Z = t.data_ptr(), z.data_ptr()
    calls = (lambda c, n: lib.ls_kv_keep(ctx.h, c, n, batch.ref, Z, Z, None),
             lambda c, n: lib.ls_kv_fork(ctx.h, c, n, 3, 4, T, T, 1, Z, Z, Z, None),
             lambda c, n: lib.ls_kv_compact(ctx.h, c, n, 3, 4, T, T, where.data_ptr(), used.data_ptr(), None))
    one = 20 * lay.H                                             # scales of an array
    note("kv arrays that overlap")

    def refused(changes, n=3):
        for call in calls:
            bad = (lodestar.ls_kv_cache * 3).from_buffer_copy(lay.caches.c)
            for i, field, value in changes:
                setattr(bad[i], field, value)
            assert call(bad, n) == lodestar.LS_ERR_INVALID and "overlap" in ctx.last_error(), (changes, ctx.last_error())

    for i, j in ((0, 1), (1, 2), (2, 0), (0, 0), (2, 2)):
        for a in FIELDS:
            for b in FIELDS:
                if (i, a) != (j, b):
                    refused([(i, a, getattr(lay.caches.c[j], b))])
    refused([(0, "k", lay.caches.c[0].v)], n=1)                  # within one cache
    refused([(0, "k_scale", lay.caches.c[0].v_scale)], n=1)
    for field, part in (("k", 16), ("v", lay.H * lay.page * lay.D), ("k_scale", 4 * one - 4), ("v_scale", 4)):
        refused([(2, field, getattr(lay.caches.c[1], field) + part)])                # in part
    torch.cuda.synchronize()
    lay.same()
    assert t.cpu().numpy().ravel().tolist() == list(range(12)) and int(used) == 0


def test_arrays_side_by_side(ctx):  # noqa: F811
    """Layers cut from one tensor, their scales from another: nothing overlaps, and nothing is refused."""
    import torch
    H, D, page, pages, n = 2, 64, 16, 6, 5
    codes = torch.zeros(n, 2, pages * H * page * D, dtype=torch.uint8, device="cuda")
    scales = torch.ones(n, 2, pages * H, device="cuda")
    layers = lodestar.KVLayers([lodestar.KVCache(pages, H, D, page_tokens=page, buffers=(*codes[i], *scales[i])) for i in range(n)])
    codes.random_(1, 100)
    want = codes.clone()
    t = i32([[5, 1, -1]])
    out, where, used = torch.empty_like(t), torch.empty(pages, dtype=torch.int32, device="cuda"), i32([0])
    note("kv arrays side by side")
    ctx.ls_kv_compact(layers, t, out, where, used)
    torch.cuda.synchronize()
    size = H * page * D
    want[..., :size] = want[..., 5 * size:]
    assert out.tolist() == [[0, 1, -1]] and torch.equal(codes, want)
