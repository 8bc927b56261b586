"""Calls on drafts and pages of the KV cache in 64 bits on the CPU, from the
definitions in include/lodestar.h (the cache itself is kv_oracle's)."""
from __future__ import annotations

import numpy as np

import kv_oracle as ko


def tree_parents(n, reach, rng):
    """A random tree of n drafts: each one's parent among the `reach` before it, -1 for the cached tokens."""
    return [max(j - 1 - int(rng.randint(0, reach)), -1) for j in range(n)]


def ancestry(parents):
    """(sees [n, n], depth [n]): a draft sees itself and its ancestors."""
    n = len(parents)
    sees, depth = np.zeros((n, n), bool), np.zeros(n, np.int64)
    for j, p in enumerate(parents):
        if p >= 0:
            sees[j], depth[j] = sees[p], depth[p] + 1
        sees[j, j] = True
    return sees, depth


def words(sees, count):
    """Rows of truth values [n, m] as `count` mask words a row, m at most 64 * count."""
    out = np.zeros((sees.shape[0], count), np.uint64)
    for j in range(sees.shape[1]):
        out[:, j // 64] |= sees[:, j].astype(np.uint64) << np.uint64(j % 64)
    return out


def attention_tree(cache, q, new_off, past, pages, sees, pos, scale, window=0, sinks=0):
    """(out, sum_j p_j |v_j|); sees[b] [n, n], pos the rows' positions."""
    T, Hq, D = q.shape
    G = Hq // cache.H
    out, mag = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    for b in range(len(past)):
        r0, n, p0 = int(new_off[b]), int(new_off[b + 1] - new_off[b]), int(past[b])
        if n == 0:
            continue
        k, there = cache.tokens("k", pages[b], p0 + n)
        v, _ = cache.tokens("v", pages[b], p0 + n)
        j = np.arange(p0)
        for i in range(n):
            near = np.ones(p0, bool)
            if window:
                p = max(int(pos[r0 + i]), p0)
                near = (j > p - window) | (j < sinks)
            seen = np.concatenate([near, sees[b][i]]) & there
            if not seen.any():
                continue
            for h in range(cache.H):
                x = (q[r0 + i, h * G:(h + 1) * G] @ k[seen, h].T) * scale
                w = np.exp(x - x.max(1, keepdims=True))
                w /= w.sum(1, keepdims=True)
                out[r0 + i, h * G:(h + 1) * G] = w @ v[seen, h]
                mag[r0 + i, h * G:(h + 1) * G] = w @ np.abs(v[seen, h])
    return out, mag


def rotate_axes(x, pos, axis, cos, sin, interleaved):
    """x [T, H, D]; pair i at pos[axis[i]] [T], held inside the table."""
    y, half = x.copy(), cos.shape[1]
    for i in range(half):
        at = np.clip(pos[axis[i]], 0, cos.shape[0] - 1)
        c, s = cos[at, i].astype(np.float64)[:, None], sin[at, i].astype(np.float64)[:, None]
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def kept_list(kept, want, n):
    """The list's part that counts."""
    out = []
    for k in kept[:max(0, min(want, n))]:
        if k >= n or k < 0 or (out and k <= out[-1]):
            break
        out.append(int(k))
    return out


def code_of(x, fmt):
    """The nearest code, as a byte, ties to even."""
    if fmt == "int8":
        return np.rint(np.clip(x, -127, 127)).astype(np.int8).view(np.uint8)
    mags = ko.E4M3[:127]
    a = np.clip(np.abs(x), 0, 448.0)
    hi = np.clip(np.searchsorted(mags, a), 1, 126)
    lo = hi - 1
    d = (a - mags[lo]) - (mags[hi] - a)
    c = np.where(d < 0, lo, np.where(d > 0, hi, np.where(lo % 2 == 0, lo, hi)))
    return (c | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def keep(cache, new_off, past, pages, kept, n_kept):
    """Changes `cache` (a kv_oracle.Cache) as ls_kv_keep does.  Products and quotients are rounded to 32 bits as the
    definition's scale and codes need it: a / 127 as a * (1 / 127), old / new scale as old * (1 / new)."""
    f32 = np.float32
    for name in "kv":
        at = ko.offsets(cache.page, cache.D, name == "v")
        codes, scale = cache.codes[name], cache.scale[name]

        def spot(b, t):
            j = t // cache.page
            p = int(pages[b][j]) if j < len(pages[b]) else -1
            return (p if 0 <= p < cache.n_pages else -1), t % cache.page

        for b in range(len(past)):
            r0, n, p0 = int(new_off[b]), int(new_off[b + 1] - new_off[b]), int(past[b])
            path = kept_list(kept[r0:r0 + n], int(n_kept[b]), n)
            for j in range(p0 // cache.page, (p0 + len(path) - 1) // cache.page + 1) if path else ():
                page = spot(b, j * cache.page)[0]
                if page < 0:
                    continue
                rows = {r: (page, r) for r in range(max(0, min(p0 + len(path) - j * cache.page, cache.page)))}
                for i, k in enumerate(path):
                    t = p0 + i - j * cache.page
                    if 0 <= t < cache.page and spot(b, p0 + k)[0] >= 0:
                        rows[t] = spot(b, p0 + k)
                old_codes, old_scale = codes.copy(), scale.copy()
                new = old_scale[page].copy()
                moved = False
                for r, (pf, rf) in rows.items():
                    if (pf, rf) != (page, r):
                        moved = True
                        top = np.abs(ko.code_values(old_codes[pf][:, at[rf]], cache.fmt)).max(1)
                        a = (top.astype(f32) * old_scale[pf].astype(f32)).astype(np.float64)
                        want = ko.scale_of(a, cache.fmt)
                        new = np.maximum(new, (a.astype(f32) * (f32(1) / f32(127))).clip(f32(ko.SCALE_MIN), f32(ko.SCALE_MAX))
                                         if cache.fmt == "int8" else want)
                if not moved:
                    continue
                scale[page] = new
                inv = f32(1) / new.astype(f32)
                for r, (pf, rf) in rows.items():
                    again = (old_scale[pf].astype(f32) * inv).astype(f32)
                    x = ko.code_values(old_codes[pf][:, at[rf]], cache.fmt).astype(f32) * again[:, None]
                    codes[page][:, at[r]] = code_of(x.astype(np.float64), cache.fmt)


def fork(cache, pages, pages_out, src, dst, tokens):
    """Changes `cache` and `pages_out` as ls_kv_fork does."""
    page = cache.page
    rows, W = pages.shape
    for s, d, t in zip(src, dst, tokens):
        if not (0 <= s < rows and 0 <= d < rows):
            continue
        t = min(max(int(t), 0), W * page)
        full, part = t // page, t % page
        pages_out[d, :full] = pages[s, :full]
        if not part:
            continue
        p, q = int(pages[s, full]), int(pages_out[d, full])
        if p == q or not (0 <= p < cache.n_pages and 0 <= q < cache.n_pages):
            continue
        held = -(-part // 16) * 16
        for name in "kv":
            at = ko.offsets(page, cache.D, name == "v")[:held].ravel()
            cache.codes[name][q][:, at] = cache.codes[name][p][:, at]
            cache.scale[name][q] = cache.scale[name][p]


def compact(n_pages, pages):
    """(new table, where, U, moves [(from, to)])."""
    named = sorted({int(p) for p in pages.ravel() if 0 <= p < n_pages})
    U = len(named)
    free = sorted(set(range(U)) - set(named))
    moves = list(zip([p for p in named if p >= U], free))
    where = np.full(n_pages, -1, np.int64)
    where[named] = named
    for a, b in moves:
        where[a] = b
    there = (pages >= 0) & (pages < n_pages)
    return np.where(there, where[np.clip(pages, 0, n_pages - 1)], pages), where, U, moves
