"""The paged 8-bit KV cache in 64 bits on the CPU: layout, codes, scales, rotation
and attention, written from the definitions in include/lodestar.h."""
from __future__ import annotations

import numpy as np

SCALE_MIN, SCALE_MAX = 2.0 ** -64, 2.0 ** 64


def e4m3_table():
    """The 256 values of OCP e4m3 (NaN for the two NaN codes)."""
    c = np.arange(256)
    sign, e, m = np.where(c & 128, -1.0, 1.0), (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    return np.where((e == 15) & (m == 7), np.nan, sign * v)


E4M3 = e4m3_table()


def code_values(codes, fmt):
    return E4M3[codes] if fmt == "fp8" else codes.view(np.int8).astype(np.float64)


def offsets(page_tokens, D, values):
    """Byte of (token, dimension) inside one page and head."""
    t, d = np.arange(page_tokens)[:, None], np.arange(D)[None, :]
    tile = ((t // 16) * (D // 64) + d // 64) * 1024
    return tile + ((t % 16 // 4) * 256 + (d % 64) * 4 + t % 4 if values else (t % 16) * 64 + d % 64)


class Cache:
    """A host copy of a cache's arrays: codes [n_pages, H, page * D], scales [n_pages, H]."""

    def __init__(self, k, v, ks, vs, n_pages, H, D, page, fmt):
        self.codes = {"k": k.reshape(n_pages, H, page * D), "v": v.reshape(n_pages, H, page * D)}
        self.scale = {"k": ks.reshape(n_pages, H).astype(np.float64), "v": vs.reshape(n_pages, H).astype(np.float64)}
        self.n_pages, self.H, self.D, self.page, self.fmt = n_pages, H, D, page, fmt

    def tokens(self, name, table, n):
        """Values [n, H, D] of a sequence's first n tokens, and which are present."""
        out, there = np.zeros((n, self.H, self.D)), np.zeros(n, bool)
        at = offsets(self.page, self.D, name == "v")
        for j in range(-(-n // self.page)):
            p = int(table[j]) if j < len(table) else -1
            if not 0 <= p < self.n_pages:
                continue
            m = min(self.page, n - j * self.page)
            x = code_values(self.codes[name][p][:, at[:m]], self.fmt) * self.scale[name][p][:, None, None]
            out[j * self.page:j * self.page + m] = x.transpose(1, 0, 2)
            there[j * self.page:j * self.page + m] = True
        return out, there


def attention(cache, q, new_off, past, pages, scale, window=0, sinks=0):
    """(out, sum_j p_j |v_j|) in 64 bits; rows of no sequence and rows that see nothing are 0."""
    T, Hq, D = q.shape
    G = Hq // cache.H
    out, mag = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    for b in range(len(past)):
        n, p0 = int(new_off[b + 1] - new_off[b]), int(past[b])
        if n == 0:
            continue
        k, there = cache.tokens("k", pages[b], p0 + n)
        v, _ = cache.tokens("v", pages[b], p0 + n)
        j = np.arange(p0 + n)
        for i in range(n):
            pos = p0 + i
            seen = (j <= pos) & there
            if window:
                seen &= (j > pos - window) | (j < sinks)
            if not seen.any():
                continue
            for h in range(Hq):
                x = (k[seen, h // G] @ q[new_off[b] + i, h]) * scale
                w = np.exp(x - x.max())
                w /= w.sum()
                out[new_off[b] + i, h] = w @ v[seen, h // G]
                mag[new_off[b] + i, h] = w @ np.abs(v[seen, h // G])
    return out, mag


def rotate(x, pos, cos, sin, interleaved):
    """x [n, H, D] at positions pos [n]."""
    y = x.copy()
    half = cos.shape[1]
    pos = np.minimum(pos, cos.shape[0] - 1)
    c, s = cos[pos][:, None].astype(np.float64), sin[pos][:, None].astype(np.float64)
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def scale_of(amax, fmt):
    if fmt == "int8":
        s = amax / 127.0
    else:
        s = 2.0 ** np.ceil(np.log2(np.maximum(amax, 1e-300) / 448.0))
    return np.clip(s, SCALE_MIN, SCALE_MAX)


def half_step(x, scale, fmt):
    """Half the distance of neighbouring representable values at x."""
    if fmt == "int8":
        return scale / 2 * np.ones_like(x)
    e = np.floor(np.log2(np.maximum(np.abs(x / scale), 2.0 ** -6)))
    return scale * 2.0 ** (e - 4)
