"""Plain 64-bit definitions of a cache in 8 bits (numpy, loops): rounding to
codes, the write of rows, what codes stand for."""
from __future__ import annotations

import numpy as np
import torch

import decode_ref as R
from paper_2609_03905_amd import ea

TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
FORM = {"e4m3": (3, -6), "e5m2": (2, -14)}  # mantissa bits, the least normal exponent
LEAST, MOST = -120, 120


def rounded(y, code):
    """y to the nearest code, ties to even (|y| up to half a step past the largest)."""
    bits, least = FORM[code]
    y = np.asarray(y, np.float64)
    ok = np.isfinite(y)
    z = np.where(ok, y, 0.0)
    step = 2.0 ** (np.maximum(np.frexp(z)[1] - 1, least) - bits)
    z = np.round(z / step) * step
    other = np.where(np.isinf(y) & (code == "e5m2"), y, np.nan)
    return np.where(ok, z, other)


def least_scale(x, code):
    """The least power of two under which the largest finite |x| has a code."""
    x = np.abs(np.asarray(x, np.float64))
    top = x[np.isfinite(x)].max(initial=0.0)
    e = LEAST
    while e < MOST and top > TOP[code] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def places(table, lengths, q_start, page, n_pages):
    """(row, sequence, position, page or -1) of every row with a key."""
    stride = table.shape[1]
    for s, length in enumerate(lengths):
        n, end = q_start[s + 1] - q_start[s], min(max(int(length), 0), stride * page)
        for i in range(n):
            at = end - n + i
            if at >= 0:
                pg = int(table[s][at // page])
                yield q_start[s] + i, s, at, pg if 0 <= pg < n_pages else -1


def write(x, codes, scale, table, lengths, q_start, code):
    """Rows x [T, H, d] into codes [P, H, page, d] (values) and scale [P, H, n], in place."""
    n_pages, heads, page, _ = codes.shape
    b = page // scale.shape[2]
    blocks = {}
    for t, s, at, pg in places(table, lengths, q_start, page, n_pages):
        if pg >= 0:
            blocks.setdefault((pg, at % page // b), []).append((at % page, t))
    for (pg, i), rows in blocks.items():
        first = min(r for r, _ in rows)
        for h in range(heads):
            new = np.stack([x[t, h] for _, t in rows])
            now = least_scale(new, code)
            old = scale[pg, h, i]
            if first > i * b and 0 < old < np.inf:
                now = max(now, 2.0 ** min(max(np.ceil(np.log2(old)), LEAST), MOST))
                codes[pg, h, i * b:first] = rounded(codes[pg, h, i * b:first] * (old / now), code)
            scale[pg, h, i] = now
            for r, t in rows:
                codes[pg, h, r] = rounded(x[t, h] / now, code)


def values(codes, scale):
    """What codes [.., page, d] stand for under scale [.., n]."""
    return codes * np.repeat(scale, codes.shape[-2] // scale.shape[-1], -1)[..., None]


def code_tensor(vals, code):
    """Codes (values that have one) as a device tensor."""
    return torch.from_numpy(np.asarray(vals, np.float32)).to(TORCH[code]).cuda()


def f64(t):
    return t.float().double().cpu().numpy()


def rel(t):
    """A relation of one block."""
    names = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16", TORCH["e4m3"]: "e4m3",
             TORCH["e5m2"]: "e5m2"}
    return ea.Relation(t.shape, names[t.dtype], ea.whole_partition(t.shape), data=t)


class Cache:
    """One layer's K or V on the device: codes with pages at 256-byte multiples,
    scales, and their relations."""

    def __init__(self, codes, scale, code):
        pages, heads, page, d = codes.shape
        self.code, self.shape = code, codes.shape
        self.rel = ea.Relation(codes.shape, code, [range(pages + 1), [0, heads], [0, page], [0, d]])
        self.scale = torch.from_numpy(np.asarray(scale, np.float32)).cuda()
        self.scale_rel = rel(self.scale)
        self.set(code_tensor(codes, code))

    def _view(self):
        pages, heads, page, d = self.shape
        n = heads * page * d
        pitch = -(-n // 256) * 256
        return self.rel.data.as_strided((pages, n), (pitch, 1))

    def set(self, t):
        self._view().copy_(t.view(torch.uint8).view(self.shape[0], -1))

    def get(self):
        return self._view().contiguous().view(TORCH[self.code]).view(self.shape)


def same(got, want, what=""):
    """Equal values, NaN where NaN."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape
    bad = ~((got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), f"{what}: {bad.sum()} differ, first {np.argwhere(bad)[0]}: {got[bad][0]}, not {want[bad][0]}"


def attention_tol(ref, info, dtype, d):
    """The store's half step; a weight times its value's scale goes to the
    product as two bf16 values, off by half a step of half a step; the score's
    f32 sum and its products with two scales are d + 10 steps of its absolute sum,
    in the exponent of numerator and denominator; 64 steps of exp2, rescaling and
    sums."""
    a, mag, _, _ = info
    u = R.HALF[dtype]
    soft = (2.0 ** -16 + 2 * (d + 10) * R.F * mag + 64 * R.F) * a
    return u * np.abs(ref) + (1 + u) * soft + R.TINY[dtype]
