"""Plain 64-bit definitions of the decoding operators (numpy, loops), and the
small helpers their GPU tests share.  Tolerances are derived here: a rounding
is off by at most half a step of its type relative to the value."""
from __future__ import annotations

import numpy as np
import torch

from paper_2609_03905_amd import ea

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a step
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}  # half the smallest fp16 step
F = 2.0 ** -24


def splits(n, b):
    return list(range(0, n, b)) + [n]


def rel(t: torch.Tensor, part=None) -> ea.Relation:
    names = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}
    return ea.Relation(t.shape, names[t.dtype], part or ea.whole_partition(t.shape), data=t)


def pages_rel(t: torch.Tensor) -> ea.Relation:
    part = ea.whole_partition(t.shape)
    for dim in range(t.dim() - 3):
        part[dim] = list(range(t.shape[dim] + 1))
    if t[(0,) * (t.dim() - 3)].numel() * t.element_size() % 256:  # pages start at 256-byte multiples: a copy
        return blocked(t, part)
    return rel(t, part)


def blocked(t: torch.Tensor, part) -> ea.Relation:
    """A relation of the values of ``t`` under ``part``."""
    names = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}
    return ea.from_dense(t, names[t.dtype], part)


def unblocked(r: ea.Relation) -> torch.Tensor:
    return ea.to_dense(r).view(TORCH[r.dtype]).view(r.shape)


def i32(values, device="cuda"):
    return torch.as_tensor(np.asarray(values), dtype=torch.int32).to(device)


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().double().cpu().numpy()


# ---- head rows -------------------------------------------------------------
def pair_index(rotary, interleaved):
    f = np.arange(rotary // 2)
    return (2 * f, 2 * f + 1) if interleaved else (f, f + rotary // 2)


def turn(n, pos, freq, interleaved, back=False):
    """Rows n [T, H, d] rotated by +-pos * freq."""
    y = n.copy()
    i, j = pair_index(2 * len(freq), interleaved)
    a = pos[:, None, None].astype(np.float64) * freq[None, None, :]
    s = -np.sin(a) if back else np.sin(a)
    y[..., i] = n[..., i] * np.cos(a) - n[..., j] * s
    y[..., j] = n[..., j] * np.cos(a) + n[..., i] * s
    return y


def spread(n, rotary, interleaved):
    """|n_i| + |n_j| of the pair an element is in: what its rotation's absolute
    errors scale with."""
    y = np.abs(n)
    i, j = pair_index(rotary, interleaved)
    both = y[..., i] + y[..., j]
    y[..., i] = both
    y[..., j] = both
    return y


def heads(x, hq, hkv, d, wq, wk, eps, freq, interleaved, pos):
    """(q, k, v) [T, H, d] and the scale of their f32 errors."""
    t = x.shape[0]
    rows = x.reshape(t, hq + 2 * hkv, d)
    out, err = [], []
    for part, w in ((rows[:, :hq], wq), (rows[:, hq:hq + hkv], wk)):
        n = part if w is None else w * part / np.sqrt((part ** 2).mean(-1, keepdims=True) + eps)
        out.append(turn(n, pos, freq, interleaved))
        err.append(spread(n, 2 * len(freq), interleaved))
    return out + [rows[:, hq + hkv:]], err + [np.zeros_like(rows[:, hq + hkv:])]


# f32 steps of one head element relative to |n_i| + |n_j|: the sum of squares
# (8 terms in a lane, 6 exchanges: 14, halved by the root), root and reciprocal
# (3), u r w (2), the angle's fraction rounded once and turned (2 pi / 4 < 2)
# and sine and cosine (2 steps), product and fused add (2): 18, taken as 32.
HEADS_STEPS = 32 * F


def heads_tol(ref, err, dtype):
    return HALF[dtype] * np.abs(ref) + (1 + HALF[dtype]) * HEADS_STEPS * err + TINY[dtype]


def heads_grad(x, dq, dk, dv, hq, hkv, d, wq, wk, eps, freq, interleaved, pos):
    """dx [T, heads, d], its error scale, and (dwq, scale, dwk, scale)."""
    t = x.shape[0]
    rows = x.reshape(t, hq + 2 * hkv, d)
    dx, scale, dws = [], [], []
    for part, w, dy in ((rows[:, :hq], wq, dq), (rows[:, hq:hq + hkv], wk, dk)):
        g = turn(dy, pos, freq, interleaved, back=True)
        ga = spread(dy, 2 * len(freq), interleaved)
        if w is None:
            dx.append(g)
            scale.append(ga)
            dws += [None, None]
            continue
        r = 1 / np.sqrt((part ** 2).mean(-1, keepdims=True) + eps)
        n = part * r
        s = w * g
        dx.append(r * (s - n * (s * n).mean(-1, keepdims=True)))
        sa = np.abs(w) * ga
        scale.append(r * (sa + np.abs(n) * (sa * np.abs(n)).mean(-1, keepdims=True)))
        dws += [(g * n).sum((0, 1)), (ga * np.abs(n)).sum((0, 1))]
    dx.append(dv)
    scale.append(np.zeros_like(dv))
    return np.concatenate(dx, 1).reshape(t, -1), np.concatenate(scale, 1).reshape(t, -1), dws


# ---- attention ----------------------------------------------------------------
def attention(q, k, v, table, lengths, page, q_start, scale):
    """Rows [T, Hq, d] in 64 bits (zeros where nothing is seen), and per element
    A = sum_j p_j |v_j|, per row the most that |scale q.k| sums absolutely."""
    t, hq, d = q.shape
    n_pages, hkv, _, _ = k.shape
    g = hq // hkv
    out, a, mag, n_keys = np.zeros_like(q), np.zeros_like(q), np.zeros((t, hq, 1)), np.zeros((t, 1, 1))
    vmax = np.zeros((t, hq, 1))
    for s, length in enumerate(lengths):
        r0, r1 = q_start[s], q_start[s + 1]
        for r in range(r0, r1):
            keys = [j for j in range(max(0, min(length, table.shape[1] * page) - (r1 - r0) + (r - r0) + 1))
                    if 0 <= table[s][j // page] < n_pages]
            if not keys:
                continue
            at = np.asarray(keys)
            pg = table[s][at // page]
            for h in range(hq):
                kk, vv = k[pg, h // g, at % page], v[pg, h // g, at % page]
                z = scale * (kk @ q[r, h])
                p = np.exp(z - z.max())
                p /= p.sum()
                out[r, h] = p @ vv
                a[r, h] = p @ np.abs(vv)
                mag[r, h] = scale * (np.abs(kk) @ np.abs(q[r, h])).max()
                vmax[r, h] = np.abs(vv).max()
            n_keys[r] = len(keys)
    return out, (a, mag, vmax, n_keys)


def attention_tol(ref, info, dtype, d):
    """The store's half step; a weight is off by half a step of its type in
    numerator and denominator (2 u A), by the score's f32 sum (d + 8 steps of
    its absolute sum, in the exponent: again twice) and by 64 steps of exp2,
    rescaling and sums; fp16 weights below the normal range lose up to half
    their smallest step, on every key."""
    a, mag, vmax, n_keys = info
    u = HALF[dtype]
    soft = (2 * u * 1.01 + 2 * (d + 8) * F * mag + 64 * F) * a + TINY[dtype] * n_keys * vmax
    return u * np.abs(ref) + (1 + u) * soft + TINY[dtype]


def check(got, ref, tol, what=""):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == ref.shape, (got.shape, ref.shape)
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    over = np.abs(got - ref) - tol
    at = np.unravel_index(np.argmax(over), over.shape) if over.size else None
    assert over.size == 0 or over.max() <= 0, \
        f"{what}: off by {abs(got[at] - ref[at]):.3e} at {at}, {np.broadcast_to(tol, ref.shape)[at]:.3e} allowed"


# ---- the page table -----------------------------------------------------------
class Pages:
    """The page calls' state and their definition, page by page."""

    def __init__(self, n_seq, stride, n_pages, page, planes=None):
        self.page, self.n_pages, self.stride = page, n_pages, stride
        self.table = np.full((n_seq, stride), -1, dtype=np.int32)
        self.len = np.zeros(n_seq, dtype=np.int32)
        self.refs = np.zeros(n_pages, dtype=np.int32)
        self.planes = planes  # numpy [planes, pages, heads, page, d] or None

    def held(self, n):
        return -(-int(n) // self.page)

    def free(self):
        return [p for p in range(self.n_pages) if self.refs[p] <= 0]

    def extend(self, add, n_tokens):
        add = np.maximum(np.asarray(add), 0)
        slots, pos = np.full(n_tokens, -1, np.int32), np.zeros(n_tokens, np.int32)
        free = self.free()
        if any(n < 0 or int(n) + int(x) > self.stride * self.page for n, x in zip(self.len, add)):
            return (ea.PAGES_TOO_LONG, len(free)), slots, pos
        need = [self.held(n + x) - self.held(n) for n, x in zip(self.len, add)]
        if sum(need) > len(free):
            return (ea.PAGES_NONE_FREE, len(free)), slots, pos
        t = 0
        for s, x in enumerate(add):
            for i in range(self.held(self.len[s]), self.held(self.len[s] + x)):
                p = free.pop(0)
                self.table[s, i] = p
                self.refs[p] = 1
            for j in range(int(self.len[s]), int(self.len[s] + x)):
                if t < n_tokens:
                    pg = self.table[s, j // self.page]
                    slots[t] = pg * self.page + j % self.page if 0 <= pg < self.n_pages else -1
                    pos[t] = j
                t += 1
            self.len[s] += x
        return (ea.PAGES_OK, len(free)), slots, pos

    def select(self, parent):
        n = len(self.len)
        if any(x < 0 or x > self.stride * self.page for x in self.len):
            return (ea.PAGES_TOO_LONG, len(self.free()))
        kids = [[i for i in range(n) if parent[i] == s] for s in range(n)]
        refs = self.refs.copy()
        for s in range(n):
            full, tail = divmod(int(self.len[s]), self.page)
            for j in range(full):
                if 0 <= self.table[s, j] < self.n_pages:
                    refs[self.table[s, j]] += len(kids[s]) - 1
            if tail and not kids[s] and 0 <= self.table[s, full] < self.n_pages:
                refs[self.table[s, full]] -= 1
        copies = [i for i in range(n) if 0 <= parent[i] < n and kids[parent[i]][0] != i
                  and self.len[parent[i]] % self.page]
        free = [p for p in range(self.n_pages) if refs[p] <= 0]
        if len(copies) > len(free):
            return (ea.PAGES_NONE_FREE, len(self.free()))
        table, length = np.full_like(self.table, -1), np.zeros_like(self.len)
        for i in range(n):
            p = parent[i]
            if not 0 <= p < n:
                continue
            length[i] = self.len[p]
            table[i, :self.held(self.len[p])] = self.table[p, :self.held(self.len[p])]
        for i in copies:
            p, to = parent[i], free.pop(0)
            full, tail = divmod(int(self.len[p]), self.page)
            if self.planes is not None and 0 <= self.table[p, full] < self.n_pages:
                self.planes[:, to, :, :tail] = self.planes[:, self.table[p, full], :, :tail]
            table[i, full] = to
            refs[to] = 1
        self.table, self.len, self.refs = table, length, refs
        return (ea.PAGES_OK, len(free))

    def compact(self):
        used = [p for p in range(self.n_pages) if self.refs[p] > 0]
        to = {p: p for p in range(self.n_pages)}
        holes = [p for p in self.free() if p < len(used)]
        for dst, src in zip(holes, [p for p in used if p >= len(used)]):
            to[src] = dst
            if self.planes is not None:
                self.planes[:, dst] = self.planes[:, src]
            self.refs[dst], self.refs[src] = self.refs[src], 0
        for s in range(len(self.len)):
            for j in range(self.stride):
                p = int(self.table[s, j])
                self.table[s, j] = -1 if j >= self.held(max(self.len[s], 0)) else to.get(p, p)
        self.refs = np.maximum(self.refs, 0)
        return (ea.PAGES_OK, self.n_pages - len(used))
