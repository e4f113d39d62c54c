"""A paged cache held in 8 bits: rows of keys and values quantised as they are
written, rows read back, and attention over the codes.  Codes are e4m3 or e5m2
[pages, heads, page size, d]; every block of `block` tokens of a page and every
head has a scale, a power of two in 32 bits [pages, heads, page size / block].
Each case has its work, a plain form in elementary torch operations and a value
in 64 bits.

A write takes each sequence's newest rows.  A block's scale is the least power
of two under which the largest finite new element has a code; a block that holds
rows from earlier calls keeps at least the scale it has, and where the scale
grows those rows' codes are rounded again.

Head counts and widths are those of the repository's configurations (32 query
heads over 8 key-value heads of width 128, and one GPU's share of them, 4 over
1); lengths, page sizes and batches are generic, and draw() spreads over the
ranges they stand for.
"""
from __future__ import annotations

import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn,
         "e5m2": torch.float8_e5m2}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
TOP = {"e4m3": 448.0, "e5m2": 57344.0}  # the largest code
LEAST, MOST = -120, 120  # exponents of a scale


def listed():
    return [
        # One decode step of 64 sequences: a token each, most into a block that
        # holds tokens already, whose scale may have to grow.  Latency counts.
        {"name": "write_decode_64", "kind": "write", "n_seq": 64, "old_lo": 0, "old_hi": 512, "lo": 1, "hi": 1,
         "hkv": 8, "d": 128, "page": 16, "block": 16, "heads": False, "dtype": "bf16", "code": "e4m3"},
        # Five drafted tokens a sequence, narrow heads, pages of an odd size
        # with five scales each, wide-range codes.
        {"name": "write_draft_5", "kind": "write", "n_seq": 21, "old_lo": 5, "old_hi": 300, "lo": 5, "hi": 5,
         "hkv": 8, "d": 64, "page": 20, "block": 4, "heads": False, "dtype": "f16", "code": "e5m2"},
        # A prompt of 8192 tokens, from the per-head rows that its attention read.
        {"name": "write_prefill_8k", "kind": "write", "n_seq": 1, "old_lo": 0, "old_hi": 0, "lo": 8192, "hi": 8192,
         "hkv": 8, "d": 128, "page": 64, "block": 64, "heads": True, "dtype": "bf16", "code": "e4m3"},
        # 32 packed prompts of ragged lengths, 65 thousand tokens.
        {"name": "write_packed_64k", "kind": "write", "n_seq": 32, "old_lo": 0, "old_hi": 0, "lo": 1, "hi": 4096,
         "hkv": 8, "d": 128, "page": 16, "block": 16, "heads": False, "dtype": "bf16", "code": "e4m3"},
        # One sequence read back, for a continued prompt.  Latency counts.
        {"name": "read_one_1k", "kind": "read", "n_seq": 1, "old_lo": 0, "old_hi": 0, "lo": 1000, "hi": 1000,
         "hkv": 8, "d": 128, "page": 16, "block": 16, "heads": True, "dtype": "bf16", "code": "e4m3"},
        # A ragged batch read back, as when sequences move to a cache of
        # another type.
        {"name": "read_ragged_48", "kind": "read", "n_seq": 48, "old_lo": 0, "old_hi": 0, "lo": 1, "hi": 8192,
         "hkv": 8, "d": 128, "page": 16, "block": 16, "heads": False, "dtype": "bf16", "code": "e4m3"},
        # One sequence answered alone: 1000 keys, one token.  Latency counts.
        {"name": "attention_one_1k", "kind": "attention", "n_seq": 1, "groups": 0, "shared": 0, "lo": 1000, "hi": 1000,
         "n_q": 1, "hq": 32, "hkv": 8, "d": 128, "page": 16, "block": 16, "dtype": "bf16", "code": "e4m3"},
        # A ragged batch that shares nothing, from one key to 8K, fp16 queries.
        {"name": "attention_ragged_48", "kind": "attention", "n_seq": 48, "groups": 0, "shared": 0, "lo": 1,
         "hi": 8192, "n_q": 1, "hq": 32, "hkv": 8, "d": 128, "page": 16, "block": 16, "dtype": "f16", "code": "e4m3"},
        # Long documents on one GPU's share of the heads: 4 over 1.
        {"name": "attention_share_128k", "kind": "attention", "n_seq": 8, "groups": 0, "shared": 0, "lo": 1024,
         "hi": 131072, "n_q": 1, "hq": 4, "hkv": 1, "d": 128, "page": 64, "block": 64, "dtype": "bf16",
         "code": "e4m3"},
        # 64 answers to one prompt of 8K tokens, up to 512 own keys each.
        {"name": "attention_prefix_8k", "kind": "attention", "n_seq": 64, "groups": 1, "shared": 8192, "lo": 1,
         "hi": 512, "n_q": 1, "hq": 32, "hkv": 8, "d": 128, "page": 64, "block": 16, "dtype": "bf16", "code": "e4m3"},
        # A long document of 64K tokens shared by 32 sequences: the largest.
        {"name": "attention_prefix_64k", "kind": "attention", "n_seq": 32, "groups": 1, "shared": 65536, "lo": 64,
         "hi": 1024, "n_q": 1, "hq": 32, "hkv": 8, "d": 128, "page": 64, "block": 64, "dtype": "bf16",
         "code": "e4m3"},
        # Five drafted tokens a sequence checked at once, narrow heads, three
        # prompts of 1500 tokens, pages of an odd size, wide-range codes.
        {"name": "attention_draft_5", "kind": "attention", "n_seq": 21, "groups": 3, "shared": 1500, "lo": 5,
         "hi": 300, "n_q": 5, "hq": 32, "hkv": 8, "d": 64, "page": 20, "block": 4, "dtype": "f16", "code": "e5m2"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "attention", "attention", "attention"])
    hkv, group = rng.choice([(8, 4), (1, 4), (2, 8), (4, 1), (12, 1), (8, 8), (3, 5)])
    page = rng.choice([8, 16, 16, 20, 32, 64, 128])
    block = rng.choice([b for b in (1, 2, 4, 5, 16, page // 2, page, page, page) if page % b == 0])
    c = {"kind": kind, "hkv": hkv, "page": page, "block": block, "code": rng.choice(["e4m3", "e4m3", "e5m2"])}
    if kind != "attention":
        c |= {"d": rng.choice([64, 96, 128, 128, 256]), "heads": rng.random() < 0.4,
              "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "n_seq": _log(rng, 1, 128)}
        old = rng.random() < 0.6
        c |= {"old_lo": 0, "old_hi": _log(rng, 1, 600) if old else 0}
        most = rng.choice([1, 1, 5, 64]) if old else _log(rng, 1, 8192)
        while c["n_seq"] > 1 and c["n_seq"] * most * hkv * c["d"] * SIZE[c["dtype"]] > 65536 * 8 * 128 * 2:
            c["n_seq"] //= 2
        return c | {"lo": max(1, most // 8), "hi": most}
    d = rng.choice([64, 128])
    n_seq, n_q = _log(rng, 1, 128), rng.choice([1, 1, 1, 2, 5, 8])
    hi = _log(rng, n_q, 8192)
    groups = min(n_seq, rng.choice([0, 0, 1, 1, 3]))
    shared = _log(rng, 64, 32768) if groups else 0
    # the plain form reads every row's whole length: keep that bounded
    while n_seq > max(1, groups) and n_seq * (shared + hi) * hkv * d > 32 * 66560 * 8 * 128 // 4:
        n_seq -= 1
    return c | {"n_seq": n_seq, "groups": groups, "shared": shared, "lo": min(hi, max(n_q, hi // 16)), "hi": hi,
                "n_q": n_q, "hq": hkv * group, "d": d, "dtype": rng.choice(["bf16", "bf16", "f16"])}


# ---- sizes that a case alone gives ------------------------------------------
def _spread(n, lo, hi):
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _pages(n, page):
    return -(-n // page)


def _news(case):
    """Rows that each sequence writes or reads, spread evenly over [lo, hi]."""
    return _spread(case["n_seq"], case["lo"], case["hi"])


def _olds(case):
    """Keys that each sequence holds before them."""
    return _spread(case["n_seq"], case["old_lo"], case["old_hi"])


def _stride(case):
    most = case["shared"] + case["hi"] if case["kind"] == "attention" else case["old_hi"] + case["hi"]
    return _pages(most, case["page"]) + 2


def _n_pages(case):
    page = case["page"]
    if case["kind"] == "attention":
        shared = case["shared"]
        mine = sum(_pages(shared + n, page) - shared // page for n in _news(case))
        return case["groups"] * (shared // page) + mine + 7
    return sum(_pages(o + n, page) for o, n in zip(_olds(case), _news(case))) + 7


def _blocks(case):
    """Blocks that the new rows lie in."""
    b = case["block"]
    return sum((o + n - 1) // b - o // b + 1 for o, n in zip(_olds(case), _news(case)))


def work(case):
    hkv, d, page = case["hkv"], case["d"], case["page"]
    if case["kind"] == "attention":
        hq, n_q, shared, news = case["hq"], case["n_q"], case["shared"], _news(case)
        keys = case["groups"] * shared + sum(news)
        seen = sum(n_q * (shared + n) - n_q * (n_q - 1) // 2 for n in news)
        pages = sum(_pages(shared + n, page) for n in news)
        return {"bytes": 2 * keys * hkv * (d + 4 / case["block"]) + 2 * case["n_seq"] * n_q * hq * d * 2 + 4 * pages,
                "flops": 4 * d * hq * seen}
    rows = sum(_news(case))
    return {"bytes": 2 * rows * hkv * d * (1 + SIZE[case["dtype"]]) + 8 * hkv * _blocks(case) + 8 * case["n_seq"],
            "flops": 2 * rows * hkv * d * (3 if case["kind"] == "write" else 1)}


# ---- inputs ------------------------------------------------------------------
def _dev():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


class _Make:
    def __init__(self, seed):
        self.dev = _dev()
        self.g = torch.Generator(device=self.dev).manual_seed(seed)
        self.host = torch.Generator().manual_seed(seed)

    def normal(self, shape, dtype=torch.float32, std=1.0):
        return (torch.randn(shape, generator=self.g, device=self.dev, dtype=torch.float32) * std).to(dtype)

    def rows(self, shape, dtype):
        """Rows of heads as a projection leaves them: tokens of different sizes,
        a few channels larger than the others."""
        size = torch.exp(0.5 * self.normal(shape[:-1] + (1,)))
        channel = torch.exp(0.7 * self.normal((shape[-1],)))
        return (self.normal(shape) * size * channel).to(dtype)

    def order(self, n):
        return torch.randperm(n, generator=self.host)

    def up(self, values, dtype=torch.int32):
        return torch.as_tensor(values).to(dtype).to(self.dev)


def _held(x, block, code):
    """Codes and scales of pages of rows x [pages, heads, page, d]."""
    pages, heads, page, d = x.shape
    cut = x.view(pages, heads, page // block, block, d)
    scale = _scale(cut.abs().amax((3, 4)), code)
    codes = (cut / scale[..., None, None]).to(TORCH[code]).view(pages, heads, page, d)
    return _apart(codes), scale


def _apart(codes):
    """The codes with pages that start at multiples of 256 bytes, as a relation's
    blocks do (a view, where a page is no such multiple)."""
    n = codes[0].numel()
    if n % 256 == 0:
        return codes
    whole = torch.zeros((len(codes), -(-n // 256) * 256), dtype=torch.uint8, device=codes.device)
    whole[:, :n] = _bytes(codes).view(len(codes), n)
    return whole.view(codes.dtype)[:, :n].view(codes.shape)


def prepare(case, seed):
    m = _Make(seed)
    s = {"case": case}
    n, page, hkv, d, n_pages = case["n_seq"], case["page"], case["hkv"], case["d"], _n_pages(case)
    order = m.order(n)
    news = torch.as_tensor(_news(case))[order]
    ids = m.order(n_pages).tolist()
    table = torch.full((n, _stride(case)), -1, dtype=torch.int32)
    if case["kind"] == "attention":
        shared, groups = case["shared"], case["groups"]
        full = shared // page  # whole pages are shared; a partly filled one is each sequence's own copy
        prefix = [[ids.pop() for _ in range(full)] for _ in range(groups)]
        keys = news + shared
        s["q"] = m.normal((n * case["n_q"], case["hq"] * d), TORCH[case["dtype"]])
        s["out"] = torch.empty_like(s["q"])
        starts = [i * case["n_q"] for i in range(n + 1)]
        if groups:  # sequence i is of group i * groups // n
            s["group_start"] = m.up([-(-g * n // groups) for g in range(groups + 1)])
            s["group_shared"] = m.up([full * page] * groups)
        else:
            s["group_start"] = s["group_shared"] = None
    else:
        full, groups = 0, 0
        keys = news + torch.as_tensor(_olds(case))[m.order(n)]
        starts = [0] + news.cumsum(0).tolist()
        t = starts[-1]
        if case["kind"] == "write":
            s["xk"], s["xv"] = m.rows((t, hkv, d), TORCH[case["dtype"]]), m.rows((t, hkv, d), TORCH[case["dtype"]])
        else:
            s["xk"], s["xv"] = (torch.empty((t, hkv, d), dtype=TORCH[case["dtype"]], device=m.dev) for _ in range(2))
        for x in ("xk", "xv"):
            s[x] = s[x].transpose(0, 1).contiguous() if case["heads"] else s[x].view(t, hkv * d)
        s["row_seq"] = m.up(torch.repeat_interleave(torch.arange(n), news), torch.int64)
    for i in range(n):
        mine = list(prefix[i * groups // n]) if groups else []
        mine += [ids.pop() for _ in range(_pages(int(keys[i]), page) - len(mine))]
        table[i, : len(mine)] = torch.as_tensor(mine, dtype=torch.int32)
    s["table"], s["len"], s["start"] = m.up(table), m.up(keys), m.up(starts)
    for x in ("k", "v"):
        s[x], s[x + "_scale"] = _held(m.rows((n_pages, hkv, page, d), torch.float32), case["block"], case["code"])
    if own:
        _handles(s, case)
    return s


def _handles(s, case):
    """The relations that a program keeps over its tensors."""
    from paper_2609_03905_amd import ea

    names = {v: k for k, v in TORCH.items()}

    def whole(t):
        return ea.Relation(t.shape, names[t.dtype], ea.whole_partition(t.shape), data=t)

    def pages(t):  # one block per page, over the memory from the first one's to the last one's end
        part = [range(t.shape[0] + 1)] + ea.whole_partition(t.shape[1:])
        return ea.Relation(t.shape, names[t.dtype], part, data=t.as_strided((len(t) * t.stride(0),), (1,)))

    rows = ("q", "out") if case["kind"] == "attention" else ("xk", "xv")
    s["rel"] = {x: whole(s[x]) for x in rows + ("k_scale", "v_scale")} | {x: pages(s[x]) for x in ("k", "v")}


# ---- one pass ------------------------------------------------------------------
def run(s):
    if own:
        return _own(s)
    return {"write": _plain_write, "read": _plain_read, "attention": _plain_attention}[s["case"]["kind"]](s)


def _own(s):
    from paper_2609_03905_amd import ea

    case, r = s["case"], s["rel"]
    cache = {"k_scale": r["k_scale"], "v_scale": r["v_scale"], "table": s["table"], "lengths": s["len"],
             "q_start": s["start"]}
    if case["kind"] == "write":
        ea.pages_write(r["xk"], r["xv"], r["k"], r["v"], **cache)
        return {x: s[x] for x in ("k", "v", "k_scale", "v_scale")}
    if case["kind"] == "read":
        ea.pages_read(r["k"], r["v"], r["xk"], r["xv"], **cache)
        return {"xk": s["xk"], "xv": s["xv"]}
    ea.attention_paged(r["q"], r["k"], r["v"], r["out"], scale=case["d"] ** -0.5, group_start=s["group_start"],
                       group_shared=s["group_shared"], **cache)
    return {"out": s["out"]}


# ---- the plain forms ---------------------------------------------------------
def _scale(top, code):
    """The least power of two under which `top` has a code: top = f 2^e with f
    in [1/2, 1), the largest code 7/8 of a power of two."""
    f, e = torch.frexp(top)
    e = e - (9 if code == "e4m3" else 16) + (f > 0.875).int()
    e = torch.where(top > 0, e, LEAST).clamp(LEAST, MOST)
    return ((e.int() + 127) << 23).view(torch.float32)


def _bytes(codes):
    return codes.view(torch.uint8)  # (indexing is by bytes: torch moves them all the same)


def _places(s):
    """Of every row: its page, its row of the page and its position."""
    case, seq = s["case"], s["row_seq"]
    start, length = s["start"].long(), s["len"].long()
    first = length - (start[1:] - start[:-1])
    at = first[seq] + torch.arange(len(seq), device=seq.device) - start[seq]
    return s["table"][seq, at // case["page"]].long(), at % case["page"], at, first


def _plain_write(s):
    case = s["case"]
    page, block, code, hkv, d = (case[x] for x in ("page", "block", "code", "hkv", "d"))
    nb = page // block
    pg, row, at, first = _places(s)
    of = pg * nb + row // block  # block of the cache
    begun = first[s["row_seq"]] <= at - row % block
    # the block that a sequence's first new row goes on with
    on = (first % block > 0)[:, None, None, None]
    on_page, on_row = s["table"].gather(1, (first // page)[:, None])[:, 0].long().clamp(min=0), first % page
    rows_of = (on_row // block * block)[:, None] + torch.arange(block, device=pg.device)[None, :]
    before = (rows_of < on_row[:, None])[:, None, :, None] & on
    for x in ("k", "v"):
        new = s["x" + x].float()
        new = new.transpose(0, 1) if case["heads"] else new.view(-1, hkv, d)
        size = new.abs()
        top = torch.where(size < math.inf, size, 0).amax(-1)  # [t, hkv]
        scale = s[x + "_scale"]
        flat = scale.transpose(1, 2).reshape(-1, hkv).clone()  # [pages * nb, hkv]
        most = torch.zeros_like(flat).scatter_reduce(0, of[:, None].expand(-1, hkv), top, "amax")[of]
        fresh = _scale(most, code)
        now = torch.where(begun[:, None], fresh, torch.maximum(flat[of], fresh))
        was = flat.clone()
        flat[of] = now  # (rows of a block agree)
        scale.copy_(flat.view(-1, nb, hkv).transpose(1, 2))
        # what the block held before, under its new scale
        b = on_page * nb + on_row // block
        kept = _bytes(s[x])[on_page[:, None], :, rows_of]  # [n, block, hkv, d]
        again = (kept.view(TORCH[code]).float() * (was[b] / flat[b])[:, None, :, None]).to(TORCH[code])
        keep = before.transpose(1, 2) & (flat[b] > was[b])[:, None, :, None]
        page_of = on_page[:, None].expand_as(rows_of)
        # (sequences without such a block write their bytes back as they are;
        # the new rows come after)
        _bytes(s[x])[page_of, :, rows_of] = torch.where(keep, _bytes(again), kept)
        _bytes(s[x])[pg, :, row] = _bytes((new / now[:, :, None]).to(TORCH[code]))
    return {x: s[x] for x in ("k", "v", "k_scale", "v_scale")}


def _plain_read(s):
    case = s["case"]
    pg, row, _, _ = _places(s)
    out = {}
    for x in ("k", "v"):
        codes = _bytes(s[x])[pg, :, row].view(TORCH[case["code"]]).float()
        y = (codes * s[x + "_scale"][pg, :, row // case["block"]][:, :, None]).to(TORCH[case["dtype"]])
        out["x" + x] = y.transpose(0, 1).contiguous() if case["heads"] else y.reshape(len(pg), -1)
    return out


def _plain_attention(s):
    case = s["case"]
    n, n_q, hq, hkv, d, block = (case[x] for x in ("n_seq", "n_q", "hq", "hkv", "d", "block"))
    g = hq // hkv
    pages = s["table"].clamp(min=0).long()

    def keys(x):  # every sequence's rows, [n, hkv, keys, d]
        scale = s[x + "_scale"][pages].repeat_interleave(block, -1)
        rows = _bytes(s[x])[pages].view(TORCH[case["code"]]).float() * scale[..., None]
        return rows.transpose(1, 2).reshape(n, hkv, -1, d)

    # query rows of one sequence and key-value head: token-major, then heads
    q = s["q"].float().view(n, n_q, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, n_q * g, d)
    scores = torch.matmul(q, keys("k").transpose(2, 3).contiguous()) * d ** -0.5
    seen = s["len"].long()[:, None] - n_q + torch.arange(1, n_q + 1, device=q.device)[None, :]
    at = torch.arange(scores.shape[-1], device=q.device)
    mask = at[None, None, :] < seen.repeat_interleave(g, 1)[:, :, None]
    scores = scores.masked_fill(~mask[:, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, keys("v")) / torch.where(total > 0, total, 1.0)
    o = o.view(n, hkv, n_q, g, d).permute(0, 2, 1, 3, 4)
    return {"out": o.reshape(n * n_q, hq * d).to(s["q"].dtype)}


# ---- 64-bit values, from the definitions ----------------------------------------
def _power(e):
    """2^e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _rounded(y, code):
    """y to the nearest multiple of the code's step where y lies, ties to even."""
    bits, least = (3, -6) if code == "e4m3" else (2, -14)  # mantissa, smallest normal exponent
    e = (torch.frexp(y).exponent - 1).clamp(min=least)
    step = _power(e - bits)
    return torch.round(y / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(s, case)
    n, page, block, hkv, d = (case[x] for x in ("n_seq", "page", "block", "hkv", "d"))
    t = len(s["row_seq"])
    value = {x: (s[x].double(), s[x + "_scale"].double()) for x in ("k", "v")}
    lens, starts, table = s["len"].tolist(), s["start"].tolist(), s["table"].tolist()
    out = {x: (torch.zeros((t, hkv, d), dtype=torch.float64, device=s["k"].device)) for x in ("xk", "xv")}
    if case["kind"] == "write" and _blocks(case) > 20000 or case["kind"] == "read" and sum(lens) // page > 20000:
        return None
    for i in range(n):
        first = lens[i] - (starts[i + 1] - starts[i])
        at = first
        while at < lens[i]:  # a block of the write, a page of the read, at a time
            unit = block if case["kind"] == "write" else page
            end = min(lens[i], (at // unit + 1) * unit)
            pg, lo, hi = table[i][at // page], at % page, (end - 1) % page + 1
            rows = slice(starts[i] + at - first, starts[i] + end - first)
            for x in ("k", "v"):
                codes, scale = value[x]
                if case["kind"] == "read":
                    each = scale[pg].repeat_interleave(block, 1)[:, lo:hi]
                    out["x" + x][rows] = (codes[pg, :, lo:hi] * each[:, :, None]).transpose(0, 1)
                    continue
                new = (s["x" + x][:, rows] if case["heads"]
                       else s["x" + x][rows].view(-1, hkv, d).transpose(0, 1)).double()
                top = new.abs().amax((1, 2)) / TOP[case["code"]]
                e = torch.ceil(torch.log2(top)).clamp(LEAST, MOST)  # or one off, where it is close
                e = torch.where(_power(e) < top, e + 1, torch.where(_power(e - 1) >= top, e - 1, e))
                least = _power(e.clamp(LEAST, MOST))
                b, begin = lo // block, lo // block * block
                if lo > begin:
                    now = torch.maximum(scale[pg, :, b], least)
                    again = _rounded(codes[pg, :, begin:lo] * (scale[pg, :, b] / now)[:, None, None], case["code"])
                    codes[pg, :, begin:lo] = again
                    least = now
                scale[pg, :, b] = least
                codes[pg, :, lo:hi] = _rounded(new / least[:, None, None], case["code"])
            at = end
    if case["kind"] == "write":
        return {"k": value["k"][0], "v": value["v"][0], "k_scale": value["k"][1], "v_scale": value["v"][1]}
    return {x: y.transpose(0, 1).contiguous() if case["heads"] else y.view(t, hkv * d) for x, y in out.items()}


def _exact_attention(s, case):
    n, n_q, hq, hkv, d, page = (case[x] for x in ("n_seq", "n_q", "hq", "hkv", "d", "page"))
    if 4 * d * hq * n_q * sum(case["shared"] + x for x in _news(case)) > 4e11:
        return None
    out = torch.zeros((n, n_q, hkv, hq // hkv, d), dtype=torch.float64, device=s["q"].device)
    lens = s["len"].tolist()
    for i, length in enumerate(lens):
        at = torch.arange(length, device=out.device)
        page_of, row = s["table"][i].long()[at // page], at % page

        def side(x):  # [hkv, keys, d]
            codes = s[x].view(torch.uint8)[page_of, :, row].view(s[x].dtype).double()
            return (codes * s[x + "_scale"][page_of, :, row // case["block"]].double()[..., None]).transpose(0, 1).contiguous()

        k, v = side("k"), side("v")
        for j in range(n_q):
            m = length - n_q + j + 1  # keys that this token sees
            if m > 0:
                q = s["q"][i * n_q + j].double().view(hkv, hq // hkv, d)
                w = torch.softmax((k[:, :m] @ q.transpose(1, 2)) / math.sqrt(d), 1)
                out[i, j] = w.transpose(1, 2) @ v[:, :m]
    return {"out": out.view(n * n_q, hq * d)}
