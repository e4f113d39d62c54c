"""The operators of decoding beside the block share: head rows normed and
rotated (with their gradient), attention over a paged cache whose batch shares
a prefix, and the page table's operations.  Each case has its work, a plain
form in elementary torch operations and a value in 64 bits.

Head counts and widths are those of the repository's configurations (32 query
heads over 8 key-value heads of width 128, and one GPU's share of them, 4 over
1); lengths, page sizes and batches are generic, and draw() spreads over the
ranges they stand for.
"""
from __future__ import annotations

import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def listed():
    return [
        # One decode step of 64 sequences: the new tokens' query and key heads
        # normed and rotated at positions far apart, keys and values written
        # to their pages.  Some rows are padding (no page).  Latency counts.
        {"name": "heads_decode_64", "kind": "heads", "t": 64, "hq": 32, "hkv": 8, "d": 128, "rotary": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "block": 0, "far": 131072, "page": 16},
        # Prefill of 8192 tokens: the QKV projection's 512-blocks to rotated
        # per-head rows, what the block chain's attention reads.
        {"name": "heads_prefill_8k", "kind": "heads", "t": 8192, "hq": 32, "hkv": 8, "d": 128, "rotary": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "block": 512, "far": 0, "page": 0},
        # fp32 rows of narrow heads, neighbouring pairs rotated over half of
        # the head only, no norm, an odd number of tokens.
        {"name": "heads_f32_partial", "kind": "heads", "t": 1537, "hq": 12, "hkv": 12, "d": 64, "rotary": 32,
         "interleaved": True, "norm": False, "dtype": "f32", "block": 0, "far": 0, "page": 0},
        # The gradient of a training batch: 4096 tokens, odd by one.
        {"name": "heads_grad_4k", "kind": "heads_grad", "t": 4097, "hq": 32, "hkv": 8, "d": 128, "rotary": 128,
         "interleaved": False, "norm": True, "dtype": "bf16"},
        # One sequence answered alone: 1000 keys, one token.  Latency counts.
        {"name": "attention_one_1k", "kind": "attention", "n_seq": 1, "groups": 0, "shared": 0, "lo": 1000, "hi": 1000,
         "n_q": 1, "hq": 32, "hkv": 8, "d": 128, "page": 16, "dtype": "bf16"},
        # A ragged batch that shares nothing, from one key to 8K, fp16.
        {"name": "attention_ragged_48", "kind": "attention", "n_seq": 48, "groups": 0, "shared": 0, "lo": 1,
         "hi": 8192, "n_q": 1, "hq": 32, "hkv": 8, "d": 128, "page": 16, "dtype": "f16"},
        # 64 answers to one prompt of 8K tokens, up to 512 own keys each.
        {"name": "attention_prefix_8k", "kind": "attention", "n_seq": 64, "groups": 1, "shared": 8192, "lo": 1,
         "hi": 512, "n_q": 1, "hq": 32, "hkv": 8, "d": 128, "page": 64, "dtype": "bf16"},
        # A long document of 64K tokens shared by 32 sequences: the largest.
        {"name": "attention_prefix_64k", "kind": "attention", "n_seq": 32, "groups": 1, "shared": 65536, "lo": 64,
         "hi": 1024, "n_q": 1, "hq": 32, "hkv": 8, "d": 128, "page": 64, "dtype": "bf16"},
        # Five drafted tokens a sequence checked at once, narrow heads, three
        # prompts of 1500 tokens, pages of an odd size.
        {"name": "attention_draft_5", "kind": "attention", "n_seq": 21, "groups": 3, "shared": 1500, "lo": 5,
         "hi": 300, "n_q": 5, "hq": 32, "hkv": 8, "d": 64, "page": 20, "dtype": "bf16"},
        # A step's new tokens get their pages and slots: 256 sequences.
        {"name": "pages_extend_256", "kind": "extend", "n_seq": 256, "lo": 1, "hi": 4096, "add": 3, "page": 16,
         "planes": 0, "hkv": 8, "d": 128},
        # A beam step: the better half of 64 sequences goes on twice, the
        # others are freed; half-filled pages are copied in all 32 layers.
        {"name": "pages_select_64", "kind": "select", "n_seq": 64, "lo": 100, "hi": 700, "page": 32, "planes": 64,
         "hkv": 8, "d": 128},
        # A cache after many sequences came and went, made dense again.
        {"name": "pages_compact", "kind": "compact", "n_seq": 32, "lo": 50, "hi": 900, "page": 16, "planes": 64,
         "hkv": 8, "d": 128},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "heads", "heads_grad", "attention", "attention", "attention", "attention", "extend",
                       "select", "compact"])
    d = rng.choice([64, 128])
    hkv, group = rng.choice([(8, 4), (1, 4), (2, 8), (4, 1), (12, 1), (8, 8), (3, 5)])
    if kind in ("heads", "heads_grad"):
        d = rng.choice([64, 96, 128, 128, 256])
        c = {"kind": kind, "t": _log(rng, 1, 8192 if kind == "heads" else 4097), "hq": hkv * group, "hkv": hkv,
             "d": d, "rotary": rng.choice([d, d, d // 2]), "interleaved": rng.random() < 0.3,
             "norm": rng.random() < 0.7, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
        while c["t"] * (c["hq"] + 2 * hkv) * d * SIZE[c["dtype"]] > 8192 * 48 * 128 * 2:
            c["t"] = c["t"] // 2
        if kind == "heads":
            c |= {"block": 0, "far": rng.choice([0, 0, 4096, 1000000]), "page": rng.choice([0, 16, 20, 64])}
        return c
    page = rng.choice([8, 16, 16, 20, 32, 64, 128])
    if kind == "attention":
        n_seq, n_q = _log(rng, 1, 128), rng.choice([1, 1, 1, 2, 5, 8])
        hi = _log(rng, n_q, 8192)
        groups = min(n_seq, rng.choice([0, 0, 1, 1, 3]))
        shared = _log(rng, 64, 32768) if groups else 0
        # the plain form reads every row's whole length: keep that bounded
        while n_seq > max(1, groups) and n_seq * (shared + hi) * hkv * d > 32 * 66560 * 8 * 128 // 4:
            n_seq -= 1
        return {"kind": kind, "n_seq": n_seq, "groups": groups, "shared": shared, "lo": min(hi, max(n_q, hi // 16)),
                "hi": hi, "n_q": n_q, "hq": hkv * group, "hkv": hkv, "d": d, "page": page,
                "dtype": rng.choice(["bf16", "bf16", "f16"])}
    if kind == "extend":
        return {"kind": kind, "n_seq": _log(rng, 1, 512), "lo": 0, "hi": _log(rng, 1, 4096),
                "add": rng.choice([1, 1, 2, 5, _log(rng, 8, 256)]), "page": page, "planes": 0, "hkv": hkv, "d": d}
    hi = _log(rng, 64, 1024)
    c = {"kind": kind, "n_seq": 2 * _log(rng, 1, 32), "lo": hi // 8, "hi": hi, "page": page,
         "planes": 2 * _log(rng, 1, 32), "hkv": hkv, "d": d}
    while c["planes"] > 2 and _n_pages(c) * c["planes"] * hkv * page * d > 1 << 29:
        c["planes"] -= 2
    return c


# ---- sizes that a case alone gives ------------------------------------------
def _lengths(case):
    """Keys of each sequence's own, spread evenly over [lo, hi]; which sequence
    has which is the seed's choice."""
    n, lo, hi = case["n_seq"], case["lo"], case["hi"]
    own_lens = [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]
    if case["kind"] == "select":  # no last page is full: every fork copies one
        own_lens = [x + 1 if x % case["page"] == 0 else x for x in own_lens]
    return own_lens


def _adds(case):
    return [1 + i % case["add"] for i in range(case["n_seq"])]


def _pages(n, page):
    return -(-n // page)


def _stride(case):
    more = case["add"] if case["kind"] == "extend" else 0
    return _pages(case.get("shared", 0) + case["hi"] + 1 + more, case["page"]) + 2


def _used(case):
    return sum(_pages(n, case["page"]) for n in _lengths(case))


def _n_pages(case):
    if case["kind"] == "attention":
        page, shared = case["page"], case["shared"]
        own_pages = sum(_pages(shared + n, page) - shared // page for n in _lengths(case))
        return case["groups"] * (shared // page) + own_pages + 7
    if case["kind"] == "extend":
        return _used(case) + sum(_adds(case)) + 5
    if case["kind"] == "select":
        return _used(case) + case["n_seq"] + 3
    return _used(case) + max(4, _used(case) // 2)  # compact: a third of the cache is holes


def work(case):
    kind = case["kind"]
    if kind in ("heads", "heads_grad"):
        rows, heads = case["t"], case["hq"] + 2 * case["hkv"]
        el = rows * heads * case["d"]
        turned = rows * (case["hq"] + case["hkv"]) * case["d"]
        if kind == "heads":
            return {"bytes": 2 * el * SIZE[case["dtype"]] + 8 * rows, "flops": 8 * turned}
        # the values' part of x is not needed
        read = el + turned
        return {"bytes": (read + el) * SIZE[case["dtype"]] + 4 * rows, "flops": 20 * turned}
    lens = _lengths(case)
    if kind == "attention":
        hq, hkv, d, n_q, shared = case["hq"], case["hkv"], case["d"], case["n_q"], case["shared"]
        keys = case["groups"] * shared + sum(lens)
        seen = sum(n_q * (shared + n) - n_q * (n_q - 1) // 2 for n in lens)
        pages = sum(_pages(shared + n, case["page"]) for n in lens)
        return {"bytes": 2 * keys * hkv * d * 2 + 2 * case["n_seq"] * n_q * hq * d * 2 + 4 * pages,
                "flops": 4 * d * hq * seen}
    n, n_pages = case["n_seq"], _n_pages(case)
    if kind == "extend":  # the reference counts, and a slot and a position a token
        return {"bytes": 4 * (2 * n_pages + 3 * n + 4 * sum(_adds(case))), "flops": n_pages}
    table = 4 * 2 * n * _stride(case) + 4 * 2 * n_pages + 12 * n
    row = case["hkv"] * case["d"] * 2 * case["planes"]
    if kind == "select":
        kept = _kept(case)
        return {"bytes": table + 2 * row * sum(lens[i] % case["page"] for i in kept), "flops": n_pages}
    return {"bytes": table + 2 * row * case["page"] * _moves(case), "flops": n_pages}


def _kept(case):
    """Which sequences of a beam step go on: every second one."""
    return list(range(0, case["n_seq"], 2))


def _holes(case):
    """Free pages of a fragmented cache: the places 0, 3, 6, ..., then from the end."""
    n_pages, free = _n_pages(case), _n_pages(case) - _used(case)
    holes = list(range(0, n_pages, 3))[:free]
    return holes + [x for x in range(n_pages - 1, -1, -1) if x % 3][: free - len(holes)]


def _moves(case):
    """Used pages behind the first _used(case): as many as the holes before them."""
    return sum(h < _used(case) for h in _holes(case))


# ---- inputs ------------------------------------------------------------------
def _dev():
    return torch.device("cuda" if torch.cuda.is_available() else "cpu")


class _Make:
    def __init__(self, seed):
        self.dev = _dev()
        self.g = torch.Generator(device=self.dev).manual_seed(seed)
        self.host = torch.Generator().manual_seed(seed)

    def normal(self, shape, dtype, std=1.0):
        return (torch.randn(shape, generator=self.g, device=self.dev, dtype=torch.float32) * std).to(dtype)

    def order(self, n):
        return torch.randperm(n, generator=self.host)

    def up(self, values, dtype=torch.int32):
        return torch.as_tensor(values).to(dtype).to(self.dev)


def prepare(case, seed):
    kind = case["kind"]
    m = _Make(seed)
    s = {"case": case}
    if kind in ("heads", "heads_grad"):
        _prepare_heads(s, case, m)
    elif kind == "attention":
        _prepare_attention(s, case, m)
    else:
        _prepare_pages(s, case, m)
    if own:
        _handles(s, case)
    return s


def _prepare_heads(s, case, m):
    t, hq, hkv, d, dt = case["t"], case["hq"], case["hkv"], case["d"], TORCH[case["dtype"]]
    w = (hq + 2 * hkv) * d
    s["x"] = m.normal((t, w), dt)
    if case.get("block"):  # as a projection leaves it: row-major blocks of the relation
        b = case["block"]
        s["x"] = s["x"].view(t // b, b, w // b, b).permute(0, 2, 1, 3).contiguous()
    s["wq"] = (1 + m.normal((d,), torch.float32, 0.1)).to(dt) if case["norm"] else None
    s["wk"] = (1 + m.normal((d,), torch.float32, 0.1)).to(dt) if case["norm"] else None
    half = case["rotary"] // 2
    s["freq"] = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().to(m.dev)
    if case.get("far"):
        s["pos"] = torch.randint(0, case["far"], (t,), generator=m.g, device=m.dev, dtype=torch.int32)
    else:
        s["pos"] = torch.arange(t, device=m.dev, dtype=torch.int32) + int(m.order(64)[0])
    if kind_grad(case):
        s["dq"] = m.normal((t, hq * d), dt)
        s["dk"] = m.normal((t, hkv * d), dt)
        s["dv"] = m.normal((t, hkv * d), dt)
        s["dx"] = torch.empty_like(s["x"])
        s["dwq"] = torch.empty(d, device=m.dev) if case["norm"] else None
        s["dwk"] = torch.empty(d, device=m.dev) if case["norm"] else None
        return
    page = case["page"]
    if page:
        n_pages = _pages(t, page) + 3
        slots = m.order(n_pages * page)[:t]
        slots[m.order(t)[: t // 16]] = -1  # padding rows
        s["real"] = m.up((slots >= 0).nonzero().view(-1), torch.int64)
        s["slots"] = m.up(slots)
        s["q"] = torch.empty((t, hq * d), device=m.dev, dtype=dt)
        s["k"] = m.normal((n_pages, hkv, page, d), dt)
        s["v"] = m.normal((n_pages, hkv, page, d), dt)
    else:
        s["slots"] = None
        s["q"] = torch.empty((hq, t, d), device=m.dev, dtype=dt)
        s["k"] = torch.empty((hkv, t, d), device=m.dev, dtype=dt)
        s["v"] = torch.empty((hkv, t, d), device=m.dev, dtype=dt)


def kind_grad(case):
    return case["kind"] == "heads_grad"


def _prepare_attention(s, case, m):
    n, page, shared, groups, hkv, d = (case[x] for x in ("n_seq", "page", "shared", "groups", "hkv", "d"))
    dt, n_pages, stride = TORCH[case["dtype"]], _n_pages(case), _stride(case)
    lens = torch.as_tensor(_lengths(case))[m.order(n)]
    ids = m.order(n_pages).tolist()
    table = torch.full((n, stride), -1, dtype=torch.int32)
    full = shared // page  # whole pages are shared; a partly filled one is each sequence's own copy
    prefix = [[ids.pop() for _ in range(full)] for _ in range(groups)]
    for i in range(n):
        mine = list(prefix[i * groups // n]) if groups else []
        mine += [ids.pop() for _ in range(_pages(shared + int(lens[i]), page) - len(mine))]
        table[i, : len(mine)] = torch.as_tensor(mine, dtype=torch.int32)
    s["table"], s["len"] = m.up(table), m.up(lens + shared)
    s["q"] = m.normal((n * case["n_q"], case["hq"] * d), dt)
    s["k"] = m.normal((n_pages, hkv, page, d), dt)
    s["v"] = m.normal((n_pages, hkv, page, d), dt)
    s["out"] = torch.empty_like(s["q"])
    s["start"] = m.up([i * case["n_q"] for i in range(n + 1)])
    if groups:  # sequence i is of group i * groups // n
        s["group_start"] = m.up([-(-g * n // groups) for g in range(groups + 1)])
        s["group_shared"] = m.up([full * page] * groups)
    else:
        s["group_start"] = s["group_shared"] = None


def _prepare_pages(s, case, m):
    n, page, n_pages, stride, planes = case["n_seq"], case["page"], _n_pages(case), _stride(case), case["planes"]
    kind = case["kind"]
    lens = torch.as_tensor(_lengths(case))
    if kind == "compact":
        holes = torch.zeros(n_pages, dtype=torch.bool)
        holes[_holes(case)] = True
        ids = (~holes).nonzero().view(-1)
        ids = ids[m.order(len(ids))]
    else:
        ids = m.order(n_pages)
    table = torch.full((n, stride), -1, dtype=torch.int32)
    at = 0
    for i in range(n):
        k = _pages(int(lens[i]), page)
        table[i, :k] = ids[at:at + k].int()
        at += k
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[ids[:at]] = 1
    s["table"], s["len"], s["refs"] = m.up(table), m.up(lens), m.up(refs)
    s["table_out"], s["len_out"], s["refs_out"] = (torch.empty_like(s[x]) for x in ("table", "len", "refs"))
    s["status"] = m.up([0, 0])
    if planes:
        s["cache"] = m.normal((planes, n_pages, case["hkv"], page, case["d"]), torch.bfloat16)
    if kind == "extend":
        adds = torch.as_tensor(_adds(case))[m.order(n)]
        s["add"], s["tokens"] = m.up(adds), int(adds.sum())
        s["slots"], s["pos"] = m.up([0] * s["tokens"]), m.up([0] * s["tokens"])
    elif kind == "select":
        kept = torch.as_tensor(_kept(case))
        parent = kept.repeat(2)[:n] if n > 1 else kept
        s["parent"], s["copies"] = m.up(parent[m.order(n)]), n - len(kept)
    else:
        s["moves"] = _moves(case)


def _handles(s, case):
    """The relations that a program keeps over its tensors."""
    from paper_2609_03905_amd import ea

    names = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}

    def whole(t, shape=None, part=None):
        if t is None:
            return None
        shape = tuple(t.shape) if shape is None else shape
        return ea.Relation(shape, names[t.dtype], part or ea.whole_partition(shape), data=t)

    def pages(t):  # one block per page
        part = ea.whole_partition(t.shape)
        for dim in range(t.dim() - 3):
            part[dim] = list(range(t.shape[dim] + 1))
        return ea.Relation(t.shape, names[t.dtype], part, data=t)

    kind, r = case["kind"], {}
    if kind in ("heads", "heads_grad"):
        t, w, b = case["t"], (case["hq"] + 2 * case["hkv"]) * case["d"], case.get("block") or 0
        r["x"] = whole(s["x"], (t, w), [list(range(0, t + 1, b)), list(range(0, w + 1, b))] if b else None)
        r["wq"], r["wk"] = whole(s["wq"]), whole(s["wk"])
        if kind_grad(case):
            r |= {x: whole(s[x]) for x in ("dq", "dk", "dv", "dx", "dwq", "dwk")}
        else:
            r["q"] = whole(s["q"])
            r["k"], r["v"] = (pages if case["page"] else whole)(s["k"]), (pages if case["page"] else whole)(s["v"])
    elif kind == "attention":
        r |= {"q": whole(s["q"]), "out": whole(s["out"]), "k": pages(s["k"]), "v": pages(s["v"])}
    elif case["planes"]:
        r["cache"] = pages(s["cache"])
    s["rel"] = r


# ---- one pass ------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s)
    return {"heads": _plain_heads, "heads_grad": _plain_heads_grad, "attention": _plain_attention,
            "extend": _plain_extend, "select": _plain_select, "compact": _plain_compact}[kind](s)


def _own(s):
    from paper_2609_03905_amd import ea

    case, r = s["case"], s["rel"]
    kind = case["kind"]
    if kind == "heads":
        ea.heads(r["x"], r["q"], r["k"], r["v"], d_head=case["d"], wq=r["wq"], wk=r["wk"], eps=EPS,
                 inv_freq=s["freq"], interleaved=case["interleaved"], positions=s["pos"], slots=s["slots"])
        return {"q": s["q"], "k": s["k"], "v": s["v"]}
    if kind == "heads_grad":
        ea.heads_backward(r["x"], r["dq"], r["dk"], r["dv"], r["dx"], d_head=case["d"], wq=r["wq"], wk=r["wk"],
                          dwq=r["dwq"], dwk=r["dwk"], eps=EPS, inv_freq=s["freq"], interleaved=case["interleaved"],
                          positions=s["pos"])
        return {"dx": s["dx"], "dwq": s["dwq"], "dwk": s["dwk"]}
    if kind == "attention":
        ea.attention_paged(r["q"], r["k"], r["v"], r["out"], scale=case["d"] ** -0.5, table=s["table"],
                           lengths=s["len"], q_start=s["start"], group_start=s["group_start"],
                           group_shared=s["group_shared"])
        return {"out": s["out"]}
    if kind == "extend":
        ea.pages_extend(s["table"], s["len"], s["refs"], s["add"], page_size=case["page"], out_lengths=s["len_out"],
                        out_refs=s["refs_out"], status=s["status"], slots=s["slots"], positions=s["pos"])
        return {"table": s["table"], "len": s["len_out"], "refs": s["refs_out"], "status": s["status"],
                "slots": s["slots"], "pos": s["pos"]}
    if kind == "select":
        ea.pages_select([r["cache"]], s["parent"], s["table"], s["len"], s["refs"], out_table=s["table_out"],
                        out_lengths=s["len_out"], out_refs=s["refs_out"], status=s["status"])
        return {"table": s["table_out"], "len": s["len_out"], "refs": s["refs_out"], "status": s["status"],
                "cache": s["cache"].view(torch.int16)}
    ea.pages_compact([r["cache"]], s["table"], s["len"], s["refs"], out_table=s["table_out"], out_refs=s["refs_out"],
                     status=s["status"])
    return {"table": s["table_out"], "refs": s["refs_out"], "status": s["status"], "cache": s["cache"].view(torch.int16)}


# ---- the plain forms ---------------------------------------------------------
def _dense(s):
    case = s["case"]
    x = s["x"]
    return x.permute(0, 2, 1, 3).reshape(case["t"], -1) if case.get("block") else x


def _angles(s):
    """cos and sin of each row's angles (in 64 bits: positions may be far)."""
    a = s["pos"].double()[:, None] * s["freq"].double()[None, :]
    return a.cos().float()[:, None, :], a.sin().float()[:, None, :]


def _turn(n, cos, sin, rot, interleaved):
    """Rows [t, h, d] with their first `rot` elements rotated in pairs."""
    if interleaved:
        a, b = n[..., 0:rot:2], n[..., 1:rot:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = n[..., : rot // 2], n[..., rot // 2:rot]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((y, n[..., rot:]), -1)


def _normed(u, w):
    if w is None:
        return u
    return u * torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS) * w.float()


def _plain_heads(s):
    case = s["case"]
    t, hq, hkv, d = case["t"], case["hq"], case["hkv"], case["d"]
    x = _dense(s).float().view(t, hq + 2 * hkv, d)
    cos, sin = _angles(s)
    q = _turn(_normed(x[:, :hq], s["wq"]), cos, sin, case["rotary"], case["interleaved"])
    k = _turn(_normed(x[:, hq:hq + hkv], s["wk"]), cos, sin, case["rotary"], case["interleaved"])
    v = x[:, hq + hkv:]
    dt = s["q"].dtype
    if not case["page"]:
        return {"q": q.to(dt).transpose(0, 1).contiguous(), "k": k.to(dt).transpose(0, 1).contiguous(),
                "v": v.to(dt).transpose(0, 1).contiguous()}
    real = s["real"]
    slot = s["slots"][real].long()
    page, at = slot // case["page"], slot % case["page"]
    s["k"][page, :, at] = k[real].to(dt)
    s["v"][page, :, at] = v[real].to(dt)
    return {"q": q.to(dt).view(t, hq * d), "k": s["k"], "v": s["v"]}


def _unturn(g, cos, sin, rot, interleaved):
    return _turn(g, cos, -sin, rot, interleaved)


def _row_grad(u, w, g):
    """dx and dw of rows u normed with w, from the gradient g of the result."""
    if w is None:
        return g, None
    r = torch.rsqrt(u.square().mean(-1, keepdim=True) + EPS)
    n, t = u * r, g * w.float()
    return r * (t - n * (t * n).mean(-1, keepdim=True)), (g * n).sum((0, 1))


def _plain_heads_grad(s):
    case = s["case"]
    t, hq, hkv, d = case["t"], case["hq"], case["hkv"], case["d"]
    x = s["x"].float().view(t, hq + 2 * hkv, d)
    cos, sin = _angles(s)
    gq = _unturn(s["dq"].float().view(t, hq, d), cos, sin, case["rotary"], case["interleaved"])
    gk = _unturn(s["dk"].float().view(t, hkv, d), cos, sin, case["rotary"], case["interleaved"])
    xq, dwq = _row_grad(x[:, :hq], s["wq"], gq)
    xk, dwk = _row_grad(x[:, hq:hq + hkv], s["wk"], gk)
    dx = torch.cat((xq, xk, s["dv"].float().view(t, hkv, d)), 1).view(t, -1).to(s["x"].dtype)
    return {"dx": dx, "dwq": dwq, "dwk": dwk}


def _plain_attention(s):
    case = s["case"]
    n, n_q, hq, hkv, d, page = (case[x] for x in ("n_seq", "n_q", "hq", "hkv", "d", "page"))
    g = hq // hkv
    pages = s["table"].clamp(min=0).long()

    def keys(c):  # every sequence's rows, [n, hkv, keys, d]
        return c[pages].float().transpose(1, 2).reshape(n, hkv, -1, d)

    # query rows of one sequence and key-value head: token-major, then heads
    q = s["q"].float().view(n, n_q, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, n_q * g, d)
    scores = torch.matmul(q, keys(s["k"]).transpose(2, 3).contiguous()) * d ** -0.5
    seen = s["len"].long()[:, None] - n_q + torch.arange(1, n_q + 1, device=q.device)[None, :]
    at = torch.arange(scores.shape[-1], device=q.device)
    mask = at[None, None, :] < seen.repeat_interleave(g, 1)[:, :, None]
    scores = scores.masked_fill(~mask[:, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(scores - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, keys(s["v"])) / torch.where(total > 0, total, 1.0)
    o = o.view(n, hkv, n_q, g, d).permute(0, 2, 1, 3, 4)
    return {"out": o.reshape(n * n_q, hq * d).to(s["q"].dtype)}


def _free(refs):
    """Page numbers, free ones first, each kind ascending."""
    return torch.sort((refs > 0).to(torch.int8), stable=True).indices


def _plain_extend(s):
    page, refs, table = s["case"]["page"], s["refs"], s["table"]
    length, add = s["len"].long(), s["add"].long()
    have, new = (length + page - 1) // page, (length + add + page - 1) // page
    need = new - have
    before = need.cumsum(0) - need
    free = _free(refs)
    col = torch.arange(table.shape[1], device=table.device)[None, :]
    rank = (before - have)[:, None] + col
    fresh = (col >= have[:, None]) & (col < new[:, None])
    table.copy_(torch.where(fresh, free[rank.clamp(0, len(free) - 1)].int(), table))
    taken = torch.arange(len(free), device=table.device) < need.sum()
    out_refs = refs.clone()
    out_refs[free] = torch.where(taken, 1, refs[free])
    ends = add.cumsum(0)
    token = torch.arange(s["tokens"], device=table.device)
    seq = torch.searchsorted(ends, token, right=True)
    pos = length[seq] + token - (ends - add)[seq]
    slots = table[seq, pos // page].long() * page + pos % page
    left = (refs == 0).sum() - need.sum()
    status = torch.stack((torch.zeros_like(left), left))
    return {"table": table, "len": (length + add).int(), "refs": out_refs, "status": status.int(),
            "slots": slots.int(), "pos": pos.int()}


def _plain_select(s):
    page, refs, table, cache = s["case"]["page"], s["refs"], s["table"], s["cache"]
    n, stride = table.shape
    length, parent = s["len"].long(), s["parent"].long()
    i = torch.arange(n, device=table.device)
    col = torch.arange(stride, device=table.device)[None, :]
    alive, p = parent >= 0, parent.clamp(min=0)
    children = torch.zeros_like(length).scatter_add(0, p, alive.long())
    first = torch.full_like(p, n).scatter_reduce(0, p, torch.where(alive, i, n), "amin")
    full, tail = length // page, length % page
    # whole pages get a count for each child, a partly filled one stays its first child's
    delta = torch.where(col < full[:, None], (children - 1)[:, None], 0)
    delta -= ((col == full[:, None]) & (tail[:, None] > 0) & (children[:, None] == 0)).long()
    out_refs = refs.long().scatter_add(0, table.clamp(min=0).long().view(-1), delta.view(-1))
    need = alive & (first[p] != i) & (tail[p] > 0)
    rank = need.cumsum(0) - 1
    dst = _free(out_refs)[rank.clamp(min=0)]
    held = torch.where(alive, (length[p] + page - 1) // page, 0)
    out = torch.where(col < held[:, None], table[p], -1)
    src = table.gather(1, full.clamp(max=stride - 1)[:, None])[p, 0].long()
    out = torch.where(need[:, None] & (col == full[p][:, None]), dst[:, None].int(), out)
    which = torch.sort((~need).to(torch.int8), stable=True).indices[: s["copies"]]
    out_refs[dst[which]] = 1
    # the rows that the sequence holds; the page's other rows keep what they held
    rows = torch.arange(page, device=table.device)[None, :] < tail[p[which]][:, None]
    old = cache[:, dst[which]]
    cache[:, dst[which]] = torch.where(rows[None, :, None, :, None], cache[:, src[which]], old)
    left = (out_refs == 0).sum()
    return {"table": out, "len": torch.where(alive, length[p], 0).int(), "refs": out_refs.int(),
            "status": torch.stack((torch.zeros_like(left), left)).int(), "cache": cache.view(torch.int16)}


def _plain_compact(s):
    page, refs, table, cache, moves = s["case"]["page"], s["refs"], s["table"], s["cache"], s["moves"]
    used = refs > 0
    n_used = used.sum()
    at = torch.arange(len(refs), device=refs.device)
    holes = torch.sort((used | (at >= n_used)).to(torch.int8), stable=True).indices[:moves]
    movers = torch.sort((~used | (at < n_used)).to(torch.int8), stable=True).indices[:moves]
    to = at.clone()
    to[movers] = holes
    held = (s["len"].long() + page - 1) // page
    col = torch.arange(table.shape[1], device=table.device)[None, :]
    out = torch.where(col < held[:, None], to[table.clamp(min=0).long()].int(), -1)
    out_refs = refs.clone()
    out_refs[holes] = refs[movers]
    out_refs[movers] = 0
    cache[:, holes] = cache[:, movers]
    left = len(refs) - n_used
    return {"table": out, "refs": out_refs, "status": torch.stack((torch.zeros_like(left), left)).int(),
            "cache": cache.view(torch.int16)}


# ---- 64-bit values, from the definitions ----------------------------------------
def exact(case, seed):
    if case["kind"] not in ("heads", "heads_grad", "attention"):
        return None
    s = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(s, case)
    t, hq, hkv, d, rot = (case[x] for x in ("t", "hq", "hkv", "d", "rotary"))
    x = _dense(s).double().view(t, -1, d)
    # pair (i, j) of a head turned as the complex number n_i + i n_j
    i = torch.arange(rot // 2, device=x.device)
    first = 2 * i if case["interleaved"] else i
    second = first + 1 if case["interleaved"] else first + rot // 2
    angle = s["pos"].double()[:, None, None] * s["freq"].double()
    turn = torch.polar(torch.ones_like(angle), angle)

    def rows(u, w):
        y = u if w is None else w * u / (u.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt()
        z = torch.complex(y[..., first], y[..., second]) * turn
        back = torch.empty(rot, dtype=torch.long, device=x.device)
        back[torch.cat((first, second))] = torch.arange(rot, device=x.device)
        return torch.cat((torch.cat((z.real, z.imag), -1)[..., back], y[..., rot:]), -1)

    wq = None if s["wq"] is None else s["wq"].double()
    wk = None if s["wk"] is None else s["wk"].double()
    if kind_grad(case):
        leaves = [u.detach().clone().requires_grad_() for u in (x[:, :hq], x[:, hq:hq + hkv])]
        weights = [None if w is None else w.clone().requires_grad_() for w in (wq, wk)]
        total = (rows(leaves[0], weights[0]) * s["dq"].double().view(t, hq, d)).sum()
        total = total + (rows(leaves[1], weights[1]) * s["dk"].double().view(t, hkv, d)).sum()
        total.backward()
        dx = torch.cat((leaves[0].grad, leaves[1].grad, s["dv"].double().view(t, hkv, d)), 1).view(t, -1)
        return {"dx": dx, "dwq": weights[0].grad if wq is not None else None,
                "dwk": weights[1].grad if wk is not None else None}
    q, k, v = rows(x[:, :hq], wq), rows(x[:, hq:hq + hkv], wk), x[:, hq + hkv:]
    if not case["page"]:
        return {"q": q.permute(1, 0, 2).contiguous(), "k": k.permute(1, 0, 2).contiguous(),
                "v": v.permute(1, 0, 2).contiguous()}
    kc, vc = s["k"].double(), s["v"].double()
    slots = s["slots"].long()
    held = (slots >= 0).nonzero().view(-1)
    for c, rows_of in ((kc, k), (vc, v)):
        c[slots[held] // case["page"], :, slots[held] % case["page"]] = rows_of[held]
    return {"q": q.reshape(t, hq * d), "k": kc, "v": vc}


def _exact_attention(s, case):
    n, n_q, hq, hkv, d, page = (case[x] for x in ("n_seq", "n_q", "hq", "hkv", "d", "page"))
    if 4 * d * hq * n_q * sum(case["shared"] + x for x in _lengths(case)) > 4e11:
        return None
    out = torch.zeros((n, n_q, hkv, hq // hkv, d), dtype=torch.float64, device=s["q"].device)
    lens = s["len"].tolist()
    for i, length in enumerate(lens):
        at = torch.arange(length, device=out.device)
        page_of = s["table"][i].long()[at // page]
        k, v = (c[page_of, :, at % page].double().transpose(0, 1).contiguous() for c in (s["k"], s["v"]))
        for j in range(n_q):
            m = length - n_q + j + 1  # keys that this token sees
            if m > 0:
                q = s["q"][i * n_q + j].double().view(hkv, hq // hkv, d)
                w = torch.softmax((k[:, :m] @ q.transpose(1, 2)) / math.sqrt(d), 1)
                out[i, j] = w.transpose(1, 2) @ v[:, :m]
    return {"out": out.view(n * n_q, hq * d)}
