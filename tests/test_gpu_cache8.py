"""Rows quantised into a cache in 8 bits and read back: equal to the definition,
code by code, over ragged batches, blocks that go on, odd pages and values that
are no numbers."""
import numpy as np
import pytest
import torch

import cache8_ref as C
import decode_ref as R
from paper_2609_03905_amd import ea

pytestmark = pytest.mark.gpu


def _state(olds, news, page, block, hkv, d, code, seed, spare=3):
    """Sequences of olds[s] keys that are to get news[s] more, over shuffled pages."""
    rng = np.random.default_rng(seed)
    n = len(olds)
    held = [-(-(o + x) // page) for o, x in zip(olds, news)]
    total = sum(held) + spare
    table = np.full((n, max(held) + 1), -1, np.int64)
    ids = list(rng.permutation(total))
    for s in range(n):
        table[s, :held[s]] = [ids.pop() for _ in range(held[s])]
    kv = []
    for _ in range(2):
        codes = C.rounded(np.clip(rng.standard_normal((total, hkv, page, d)) * 100, -448, 448), code)  # what has a code
        kv.append((codes, 2.0 ** rng.integers(-6, 3, (total, hkv, page // block))))
    lens = [o + x for o, x in zip(olds, news)]
    return kv, table, lens, [0] + list(np.cumsum(news)), rng


def _rows(rng, t, hkv, d, dtype):
    x = rng.standard_normal((t, hkv, d)) * np.exp(rng.standard_normal((t, hkv, 1)) * 2)
    return torch.from_numpy(x.astype(np.float32)).to(R.TORCH[dtype]).cuda()


def _laid(x, form):
    t, h, d = x.shape
    if form == "tokens":
        return C.rel(x.reshape(t, h * d)), lambda r: r.data.view(x.dtype).view(t, h, d)
    if form == "heads":
        y = x.transpose(0, 1).contiguous()
        return C.rel(y), lambda r: y.transpose(0, 1)
    # blocks of 5 rows, of a head each
    part = [list(range(0, t, 5)) + [t], list(range(0, (h + 1) * d, d))]
    return R.blocked(x.reshape(t, h * d), part), lambda r: R.unblocked(r).view(t, h, d)


def _write(xk, xv, k, v, table, lens, starts, forms=("tokens", "tokens")):
    ea.pages_write(_laid(xk, forms[0])[0], _laid(xv, forms[1])[0], k.rel, v.rel, k_scale=k.scale_rel,
                   v_scale=v.scale_rel, table=R.i32(table), lengths=R.i32(lens),
                   q_start=None if starts is None else R.i32(starts))


def _check_write(kv, xs, table, lens, starts, code, forms=("tokens", "tokens"), null=False):
    dev = [C.Cache(codes, scale, code) for codes, scale in kv]
    _write(xs[0], xs[1], *dev, table, lens, None if null else starts, forms)
    for x, (codes, scale), c, what in zip(xs, kv, dev, "KV"):
        C.write(C.f64(x), codes, scale, table, lens, starts, code)
        C.same(c.scale.cpu().numpy(), scale, what + " scale")
        C.same(C.f64(c.get()), codes, what)
    return dev


CASES = [
    # olds, news, page, block, hkv, d, code, dtype, forms
    ([0], [1], 16, 16, 1, 128, "e4m3", "bf16", ("tokens", "tokens")),
    ([3], [1], 16, 16, 2, 64, "e5m2", "f16", ("heads", "tokens")),
    ([0, 15, 16, 17, 31, 7], [1, 1, 1, 1, 1, 1], 16, 16, 3, 128, "e4m3", "bf16", ("tokens", "heads")),
    ([5, 0, 300, 20], [5, 5, 5, 5], 20, 4, 2, 64, "e5m2", "bf16", ("blocks", "tokens")),
    ([0, 2, 40], [33, 0, 70], 8, 8, 1, 96, "e4m3", "f32", ("tokens", "blocks")),
    ([0], [257], 64, 64, 2, 128, "e4m3", "bf16", ("heads", "heads")),
    ([100], [300], 128, 128, 1, 256, "e4m3", "f32", ("tokens", "tokens")),  # more rows than stay in registers
    ([1, 9], [90, 3], 7, 1, 5, 16, "e5m2", "f16", ("tokens", "tokens")),    # a scale a row
    ([0, 4], [50, 5], 6, 3, 2, 512, "e4m3", "bf16", ("tokens", "heads")),
    ([11] * 70, [1] * 70, 16, 8, 1, 48, "e4m3", "f16", ("tokens", "tokens")),
    ([4], [200], 4096, 4096, 1, 32, "e4m3", "bf16", ("tokens", "tokens")),
]


@pytest.mark.parametrize("case", CASES, ids=[f"n{len(c[0])}_p{c[2]}_b{c[3]}_h{c[4]}_d{c[5]}_{c[6]}_{c[7]}" for c in CASES])
def test_write(case):
    olds, news, page, block, hkv, d, code, dtype, forms = case
    kv, table, lens, starts, rng = _state(olds, news, page, block, hkv, d, code, 1)
    xs = [_rows(rng, starts[-1], hkv, d, dtype) for _ in range(2)]
    _check_write(kv, xs, table, lens, starts, code, forms, null=all(x == 1 for x in news))


@pytest.mark.parametrize("case", CASES, ids=[f"n{len(c[0])}_p{c[2]}_b{c[3]}_h{c[4]}_d{c[5]}_{c[6]}_{c[7]}" for c in CASES])
def test_read(case):
    olds, news, page, block, hkv, d, code, dtype, forms = case
    kv, table, lens, starts, rng = _state(olds, news, page, block, hkv, d, code, 2)
    if len(table) > 1:
        table[1, 0] = len(kv[0][0]) + 5  # outside the cache: zeros
    dev = [C.Cache(codes, scale, code) for codes, scale in kv]
    t = starts[-1] + 3  # rows behind the last sequence stay
    outs = [_laid(torch.full((t, hkv, d), 7.0, device="cuda").to(R.TORCH[dtype]), f) for f in forms]
    ea.pages_read(dev[0].rel, dev[1].rel, outs[0][0], outs[1][0], k_scale=dev[0].scale_rel, v_scale=dev[1].scale_rel,
                  table=R.i32(table), lengths=R.i32(lens), q_start=R.i32(starts))
    for (codes, scale), (r, get) in zip(kv, outs):
        want = np.full((t, hkv, d), 7.0)
        want[:starts[-1]] = 0
        vals = C.values(codes, scale)
        for row, _, at, pg in C.places(table, lens, starts, page, len(codes)):
            if pg >= 0:
                want[row] = vals[pg, :, at % page]
        want = torch.from_numpy(want).to(R.TORCH[dtype]).double().numpy()  # one rounding
        C.same(C.f64(get(r)), want)


@pytest.mark.parametrize("major", ["tokens", "heads"])
@pytest.mark.parametrize("hb,tb", [(2, 7), (3, 1), (1, 64), (5, 6)])
def test_partitions_of_the_rows(major, hb, tb):
    """K's rows in blocks of hb of 5 heads and tb rows, the last ones shorter; V's
    in one block."""
    news, page, block, hkv, d = [40, 3, 25], 12, 6, 5, 48
    kv, table, lens, starts, rng = _state([5, 0, 9], news, page, block, hkv, d, "e4m3", 21)
    t = starts[-1]
    cut = lambda n, b: list(range(0, n, b)) + [n]
    lay = lambda x: R.blocked(x.reshape(t, hkv * d), [cut(t, tb), [i * d for i in cut(hkv, hb)]]) if major == "tokens" else \
        R.blocked(x.transpose(0, 1).contiguous(), [cut(hkv, hb), cut(t, tb), [0, d]])
    dense = lambda r: R.unblocked(r).view(t, hkv, d) if major == "tokens" else R.unblocked(r).transpose(0, 1)
    xs = [_rows(rng, t, hkv, d, "bf16") for _ in range(2)]
    dev = [C.Cache(codes, scale, "e4m3") for codes, scale in kv]
    batch = dict(k_scale=dev[0].scale_rel, v_scale=dev[1].scale_rel, table=R.i32(table), lengths=R.i32(lens),
                 q_start=R.i32(starts))
    ea.pages_write(lay(xs[0]), _laid(xs[1], "tokens")[0], dev[0].rel, dev[1].rel, **batch)
    for x, (codes, scale), c in zip(xs, kv, dev):
        C.write(C.f64(x), codes, scale, table, lens, starts, "e4m3")
        C.same(c.scale.cpu().numpy(), scale)
        C.same(C.f64(c.get()), codes)
    outs = [lay(torch.full_like(xs[0], 7.0)), _laid(torch.full_like(xs[1], 7.0), "tokens")]
    ea.pages_read(dev[0].rel, dev[1].rel, outs[0], outs[1][0], **batch)
    for (codes, scale), got in zip(kv, (dense(outs[0]), outs[1][1](outs[1][0]))):
        vals, want = C.values(codes, scale), np.zeros((t, hkv, d))
        for row, _, at, pg in C.places(table, lens, starts, page, len(codes)):
            want[row] = vals[pg, :, at % page]
        C.same(C.f64(got), torch.from_numpy(want).bfloat16().double().numpy())


def test_the_most_sequences():
    """As many sequences as a call takes, of no row to three."""
    n = ea.PAGED_MAX_SEQ
    rng = np.random.default_rng(22)
    olds, news = rng.integers(0, 9, n), rng.integers(0, 4, n)
    kv, table, lens, starts, rng = _state(list(olds), list(news), 4, 2, 1, 16, "e5m2", 23)
    xs = [_rows(rng, starts[-1], 1, 16, "f16") for _ in range(2)]
    dev = _check_write(kv, xs, table, lens, starts, "e5m2")
    outs = [_laid(torch.zeros_like(xs[0]), "tokens") for _ in range(2)]
    ea.pages_read(dev[0].rel, dev[1].rel, outs[0][0], outs[1][0], k_scale=dev[0].scale_rel, v_scale=dev[1].scale_rel,
                  table=R.i32(table), lengths=R.i32(lens), q_start=R.i32(starts))
    for (codes, scale), (r, get) in zip(kv, outs):
        vals, want = C.values(codes, scale), np.zeros((starts[-1], 1, 16))
        for row, _, at, pg in C.places(table, lens, starts, 4, len(codes)):
            want[row] = vals[pg, :, at % 4]
        C.same(C.f64(get(r)), torch.from_numpy(want).half().double().numpy())


def test_rows_that_do_not_ascend_or_overlap():
    """First rows that fall back (a sequence without rows, one that has a row twice):
    as many rows as the call has are written by those whose they are; more are not."""
    page, block, hkv, d = 4, 4, 2, 32
    kv, table, lens, _, rng = _state([0, 0, 0], [5, 4, 6], page, block, hkv, d, "e4m3", 24)
    x = _rows(rng, 12, hkv, d, "bf16")
    # sequence 0 rows 0-4, sequence 1 none, sequence 2 rows 2-7: 11 of 12
    dev = [C.Cache(codes, scale, "e4m3") for codes, scale in kv]
    _write(x, x, *dev, table, lens, [0, 5, 2, 8])
    for (codes, scale), c in zip(kv, dev):
        want = [codes.copy(), scale.copy()]
        C.write(C.f64(x[:5]), *want, table[:1], lens[:1], [0, 5], "e4m3")
        C.write(C.f64(x[2:8]), *want, table[2:], lens[2:], [0, 6], "e4m3")
        C.same(c.scale.cpu().numpy(), want[1])
        C.same(C.f64(c.get()), want[0])
    # 15 rows of 12: none
    dev = [C.Cache(codes, scale, "e4m3") for codes, scale in kv]
    _write(x, x, *dev, table, lens, [0, 9, 2, 8])
    for (codes, scale), c in zip(kv, dev):
        C.same(c.scale.cpu().numpy(), scale)
        C.same(C.f64(c.get()), codes)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_every_value_is_rounded_as_defined(code, dtype):
    """All values of 16 bits that a code reaches under the scale 1, the ties and
    the subnormal codes among them (f32: those of fp16)."""
    t = R.TORCH[dtype]
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16 if dtype == "bf16" else torch.float16)
    x = bits[bits.float().abs() <= C.TOP[code]].cuda().to(t)
    d = 512
    n = -(-len(x) // (d - 1))
    rows = torch.zeros(n, 1, d, dtype=t, device="cuda")
    flat = torch.zeros(n * (d - 1), dtype=t, device="cuda")
    flat[:len(x)] = x
    rows[:, 0, 1:] = flat.view(n, d - 1)
    rows[:, 0, 0] = C.TOP[code]  # so the scale is 1
    kv, table, lens, starts, _ = _state([0], [n], 8, 1, 1, d, code, 3)
    dev = _check_write(kv, [rows, rows], table, lens, starts, code)
    assert (dev[0].scale[table[0, 0]] == 1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_scales_at_their_borders(code, dtype):
    """The largest element at, just above and far below a code's reach, zero,
    the smallest numbers, infinities and NaN: a row each, a scale each; and with
    a number of about a third beside it."""
    top = C.TOP[code]
    tops = [top, np.nextafter(np.float32(top), np.float32(np.inf)), top * 1.0078125, top * 2, top / 2, 1.0, 1.75,
            1.7500001, 1.7578125, 0.0, -0.0, 2.0 ** -149, 2.0 ** -133, 2.0 ** -126, 2.0 ** -112, 2.0 ** -111, 2.0 ** -24,
            2.0 ** -14, 65504.0, 3e38, 2.0 ** 127, -top * 1.01, np.inf, -np.inf, np.nan]
    x = np.zeros((len(tops), 1, 16), np.float32)
    x[:, 0, 5] = tops
    x[:, 0, 7] = np.float32(0.3) * np.where(np.isfinite(tops), tops, 1)
    x = torch.from_numpy(x).to(R.TORCH[dtype]).cuda()
    kv, table, lens, starts, _ = _state([0], [len(tops)], 4, 1, 1, 16, code, 4)
    _check_write(kv, [x, -x], table, lens, starts, code)


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_a_scale_grows_and_keeps(code):
    """One token a step into blocks of 8: smaller ones keep the scale, larger
    ones grow it and the codes before are rounded again, into the subnormal ones
    at last; scales that another program left."""
    page, block, hkv, d = 16, 8, 2, 32
    kv, table, lens, _, rng = _state([0, 3], [24, 20], page, block, hkv, d, code, 5)
    dev = [C.Cache(codes, scale, code) for codes, scale in kv]
    at = [0, 3]
    for i in range(18):
        size = 2.0 ** np.where(rng.random() < 0.3, rng.integers(0, 9 + i), rng.integers(-4, 2))
        xs = [_rows(rng, 2, hkv, d, "f32") * float(size) for _ in range(2)]
        at = [n + 1 for n in at]
        if i == 9:
            for (_, scale), c in zip(kv, dev):
                scale *= 0.7
                c.scale.mul_(0.7)
                scale[...] = c.scale.cpu().numpy()
        if i in (3, 13):  # no scale at all: the block's is the new row's
            for (_, scale), c in zip(kv, dev):
                scale[:, 1] = [np.nan, np.inf, -1.0, 0.0][i // 4]
                c.scale[:, 1] = float(scale[0, 1, 0])
        _write(xs[0], xs[1], *dev, table, at, None)
        for x, (codes, scale), c in zip(xs, kv, dev):
            C.write(C.f64(x), codes, scale, table, at, [0, 1, 2], code)
            C.same(c.scale.cpu().numpy(), scale, f"scale, step {i}")
            C.same(C.f64(c.get()), codes, f"step {i}")


def test_rows_without_a_place_are_not_written():
    """More rows than keys, lengths past a table row and below zero, pages
    outside the cache, rows of no sequence; starts that do not ascend and
    tables of any numbers write inside the cache alone."""
    page, hkv, d, code = 8, 1, 16, "e4m3"
    kv, table, _, _, rng = _state([0] * 6, [24] * 6, page, page, hkv, d, code, 6)
    table[2, 1] = -7
    table[3, 0] = len(kv[0][0])
    lens, starts = [3, -4, 20, 10, 10 ** 6, 2 ** 31 - 1], [2, 9, 11, 31, 33, 60, 61]
    xs = [_rows(rng, 70, hkv, d, "bf16") for _ in range(2)]
    _check_write(kv, xs, table, lens, starts, code)
    dev = [C.Cache(codes, scale, code) for codes, scale in kv]
    table = rng.integers(-2 ** 31, 2 ** 31 - 1, table.shape)
    before = [(c.get().view(torch.uint8), c.scale.clone()) for c in dev]
    _write(xs[0], xs[1], *dev, table, lens, [40, -9, 2 ** 31 - 1, 7, -2 ** 31, 60, 90])
    for c, (codes, scale) in zip(dev, before):
        assert torch.equal(c.get().view(torch.uint8), codes) and torch.equal(c.scale, scale)


def test_what_is_read_stands_when_written_again():
    """Values read back and written again are the same (their scale may be half
    as large, where the largest was rounded down to what the next one reaches)."""
    for code, dtype in (("e4m3", "bf16"), ("e5m2", "f32")):
        kv, table, lens, starts, rng = _state([0, 0], [100, 37], 16, 8, 3, 64, code, 7)
        xs = [_rows(rng, starts[-1], 3, 64, dtype) for _ in range(2)]
        dev = _check_write(kv, xs, table, lens, starts, code)
        args = dict(k_scale=dev[0].scale_rel, v_scale=dev[1].scale_rel, table=R.i32(table), lengths=R.i32(lens),
                    q_start=R.i32(starts))
        seen = []
        for _ in range(2):
            back = [_laid(torch.empty_like(x), "tokens") for x in xs]
            ea.pages_read(dev[0].rel, dev[1].rel, back[0][0], back[1][0], **args)
            seen.append([get(r).clone() for r, get in back])
            ea.pages_write(back[0][0], back[1][0], dev[0].rel, dev[1].rel, **args)
        assert all(torch.equal(x, y) for x, y in zip(*seen))


def test_codes_past_four_gib():
    """Pages at both ends of caches of more than 2^32 bytes."""
    page, hkv, d, pages = 64, 8, 128, 66000
    part = [range(pages + 1), [0, hkv], [0, page], [0, d]]
    k, v = (ea.Relation((pages, hkv, page, d), "e4m3", part) for _ in range(2))
    assert k.nbytes > 2 ** 32
    ks, vs = (torch.zeros(pages, hkv, 4, device="cuda") for _ in range(2))
    table = R.i32([[pages - 1, 0, pages - 2]])
    rng = np.random.default_rng(8)
    xs = [_rows(rng, 150, hkv, d, "bf16") for _ in range(2)]
    args = dict(k_scale=C.rel(ks), v_scale=C.rel(vs), table=table, lengths=R.i32([150]), q_start=R.i32([0, 150]))
    ea.pages_write(_laid(xs[0], "tokens")[0], _laid(xs[1], "tokens")[0], k, v, **args)
    back = [_laid(torch.zeros_like(x), "heads") for x in xs]
    ea.pages_read(k, v, back[0][0], back[1][0], **args)
    for x, (r, get) in zip(xs, back):
        codes = np.zeros((3, hkv, page, d))
        scale = np.zeros((3, hkv, 4))
        C.write(C.f64(x), codes, scale, np.array([[2, 0, 1]]), [150], [0, 150], "e4m3")
        vals = C.values(codes, scale)[[2, 0, 1]].transpose(0, 2, 1, 3).reshape(-1, hkv, d)[:150]
        C.same(C.f64(get(r)), torch.from_numpy(vals).bfloat16().double().numpy())


def test_captured_writes_follow_lengths_on_their_stream():
    """A captured write of one token a sequence, replayed while lengths grow, on
    another stream: as the definition, every replay."""
    page, hkv, d, code = 16, 2, 64, "e4m3"
    kv, table, lens, _, rng = _state([0, 5, 30], [40, 40, 40], page, 8, hkv, d, code, 9)
    dev = [C.Cache(codes, scale, code) for codes, scale in kv]
    at = R.i32([0, 5, 30])
    tab = R.i32(table)
    xs = [_rows(rng, 3, hkv, d, "bf16") for _ in range(2)]
    rels = [_laid(x, "tokens")[0] for x in xs]
    out = [_laid(torch.zeros_like(x), "tokens") for x in xs]
    args = dict(k_scale=dev[0].scale_rel, v_scale=dev[1].scale_rel, table=tab, lengths=at)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        at.add_(1)
        ea.pages_write(*rels, dev[0].rel, dev[1].rel, **args)
        ea.pages_read(dev[0].rel, dev[1].rel, out[0][0], out[1][0], **args)
    lens = [0, 5, 30]
    for i in range(20):
        for x in xs:
            x.copy_(_rows(rng, 3, hkv, d, "bf16"))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        torch.cuda.synchronize()
        lens = [n + 1 for n in lens]
        assert at.tolist() == lens
        for x, (codes, scale), c, (r, get) in zip(xs, kv, dev, out):
            C.write(C.f64(x), codes, scale, table, lens, [0, 1, 2, 3], code)
            C.same(c.scale.cpu().numpy(), scale)
            C.same(C.f64(c.get()), codes)
            vals = C.values(codes, scale)
            want = np.stack([vals[table[s][(lens[s] - 1) // page], :, (lens[s] - 1) % page] for s in range(3)])
            C.same(C.f64(get(r)), torch.from_numpy(want).bfloat16().double().numpy())


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
@pytest.mark.parametrize("old", [np.nan, np.inf, -np.inf, -1.0, 0.0, 2.0 ** -149, 2.0 ** -130, 1.5 * 2.0 ** -121,
                                 2.0 ** 120, 2.0 ** 121, 1.5 * 2.0 ** 121, 2.0 ** 126, 2.0 ** 127, 1.75 * 2.0 ** 127])
def test_scales_that_another_program_left(code, old):
    """Blocks that go on under any scale: one that is no positive number counts as
    none, one that is no power of two as the next, one past 2^120 as 2^120, and the
    codes before stand for what they stood for (they are at most 1: 224 under the
    largest)."""
    kv, table, lens, starts, rng = _state([5, 8], [2, 3], 8, 4, 2, 32, code, 31)
    for i, (codes, scale) in enumerate(kv):
        kv[i] = (C.rounded(codes / 2 ** 18 if code == "e5m2" else codes / 512, code), np.full(scale.shape, old))
        assert np.abs(kv[i][0]).max() <= 1
    before = C.values(kv[0][0], kv[0][1]) if 2.0 ** 120 <= old < np.inf else None
    xs = [_rows(rng, starts[-1], 2, 32, "f32") for _ in range(2)]
    dev = _check_write(kv, xs, table, lens, starts, code)
    assert (dev[0].scale[table[0, 0], :, 1] <= 2.0 ** 120).all()
    if before is not None and np.log2(old) % 1 == 0:  # nothing is lost: the same values, exactly
        now = C.values(C.f64(dev[0].get()), dev[0].scale.double().cpu().numpy())
        C.same(now[table[0, 0], :, 4], before[table[0, 0], :, 4])


def _once(y, bits, least):
    """y to the nearest number of `bits` significant bits, ties to even; the least
    step is 2^least."""
    step = 2.0 ** np.maximum(np.frexp(y)[1] - bits, least)
    return np.round(y / step) * step


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_values_are_rounded_once_under_any_scale(code, dtype):
    """Scales that are no powers of two: code times scale just beside a tie of the
    output's type, nearer than 32 bits tell, and among its subnormal numbers."""
    bits, least = {"bf16": (8, -133), "f16": (11, -24)}[dtype]
    parts = 2 ** C.FORM[code][0]
    pairs = []
    for c in [1 + i / parts for i in range(1, parts)]:
        for i in range(0, 2 ** (bits - 1), 1 if bits == 8 else 8):
            pairs.append((c, np.float32((1 + (2 * i + 1) * 2.0 ** -bits) / c)))
    normal = len(pairs)
    for i in range(64):
        pairs.append((pairs[i][0], np.float32((1 + i / 64) * 2.0 ** (least + 1 - i % 4))))
    n, d = len(pairs), 16
    kv, table, lens, starts, _ = _state([0], [n], 8, 1, 1, d, code, 32)
    for codes, scale in kv:
        for r, (c, s) in enumerate(pairs):
            codes[table[0, r // 8], 0, r % 8] = c * np.where(np.arange(d) % 2, -1, 1)
            scale[table[0, r // 8], 0, r % 8] = s
    y = np.array([c * np.float64(s) for c, s in pairs])  # exact: 28 bits
    want = _once(y, bits, least)
    twice = _once(y.astype(np.float32).astype(np.float64), bits, least)
    assert (want != twice)[:normal].sum() > normal // 8  # what the test is about
    dev = [C.Cache(codes, scale, code) for codes, scale in kv]
    outs = [_laid(torch.zeros((n, 1, d), device="cuda").to(R.TORCH[dtype]), "tokens") for _ in range(2)]
    ea.pages_read(dev[0].rel, dev[1].rel, outs[0][0], outs[1][0], k_scale=dev[0].scale_rel, v_scale=dev[1].scale_rel,
                  table=R.i32(table), lengths=R.i32(lens), q_start=R.i32(starts))
    for r, get in outs:
        C.same(C.f64(get(r))[:, 0], want[:, None] * np.where(np.arange(d) % 2, -1, 1))
