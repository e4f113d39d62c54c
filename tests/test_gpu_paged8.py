"""Attention over a paged cache in 8 bits against the 64-bit definition: both
codes, both query types, scales of one row to a page, with and without shared
prefixes, whatever the rows and scales hold that nothing sees."""
import numpy as np
import pytest
import torch

import cache8_ref as C
import decode_ref as R
from paper_2609_03905_amd import ea

pytestmark = pytest.mark.gpu


def _batch(lens, groups, page, block, hkv, d, code, seed, spare=3, spread=2):
    """Codes and scales of K and V, and the page table; groups is a list of
    (first, last + 1, keys shared)."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    own = [-(-max(x, 0) // page) for x in lens]
    table = np.full((n, max(1, max(own)) + 1), -1, np.int64)
    total = sum(own) + spare
    ids = list(rng.permutation(total))
    prefix = {}
    for first, _, keys in groups:
        prefix[first] = [ids.pop() for _ in range(keys // page)]
    for s in range(n):
        g = next((f for f, e, _ in groups if f <= s < e), None)
        mine = list(prefix.get(g, []))[:own[s]]
        mine += [ids.pop() for _ in range(own[s] - len(mine))]
        table[s, :own[s]] = mine
    kv = []
    for _ in range(2):
        x = rng.standard_normal((total, hkv, page, d)) * C.TOP[code] / 5
        x = np.clip(x, -C.TOP[code], C.TOP[code])
        # keys of about 1, whatever the code's reach; scales up to 2^spread apart
        one = {"e4m3": -7, "e5m2": -14}[code]
        kv.append((C.rounded(x, code), 2.0 ** (one + rng.integers(-spread, spread + 1, (total, hkv, page // block)))))
    return kv, table, rng


def _run(q, dev, table, lens, q_start, groups, scale, out=None, form="tokens", **more):
    t, hq, d = q.shape
    src = q.reshape(t, hq * d) if form == "tokens" else q.transpose(0, 1).contiguous()
    out = torch.full_like(src, float("nan")) if out is None else out
    kw = dict(more)
    if groups:
        kw |= {"group_start": R.i32([g[0] for g in groups] + [groups[-1][1]]),
               "group_shared": R.i32([g[2] for g in groups])}
    ea.attention_paged(C.rel(src), dev[0].rel, dev[1].rel, C.rel(out), scale=scale, table=R.i32(table),
                       lengths=R.i32(lens), q_start=None if q_start is None else R.i32(q_start),
                       k_scale=dev[0].scale_rel, v_scale=dev[1].scale_rel, **kw)
    return out.view(t, hq, d) if form == "tokens" else out.transpose(0, 1)


def _check(q, kv, table, lens, q_start, groups, code, dtype, scale=None, form="tokens", dev=None):
    t, hq, d = q.shape
    page = kv[0][0].shape[2]
    scale = d ** -0.5 if scale is None else scale
    dev = dev or [C.Cache(codes, s, code) for codes, s in kv]
    got = _run(q, dev, table, lens, q_start, groups, scale, form=form)
    starts = list(range(len(lens) + 1)) if q_start is None else q_start
    ref, info = R.attention(R.f64(q), C.values(*kv[0]), C.values(*kv[1]), table, lens, page, starts, scale)
    n = starts[-1]
    R.check(R.f64(got)[:n], ref[:n], C.attention_tol(ref, info, dtype, d)[:n])
    return got


CASES = [
    # lens, groups, n_q, hq, hkv, d, page, block, code, dtype
    ([1], [], 1, 1, 1, 64, 16, 16, "e4m3", "bf16"),
    ([0], [], 1, 4, 1, 128, 16, 4, "e5m2", "f16"),
    ([0, 3, 0, 128, 129, 1], [], 1, 4, 2, 128, 16, 16, "e4m3", "bf16"),
    ([700], [], 1, 8, 2, 128, 64, 64, "e4m3", "f16"),
    ([333, 17, 1, 64], [], 1, 6, 2, 64, 20, 5, "e5m2", "f16"),
    ([31, 32, 33, 127], [], 1, 5, 1, 128, 1, 1, "e4m3", "bf16"),
    ([90, 45], [], 1, 40, 1, 64, 7, 1, "e4m3", "f16"),               # more heads a group than a tile's columns
    ([90, 145], [], 1, 24, 1, 128, 16, 8, "e5m2", "bf16"),           # two column tiles
    ([200, 210, 205], [(0, 3, 192)], 1, 4, 1, 128, 16, 16, "e4m3", "bf16"),
    ([128, 128], [(0, 2, 128)], 1, 4, 1, 64, 16, 2, "e5m2", "f16"),  # nothing of their own
    ([50, 300, 310, 290, 12], [(1, 4, 288)], 1, 8, 2, 128, 32, 32, "e5m2", "bf16"),
    ([130, 140, 150, 60, 70], [(0, 3, 128), (3, 5, 48)], 1, 3, 3, 64, 16, 8, "e4m3", "bf16"),
    ([40, 41, 42, 43], [(0, 2, 0), (2, 4, 40)], 1, 4, 2, 64, 8, 8, "e4m3", "f16"),  # a group that shares nothing
    ([64, 100, 64], [(0, 3, 64)], 5, 8, 2, 64, 16, 16, "e4m3", "bf16"),  # drafts that end in the shared keys
    ([3, 9, 1], [], 4, 4, 1, 128, 16, 16, "e4m3", "bf16"),           # more tokens than keys: rows that see none
    ([300, 90], [], 30, 8, 2, 128, 16, 4, "e4m3", "f16"),            # many columns, nothing shared
    ([300, 290], [(0, 2, 256)], 20, 8, 1, 128, 64, 16, "e5m2", "f16"),  # and both
]


@pytest.mark.parametrize("case", CASES, ids=[f"n{len(c[0])}_g{len(c[1])}_q{c[2]}_h{c[3]}_{c[4]}_d{c[5]}_p{c[6]}_b{c[7]}_"
                                             f"{c[8]}_{c[9]}" for c in CASES])
def test_paged8(case):
    lens, groups, n_q, hq, hkv, d, page, block, code, dtype = case
    kv, table, rng = _batch(lens, groups, page, block, hkv, d, code, 1)
    q = torch.from_numpy(rng.standard_normal((len(lens) * n_q, hq, d))).to(R.TORCH[dtype]).cuda()
    starts = None if n_q == 1 else [n_q * i for i in range(len(lens) + 1)]
    _check(q, kv, table, lens, starts, groups, code, dtype)


@pytest.mark.parametrize("shared", [0, 96])
@pytest.mark.parametrize("d,code,dtype", [(64, "e4m3", "bf16"), (64, "e5m2", "f16"), (128, "e4m3", "f16"), (128, "e5m2", "bf16")])
@pytest.mark.parametrize("n_q", [8, 9, 16, 17, 32, 33, 64, 65])
def test_columns_about_the_tiles(n_q, d, code, dtype, shared):
    """Twice 8 to 65 columns a sequence: either side of tiles of 16, 32, 64 and 128
    in both walks, keys that end inside a step and a page."""
    lens = [shared + n_q + 3, shared + 150, shared + n_q]
    groups = [(0, 3, shared)] if shared else []
    kv, table, rng = _batch(lens, groups, 12, 6, 1, d, code, 30 + n_q)
    q = torch.from_numpy(rng.standard_normal((3 * n_q, 2, d))).to(R.TORCH[dtype]).cuda()
    _check(q, kv, table, lens, [n_q * i for i in range(4)], groups, code, dtype)


@pytest.mark.parametrize("code,dtype", [("e4m3", "bf16"), ("e5m2", "f16")])
def test_ragged_query_rows_and_rows_behind(code, dtype):
    """0, 1, 7 and 40 newest tokens a sequence; rows behind the last sequence
    stay as they were; head-major q and out."""
    lens, starts = [30, 5, 260, 40], [0, 0, 1, 41, 48]
    kv, table, rng = _batch(lens, [], 16, 8, 2, 128, code, 2)
    q = torch.from_numpy(rng.standard_normal((53, 4, 128))).to(R.TORCH[dtype]).cuda()
    got = _check(q, kv, table, lens, starts, [], code, dtype, form="heads")
    assert torch.isnan(got[48:].float()).all()


@pytest.mark.parametrize("shared", [0, 6000])
def test_long_walks_and_repeatable(shared):
    """Long walks over many workgroups: against the definition, and the same
    bits on every run."""
    n, page, hkv, hq, d = 5, 16, 2, 8, 128
    lens = [6000 + 40 * i + 1 for i in range(n)]
    groups = [(0, n, shared)] if shared else []
    kv, table, rng = _batch(lens, groups, page, page, hkv, d, "e4m3", 3)
    q = torch.from_numpy(rng.standard_normal((n, hq, d))).bfloat16().cuda()
    dev = [C.Cache(codes, s, "e4m3") for codes, s in kv]
    got = _check(q, kv, table, lens, None, groups, "e4m3", "bf16", dev=dev)
    for _ in range(3):
        assert torch.equal(_run(q, dev, table, lens, None, groups, d ** -0.5), got)


@pytest.mark.parametrize("big", [-100, -60, 60, 100])
def test_scales_far_apart(big):
    """V's scales near the ends of their range and 2^24 apart, K's so that the
    scores stay in reach: the output is as large."""
    lens, page, block, d = [70, 300], 16, 4, 64
    kv, table, rng = _batch(lens, [], page, block, 1, d, "e4m3", 4, spread=12)
    (kc, ks), (vc, vs) = kv
    ks[...] = 2.0 ** rng.integers(-14, -8, ks.shape)
    vs[...] = 2.0 ** (big + rng.integers(-12, 12, vs.shape))
    q = torch.from_numpy(rng.standard_normal((2, 4, d))).bfloat16().cuda()
    _check(q, kv, table, lens, None, [], "e4m3", "bf16")


def _garbage(kv, table, lens, code, seed, number):
    """NaN codes in all rows that nothing sees, and `number` for scales of
    blocks without a row that is seen."""
    (kc, ks), (vc, vs) = kv
    page, block = kc.shape[2], kc.shape[2] // ks.shape[2]
    seen = np.zeros((len(kc), page), bool)
    for s, n in enumerate(lens):
        for j in range(n):
            seen[table[s, j // page], j % page] = True
    blocks = seen.reshape(len(kc), -1, block).any(-1)
    dirty = []
    for codes, scale in kv:
        c, s = codes.copy(), scale.copy()
        c[np.broadcast_to(~seen[:, None, :, None], c.shape)] = np.nan
        s[np.broadcast_to(~blocks[:, None], s.shape)] = number
        dirty.append(C.Cache(c, s, code))
    return dirty


@pytest.mark.parametrize("number", [float("nan"), float("inf"), 3e38, -1.0, 0.0])
@pytest.mark.parametrize("case", [0, 1, 2])
def test_what_nothing_sees_does_not_matter(case, number):
    lens, groups, n_q, hq, hkv, d, page, block, code, dtype = [
        ([33, 1, 150], [], 1, 4, 2, 128, 16, 4, "e4m3", "bf16"),
        ([70, 90, 80], [(0, 3, 64)], 5, 8, 2, 64, 16, 8, "e5m2", "f16"),
        ([300, 90], [], 30, 8, 2, 128, 20, 1, "e4m3", "bf16"),
    ][case]
    kv, table, rng = _batch(lens, groups, page, block, hkv, d, code, 5, spare=6)
    table[0, -1] = 10 ** 6  # behind the keys: not read
    q = torch.from_numpy(rng.standard_normal((len(lens) * n_q, hq, d))).to(R.TORCH[dtype]).cuda()
    starts = [n_q * i for i in range(len(lens) + 1)]
    _check(q, kv, table, lens, starts, groups, code, dtype, dev=_garbage(kv, table, lens, code, 6, number))


@pytest.mark.parametrize("walk", ["few", "many", "both"])
@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_what_one_row_sees_another_does_not(walk, code):
    """The last key of a draft, seen by the last row alone: NaN in an element of
    its V, in its V's scale, in its K, infinities in V (e5m2): the other rows are
    as without; the last row's element, or row, shows them."""
    n_q, hq, d, page = {"few": 3, "many": 20, "both": 5}[walk], 4, 128, 16
    lens = [200, 170]
    groups = [(0, 2, 160)] if walk == "both" else []
    if walk == "both":  # the last shared key is the last that a first draft sees
        lens = [160, 170]
    kv, table, rng = _batch(lens, groups, page, 1, 1, d, code, 7)
    q = torch.from_numpy(rng.standard_normal((2 * n_q, hq, d))).bfloat16().cuda()
    starts = [0, n_q, 2 * n_q]
    clean = _check(q, kv, table, lens, starts, groups, code, "bf16")
    last = lens[0] - 1
    pg, row = table[0, last // page], last % page
    # (shared pages are the other sequence's too: its rows all see that key)
    others = [i for i in range(2 * n_q) if i != n_q - 1 and (walk != "both" or i < n_q)]
    for what in ["code", "scale", "half", "key"] + (["inf"] if code == "e5m2" else []):
        dev = []
        for i, (codes, scale) in enumerate(kv):
            c, s = codes.copy(), scale.copy()
            if what == "code" and i == 1:
                c[pg, 0, row, 9] = np.nan
            if what == "inf" and i == 1:
                c[pg, 0, row, 9] = -np.inf
            if what == "scale" and i == 1:
                s[pg, 0, row] = np.nan
            if what == "half" and i == 0:
                s[pg, 0, row] = 1.5  # no power of two: no number
            if what == "key" and i == 0:
                c[pg, 0, row, 3] = np.nan
            dev.append(C.Cache(c, s, code))
        got = _run(q, dev, table, lens, starts, groups, d ** -0.5)
        assert torch.equal(got[others], clean[others]), what
        mine = got[n_q - 1].float()
        if what == "code":
            assert mine[:, 9].isnan().all() and torch.equal(got[n_q - 1, :, 10:], clean[n_q - 1, :, 10:])
        elif what == "inf":
            assert (mine[:, 9] == -float("inf")).all() and torch.equal(got[n_q - 1, :, :9], clean[n_q - 1, :, :9])
        else:
            assert mine.isnan().all()


@pytest.mark.parametrize("walk", ["few", "many", "both"])
@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_values_past_the_range_of_32_bits_stay_with_who_sees_them(walk, code):
    """The last key of a draft, seen by the last row alone, has V codes up to the
    largest under the largest scale, 2^128 and more among them: the other rows are
    as without, and the last row has an infinity of its sign where a value is one
    (the walk over few columns, which scales the weights: at least 2^110, or one)."""
    n_q, hq, d, page = {"few": 3, "many": 20, "both": 5}[walk], 4, 128, 16
    lens = [200, 170]
    groups = [(0, 2, 160)] if walk == "both" else []
    if walk == "both":
        lens = [160, 170]
    kv, table, rng = _batch(lens, groups, page, 1, 1, d, code, 12)
    q = torch.from_numpy(rng.standard_normal((2 * n_q, hq, d))).bfloat16().cuda()
    starts = [0, n_q, 2 * n_q]
    clean = _check(q, kv, table, lens, starts, groups, code, "bf16")
    last = lens[0] - 1
    pg, row = table[0, last // page], last % page
    (vc, vs), top = kv[1], C.TOP[code]
    vc[pg, 0, row] = 0
    vc[pg, 0, row, :4] = [top, -top, 1, -1]
    vs[pg, 0, row] = 2.0 ** 120
    got = _run(q, [C.Cache(*x, code) for x in kv], table, lens, starts, groups, d ** -0.5)
    others = [i for i in range(2 * n_q) if i != n_q - 1 and (walk != "both" or i < n_q)]
    assert torch.equal(got[others], clean[others])
    mine = got[n_q - 1].float()
    assert (mine[:, 0] > 2.0 ** 110).all() and (mine[:, 1] < -2.0 ** 110).all()
    if walk != "few":
        assert mine[:, :2].isinf().all()


def test_pages_outside_the_cache_are_invisible():
    lens, page = [100, 64], 16
    kv, table, rng = _batch(lens, [], page, 16, 2, 64, "e4m3", 8)
    table[0, 2], table[1, 0] = -5, len(kv[0][0])
    q = torch.from_numpy(rng.standard_normal((2, 4, 64))).bfloat16().cuda()
    _check(q, kv, table, lens, None, [], "e4m3", "bf16")
    _check(q, kv, table, [10 ** 9, -3], None, [], "e4m3", "bf16")  # a table row's keys; none


def test_as_sixteen_bits():
    """Codes and scales of a bf16 cache's values exactly: both calls agree within
    what they may each be off."""
    lens, page, hq, hkv, d = [500, 77, 1300], 32, 8, 2, 128
    kv, table, rng = _batch(lens, [], page, page, hkv, d, "e4m3", 9)
    for i, (codes, scale) in enumerate(kv):
        scale[...] = 2.0 ** -8
    q = torch.from_numpy(rng.standard_normal((3, hq, d))).bfloat16().cuda()
    got = _check(q, kv, table, lens, None, [], "e4m3", "bf16")
    wide = [R.pages_rel(torch.from_numpy(C.values(*x)).bfloat16().cuda()) for x in kv]
    src, out = q.reshape(3, -1), torch.empty(3, hq * d, dtype=torch.bfloat16, device="cuda")
    ea.attention_paged(R.rel(src), *wide, R.rel(out), scale=d ** -0.5, table=R.i32(table), lengths=R.i32(lens))
    ref, info = R.attention(R.f64(q), C.values(*kv[0]), C.values(*kv[1]), table, lens, page, [0, 1, 2, 3], d ** -0.5)
    assert np.all(np.abs(R.f64(got) - R.f64(out).reshape(ref.shape)) <= 2 * C.attention_tol(ref, info, "bf16", d))


def test_the_most_sequences():
    """As many sequences and groups as a call takes, most of a key or none, their
    schedule in shared memory beside both walks' buffers."""
    n, page, hq, hkv, d = ea.PAGED_MAX_SEQ - 4, 4, 4, 1, 128
    rng = np.random.default_rng(13)
    lens = [int(x) for x in rng.integers(0, 12, n)]
    groups = []
    for i in range(4):
        groups.append((i * 20, (i + 1) * 20, 8 * (i + 1)))
        for s in range(i * 20, (i + 1) * 20):
            lens[s] += 8 * (i + 1)
    kv, table, rng = _batch(lens, groups, page, 2, hkv, d, "e4m3", 14)
    q = torch.from_numpy(rng.standard_normal((n, hq, d))).bfloat16().cuda()
    _check(q, kv, table, lens, None, groups, "e4m3", "bf16")
    _check(q, kv, table, lens, None, [], "e4m3", "bf16")


def test_the_most_sequences_of_many_columns():
    """The same beside the buffers of the walk over many columns: 40 heads over one."""
    n, page, hq, d = ea.PAGED_MAX_SEQ, 4, 40, 64
    rng = np.random.default_rng(16)
    lens = [int(x) for x in rng.integers(0, 9, n)]
    kv, table, rng = _batch(lens, [], page, 4, 1, d, "e5m2", 17)
    q = torch.from_numpy(rng.standard_normal((n, hq, d))).to(torch.float16).cuda()
    _check(q, kv, table, lens, None, [], "e5m2", "f16")
    _check(q, kv, table[:-1], lens[:-1], [0] * n, [], "e5m2", "f16")  # and none with a row


@pytest.mark.parametrize("lens", [[4000], [4090, 1], [4200], [2000, 3900, 0, 300]])
def test_walks_joined_by_their_last_part(lens):
    """Table rows about as long as those whose parts the last one joins; the same
    bits on every run, the arrival counters left at zero."""
    hq, hkv, d, page = 8, 2, 128, 16
    kv, table, rng = _batch(lens, [], page, 16, hkv, d, "e4m3", 15)
    table = table[:, :max(-(-n // page) for n in lens)]
    q = torch.from_numpy(rng.standard_normal((len(lens), hq, d))).bfloat16().cuda()
    dev = [C.Cache(codes, s, "e4m3") for codes, s in kv]
    got = _check(q, kv, table, lens, None, [], "e4m3", "bf16", dev=dev)
    ws = ea.new_workspace(ea.attention_paged_workspace(C.rel(q.view(len(lens), -1)), dev[0].rel, len(lens)))
    for _ in range(3):
        assert torch.equal(_run(q, dev, table, lens, None, [], d ** -0.5, workspace=ws), got)
        assert not ws[:ea.WS_COUNTER_BYTES].any()


def test_codes_past_four_gib():
    """Pages at both ends of caches of more than 2^32 bytes."""
    page, hkv, d, pages = 64, 8, 128, 66000
    lens = [300, 40]
    kv, table, rng = _batch(lens, [], page, 16, hkv, d, "e4m3", 10)
    n = len(kv[0][0])
    where = np.array([pages - 1 - i if i % 2 else i for i in range(n)])
    part = [range(pages + 1), [0, hkv], [0, page], [0, d]]
    rels, scales = [], []
    for codes, scale in kv:
        r = ea.Relation((pages, hkv, page, d), "e4m3", part)
        assert r.nbytes > 2 ** 32
        r.data.view(pages, -1)[torch.from_numpy(where).cuda()] = C.code_tensor(codes, "e4m3").view(torch.uint8).view(n, -1)
        s = torch.zeros(pages, hkv, page // 16, device="cuda")
        s[torch.from_numpy(where).cuda()] = torch.from_numpy(scale).float().cuda()
        rels.append(r)
        scales.append(C.rel(s))
    q = torch.from_numpy(rng.standard_normal((2, 2 * hkv, d))).bfloat16().cuda()
    out = torch.empty_like(q)
    far = np.where(table >= 0, where[np.maximum(table, 0)], -1)
    ea.attention_paged(C.rel(q.view(2, -1)), *rels, C.rel(out.view(2, -1)), scale=0.1, table=R.i32(far),
                       lengths=R.i32(lens), k_scale=scales[0], v_scale=scales[1])
    ref, info = R.attention(R.f64(q), C.values(*kv[0]), C.values(*kv[1]), table, lens, page, [0, 1, 2], 0.1)
    R.check(R.f64(out), ref, C.attention_tol(ref, info, "bf16", d))


def test_captured_calls_follow_lengths_with_workspaces_of_their_own():
    """Two captured calls on two streams, replayed together while lengths grow:
    the bits of eager calls, every replay."""
    lens, page, hq, hkv, d = [[500, 3, 40], [7, 2000, 64]], 16, 8, 2, 128
    sets = []
    for i in range(2):
        kv, table, rng = _batch([n + 40 for n in lens[i]], [], page, 8, hkv, d, ["e4m3", "e5m2"][i], 11 + i)
        dev = [C.Cache(codes, s, ["e4m3", "e5m2"][i]) for codes, s in kv]
        q = torch.from_numpy(rng.standard_normal((3, hq, d))).bfloat16().cuda().view(3, -1)
        out = torch.empty_like(q)
        at = R.i32(lens[i])
        ws = ea.new_workspace(ea.attention_paged_workspace(C.rel(q), dev[0].rel, 3))
        sets.append((dev, q, out, at, R.i32(table), ws, [C.rel(q), dev[0].rel, dev[1].rel, C.rel(out)]))

    def call(s, out=None, ws=None):
        dev, q, o, at, table, w, rels = s
        rels = rels if out is None else rels[:3] + [C.rel(out)]
        ea.attention_paged(*rels, scale=0.1, table=table, lengths=at, k_scale=dev[0].scale_rel, v_scale=dev[1].scale_rel,
                           workspace=w if ws is None else ws)

    streams, graphs = [torch.cuda.Stream() for _ in sets], []
    torch.cuda.synchronize()
    for s, st in zip(sets, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            s[3].add_(1)
            call(s)
        graphs.append(g)
    for _ in range(6):
        torch.cuda.synchronize()
        for st, g in zip(streams, graphs):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s in sets:
            want = torch.empty_like(s[2])
            call(s, want, ea.new_workspace(s[5].numel()))
            assert torch.equal(s[2], want) and want.isfinite().all()
            assert not s[5][:ea.WS_COUNTER_BYTES].any()


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
@pytest.mark.parametrize("walk", ["few", "many", "both"])
@pytest.mark.parametrize("keys,scale,top", [(6000, 97, 448.0), (400, 119, 2.0 ** -9)])
def test_large_values_of_many_keys(keys, scale, top, walk, code):
    """V of one sign under a scale of up to 2^119, the largest value times the keys
    just under 2^119, and later keys whose weights are 2^7.2 of the first ones': all
    finite, as in 64 bits."""
    n_q, d, page = {"few": 1, "many": 20, "both": 1}[walk], 64, 16
    lens = [keys, keys - 1]
    groups = [(0, 2, keys // 2 // page * page)] if walk == "both" else []
    kv, table, rng = _batch(lens, groups, page, 1, 1, d, code, 40)
    (kc, ks), (vc, vs) = kv
    kc[...], ks[...], vs[...] = 0, 1, 2.0 ** scale
    vc[...] = C.rounded(rng.uniform(top / 2, top, vc.shape), code) if top > 1 else top
    assert vc.max() * 2.0 ** scale * keys < 2.0 ** 119
    for s, n in enumerate(lens):
        for j in range(256, n):
            kc[table[s, j // page], 0, j % page, 0] = 5
    q = torch.zeros(2 * n_q, 4, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1
    got = _check(q, kv, table, lens, [n_q * i for i in range(3)], groups, code, "bf16", scale=1.0)
    assert got.isfinite().all()


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
@pytest.mark.parametrize("walk", ["few", "many", "both"])
@pytest.mark.parametrize("scale", [-120, -112])
def test_small_values_of_many_keys(scale, walk, code):
    """V under the smallest scales, most keys of weights of 2^-7.2: off by half of
    bf16's smallest number (2^-134) times a code for every key, and in the store by
    as much."""
    keys, n_q, d, page = 700, {"few": 1, "many": 20, "both": 1}[walk], 64, 16
    lens = [keys, keys - 1]
    groups = [(0, 2, 320)] if walk == "both" else []
    kv, table, rng = _batch(lens, groups, page, 1, 1, d, code, 41)
    (kc, ks), (vc, vs) = kv
    kc[...], ks[...], vs[...] = 0, 1, 2.0 ** scale
    vc[...] = C.rounded(rng.uniform(-C.TOP[code], C.TOP[code], vc.shape) * 2.0 ** -rng.integers(0, 20, vc.shape), code)
    for s in range(2):
        for j in range(0, 300, 7):
            kc[table[s, j // page], 0, j % page, 0] = 5
    q = torch.zeros(2 * n_q, 4, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1
    starts = [n_q * i for i in range(3)]
    dev = [C.Cache(codes, s, code) for codes, s in kv]
    got = _run(q, dev, table, lens, starts, groups, 1.0)
    ref, info = R.attention(R.f64(q), C.values(*kv[0]), C.values(*kv[1]), table, lens, page, starts, 1.0)
    R.check(R.f64(got), ref, C.attention_tol(ref, info, "bf16", d) + 2.0 ** -134 * (1 + keys * C.TOP[code]))
