"""Attention over a paged cache, with and without shared prefixes, against the
64-bit definition: lengths from none to several chunks, odd pages, ragged
query rows, tables with pages outside the cache."""
import numpy as np
import pytest
import torch

import decode_ref as R
from paper_2609_03905_amd import ea

pytestmark = pytest.mark.gpu


def _batch(lens, shared, groups, page, hkv, d, dtype, seed, spare=3, garbage=None):
    """K, V, the page table and host copies: groups is a list of (first, last
    + 1, keys shared).  Rows no sequence holds are `garbage` if given."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    stride = max(1, max((-(-x // page) for x in lens), default=1)) + 1
    table = np.full((n, stride), -1, np.int64)
    own = [-(-x // page) for x in lens]
    total = sum(own) + spare
    ids = list(rng.permutation(total))
    prefix = {}
    for first, last, keys in groups:
        prefix[first] = [ids.pop() for _ in range(keys // page)]
    for s in range(n):
        g = next((f for f, e, _ in groups if f <= s < e), None)
        mine = list(prefix.get(g, []))[: own[s]]
        mine += [ids.pop() for _ in range(own[s] - len(mine))]
        table[s, :own[s]] = mine
    gen = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((total, hkv, page, d), generator=gen, device="cuda").to(R.TORCH[dtype]) for _ in range(2))
    if garbage is not None:
        seen = np.zeros((total, page), bool)
        for s in range(n):
            for j in range(lens[s]):
                seen[table[s, j // page], j % page] = True
        dead = torch.from_numpy(~seen).cuda()[:, None, :, None].expand_as(k)
        k[dead] = garbage
        v[dead] = garbage
    return k, v, table


def _run(q, k, v, table, lens, q_start, groups, scale, out=None, form="tokens"):
    t, hq, d = q.shape
    src = q.reshape(t, hq * d) if form == "tokens" else q.transpose(0, 1).contiguous()
    out = torch.full_like(src, float("nan")) if out is None else out
    kw = {}
    if groups:
        kw = {"group_start": R.i32([g[0] for g in groups] + [groups[-1][1]]),
              "group_shared": R.i32([g[2] for g in groups])}
    ea.attention_paged(R.rel(src), R.pages_rel(k), R.pages_rel(v), R.rel(out), scale=scale, table=R.i32(table),
                       lengths=R.i32(lens), q_start=None if q_start is None else R.i32(q_start), **kw)
    return out.view(t, hq, d) if form == "tokens" else out.transpose(0, 1)


def _check(q, k, v, table, lens, q_start, groups, page, dtype, scale=None, form="tokens"):
    t, hq, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    got = _run(q, k, v, table, lens, q_start, groups, scale, form=form)
    starts = list(range(len(lens) + 1)) if q_start is None else q_start
    hide = lambda z: np.nan_to_num(R.f64(z), nan=0.0, posinf=0.0, neginf=0.0)
    ref, info = R.attention(R.f64(q), hide(k), hide(v), table, lens, page, starts, scale)
    n = starts[-1]
    R.check(R.f64(got)[:n], ref[:n], R.attention_tol(ref, info, dtype, d)[:n])
    return got


CASES = [
    # lens, groups, n_q, hq, hkv, d, page, dtype
    ([1], [], 1, 1, 1, 64, 16, "bf16"),
    ([0], [], 1, 4, 1, 128, 16, "f16"),
    ([0, 3, 0, 128, 129, 1], [], 1, 4, 2, 128, 16, "bf16"),
    ([700], [], 1, 8, 2, 128, 64, "bf16"),
    ([333, 17, 1, 64], [], 1, 6, 2, 64, 20, "f16"),
    ([31, 32, 33, 127], [], 1, 5, 1, 128, 1, "bf16"),
    ([90, 45], [], 1, 40, 1, 64, 7, "f16"),             # more heads a group than a tile's columns
    ([200, 210, 205], [(0, 3, 192)], 1, 4, 1, 128, 16, "bf16"),
    ([128, 128], [(0, 2, 128)], 1, 4, 1, 64, 16, "f16"),  # nothing of their own
    ([50, 300, 310, 290, 12], [(1, 4, 288)], 1, 8, 2, 128, 32, "bf16"),
    ([130, 140, 150, 60, 70], [(0, 3, 128), (3, 5, 48)], 1, 3, 3, 64, 16, "bf16"),
    ([40, 41, 42, 43], [(0, 2, 0), (2, 4, 40)], 1, 4, 2, 64, 8, "f16"),  # a group that shares nothing
    ([64, 100, 64], [(0, 3, 64)], 5, 8, 2, 64, 16, "bf16"),  # drafts that end in the shared keys
    ([3, 9, 1], [], 4, 4, 1, 128, 16, "bf16"),             # more tokens than keys: rows that see none
]


@pytest.mark.parametrize("case", CASES, ids=[f"n{len(c[0])}_g{len(c[1])}_q{c[2]}_h{c[3]}_{c[4]}_d{c[5]}_p{c[6]}_{c[7]}"
                                             for c in CASES])
def test_paged(case):
    lens, groups, n_q, hq, hkv, d, page, dtype = case
    k, v, table = _batch(lens, None, groups, page, hkv, d, dtype, 1)
    q = torch.randn((len(lens) * n_q, hq, d), device="cuda").to(R.TORCH[dtype])
    starts = None if n_q == 1 else [n_q * i for i in range(len(lens) + 1)]
    _check(q, k, v, table, lens, starts, groups, page, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_ragged_query_rows_and_rows_behind(dtype):
    """0, 1, 7 and 40 newest tokens a sequence; rows behind the last sequence
    stay as they were; head-major q and out."""
    lens, starts = [30, 5, 260, 40], [0, 0, 1, 41, 48]
    k, v, table = _batch(lens, None, [], 16, 2, 128, dtype, 2)
    q = torch.randn((53, 4, 128), device="cuda").to(R.TORCH[dtype])
    got = _check(q, k, v, table, lens, starts, [], 16, dtype, form="heads")
    assert torch.isnan(got[48:].float()).all()


def test_many_chunks_and_repeatable():
    """A long shared prefix split over many workgroups: against the definition
    on a few rows, and the same bits on every run."""
    n, shared, page, hkv, hq, d = 9, 6000, 16, 2, 8, 128
    lens = [shared + 40 * i + 1 for i in range(n)]
    groups = [(0, n, shared)]
    k, v, table = _batch(lens, None, groups, page, hkv, d, "bf16", 3)
    q = torch.randn((n, hq, d), device="cuda").to(torch.bfloat16)
    got = _check(q, k, v, table, lens, None, groups, page, "bf16")
    for _ in range(3):
        assert torch.equal(_run(q, k, v, table, lens, None, groups, d ** -0.5), got)
    # without the groups the same sequences, the same values
    _check(q, k, v, table, lens, None, [], page, "bf16")


@pytest.mark.parametrize("garbage", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_nobody_holds_are_never_seen(garbage):
    lens = [70, 33, 1]
    k, v, table = _batch(lens, None, [], 16, 1, 64, "bf16", 4, garbage=garbage)
    q = torch.randn((3, 4, 64), device="cuda").to(torch.bfloat16)
    _check(q, k, v, table, lens, None, [], 16, "bf16")


def test_pages_outside_the_cache_are_invisible():
    """Entries -1, beyond the cache and far off inside a sequence: its keys are
    not seen, even where page 0 holds NaN; a row of them only gives zeros."""
    lens = [64, 48, 300]
    k, v, table = _batch(lens, None, [(0, 3, 16)], 16, 1, 64, "bf16", 5)
    used = set(table[table >= 0].tolist())
    table[0, 2] = -1
    table[1, :3] = [k.shape[0], 2 ** 31 - 1, -2 ** 31]
    table[2, 5] = k.shape[0] + 7
    for s in (0, 2):
        table[s, 0] = table[1, 0]
    spare = next(p for p in range(k.shape[0]) if p not in used)
    k[spare], v[spare] = float("nan"), float("nan")
    # the spare page becomes page 0, what a missing row's address falls back to
    if spare:
        for z in (k, v):
            z[[0, spare]] = z[[spare, 0]]
        a, b = table == 0, table == spare
        table[a], table[b] = spare, 0
    q = torch.randn((3, 2, 64), device="cuda").to(torch.bfloat16)
    got = _check(q, k, v, table, lens, None, [(0, 3, 16)], 16, "bf16")
    assert (got[1] == 0).all()


def test_lengths_beyond_the_table_and_below_zero():
    lens = [64, 64]
    k, v, table = _batch(lens, None, [], 16, 1, 64, "f16", 6)
    table = table[:, :4]  # rows of exactly 64 keys
    q = torch.randn((2, 1, 64), device="cuda").half()
    got = _run(q, k, v, table, [2 ** 31 - 1, -5], None, [], 0.125)
    ref = _run(q, k, v, table, [64, 0], None, [], 0.125)
    assert torch.equal(got, ref) and (got[1] == 0).all()


def test_large_scores_and_equal_values():
    """Scores far apart and large: the largest key wins; equal values come out
    as they are."""
    lens = [400]
    k, v, table = _batch(lens, None, [], 16, 1, 128, "bf16", 7)
    q = torch.randn((1, 4, 128), device="cuda").to(torch.bfloat16)
    _check(q, k, v, table, lens, None, [], 16, "bf16", scale=30.0)
    v.fill_(3.0)
    assert (_run(q, k, v, table, lens, None, [], 0.1) == 3.0).all()


def test_a_cache_past_4_gib():
    """Pages whose byte offsets pass 2^32."""
    page, hkv, d = 256, 8, 128
    n_pages = (4 << 30) // (page * hkv * d * 2) + 40
    k = torch.empty((n_pages, hkv, page, d), device="cuda", dtype=torch.bfloat16)
    v = torch.empty_like(k)
    table = np.asarray([[n_pages - 1, 3, n_pages - 7], [0, n_pages - 2, -1]])
    for p in (0, 3, n_pages - 1, n_pages - 2, n_pages - 7):
        k[p] = torch.randn((hkv, page, d), device="cuda").to(torch.bfloat16)
        v[p] = torch.randn((hkv, page, d), device="cuda").to(torch.bfloat16)
    lens = [600, 300]
    q = torch.randn((2, hkv, d), device="cuda").to(torch.bfloat16)
    got = _run(q, k, v, table, lens, None, [], d ** -0.5)
    small = [0, 3, n_pages - 7, n_pages - 2, n_pages - 1]
    t2 = np.asarray([[4, 1, 2], [0, 3, -1]])
    ref, info = R.attention(R.f64(q), R.f64(k[small]), R.f64(v[small]), t2, lens, page, [0, 1, 2], d ** -0.5)
    R.check(R.f64(got), ref, R.attention_tol(ref, info, "bf16", d))


def test_captured_call_follows_lengths():
    """Captured once, replayed with other lengths and queries: every replay is
    the eager call's, with eager work of the same stream workspace in between."""
    page, hkv, hq, d, n = 16, 2, 8, 128, 5
    lens = [300, 20, 170, 1, 64]
    k, v, table = _batch([320] * n, None, [(1, 4, 64)], page, hkv, d, "bf16", 8)
    groups = [(1, 4, 64)]
    q = torch.randn((n, hq * d), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    tab, ln = R.i32(table), R.i32(lens)
    gs, gk = R.i32([1, 4]), R.i32([64])
    ws = ea.new_workspace(ea.attention_paged_workspace(R.rel(q), R.pages_rel(k), n, 1))
    rq, rk, rv, ro = R.rel(q), R.pages_rel(k), R.pages_rel(v), R.rel(out)
    call = lambda: ea.attention_paged(rq, rk, rv, ro, scale=0.1, table=tab, lengths=ln, group_start=gs,
                                      group_shared=gk, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        new = [min(320, x + 37 * step) for x in lens]
        ln.copy_(R.i32(new))
        q.copy_(torch.randn_like(q.float()).to(torch.bfloat16))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        eager = _run(q.view(n, hq, d), k, v, table, new, None, groups, 0.1)
        assert torch.equal(out.view(n, hq, d), eager)


def test_two_streams_with_workspaces_of_their_own():
    page, hkv, hq, d, n = 16, 2, 8, 128, 6
    lens = [900, 800, 700, 600, 500, 400]
    k, v, table = _batch(lens, None, [], page, hkv, d, "f16", 9)
    qs = [torch.randn((n, hq, d), device="cuda").half() for _ in range(2)]
    ref = [_run(q, k, v, table, lens, None, [], 0.1).clone() for q in qs]
    tab, ln = R.i32(table), R.i32(lens)
    rk, rv = R.pages_rel(k), R.pages_rel(v)
    outs = [torch.empty((n, hq * d), device="cuda", dtype=torch.float16) for _ in qs]
    rels = [(R.rel(q.view(n, hq * d)), R.rel(o)) for q, o in zip(qs, outs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(5):
        for s, (rq, ro) in zip(streams, rels):
            with torch.cuda.stream(s):
                ea.attention_paged(rq, rk, rv, ro, scale=0.1, table=tab, lengths=ln)
    torch.cuda.synchronize()
    for o, r in zip(outs, ref):
        assert torch.equal(o.view(n, hq, d), r)


WIDE = [
    # lens, groups, n_q, hq, hkv, d, page, dtype: more than 32 columns a tile
    ([200] * 9, [(0, 9, 160)], 1, 8, 2, 128, 16, "bf16"),            # 36 columns
    ([130] * 17, [(0, 17, 128)], 1, 4, 1, 64, 64, "f16"),            # 68
    ([300, 310, 320], [], 40, 4, 1, 128, 16, "bf16"),                # long drafts, 160 columns each
    ([33, 1, 64, 65], [], 20, 4, 2, 64, 7, "f16"),                   # rows that see none, odd pages
    ([700 + 3 * i for i in range(40)], [(0, 40, 640)], 1, 8, 1, 128, 20, "bf16"),  # 320 columns
    ([90 + i for i in range(30)], [(0, 15, 64), (15, 30, 80)], 2, 6, 1, 64, 8, "bf16"),
]


@pytest.mark.parametrize("case", WIDE, ids=[f"n{len(c[0])}_g{len(c[1])}_q{c[2]}_h{c[3]}_{c[4]}_d{c[5]}_p{c[6]}_{c[7]}"
                                            for c in WIDE])
def test_many_columns(case):
    lens, groups, n_q, hq, hkv, d, page, dtype = case
    k, v, table = _batch(lens, None, groups, page, hkv, d, dtype, 21, garbage=float("nan"))
    q = torch.randn((len(lens) * n_q, hq, d), device="cuda").to(R.TORCH[dtype])
    starts = None if n_q == 1 else [n_q * i for i in range(len(lens) + 1)]
    got = _check(q, k, v, table, lens, starts, groups, page, dtype)
    assert torch.equal(got, _run(q, k, v, table, lens, starts, groups, d ** -0.5))


def test_many_columns_with_pages_outside_the_cache():
    lens, groups = [210] * 12, [(0, 12, 128)]
    k, v, table = _batch(lens, None, groups, 16, 1, 128, "bf16", 22, garbage=float("nan"))
    for s in range(12):
        table[s, 3] = -1          # inside the shared keys
        table[s, 10] = k.shape[0]  # and inside the own ones
    q = torch.randn((12, 4, 128), device="cuda").to(torch.bfloat16)
    _check(q, k, v, table, lens, None, groups, 16, "bf16")


def test_the_largest_batch():
    """As many sequences as a call takes: lengths 0 to 6, some with none."""
    n = ea.PAGED_MAX_SEQ - 1
    lens = [i % 7 for i in range(n)]
    k, v, table = _batch(lens, None, [], 4, 1, 64, "bf16", 23)
    q = torch.randn((n, 1, 64), device="cuda").to(torch.bfloat16)
    _check(q, k, v, table, lens, None, [], 4, "bf16")
    groups = [(100, 900, 0)]
    _check(q, k, v, table, lens, None, groups, 4, "bf16")


def test_query_rows_that_do_not_ascend_stay_inside():
    """A bad q_start gives no defined values; the call ends, writes no row
    behind the last and leaves the workspace usable."""
    lens = [100, 200, 300]
    k, v, table = _batch(lens, None, [], 16, 1, 64, "bf16", 24)
    q = torch.randn((8, 4, 64), device="cuda").to(torch.bfloat16)
    good = _run(q, k, v, table, lens, [0, 2, 5, 8], [], 0.1).clone()
    for bad in ([0, 8, 0, 8], [8, 0, 8, 0], [-5, 2 ** 31 - 1, -2 ** 31, 8], [3, 3, 3, 3]):
        out = torch.full((9, 4 * 64), 7.0, device="cuda", dtype=torch.bfloat16)
        _run(q, k, v, table, lens, bad, [], 0.1, out=out[:8])
        assert (out[8] == 7.0).all()
        assert torch.equal(_run(q, k, v, table, lens, [0, 2, 5, 8], [], 0.1), good)


@pytest.mark.parametrize("lens,groups", [([70000], []), ([20000, 3], []), ([30010, 30001, 29990], [(0, 3, 29984)])])
def test_long_walks_of_few_tiles(lens, groups):
    """One key-value head and few sequences: every tile's walk is cut in
    hundreds of parts, whose results all the waves of a workgroup join."""
    k, v, table = _batch(lens, None, groups, 16, 1, 128, "f16", 25)
    q = torch.randn((len(lens), 4, 128), device="cuda").half()
    _check(q, k, v, table, lens, None, groups, 16, "f16")


def test_partitions_of_queries_and_output():
    """Queries in blocks of 3 rows and 2 heads, the last ones shorter; the output
    head-major in blocks of 4 rows."""
    lens, hq, hkv, d, page = [40, 7, 0, 130, 64], 6, 2, 64, 16
    k, v, table = _batch(lens, None, [], page, hkv, d, "bf16", 26)
    q = torch.randn((5, hq, d), device="cuda").to(torch.bfloat16)
    rq = R.blocked(q.view(5, hq * d), [R.splits(5, 3), R.splits(hq * d, 2 * d)])
    out = ea.Relation((1, hq, 5, d), "bf16", [[0, 1], R.splits(hq, 4), R.splits(5, 4), [0, d]])
    out.data.fill_(0xFF)
    ea.attention_paged(rq, R.pages_rel(k), R.pages_rel(v), out, scale=0.2, table=R.i32(table), lengths=R.i32(lens))
    ref, info = R.attention(R.f64(q), R.f64(k), R.f64(v), table, lens, page, list(range(6)), 0.2)
    R.check(R.f64(R.unblocked(out)[0].transpose(0, 1)), ref, R.attention_tol(ref, info, "bf16", d))


@pytest.mark.parametrize("groups", [[], [(0, 3, 48)]])
def test_a_nan_query_is_its_own(groups):
    lens = [60, 50, 90]
    k, v, table = _batch(lens, None, groups, 16, 1, 64, "bf16", 27)
    q = torch.randn((3, 4, 64), device="cuda").to(torch.bfloat16)
    clean = _run(q, k, v, table, lens, None, groups, 0.125).clone()
    q[1, 2, 5] = float("nan")
    got = _run(q, k, v, table, lens, None, groups, 0.125)
    assert torch.isnan(got[1, 2]).all()
    got[1, 2] = clean[1, 2]
    assert torch.equal(got, clean)


HIDDEN = [
    # lens, groups, n_q, hq, hkv, d, dtype, key of sequence 0 (as the last of all the first rows do not see it)
    ([70, 45], [], 3, 4, 2, 128, "bf16", 69),
    ([300, 200], [], 2, 4, 1, 64, "f16", 299),
    ([161, 40], [], 5, 4, 1, 128, "f16", 158),
    ([129, 40], [], 5, 8, 2, 64, "bf16", 126),
    ([90, 200], [], 12, 4, 1, 128, "bf16", 80),
    ([64, 20], [], 12, 8, 2, 64, "f16", 60),
    ([130, 70], [], 30, 4, 1, 128, "f16", 128),
    ([500, 70], [], 30, 4, 1, 64, "bf16", 480),
    ([64, 100, 64], [(0, 3, 64)], 5, 8, 2, 64, "bf16", 62),
    ([64, 100, 80], [(0, 3, 64)], 5, 8, 1, 128, "f16", 61),  # 120 columns
    ([64, 200, 210, 220, 230], [(0, 5, 64)], 5, 8, 1, 128, "bf16", 63),
]


@pytest.mark.parametrize("case", HIDDEN, ids=[f"n{len(c[0])}_g{len(c[1])}_q{c[2]}_h{c[3]}_{c[4]}_d{c[5]}_{c[6]}"
                                              for c in HIDDEN])
def test_what_a_row_does_not_see_may_be_anything(case):
    """A value's infinities and NaN reach the rows that see its key, in their own
    elements, and no other; then its key is NaN too."""
    lens, groups, n_q, hq, hkv, d, dtype, key = case
    page, h, g = 16, hkv - 1, hq // hkv
    k, v, table = _batch(lens, None, groups, page, hkv, d, dtype, 28)
    q = torch.randn((len(lens) * n_q, hq, d), device="cuda").to(R.TORCH[dtype])
    starts = [n_q * i for i in range(len(lens) + 1)]
    at = (table[0, key // page], h, key % page)
    v[at][3], v[at][d // 2], v[at][d - 1] = float("inf"), -float("inf"), float("nan")
    finite = torch.nan_to_num(v.double(), nan=0.0, posinf=0.0, neginf=0.0)
    ref, info = R.attention(R.f64(q), R.f64(k), R.f64(finite), table, lens, page, starts, 0.125)
    tol = R.attention_tol(ref, info, dtype, d)
    sees = np.zeros(len(q), bool)
    for s, n in enumerate(lens):
        for i in range(n_q):
            sees[s * n_q + i] = table[s, key // page] == at[0] and key < n - n_q + i + 1
    assert sees.any() and not sees[:n_q].all()
    heads = slice(h * g, (h + 1) * g)
    for _ in range(2):
        got = R.f64(_run(q, k, v, table, lens, starts, groups, 0.125))
        rows = got[sees][:, heads]
        if not np.isnan(R.f64(k)).any():
            assert (rows[..., 3] == np.inf).all() and (rows[..., d // 2] == -np.inf).all()
            assert np.isnan(rows[..., d - 1]).all()
            rows[..., [3, d // 2, d - 1]] = ref[sees][:, heads][..., [3, d // 2, d - 1]]
        else:
            assert np.isnan(rows).all()
            rows = ref[sees][:, heads]
        got[np.ix_(np.flatnonzero(sees), np.arange(hq)[heads])] = rows
        R.check(got, ref, tol)
        k[at][5] = float("nan")


def test_query_rows_that_do_not_ascend_under_a_group():
    """As without groups: rows of a sequence that are not its group's join no
    part of the group's walk."""
    lens, groups = [100, 200, 300], [(0, 3, 96)]
    k, v, table = _batch(lens, None, groups, 16, 1, 64, "bf16", 24)
    q = torch.randn((8, 4, 64), device="cuda").to(torch.bfloat16)
    good = _run(q, k, v, table, lens, [0, 2, 5, 8], groups, 0.1).clone()
    for bad in ([0, 8, 0, 8], [8, 0, 8, 0], [5, 0, 6, 6], [-5, 2 ** 31 - 1, -2 ** 31, 8], [3, 3, 3, 3]):
        out = torch.full((9, 4 * 64), 7.0, device="cuda", dtype=torch.bfloat16)
        _run(q, k, v, table, lens, bad, groups, 0.1, out=out[:8])
        assert (out[8] == 7.0).all()
        assert torch.equal(_run(q, k, v, table, lens, [0, 2, 5, 8], groups, 0.1), good)
