"""What the softmax weights of attention over pages keep on their way through
the product with V: sums that cancel show every bit that a weight has lost."""
import numpy as np
import pytest
import torch

import decode_ref as R
from paper_2609_03905_amd import ea

pytestmark = pytest.mark.gpu

# A weight is held as two values of the cache's type, the second what the first
# leaves: each rounding is off by at most half a step, so the two by half a step
# of half a step.  The denominator is summed in f32.  In fp16 the largest weight
# of a row is 2^7 or more, so that half the smallest step is 2^-25 / 2^7 of it.
WEIGHT = {"bf16": 2.0 ** -16, "f16": 2.0 ** -22}
SMALLEST = {"bf16": 0.0, "f16": 2.0 ** -32}


def _tol(ref, info, dtype, d):
    a, mag, vmax, n_keys = info
    u = R.HALF[dtype]
    soft = (WEIGHT[dtype] + 2 * (d + 8) * R.F * mag + 64 * R.F) * a + SMALLEST[dtype] * n_keys * vmax
    return u * np.abs(ref) + (1 + u) * soft + R.TINY[dtype]


CASES = [
    # lens, groups, n_q, hq, hkv, d: tiles of 16, 32, 64 and 128 columns, with and without shared keys
    ([2, 3, 5, 9, 17, 40], [], 1, 4, 1, 128),
    ([3, 6, 200], [], 4, 8, 2, 64),
    ([40, 70], [], 12, 4, 1, 128),
    ([33, 90], [], 30, 4, 1, 64),
    ([20, 21, 22], [(0, 3, 16)], 5, 8, 2, 64),
    ([40, 36, 39, 33], [(0, 4, 32)], 5, 8, 1, 128),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", CASES, ids=[f"n{len(c[0])}_g{len(c[1])}_q{c[2]}_h{c[3]}_{c[4]}_d{c[5]}" for c in CASES])
def test_weights_keep_more_than_the_cache_type(case, dtype):
    lens, groups, n_q, hq, hkv, d = case
    page = 4
    rng = np.random.default_rng(5)
    held = [-(-n // page) for n in lens]
    table = np.full((len(lens), max(held)), -1, np.int64)
    ids = list(rng.permutation(sum(held)))
    for s, n in enumerate(held):
        table[s, :n] = [ids.pop() for _ in range(n)]
    for first, last, keys in groups:
        table[first:last, :keys // page] = table[first, :keys // page]
    g = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn((sum(held), hkv, page, d), generator=g, device="cuda").to(R.TORCH[dtype]) for _ in range(2))
    q = torch.randn((len(lens) * n_q, hq, d), generator=g, device="cuda").to(R.TORCH[dtype])
    out = torch.empty((len(q), hq * d), device="cuda", dtype=R.TORCH[dtype])
    starts = [n_q * i for i in range(len(lens) + 1)]
    kw = {"group_start": R.i32([groups[0][0], groups[0][1]]), "group_shared": R.i32([groups[0][2]])} if groups else {}
    ea.attention_paged(R.rel(q.view(len(q), -1)), R.pages_rel(k), R.pages_rel(v), R.rel(out), scale=d ** -0.5,
                       table=R.i32(table), lengths=R.i32(lens), q_start=R.i32(starts), **kw)
    ref, info = R.attention(R.f64(q), R.f64(k), R.f64(v), table, lens, page, starts, d ** -0.5)
    R.check(R.f64(out.view(q.shape)), ref, _tol(ref, info, dtype, d))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n_q,hq,d", [(1, 4, 128), (3, 8, 64), (12, 4, 128), (30, 4, 64)])
def test_an_infinite_value_that_every_row_sees(n_q, hq, d, dtype):
    """Equal weights, held without a rest: infinities come out as they are, the
    other elements' means beside them."""
    n, page = 256 + n_q, 16
    k = torch.randn((20, 1, page, d), device="cuda").to(R.TORCH[dtype])
    v = torch.ones_like(k)
    v[2, 0, 3, 5], v[4, 0, 7, 6], v[1, 0, 0, d - 1] = float("inf"), -float("inf"), float("nan")
    q = torch.zeros((n_q, hq * d), device="cuda", dtype=R.TORCH[dtype])
    out = torch.empty_like(q)
    ea.attention_paged(R.rel(q), R.pages_rel(k), R.pages_rel(v), R.rel(out), scale=1.0,
                       table=R.i32([list(range(20))]), lengths=R.i32([n]), q_start=R.i32([0, n_q]))
    got = R.f64(out).reshape(n_q, hq, d)
    assert (got[..., 5] == np.inf).all() and (got[..., 6] == -np.inf).all() and np.isnan(got[..., d - 1]).all()
    assert (got[..., [i for i in range(d) if i not in (5, 6, d - 1)]] == 1.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("n,n_q,hq,d,shared", [(64, 1, 4, 128, 0), (900, 2, 8, 64, 0), (320, 12, 4, 128, 0),
                                               (200, 30, 4, 64, 0), (320, 8, 8, 128, 256)])
def test_many_small_weights_beside_large_ones(n, n_q, hq, d, shared, dtype):
    """Every 32nd key's score is 26 octaves above the others', whose values make
    the sum: weights of 2^-26 count, below what one fp16 number holds beside 1."""
    page, seqs = 16, 2
    held = -(-n // page)
    key = torch.arange(held * page, device="cuda").view(held, 1, page, 1)
    k = torch.zeros((held, 1, page, d), device="cuda")
    k[..., 0:1] = 26.0 * (key % 32 == 0)
    v = torch.where(key % 32 == 0, 0.0, 48000.0 + 1024 * (key % 7)).expand(-1, -1, -1, d).contiguous()
    k, v = k.to(R.TORCH[dtype]), v.to(R.TORCH[dtype])
    q = torch.zeros((seqs * n_q, hq, d), device="cuda", dtype=R.TORCH[dtype])
    q[..., 0] = 1.0
    table, starts = np.arange(held)[None].repeat(seqs, 0), [0, n_q, 2 * n_q]
    out = torch.empty((len(q), hq * d), device="cuda", dtype=R.TORCH[dtype])
    kw = {"group_start": R.i32([0, seqs]), "group_shared": R.i32([shared])} if shared else {}
    ea.attention_paged(R.rel(q.view(len(q), -1)), R.pages_rel(k), R.pages_rel(v), R.rel(out), scale=float(np.log(2)),
                       table=R.i32(table), lengths=R.i32([n] * seqs), q_start=R.i32(starts), **kw)
    scale = float(np.float32(np.log(2)))
    ref, info = R.attention(R.f64(q), R.f64(k), R.f64(v), table, [n] * seqs, page, starts, scale)
    assert ref.min() > 0.01
    R.check(R.f64(out.view(q.shape)), ref, _tol(ref, info, dtype, d))


LONG = [
    # lens, groups, n_q, hq, hkv, d
    ([70000], [], 1, 4, 1, 128),                                       # parts joined by the waves of a workgroup
    ([20000, 3], [], 1, 4, 1, 128),
    ([30010, 30001, 29990], [(0, 3, 29984)], 1, 4, 1, 128),            # shared and own parts
    ([9000 + i for i in range(12)], [(0, 12, 8960)], 1, 8, 1, 64),
    ([131072, 5, 900, 1, 70, 300, 64, 2], [], 1, 4, 1, 128),
    ([131072] + [3] * 299, [], 1, 4, 1, 128),                          # the last to arrive joins hundreds of parts
    ([32000 - 100 * i for i in range(8)], [], 1, 4, 1, 64),
    ([40000, 17], [], 12, 4, 1, 128),                                  # 48 columns a sequence
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", LONG, ids=[f"n{len(c[0])}_{c[0][0]}_g{len(c[1])}_q{c[2]}_d{c[5]}" for c in LONG])
def test_every_stretch_of_a_long_walk_counts(case, dtype):
    """Each 64 keys add to an element of their own (one of d, in turn) with a
    weight of 1, 2 or 4: a stretch that is lost, counted twice or joined with
    another's maximum changes its element by far more than the tolerance."""
    lens, groups, n_q, hq, hkv, d = case
    page, longest = 64, max(lens)
    held = -(-longest // page)
    rng = np.random.default_rng(9)
    octave = rng.integers(0, 3, held)
    octave[0], octave[-1] = 2, 2
    # every sequence reads the same pages, in an order of their own
    order = rng.permutation(held)
    place = torch.from_numpy(order).cuda()
    k = torch.zeros((held, hkv, page, d), device="cuda")
    v = torch.zeros_like(k)
    k[place, :, :, 0] = torch.from_numpy(octave).cuda().float()[:, None, None]
    v[place, :, :, torch.arange(held, device="cuda") % d] = 1.0
    k, v = k.to(R.TORCH[dtype]), v.to(R.TORCH[dtype])
    q = torch.zeros((len(lens) * n_q, hq, d), device="cuda", dtype=R.TORCH[dtype])
    q[..., 0] = 1.0
    starts = [n_q * i for i in range(len(lens) + 1)]
    table = order[None].repeat(len(lens), 0)
    kw = {"group_start": R.i32([groups[0][0], groups[0][1]]), "group_shared": R.i32([groups[0][2]])} if groups else {}
    scale = float(np.float32(np.log(2)))
    outs = []
    for _ in range(3):
        out = torch.full((len(q), hq * d), float("nan"), device="cuda", dtype=R.TORCH[dtype])
        ea.attention_paged(R.rel(q.view(len(q), -1)), R.pages_rel(k), R.pages_rel(v), R.rel(out), scale=scale,
                           table=R.i32(table), lengths=R.i32(lens), q_start=R.i32(starts), **kw)
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    got = R.f64(outs[0].view(q.shape))
    for s, n in enumerate(lens):
        for i in range(n_q):
            seen = max(0, n - n_q + i + 1)
            keys = np.clip(seen - page * np.arange(held), 0, page)   # of each stretch
            add = keys * np.exp(scale * octave)
            ref = np.zeros(d)
            np.add.at(ref, np.arange(held) % d, add / max(add.sum(), 1e-300))
            # A is the value itself, one key's score is at most scale * 2
            info = (ref, 2 * scale, 1.0, seen)
            tol = _tol(ref, info, dtype, d)
            if seen > page * d:  # the smallest whole stretch changes its element by four tolerances and more
                assert (add[keys == page] / add.sum() > 4 * tol[np.flatnonzero(keys == page) % d]).all()
            R.check(got[s * n_q + i], np.broadcast_to(ref, (hq, d)), tol)
