"""Head rows normed, rotated and moved (ea.heads) and their gradient against
the 64-bit definition, over types, widths, partitions, positions and pages."""
import numpy as np
import pytest
import torch

import decode_ref as R
from paper_2609_03905_amd import ea

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _freq(rotary):
    n = rotary // 2
    return (10000.0 ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))).float().cuda()


def _inputs(t, hq, hkv, d, rotary, dtype, norm, far, seed, wdtype=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = R.TORCH[dtype]
    x = torch.randn((t, (hq + 2 * hkv) * d), generator=g, device="cuda").to(dt)
    w = [(1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(R.TORCH[wdtype or dtype]) if norm else None
         for _ in range(2)]
    pos = torch.randint(0, far, (t,), generator=g, device="cuda", dtype=torch.int32) if far else None
    return x, w[0], w[1], _freq(rotary), pos


def _np(t):
    return None if t is None else R.f64(t)


def _relw(w):
    return None if w is None else R.rel(w)


CASES = [
    # t, hq, hkv, d, rotary, interleaved, norm, dtype, far
    (1, 1, 1, 8, 8, False, True, "bf16", 0),
    (1, 4, 1, 128, 128, False, True, "bf16", 1 << 30),
    (7, 5, 3, 128, 128, False, True, "f16", 1000),
    (33, 4, 4, 64, 64, False, False, "f32", 1 << 20),
    (65, 8, 2, 96, 96, False, True, "bf16", 131072),
    (19, 3, 1, 80, 32, False, True, "f32", 4096),
    (19, 3, 1, 80, 40, False, True, "f16", 4096),   # rotary / 2 no multiple of 8
    (40, 2, 2, 256, 64, True, True, "bf16", 4096),
    (5, 6, 2, 64, 6, True, True, "f32", 4096),      # rotation ends inside a lane's eight
    (5, 6, 2, 64, 6, False, True, "f32", 4096),
    (11, 2, 1, 512, 512, False, True, "bf16", 100),
    (11, 2, 1, 264, 0, False, True, "f16", 0),      # no rotation
    (300, 12, 12, 72, 72, False, True, "bf16", 0),  # the row's index
    (23, 3, 2, 72, 16, False, True, "f32", 300),    # an odd number of eights stays unrotated
    (23, 9, 3, 88, 64, False, False, "f16", 300),
    (2000, 6, 1, 64, 64, True, True, "bf16", 300),
]


@pytest.mark.parametrize("case", CASES, ids=[f"t{c[0]}_h{c[1]}_{c[2]}_d{c[3]}_r{c[4]}_{c[7]}" for c in CASES])
@pytest.mark.parametrize("form", ["tokens", "heads"])
def test_heads(case, form):
    t, hq, hkv, d, rotary, inter, norm, dtype, far = case
    x, wq, wk, freq, pos = _inputs(t, hq, hkv, d, rotary, dtype, norm, far, 1)
    dt = R.TORCH[dtype]
    shape = (lambda h: (t, h * d)) if form == "tokens" else (lambda h: (h, t, d))
    q, k, v = (torch.full(shape(h), float("nan"), device="cuda", dtype=dt) for h in (hq, hkv, hkv))
    ea.heads(R.rel(x), R.rel(q), R.rel(k), R.rel(v), d_head=d, wq=_relw(wq), wk=_relw(wk), eps=EPS,
             inv_freq=freq if rotary else None, interleaved=inter, positions=pos)
    p = np.arange(t) if pos is None else pos.cpu().numpy()
    ref, err = R.heads(R.f64(x), hq, hkv, d, _np(wq), _np(wk), EPS, R.f64(freq), inter, p)
    for got, r, e, what in zip((q, k, v), ref, err, "qkv"):
        got = R.f64(got).reshape(t, -1, d) if form == "tokens" else R.f64(got).transpose(1, 0, 2)
        R.check(got, r, R.heads_tol(r, e, dtype), what)
    assert torch.equal(v.transpose(0, 1).reshape(t, -1) if form == "heads" else v, x[:, (hq + hkv) * d:])


@pytest.mark.parametrize("dtype,t,hq,hkv,d,tb,hb", [("bf16", 70, 8, 2, 128, 32, 4), ("f16", 131, 4, 3, 40, 64, 3),
                                                    ("f32", 9, 6, 2, 8, 4, 4)])
def test_heads_partitions(dtype, t, hq, hkv, d, tb, hb):
    """Blocks on both sides, the last ones shorter, and rank-4 outputs as the
    block chain's attention takes them; norm weights of another type."""
    x, wq, wk, freq, pos = _inputs(t, hq, hkv, d, d, dtype, True, 500, 2, wdtype="f32")
    X = R.blocked(x, [R.splits(t, tb), R.splits(x.shape[1], hb * d)])
    dt = R.TORCH[dtype]
    mk = lambda shape, part: ea.Relation(shape, dtype, part)
    q = mk((1, hq, t, d), [[0, 1], R.splits(hq, 1), R.splits(t, tb), [0, d]])
    k = mk((hkv, t, d), [R.splits(hkv, 2), R.splits(t, tb), [0, d]])
    v = mk((t, hkv * d), [R.splits(t, tb + 1), R.splits(hkv * d, 2 * d)])
    for r in (q, k, v):
        r.data.fill_(0xFF)
    ea.heads(X, q, k, v, d_head=d, wq=R.rel(wq), wk=R.rel(wk), eps=EPS, inv_freq=freq, positions=pos)
    ref, err = R.heads(R.f64(x), hq, hkv, d, _np(wq), _np(wk), EPS, R.f64(freq), False, pos.cpu().numpy())
    got = [R.unblocked(q)[0].transpose(0, 1), R.unblocked(k).transpose(0, 1), R.unblocked(v).reshape(t, hkv, d)]
    for g, r, e in zip(got, ref, err):
        R.check(R.f64(g), r, R.heads_tol(r, e, dtype))
    assert got[0].dtype == dt


@pytest.mark.parametrize("page", [1, 5, 16, 64])
def test_heads_into_pages(page):
    t, hq, hkv, d, n_pages = 37, 4, 2, 64, 80 // page + 2
    x, wq, wk, freq, pos = _inputs(t, hq, hkv, d, d, "bf16", True, 9000, 3)
    g = torch.Generator().manual_seed(4)
    slots = torch.randperm(n_pages * page, generator=g)[:t].int()
    slots[3], slots[11], slots[20] = -1, n_pages * page, -2 ** 31  # nowhere
    kc, vc = (torch.randn((n_pages, hkv, page, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    k0, v0 = kc.clone(), vc.clone()
    q = torch.empty((t, hq * d), device="cuda", dtype=torch.bfloat16)
    ea.heads(R.rel(x), R.rel(q), R.pages_rel(kc), R.pages_rel(vc), d_head=d, wq=R.rel(wq), wk=R.rel(wk), eps=EPS,
             inv_freq=freq, positions=pos, slots=slots.cuda())
    ref, err = R.heads(R.f64(x), hq, hkv, d, _np(wq), _np(wk), EPS, R.f64(freq), False, pos.cpu().numpy())
    R.check(R.f64(q).reshape(t, hq, d), ref[0], R.heads_tol(ref[0], err[0], "bf16"))
    want_k, want_v, tol_k = R.f64(k0), R.f64(v0), np.zeros(k0.shape)
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < n_pages * page:
            want_k[s // page, :, s % page] = ref[1][i]
            want_v[s // page, :, s % page] = ref[2][i]
            tol_k[s // page, :, s % page] = R.heads_tol(ref[1][i], err[1][i], "bf16")
    R.check(R.f64(kc), want_k, tol_k)  # rows that no slot names stay to the bit
    R.check(R.f64(vc), want_v, np.zeros(v0.shape))


def test_heads_rows_are_independent():
    """A NaN in one head row, an infinity in another: only those rows see it."""
    t, hq, hkv, d = 6, 3, 1, 64
    x, wq, wk, freq, pos = _inputs(t, hq, hkv, d, 6, "f32", True, 50, 5)
    clean, bad = [torch.empty((t, h * d), device="cuda") for h in (hq, hkv, hkv)], None
    run = lambda src, o: ea.heads(R.rel(src), *[R.rel(z) for z in o], d_head=d, wq=R.rel(wq), wk=R.rel(wk), eps=EPS,
                                  inv_freq=freq, interleaved=True, positions=pos)
    run(x, clean)
    y = x.clone()
    y[2, 3] = float("nan")
    y[4, d + 7] = float("inf")
    bad = [torch.empty_like(z) for z in clean]
    run(y, bad)
    same = (bad[0] == clean[0]).view(t, hq, d).all(-1).cpu()
    assert same.sum() == t * hq - 2 and not same[2, 0] and not same[4, 1]
    assert torch.equal(bad[1], clean[1]) and torch.equal(bad[2], clean[2])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [16, 18])
def test_elements_past_the_rotated_part_stay(rotary, interleaved):
    """Without a norm an infinity among them reaches no other element."""
    t, d = 3, 64
    x, _, _, freq, _ = _inputs(t, 1, 1, d, rotary, "f32", False, 0, 12)
    x[1, 40], x[1, rotary] = float("inf"), float("nan")
    out = [torch.empty((t, d), device="cuda") for _ in range(3)]
    ea.heads(R.rel(x), *[R.rel(o) for o in out], d_head=d, inv_freq=freq, interleaved=interleaved)
    assert torch.equal(out[0][1, rotary + 1:], x[1, rotary + 1:d]) and torch.isfinite(out[0][1, :rotary]).all()


GRAD = [
    (1, 1, 1, 8, 8, False, True, "f32", 0),
    (50, 4, 2, 128, 128, False, True, "bf16", 5000),
    (33, 3, 3, 96, 48, False, True, "f32", 5000),
    (20, 2, 1, 80, 40, False, True, "f16", 100),
    (70, 5, 1, 64, 10, True, True, "f32", 100),
    (9, 2, 2, 256, 256, True, False, "f32", 100),
    (9, 2, 1, 512, 0, False, True, "bf16", 0),
    (23, 3, 2, 72, 16, False, True, "f32", 300),
    (300, 7, 3, 40, 40, True, True, "f16", 300),
]


@pytest.mark.parametrize("case", GRAD, ids=[f"t{c[0]}_h{c[1]}_{c[2]}_d{c[3]}_r{c[4]}_{c[7]}" for c in GRAD])
def test_heads_backward(case):
    t, hq, hkv, d, rotary, inter, norm, dtype, far = case
    x, wq, wk, freq, pos = _inputs(t, hq, hkv, d, rotary, dtype, norm, far, 6)
    g = torch.Generator(device="cuda").manual_seed(7)
    dt = R.TORCH[dtype]
    dq, dk, dv = (torch.randn((h, t, d), generator=g, device="cuda").to(dt) for h in (hq, hkv, hkv))
    part = [R.splits(t, 16), R.splits(x.shape[1], d)]
    dx = ea.Relation(x.shape, dtype, part)
    dx.data.fill_(0xFF)
    dwq, dwk = (torch.full((d,), float("nan"), device="cuda") for _ in range(2))
    ea.heads_backward(R.blocked(x, part), R.rel(dq), R.rel(dk), R.rel(dv), dx, d_head=d, wq=_relw(wq), wk=_relw(wk),
                      dwq=R.rel(dwq) if norm else None, dwk=R.rel(dwk) if norm else None, eps=EPS,
                      inv_freq=freq if rotary else None, interleaved=inter, positions=pos)
    p = np.arange(t) if pos is None else pos.cpu().numpy()
    tm = lambda z: R.f64(z).transpose(1, 0, 2)
    ref, scale, dws = R.heads_grad(R.f64(x), tm(dq), tm(dk), tm(dv), hq, hkv, d, _np(wq), _np(wk), EPS, R.f64(freq),
                                   inter, p)
    # dx: the forward's 32 steps in n and in g, and the mean of s n over the row
    # (14 steps) with its few products: 96
    R.check(R.f64(R.unblocked(dx)), ref, R.HALF[dtype] * np.abs(ref) + 1.01 * 96 * R.F * scale + R.TINY[dtype], "dx")
    if norm:  # a term's 64 steps; sums of fewer than 64 terms a lane, then of lanes and workgroups
        R.check(R.f64(dwq), dws[0], 160 * R.F * dws[1], "dwq")
        R.check(R.f64(dwk), dws[2], 160 * R.F * dws[3], "dwk")


def test_heads_backward_against_differences():
    """The gradient of sum(y c) along one direction of x and of the weights,
    against differences of the 64-bit forward."""
    t, hq, hkv, d = 3, 2, 1, 64
    x, wq, wk, freq, pos = _inputs(t, hq, hkv, d, d, "f32", True, 50, 8)
    g = torch.Generator(device="cuda").manual_seed(9)
    cq, ck, cv = (torch.randn((t, h * d), generator=g, device="cuda") for h in (hq, hkv, hkv))
    dx, dwq, dwk = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    ea.heads_backward(R.rel(x), R.rel(cq), R.rel(ck), R.rel(cv), R.rel(dx), d_head=d, wq=R.rel(wq), wk=R.rel(wk),
                      dwq=R.rel(dwq), dwk=R.rel(dwk), eps=EPS, inv_freq=freq, positions=pos)
    rng = np.random.default_rng(10)
    ux, uq, uk = rng.standard_normal(x.shape), rng.standard_normal(d), rng.standard_normal(d)

    def value(h):
        y, _ = R.heads(R.f64(x) + h * ux, hq, hkv, d, R.f64(wq) + h * uq, R.f64(wk) + h * uk, EPS, R.f64(freq), False,
                       pos.cpu().numpy())
        return sum((a * R.f64(b).reshape(a.shape)).sum() for a, b in zip(y, (cq, ck, cv)))

    slope = (value(1e-5) - value(-1e-5)) / 2e-5
    got = (R.f64(dx) * ux).sum() + (R.f64(dwq) * uq).sum() + (R.f64(dwk) * uk).sum()
    # differences: curvature of order one over 1e-10; the sum's f32 terms
    size = (np.abs(R.f64(dx)) * np.abs(ux)).sum() + (np.abs(R.f64(dwq) * uq)).sum() + (np.abs(R.f64(dwk) * uk)).sum()
    assert abs(slope - got) <= 1e-6 * size


def test_heads_backward_repeats_to_the_bit():
    t, hq, hkv, d = 2500, 8, 2, 128
    x, wq, wk, freq, pos = _inputs(t, hq, hkv, d, d, "bf16", True, 5000, 11)
    dq, dk, dv = (torch.randn((t, h * d), device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    out = []
    for _ in range(3):
        dx, dwq, dwk = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        ea.heads_backward(R.rel(x), R.rel(dq), R.rel(dk), R.rel(dv), R.rel(dx), d_head=d, wq=R.rel(wq), wk=R.rel(wk),
                          dwq=R.rel(dwq), dwk=R.rel(dwk), eps=EPS, inv_freq=freq, positions=pos)
        out.append((dx.clone(), dwq.clone(), dwk.clone()))
    for o in out[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, out[0]))


def test_heads_into_padded_pages_on_another_stream():
    """Pages of 240 bytes at 256-byte multiples, the call on a stream of its own."""
    t, hq, hkv, d, page, n_pages = 10, 2, 1, 40, 3, 5
    x, wq, wk, freq, pos = _inputs(t, hq, hkv, d, d, "f16", True, 90, 13)
    slots = torch.tensor([14, 0, 3, 7, -1, 8, 2, 13, 5, 10], dtype=torch.int32, device="cuda")
    kc, vc = (R.pages_rel(torch.zeros((n_pages, hkv, page, d), device="cuda", dtype=torch.float16)) for _ in range(2))
    q = torch.empty((t, hq * d), device="cuda", dtype=torch.float16)
    args = (R.rel(x), R.rel(q), kc, vc)
    kw = dict(d_head=d, wq=R.rel(wq), wk=R.rel(wk), eps=EPS, inv_freq=freq, positions=pos, slots=slots)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ea.heads(*args, stream=s, **kw)
    s.synchronize()
    ref, err = R.heads(R.f64(x), hq, hkv, d, _np(wq), _np(wk), EPS, R.f64(freq), False, pos.cpu().numpy())
    R.check(R.f64(q).reshape(t, hq, d), ref[0], R.heads_tol(ref[0], err[0], "f16"))
    k, v = R.f64(R.unblocked(kc)), R.f64(R.unblocked(vc))
    for i, s in enumerate(slots.tolist()):
        if s >= 0:
            R.check(k[s // page, :, s % page], ref[1][i], R.heads_tol(ref[1][i], err[1][i], "f16"))
            assert np.array_equal(v[s // page, :, s % page], ref[2][i])
    assert not k[4, 0, 0].any() and not k[0, 0, 1].any()  # rows that no slot names


def test_heads_rows_past_4_gib():
    """The last rows of an activation whose offsets pass 2^32."""
    t, hq, hkv, d = 360001, 32, 8, 128
    x = torch.empty((t, (hq + 2 * hkv) * d), device="cuda", dtype=torch.bfloat16)
    assert x.numel() * 2 > 1 << 32
    rows = [0, 174762, 174763, 349525, 349526, t - 1]
    x[rows] = torch.randn((len(rows), x.shape[1]), device="cuda").to(torch.bfloat16)
    freq = _freq(d)
    q, k, v = (torch.empty((t, h * d), device="cuda", dtype=torch.bfloat16) for h in (hq, hkv, hkv))
    ea.heads(R.rel(x), R.rel(q), R.rel(k), R.rel(v), d_head=d, inv_freq=freq)
    ref, err = R.heads(R.f64(x[rows]), hq, hkv, d, None, None, 0.0, R.f64(freq), False, np.asarray(rows))
    for got, r, e in zip((q, k, v), ref, err):
        R.check(R.f64(got[rows]).reshape(len(rows), -1, d), r, R.heads_tol(r, e, "bf16"))


def test_weights_and_their_gradients_of_other_types():
    t, hq, hkv, d = 30, 4, 2, 64
    x, _, _, freq, pos = _inputs(t, hq, hkv, d, d, "bf16", True, 50, 14)
    g = torch.Generator(device="cuda").manual_seed(15)
    wq, wk = torch.randn(d, generator=g, device="cuda").half(), torch.randn(d, generator=g, device="cuda")
    dq, dk, dv = (torch.randn((t, h * d), generator=g, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    dx, dwq = torch.empty_like(x), torch.empty(d, device="cuda", dtype=torch.bfloat16)
    # the keys' weight gradient is not wanted
    ea.heads_backward(R.rel(x), R.rel(dq), R.rel(dk), R.rel(dv), R.rel(dx), d_head=d, wq=R.rel(wq), wk=R.rel(wk),
                      dwq=R.rel(dwq), eps=EPS, inv_freq=freq, positions=pos)
    tm = lambda z: R.f64(z).reshape(t, -1, d)
    ref, scale, dws = R.heads_grad(R.f64(x), tm(dq), tm(dk), tm(dv), hq, hkv, d, R.f64(wq), R.f64(wk), EPS,
                                   R.f64(freq), False, pos.cpu().numpy())
    R.check(R.f64(dx), ref, R.HALF["bf16"] * np.abs(ref) + 1.01 * 96 * R.F * scale)
    R.check(R.f64(dwq), dws[0], R.HALF["bf16"] * np.abs(dws[0]) + 1.01 * 160 * R.F * dws[1])


MANY = [
    # more tokens than a launch has waves (768 workgroups of 4 in 16 bits, 512 in
    # f32), so that a wave goes on to others; the last round is partly filled
    (3500, 2, 1, 64, 64, False, True, "bf16", 5000),
    (6201, 3, 1, 128, 128, False, True, "f16", 5000),
    (4100, 2, 1, 80, 40, False, True, "f32", 5000),    # rotary / 2 no multiple of 8
    (2500, 4, 2, 64, 32, True, True, "f32", 0),
    (3300, 1, 1, 96, 96, True, True, "bf16", 0),
    (3100, 1, 1, 512, 512, False, True, "bf16", 5000),
]


@pytest.mark.parametrize("case", MANY, ids=[f"t{c[0]}_h{c[1]}_{c[2]}_d{c[3]}_r{c[4]}_{c[7]}" for c in MANY])
def test_heads_backward_over_many_tokens(case):
    test_heads_backward(case)


@pytest.mark.parametrize("form", ["tokens", "heads"])
@pytest.mark.parametrize("case", MANY[:2] + MANY[3:5], ids=[f"t{c[0]}_d{c[3]}_{c[7]}" for c in MANY[:2] + MANY[3:5]])
def test_heads_over_many_tokens(case, form):
    test_heads(case, form)


def test_heads_over_more_rows_than_a_launch_holds():
    """Past 2^20 workgroups of four rows the first waves go round again."""
    t, hq, hkv, d = (1 << 22) + 70003, 1, 1, 8
    g = torch.Generator(device="cuda").manual_seed(16)
    x = torch.randn((t, 3 * d), generator=g, device="cuda").to(torch.bfloat16)
    wq, wk = (torch.randn(d, generator=g, device="cuda") for _ in range(2))
    freq = _freq(d)
    q, k, v = (torch.full((t, d), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(3))
    ea.heads(R.rel(x), R.rel(q), R.rel(k), R.rel(v), d_head=d, wq=R.rel(wq), wk=R.rel(wk), eps=EPS, inv_freq=freq)
    assert torch.equal(v, x[:, 2 * d:]) and torch.isfinite(q).all() and torch.isfinite(k).all()
    rows = np.r_[0:40, (1 << 22) - 40:(1 << 22) + 40, t - 40:t]
    ref, err = R.heads(R.f64(x[rows]), hq, hkv, d, R.f64(wq), R.f64(wk), EPS, R.f64(freq), False, rows)
    for got, r, e in zip((q, k), ref, err):
        R.check(R.f64(got[rows]).reshape(len(rows), 1, d), r, R.heads_tol(r, e, "bf16"))
