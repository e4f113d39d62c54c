"""What the calls on a cache in 8 bits refuse, host only: every check precedes HIP."""
import ctypes

import numpy as np
import pytest
import torch

ea = pytest.importorskip("paper_2609_03905_amd")
from paper_2609_03905_amd import ea as E  # noqa: E402
from test_decode_cpu import cache, fake, heads, paged  # noqa: E402
import cache8_ref as C  # noqa: E402

OK, ARG, DTYPE, CAPACITY, UNSUPPORTED = 0, -1, -2, -4, -7
NODATA = object()


def scales(pages=30, h=2, n=4, dtype="f32", part=None):
    return fake([pages, h, n], dtype, part)


def bare(shape, dtype, part=None):
    return ea.Relation(shape, dtype, part or E.whole_partition(shape), allocate=False)


def rows(call, **change):
    a = dict(xk=fake([9, 2 * 64]), xv=fake([2, 9, 64]), k=cache(30, 2, 16, 64, "e4m3"), v=cache(30, 2, 16, 64, "e4m3"),
             ks=scales(), vs=scales(), n_seq=3, stride=5, start=256, lengths=512, table=1024)
    a.update({n: v() if callable(v) else v for n, v in change.items()})
    b = E._PageRows(a["n_seq"], a["stride"], a["start"], a["lengths"], a["table"])
    h = lambda r: None if r is None else r._h
    order = ("xk", "xv", "k", "v", "ks", "vs") if call == "write" else ("k", "v", "ks", "vs", "xk", "xv")
    return getattr(ea.lib(), "ea_pages_" + call)(*[h(a[x]) for x in order], None if a.get("no_rows") else ctypes.byref(b),
                                                 None)


@pytest.mark.parametrize("call", ["write", "read"])
@pytest.mark.parametrize("code,change", [
    (ARG, dict(no_rows=True)), (ARG, dict(xk=None)), (ARG, dict(xv=None)), (ARG, dict(k=None)), (ARG, dict(v=None)),
    (ARG, dict(ks=None)), (ARG, dict(vs=None)),
    (ARG, dict(xk=lambda: bare([9, 128], "bf16"))), (ARG, dict(ks=lambda: bare([30, 2, 4], "f32"))),
    (ARG, dict(n_seq=0)), (ARG, dict(stride=0)), (UNSUPPORTED, dict(n_seq=2049)), (UNSUPPORTED, dict(stride=2 ** 27)),
    (ARG, dict(lengths=None)), (ARG, dict(table=None)), (ARG, dict(n_seq=10, start=None)),
    (DTYPE, dict(k=lambda: cache(30, 2, 16, 64), v=lambda: cache(30, 2, 16, 64))),   # not in 8 bits
    (DTYPE, dict(v=lambda: cache(30, 2, 16, 64, "e5m2"))),
    (DTYPE, dict(xv=lambda: fake([9, 128], "f16"))),
    (DTYPE, dict(xk=lambda: fake([9, 128], "e4m3"), xv=lambda: fake([9, 128], "e4m3"))),
    (DTYPE, dict(ks=lambda: scales(dtype="bf16"))),
    (ARG, dict(v=lambda: cache(31, 2, 16, 64, "e4m3"))),
    (UNSUPPORTED, dict(k=lambda: fake([30, 2, 16, 64], "e4m3"))),                    # a block that is not one page
    (ARG, dict(ks=lambda: scales(pages=31))), (ARG, dict(ks=lambda: scales(h=1))), (ARG, dict(ks=lambda: scales(n=3))),
    (ARG, dict(ks=lambda: scales(n=32))), (ARG, dict(vs=lambda: scales(n=8))), (ARG, dict(ks=lambda: fake([30, 8], "f32"))),
    (UNSUPPORTED, dict(ks=lambda: scales(part=[[0, 15, 30], [0, 2], [0, 4]]))),
    (UNSUPPORTED, dict(k=lambda: cache(30, 2, 16, 8, "e4m3"), v=lambda: cache(30, 2, 16, 8, "e4m3"))),
    (UNSUPPORTED, dict(k=lambda: cache(30, 2, 16, 24, "e4m3"), v=lambda: cache(30, 2, 16, 24, "e4m3"))),
    (UNSUPPORTED, dict(k=lambda: cache(30, 2, 16, 528, "e4m3"), v=lambda: cache(30, 2, 16, 528, "e4m3"))),
    (ARG, dict(xk=lambda: fake([9, 64]))), (ARG, dict(xk=lambda: fake([8, 128]))), (ARG, dict(xv=lambda: fake([9, 100]))),
    (UNSUPPORTED, dict(xk=lambda: fake([9, 128], "bf16", [[0, 9], [0, 32, 128]]))),
])
def test_rows_refusals(call, code, change):
    assert rows(call, **change) == code, ea.lib().ea_last_error()


def test_rows_slots():
    """Slots lie under no output."""
    xk, xv = (_at(bare([9, 128], "bf16"), BASE + i * (1 << 20)) for i in range(2))
    part = [range(31), [0, 2], [0, 16], [0, 64]]
    k, v = (_at(bare([30, 2, 16, 64], "e4m3", part), BASE + i * (1 << 20)) for i in (2, 3))
    ks, vs = (_at(bare([30, 2, 4], "f32"), BASE + i * (1 << 20)) for i in (4, 5))
    for call, rels, outs in (("write", (xk, xv, k, v, ks, vs), (k, v, ks, vs)), ("read", (k, v, ks, vs, xk, xv), (xk, xv))):
        for o in outs:
            at = BASE + (xk, xv, k, v, ks, vs).index(o) * (1 << 20)
            b = E._PageRows(3, 5, 256, 512, 1024, at + o.nbytes - 4)
            assert getattr(ea.lib(), "ea_pages_" + call)(*[r._h for r in rels], ctypes.byref(b), None) == ARG
            assert b"slots" in ea.lib().ea_last_error()


@pytest.mark.parametrize("call", ["write", "read"])
def test_rows_of_more_elements_than_are_counted(call):
    """(rows of 2^26 elements; and one head less, whose batch is then looked at)"""
    for h, want, change in ((2 ** 20, UNSUPPORTED, {}), (2 ** 20 - 1, ARG, dict(table=None))):
        part = [[0, 1], [0, h], [0, 1], [0, 64]]
        got = rows(call, xk=_at(bare([3, h * 64], "bf16"), BASE), xv=_at(bare([3, h * 64], "bf16"), BASE + (1 << 32)),
                   k=_at(bare([1, h, 1, 64], "e4m3", part), BASE + (2 << 32)),
                   v=_at(bare([1, h, 1, 64], "e4m3", part), BASE + (3 << 32)),
                   ks=_at(bare([1, h, 1], "f32"), BASE + (4 << 32)), vs=_at(bare([1, h, 1], "f32"), BASE + (5 << 32)),
                   **change)
        assert got == want, ea.lib().ea_last_error()


def _at(r, address):
    assert ea.lib().ea_relation_set_data(r.handle, ctypes.c_void_p(address), r.nbytes) == OK
    return r


BASE = 1 << 44  # addresses that no other relation of these tests has


def test_rows_overlap():
    xk, xv = (_at(bare([9, 128], "bf16"), BASE + i * (1 << 20)) for i in range(2))
    for call, bad in (("write", "k"), ("write", "v"), ("write", "ks"), ("write", "vs")):
        r = bare([30, 2, 4], "f32") if bad in ("ks", "vs") else \
            bare([30, 2, 16, 64], "e4m3", [range(31), [0, 2], [0, 16], [0, 64]])
        assert rows(call, xk=xk, xv=xv, **{bad: _at(r, BASE)}) == ARG
        at = BASE + (1 << 24)
        for array in ("start", "lengths", "table"):
            assert rows(call, **{bad: _at(r, at), array: at + r.nbytes - 4}) == ARG
    for bad in ("xk", "xv"):
        x = _at(bare([9, 128], "bf16"), BASE + (1 << 25))
        for array in ("start", "lengths", "table"):
            assert rows("read", **{bad: x, array: BASE + (1 << 25)}) == ARG
        assert rows("read", **{bad: x}, ks=_at(bare([30, 2, 4], "f32"), BASE + (1 << 25) + 256)) == ARG
    same = fake([9, 128])
    assert rows("read", xk=same, xv=same) == ARG
    k, s = cache(30, 2, 16, 64, "e4m3"), scales()
    assert rows("write", k=k, v=k) == ARG and rows("write", ks=s, vs=s) == ARG


def paged8(ws=256, n=None, **change):
    a = dict(q=fake([5, 8 * 128]), k=cache(30, 2, 16, 128, "e4m3"), v=cache(30, 2, 16, 128, "e4m3"), ks=scales(),
             vs=scales(), out=fake([8, 5, 128]), scale=0.1, n_seq=5, lengths=256, table=256, stride=4)
    a.update({x: v() if callable(v) else v for x, v in change.items()})
    b = E._Paged(a["scale"], a["n_seq"], None, a["lengths"], a["table"], a["stride"], 0, None, None)
    h = lambda r: None if r is None else r._h
    if n is None:
        need = ctypes.c_int64()
        rc = ea.lib().ea_attention_paged_workspace(h(a["q"]), h(a["k"]), ctypes.byref(b), ctypes.byref(need))
        n = need.value if rc == OK else 0
    return ea.lib().ea_attention_paged8(*[h(a[x]) for x in ("q", "k", "v", "ks", "vs", "out")], ctypes.byref(b), ws, n,
                                        None)


@pytest.mark.parametrize("code,change", [
    (ARG, dict(ks=None)), (ARG, dict(vs=None)), (ARG, dict(scale=0.0)), (ARG, dict(ws=None)), (CAPACITY, dict(n=4096)),
    (DTYPE, dict(k=lambda: cache(30, 2, 16, 128), v=lambda: cache(30, 2, 16, 128))),
    (DTYPE, dict(q=lambda: fake([5, 1024], "f32"))), (DTYPE, dict(out=lambda: fake([5, 1024], "f16"))),
    (DTYPE, dict(q=lambda: fake([5, 1024], "e4m3"))),
    (DTYPE, dict(v=lambda: cache(30, 2, 16, 128, "e5m2"))), (DTYPE, dict(vs=lambda: scales(dtype="f16"))),
    (ARG, dict(ks=lambda: scales(n=5))), (ARG, dict(vs=lambda: scales(n=2))),
    (UNSUPPORTED, dict(k=lambda: cache(30, 2, 16, 96, "e4m3"), v=lambda: cache(30, 2, 16, 96, "e4m3"))),
])
def test_attention_refusals(code, change):
    assert paged8(**change) == code, ea.lib().ea_last_error()


def test_attention_overlap():
    q = fake([5, 1024])
    assert paged8(q=q, out=q) == ARG
    s = _at(bare([30, 2, 4], "f32"), BASE)
    assert paged8(ks=s, out=_at(bare([5, 1024], "bf16"), BASE + 256)) == ARG
    assert paged8(vs=s, ws=BASE + 256) == ARG


def test_other_calls_refuse_eight_bits():
    assert paged(k=cache(30, 2, 16, 128, "e4m3"), v=cache(30, 2, 16, 128, "e4m3")) == DTYPE  # no scales
    eight = lambda *s: fake(list(s), "e5m2")
    assert heads(x=eight(9, 512), q=eight(9, 256), k=eight(9, 128), v=eight(2, 9, 64)) == DTYPE
    assert heads(wq=fake([64], "e4m3")) == DTYPE and heads(wk=fake([64], "e4m3")) == DTYPE
    for dtype in ("e4m3", "e5m2"):
        assert ea.lib().ea_dtype_size(E.DTYPES[dtype]) == 1
        a, b, c = (fake([256, 256], dtype) for _ in range(3))
        for op, agg, ins, spec in ((E.JOIN_MUL, E.AGG_SUM, [a, b], "ij,jk->ik"), (E.JOIN_ADD, E.AGG_NONE, [a, b], "ij,ij->ij"),
                                   (E.OP_SOFTMAX, E.AGG_LSE, [a], "ij->ij")):
            with pytest.raises(E.EAError) as e:
                E.joinagg(spec, op, agg, ins, c)
            assert e.value.code == DTYPE
        with pytest.raises(E.EAError) as e:  # an output, a residual
            E.joinagg("ij,jk->ik", E.JOIN_MUL, E.AGG_SUM, [fake([256, 256]), fake([256, 256])], c)
        assert e.value.code == DTYPE


def test_binding_refuses():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    k = cache(30, 2, 16, 64, "e4m3")
    with pytest.raises(E.EAError, match="both or neither"):
        E.attention_paged(fake([3, 256]), k, k, fake([3, 256]), scale=1.0, table=i(3, 5), lengths=i(3), k_scale=scales())
    for bad in (dict(table=i(3)), dict(table=i(3, 5)), dict(lengths=None)):
        with pytest.raises(E.EAError):  # a table of one dim; arrays that are not on a GPU
            E.pages_write(fake([9, 128]), fake([9, 128]), k, k, k_scale=scales(), v_scale=scales(),
                          **{"table": i(3, 5), "lengths": i(3), **bad})


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
def test_the_reference_rounds_as_the_type_does(code):
    x = torch.from_numpy(np.random.default_rng(1).standard_normal(50000) * 10.0 ** np.linspace(-8, 5, 50000)).float()
    x = x[x.abs() <= C.TOP[code]]
    C.same(x.to(C.TORCH[code]).float().numpy(), C.rounded(x.double().numpy(), code))
    for top in (448, 57344, 1, 1.75, 1.76, 3.5, 2.0 ** -130, 0):
        s = C.least_scale(np.array([top, -np.inf, np.nan]), code)
        assert top <= C.TOP[code] * s and (s == 2.0 ** C.LEAST or top > C.TOP[code] * s / 2)


# ---- pages that move with their scales ---------------------------------------------
def moved(call, caches, given, ws=256, n=None, parent=(1 << 40) + (7 << 20), **change):
    from test_decode_cpu import state

    s, need = state(**({"out_lengths": None} if call == "compact" else {}) | change), ctypes.c_int64()
    ea.lib().ea_pages_workspace(4, 30, ctypes.byref(need))
    z = (ctypes.c_void_p * max(1, len(given)))(*[None if r is None else r._h for r in given])
    args = [len(caches), E._handles(caches), z, ctypes.byref(s)] + ([parent] if call == "select" else [])
    return getattr(ea.lib(), f"ea_pages_{call}_scaled")(*args, ws, need.value if n is None else n, None)


def planes(p, n=4, dtype="f32", split=True):
    return fake([p, 30, 2, n], dtype, [list(range(p + 1)) if split else [0, p], [0, 30], [0, 2], [0, n]])


@pytest.mark.parametrize("call", ["select", "compact"])
def test_scaled_moves_refuse(call):
    eight, wide = cache(30, 2, 16, 64, "e4m3"), cache(30, 2, 16, 64)
    five = cache(30, 2, 16, 64, "e5m2", planes=3)
    bad = lambda code, caches, given, **kw: moved(call, caches, given, n=100, **kw) == code
    assert bad(CAPACITY, [eight, wide, five], [scales(), None, planes(3)])  # all well but the workspace
    assert bad(DTYPE, [eight], [None]) and bad(DTYPE, [wide], [scales()]) and bad(DTYPE, [eight], [scales(dtype="bf16")])
    assert bad(ARG, [eight], [scales(pages=31)]) and bad(ARG, [eight], [scales(h=1)]) and bad(ARG, [eight], [scales(n=3)])
    assert bad(ARG, [eight], [planes(1)]) and bad(ARG, [five], [planes(2)]) and bad(ARG, [five], [scales()])
    assert bad(UNSUPPORTED, [five], [planes(3, split=False)])
    assert bad(UNSUPPORTED, [eight], [scales(part=[[0, 15, 30], [0, 2], [0, 4]])])
    z = scales()
    assert bad(ARG, [eight, cache(30, 2, 16, 64, "e4m3")], [z, z])
    over = _at(bare([30, 2, 4], "f32"), BASE)
    under = _at(bare([30, 2, 16, 64], "e4m3", [range(31), [0, 2], [0, 16], [0, 64]]), BASE)
    assert bad(ARG, [under], [over]) and bad(ARG, [eight, under], [over, scales()])
    for array in ("table", "lengths", "refs", "status"):
        assert bad(ARG, [eight], [over], **{array: BASE + 256})
    if call == "select":
        assert bad(ARG, [eight], [over], parent=BASE + 128)
    assert moved(call, [eight], [over], ws=BASE) == ARG
    # the calls without scales take no cache in 8 bits
    from test_decode_cpu import compact, select

    assert (select if call == "select" else compact)(caches=[eight]) == DTYPE


def test_kv_cache_refuses():
    from paper_2609_03905_amd.cache import KVCache

    for more in (dict(dtype="e4m3", block=3), dict(dtype="e4m3", block=0), dict(dtype="bf16", block=8)):
        with pytest.raises(E.EAError) as e:
            KVCache(1, 4, 1, 16, 64, 2, 2, device="meta", **more)
        assert e.value.code == ARG
    c = KVCache(1, 4, 1, 16, 64, 2, 2, device="meta")
    for call in (c.write, c.read):
        with pytest.raises(E.EAError, match="ea.heads"):
            call(0, None, None)
    c = KVCache(3, 4, 2, 16, 64, 2, 2, dtype="e5m2", block=4, device="meta")
    assert c.scales.shape == (6, 4, 2, 4) and c.k_scale[2].shape == (4, 2, 4) and c.k[1].dtype == "e5m2"
    assert c.v_scale[1]._byte_offset == c.scales.block(3)[2]
    with pytest.raises(E.EAError):  # one list entry a cache
        E.pages_select([c.data], c.lengths, c.table, c.lengths, c.refs, out_table=c.table, out_lengths=c.lengths,
                       out_refs=c.refs, status=c.status, scales=[])


def test_store_to_eight_bits_needs_the_sequences():
    """Slots place every token of a prompt in a cache in 16 bits; in 8 bits they
    place none: without q_start it would be a token a sequence."""
    from paper_2609_03905_amd.block import LlamaBlockShare
    from paper_2609_03905_amd.cache import KVCache

    share = LlamaBlockShare(8, 256, 2, 128, 256, device="meta")
    slots = torch.zeros(8, dtype=torch.int32)
    for sequences in (2, 8):  # fewer than the tokens, and as many
        cache = KVCache(1, 4, 2, 16, 128, sequences, 2, dtype="e4m3", device="meta")
        for given in (slots, None):
            with pytest.raises(E.EAError, match="q_start") as e:
                share.store(cache, given)
            assert e.value.code == ARG


def test_steps_are_counted_as_they_are_walked():
    """2500 tiles over table rows of 160 million keys: 2^31 steps of 128 keys and
    more, but not of 256, as the walk over codes takes them.  (What is refused then
    is the workspace, which is looked at after the steps.)"""
    q, out = fake([1000, 1024]), fake([8, 1000, 128])
    for keys, want in ((160_000_000, CAPACITY), (230_000_000, UNSUPPORTED)):
        assert paged8(q=q, out=out, n_seq=1000, stride=keys // 16, n=4096) == want, ea.lib().ea_last_error()
    sixteen = dict(k=cache(30, 2, 16, 128), v=cache(30, 2, 16, 128))
    assert paged(q=q, out=out, n_seq=1000, stride=10_000_000, n=4096, **sixteen) == UNSUPPORTED


def test_drawn_codes_lie_as_page_relations_do():
    """Every page size that the measured cases draw: pages at multiples of 256 bytes,
    in no less memory than their relation has."""
    import random

    from perf import more_operators as M

    rng, odd = random.Random(3), 0
    cases = {(c["hkv"], c["page"], c["d"], c["code"]) for c in M.listed() + [M.draw(rng) for _ in range(4000)]}
    for h, page, d, code in cases:
        n = h * page * d
        odd += n % 256 != 0
        codes = torch.randint(0, 100, (3, h, page, d), dtype=torch.uint8).view(C.TORCH[code])
        x = M._apart(codes)
        assert torch.equal(x.view(torch.uint8), codes.view(torch.uint8)) and x.stride(0) % 256 == 0
        assert 3 * x.stride(0) >= ea.layout_nbytes(x.shape, code, [range(4), [0, h], [0, page], [0, d]])
    assert odd > 1
