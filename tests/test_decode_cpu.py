"""What the decoding calls refuse, host only: every check precedes HIP."""
import ctypes

import pytest
import torch

ea = pytest.importorskip("paper_2609_03905_amd")
from paper_2609_03905_amd import ea as E  # noqa: E402

OK, ARG, DTYPE, CAPACITY, UNSUPPORTED = 0, -1, -2, -4, -7
_next = [1 << 30]


def fake(shape, dtype="bf16", part=None):
    """A relation over an address that host-side checks never dereference."""
    r = ea.Relation(shape, dtype, part or E.whole_partition(shape), allocate=False)
    at = _next[0]
    _next[0] += (r.nbytes + 511) // 256 * 256
    assert ea.lib().ea_relation_set_data(r.handle, ctypes.c_void_p(at), r.nbytes) == 0
    return r


def cache(pages, h, page, d, dtype="bf16", planes=None):
    shape = ([planes] if planes else []) + [pages, h, page, d]
    part = E.whole_partition(shape)
    for i in range(len(shape) - 3):
        part[i] = list(range(shape[i] + 1))
    return fake(shape, dtype, part)


def splits(n, b):
    return list(range(0, n, b)) + [n]


# ---- head rows -----------------------------------------------------------------
def heads(**change):
    a = dict(x=fake([9, 8 * 64]), wq=fake([64]), wk=fake([64], "f32"), q=fake([9, 4 * 64]), k=fake([9, 2 * 64]),
             v=fake([2, 9, 64]), d=64, eps=1e-6, rotary=64, inter=0, freq=256, slots=None)
    a.update(change)
    prm = E._HeadsParams(a["d"], a["eps"], a["rotary"], a["inter"], a["freq"], None, a["slots"])
    h = lambda r: None if r is None else r._h
    return ea.lib().ea_heads(h(a["x"]), h(a["wq"]), h(a["wk"]), h(a["q"]), h(a["k"]), h(a["v"]),
                             None if change.get("no_params") else ctypes.byref(prm), None)


NODATA = object()


@pytest.mark.parametrize("code,change", [
    (ARG, dict(no_params=True)),
    (ARG, dict(x=None)), (ARG, dict(q=None)), (ARG, dict(k=None)), (ARG, dict(v=None)),
    (ARG, dict(q=NODATA)),
    (UNSUPPORTED, dict(d=0)), (UNSUPPORTED, dict(d=12)), (UNSUPPORTED, dict(d=520)), (UNSUPPORTED, dict(d=-8)),
    (ARG, dict(d=40)),                       # columns are no heads of 40
    (ARG, dict(rotary=3)), (ARG, dict(rotary=-2)), (ARG, dict(rotary=66)), (ARG, dict(freq=None)),
    (ARG, dict(inter=2)), (ARG, dict(wk=None)), (ARG, dict(wq=None)),
    (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))), (ARG, dict(eps=float("inf"))),
    (ARG, dict(wq=lambda: fake([128]))), (ARG, dict(wq=lambda: fake([1, 64]))),
    (UNSUPPORTED, dict(wq=lambda: fake([64], "f32", [[0, 32, 64]]))),
    (DTYPE, dict(q=lambda: fake([9, 256], "f16"))), (DTYPE, dict(v=lambda: fake([9, 128], "f32"))),
    (ARG, dict(q=lambda: fake([8, 256]))),   # fewer rows
    (ARG, dict(q=lambda: fake([9, 320]))),   # another head
    (ARG, dict(k=lambda: fake([9, 64]))),    # k and v differ
    (ARG, dict(v=lambda: fake([2, 8, 64]))),
    (ARG, dict(v=lambda: fake([2, 9, 128]))),
    (ARG, dict(v=lambda: fake([2, 2, 9, 64]))),  # leading extent
    (ARG, dict(v=lambda: fake([9]))),
    (ARG, dict(x=lambda: fake([1, 9, 512]))),
    (UNSUPPORTED, dict(x=lambda: fake([9, 512], "bf16", [[0, 9], [0, 96, 512]]))),
    (UNSUPPORTED, dict(x=lambda: fake([9, 512], "bf16", [[0, 9], splits(512, 32)]))),
    (UNSUPPORTED, dict(x=lambda: fake([9, 512], "bf16", [[0, 4, 6, 9], [0, 512]]))),
    (UNSUPPORTED, dict(x=lambda: fake([9, 512], "bf16", [[0, 2, 9], [0, 512]]))),
    (UNSUPPORTED, dict(v=lambda: fake([2, 9, 64], "bf16", [[0, 2], [0, 9], [0, 32, 64]]))),
    # slots: k and v are caches
    (ARG, dict(slots=256)),
    (UNSUPPORTED, dict(slots=256, k=lambda: fake([4, 2, 16, 64]), v=lambda: fake([4, 2, 16, 64]))),
    (ARG, dict(slots=256, k=lambda: cache(4, 2, 16, 128), v=lambda: cache(4, 2, 16, 128))),
    (ARG, dict(slots=256, k=lambda: cache(4, 2, 16, 64), v=lambda: cache(5, 2, 16, 64))),
    (ARG, dict(slots=256, k=lambda: cache(4, 3, 16, 64), v=lambda: cache(4, 3, 16, 64))),
])
def test_heads_refusals(code, change):
    change = {n: (v() if callable(v) else v) for n, v in change.items()}
    if change.get("q") is NODATA:
        change["q"] = ea.Relation([9, 256], "bf16", E.whole_partition([9, 256]), allocate=False)
    assert heads(**change) == code, ea.lib().ea_last_error()


def test_heads_overlap():
    x = fake([9, 512])
    q = ea.Relation([9, 256], "bf16", E.whole_partition([9, 256]), allocate=False)
    base = _next[0] - (x.nbytes + 511) // 256 * 256
    ea.lib().ea_relation_set_data(q.handle, ctypes.c_void_p(base + 256), q.nbytes)
    assert heads(x=x, q=q) == ARG
    k = fake([9, 128])
    assert heads(k=k, v=k) == ARG


def grad(ws=256, n=None, **change):
    a = dict(x=fake([9, 512]), wq=fake([64]), wk=fake([64]), dq=fake([9, 256]), dk=fake([9, 128]), dv=fake([9, 128]),
             dx=fake([9, 512]), dwq=fake([64], "f32"), dwk=fake([64], "f32"), slots=None)
    a.update(change)
    prm = E._HeadsParams(64, 1e-6, 64, 0, 256, None, a["slots"])
    need = ctypes.c_int64()
    assert ea.lib().ea_heads_backward_workspace(64, ctypes.byref(need)) == OK
    h = lambda r: None if r is None else r._h
    return ea.lib().ea_heads_backward(*[h(a[x]) for x in ("x", "wq", "wk", "dq", "dk", "dv", "dx", "dwq", "dwk")],
                                      ctypes.byref(prm), ws, need.value if n is None else n, None)


def test_heads_backward_refusals():
    x = fake([9, 512])
    ea.plan_cache_clear()  # (also forgets layouts: an equal one is given another id)
    assert grad(x=x, n=1000) == CAPACITY  # dx's layout passes as qkv's
    assert grad(dx=None) == ARG and grad(dx=fake([9, 512], "bf16", [[0, 9], [0, 64, 512]])) == ARG
    assert grad(dx=fake([9, 512], "f16")) == ARG
    assert grad(slots=256) == ARG
    assert grad(wq=None, wk=None) == ARG          # gradients of weights that are not there
    assert grad(dwq=fake([32], "f32")) == ARG
    assert grad(ws=None) == ARG and grad(ws=128) == ARG and grad(n=1000) == CAPACITY
    x = fake([9, 512])
    assert grad(x=x, dx=x) == ARG
    w = fake([64], "f32")
    assert grad(dwq=w, dwk=w) == ARG
    assert grad(dq=fake([9, 256], "f32")) == DTYPE
    L, n = ea.lib(), ctypes.c_int64()
    assert L.ea_heads_backward_workspace(64, None) == ARG
    assert L.ea_heads_backward_workspace(12, ctypes.byref(n)) == UNSUPPORTED


# ---- attention over pages ---------------------------------------------------------
def paged(ws=256, n=None, **change):
    a = dict(q=fake([5, 8 * 128]), k=cache(30, 2, 16, 128), v=cache(30, 2, 16, 128), out=fake([8, 5, 128]), scale=0.1,
             n_seq=5, start=None, lengths=256, table=256, stride=4, n_group=0, gs=None, gk=None)
    a.update(change)
    b = E._Paged(a["scale"], a["n_seq"], a["start"], a["lengths"], a["table"], a["stride"], a["n_group"], a["gs"],
                 a["gk"])
    h = lambda r: None if r is None else r._h
    if n is None:
        need = ctypes.c_int64()
        rc = ea.lib().ea_attention_paged_workspace(h(a["q"]), h(a["k"]), ctypes.byref(b), ctypes.byref(need))
        n = need.value if rc == OK else 0
    return ea.lib().ea_attention_paged(h(a["q"]), h(a["k"]), h(a["v"]), h(a["out"]),
                                       None if change.get("no_batch") else ctypes.byref(b), ws, n, None)


@pytest.mark.parametrize("code,change", [
    (ARG, dict(no_batch=True)), (ARG, dict(q=None)), (ARG, dict(k=None)), (ARG, dict(v=None)), (ARG, dict(out=None)),
    (ARG, dict(scale=0.0)), (ARG, dict(scale=-1.0)), (ARG, dict(scale=float("nan"))), (ARG, dict(scale=float("inf"))),
    (ARG, dict(n_seq=0)), (ARG, dict(n_group=-1)), (UNSUPPORTED, dict(n_seq=2049)),
    (UNSUPPORTED, dict(n_seq=2000, n_group=49)),
    (ARG, dict(lengths=None)), (ARG, dict(table=None)), (ARG, dict(stride=0)), (UNSUPPORTED, dict(stride=2 ** 27)),
    (ARG, dict(n_group=1)), (ARG, dict(n_group=1, gs=256)),
    (ARG, dict(n_seq=6)),                               # fewer rows than sequences, one row each
    (DTYPE, dict(q=lambda: fake([5, 1024], "f16"))), (DTYPE, dict(out=lambda: fake([5, 1024], "f16"))),
    (DTYPE, dict(k=lambda: cache(30, 2, 16, 128, "f32"), q=lambda: fake([5, 1024], "f32"))),
    (ARG, dict(v=lambda: cache(31, 2, 16, 128))), (DTYPE, dict(v=lambda: cache(30, 2, 16, 128, "f16"))),
    (UNSUPPORTED, dict(k=lambda: cache(30, 2, 16, 96), v=lambda: cache(30, 2, 16, 96))),
    (UNSUPPORTED, dict(k=lambda: fake([30, 2, 16, 128]))),  # a block that is not one page
    (ARG, dict(k=lambda: cache(30, 2, 16, 128, planes=2))),
    (ARG, dict(k=lambda: cache(30, 3, 16, 128), v=lambda: cache(30, 3, 16, 128))),  # 8 heads over 3
    (ARG, dict(out=lambda: fake([5, 512]))), (ARG, dict(out=lambda: fake([6, 1024]))),
    (ARG, dict(ws=None)), (ARG, dict(ws=100)), (CAPACITY, dict(n=4096)),
])
def test_paged_refusals(code, change):
    change = {n: (v() if callable(v) else v) for n, v in change.items()}
    assert paged(**change) == code, ea.lib().ea_last_error()


def test_paged_workspace_refusals_and_overlap():
    q = fake([5, 1024])
    assert paged(q=q, out=q) == ARG
    n = ctypes.c_int64()
    b = E._Paged(1.0, 5, None, None, None, 1, 0, None, None)
    k = cache(30, 2, 16, 128)
    assert ea.lib().ea_attention_paged_workspace(q._h, k._h, ctypes.byref(b), None) == ARG
    assert ea.lib().ea_attention_paged_workspace(q._h, k._h, None, ctypes.byref(n)) == ARG
    assert ea.attention_paged_workspace(q, k, 5) > E.WS_COUNTER_BYTES


# ---- the page table -----------------------------------------------------------------
A = 1 << 40  # device addresses, 1 MiB apart


def state(**change):
    f = dict(n_seq=4, stride=5, n_pages=30, page_size=16, table=A, lengths=A + (1 << 20), refs=A + (2 << 20),
             out_table=A + (3 << 20), out_lengths=A + (4 << 20), out_refs=A + (5 << 20), status=A + (6 << 20))
    f.update(change)
    return E._Pages(*[f[n] for n, _ in E._Pages._fields_])


def extend(add=A + (7 << 20), n_tokens=3, ws=256, n=None, **change):
    s, need = state(**{"out_table": A, **change}), ctypes.c_int64()
    ea.lib().ea_pages_workspace(max(s.n_seq, 1), max(s.n_pages, 1), ctypes.byref(need))
    return ea.lib().ea_pages_extend(ctypes.byref(s), add, A + (8 << 20), None, n_tokens, ws,
                                    need.value if n is None else n, None)


def select(caches=(), parent=A + (7 << 20), ws=256, n=None, **change):
    s, need = state(**change), ctypes.c_int64()
    ea.lib().ea_pages_workspace(max(s.n_seq, 1), max(s.n_pages, 1), ctypes.byref(need))
    return ea.lib().ea_pages_select(len(caches), E._handles(caches), ctypes.byref(s), parent, ws,
                                    need.value if n is None else n, None)


def compact(caches=(), ws=256, n=None, **change):
    s, need = state(**{"out_lengths": None, **change}), ctypes.c_int64()
    ea.lib().ea_pages_workspace(max(s.n_seq, 1), max(s.n_pages, 1), ctypes.byref(need))
    return ea.lib().ea_pages_compact(len(caches), E._handles(caches), ctypes.byref(s), ws,
                                     need.value if n is None else n, None)


@pytest.mark.parametrize("call", [extend, select, compact])
@pytest.mark.parametrize("code,change", [
    (ARG, dict(n_seq=0)), (ARG, dict(stride=0)), (ARG, dict(n_pages=0)), (ARG, dict(page_size=0)),
    (ARG, dict(n_pages=-5)), (UNSUPPORTED, dict(n_seq=2049)), (UNSUPPORTED, dict(n_seq=2048, stride=1 << 20)),
    (UNSUPPORTED, dict(n_pages=1 << 28)), (UNSUPPORTED, dict(n_pages=(1 << 30) + 1, page_size=1)),
    (UNSUPPORTED, dict(stride=1 << 27, n_seq=1)),
    (ARG, dict(table=None)), (ARG, dict(lengths=None)), (ARG, dict(refs=None)), (ARG, dict(out_refs=None)),
    (ARG, dict(status=None)), (ARG, dict(out_refs=A + 4)), (ARG, dict(status=A + (2 << 20))),
    (ARG, dict(out_refs=A + (2 << 20) + 4)),
])
def test_pages_refusals(call, code, change):
    assert call(**change) == code, ea.lib().ea_last_error()


def test_pages_refusals_of_one_call():
    assert extend(add=None) == ARG and extend(n_tokens=-1) == ARG and extend(out_lengths=None) == ARG
    assert extend(out_table=A + (3 << 20)) == ARG  # it works in its table
    for bad in (A, A + (1 << 20), A + (2 << 20), A + (6 << 20), A + (7 << 20)):  # slots over another array
        s = state(out_table=A)
        assert ea.lib().ea_pages_extend(ctypes.byref(s), A + (7 << 20), bad, None, 3, 256, 1 << 30, None) == ARG
        assert ea.lib().ea_pages_extend(ctypes.byref(s), A + (7 << 20), None, bad, 3, 256, 1 << 30, None) == ARG
    assert extend(add=A + (4 << 20)) == ARG and extend(add=A + (5 << 20)) == ARG and extend(add=A) == ARG
    for bad in (3, 4, 5, 6):
        assert select(parent=A + (bad << 20)) == ARG
    assert select(parent=None) == ARG and select(out_lengths=None) == ARG
    for same in (dict(out_table=A), dict(out_lengths=A + (1 << 20)), dict(out_refs=A + (2 << 20))):
        assert select(**same) == ARG
    assert extend(ws=None) == ARG and extend(ws=64) == ARG and extend(n=100) == CAPACITY
    for call in (select, compact):
        assert call(ws=None) == ARG and call(ws=64) == ARG and call(n=100) == CAPACITY
        c = cache(30, 2, 16, 64, planes=3)
        assert call([c, c]) == ARG                                   # the same cache twice
        assert call([cache(30, 2, 16, 64) for _ in range(5)]) == ARG
        assert call([cache(31, 2, 16, 64)]) == ARG and call([cache(30, 2, 8, 64)]) == ARG
        assert call([fake([30, 2, 16, 64])]) == UNSUPPORTED
        assert call([cache(30, 2, 16, 12)]) == UNSUPPORTED           # rows of 24 bytes
        assert call([fake([30, 2, 16])]) == ARG
    assert ea.lib().ea_pages_workspace(0, 5, ctypes.byref(ctypes.c_int64())) == ARG
    assert ea.lib().ea_pages_workspace(5, 5, None) == ARG


# ---- the binding ------------------------------------------------------------------------
def _raises(code, f):
    with pytest.raises(ea.EAError) as e:
        f()
    assert e.value.code == code


def test_binding_checks_device_arrays():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    q, k = fake([5, 1024]), cache(30, 2, 16, 128)
    call = lambda **kw: ea.attention_paged(q, k, k, q, **{**dict(scale=0.1, table=i(5, 4), lengths=i(5)), **kw})
    _raises(ARG, lambda: call(table=i(20)))
    _raises(ARG, lambda: call(table=i(5, 4).long()))
    _raises(ARG, lambda: call(lengths=i(4)))
    _raises(ARG, lambda: call(lengths=None))
    _raises(ARG, lambda: call(q_start=i(5)))
    _raises(ARG, lambda: call(group_start=i(2)))
    _raises(ARG, call)  # on the host
    x = fake([9, 512])
    _raises(ARG, lambda: ea.heads(x, x, x, x, d_head=64, inv_freq=torch.zeros(32)))
    _raises(ARG, lambda: ea.heads(x, x, x, x, d_head=64, inv_freq=i(32)))
    _raises(ARG, lambda: ea.heads(x, x, x, x, d_head=64, positions=i(8)))
    st = dict(page_size=16, status=i(2))
    _raises(ARG, lambda: ea.pages_extend(i(20), i(4), i(30), i(4), **st))
    _raises(ARG, lambda: ea.pages_extend(i(4, 5), i(4), None, i(4), **st))
    _raises(ARG, lambda: ea.pages_extend(i(4, 5), i(4), i(30), i(4), **st))


def test_a_workspace_of_the_host_is_refused():
    with pytest.raises(ea.EAError, match="workspace"):
        E._workspace(256, torch.zeros(512, dtype=torch.uint8), None)


def test_paged_refuses_more_steps_than_it_counts():
    """Tiles of 128 columns times steps of 64 keys, and of 16 times 128, 2^31 or
    more of them; one page less passes that check and fails for its workspace."""
    # 65536 rows of 4 heads a key-value head: (262144 / 128 + 5) * 2 tiles
    big = dict(q=fake([65536, 1024]), out=fake([65536, 1024]), start=256, n=4096)
    most = (2 ** 31 - 1) // ((262144 // 128 + 5) * 2) * 64 // 16
    assert paged(stride=most + 4, **big) == UNSUPPORTED and paged(stride=most, **big) == CAPACITY
    # 5 sequences of 4 columns: (20 / 16 + 5) * 2 tiles over 2^31 keys are within
    assert paged(stride=2 ** 27 - 128, n=4096) == CAPACITY
    # 2000 sequences over 8 heads, groups among them
    q = fake([2000, 4096])
    few = dict(q=q, out=fake([2000, 4096]), k=cache(30, 8, 16, 128), v=cache(30, 8, 16, 128), n_seq=2000, n=4096)
    tiles = (8000 // 16 + 2000) * 8
    most = (2 ** 31 - 1) // tiles * 128 // 16
    assert paged(stride=most + 8, **few) == UNSUPPORTED and paged(stride=most, **few) == CAPACITY
    # 40 groups' tiles of 128 columns, in steps of 64 keys
    assert paged(stride=most // 2, n_group=40, gs=256, gk=256, **few) == CAPACITY


def test_decoders_have_workspaces_of_their_own(monkeypatch):
    """Every call of a step that takes a workspace is given the decoder's, which
    holds what attention needs for any number of groups."""
    from paper_2609_03905_amd.block import LlamaBlockDecode, LlamaBlockShare
    from paper_2609_03905_amd.cache import KVCache

    share = LlamaBlockShare(16, 256, 2, 128, 256, block=128, heads_kv=1, device="meta")
    c = KVCache(1, 20, 1, 16, 128, 6, 3, device="meta")
    decoders = [LlamaBlockDecode(share, c, 6, device="meta") for _ in range(2)]
    assert decoders[0].workspace is not decoders[1].workspace
    for d in decoders:
        assert all(ea.attention_paged_workspace(d.q, c.k[0], 6, g) <= d.workspace.numel() for g in range(7))
    seen = []
    for name in ("joinagg", "attention_paged"):
        monkeypatch.setattr(E, name, lambda *a, **kw: seen.append(kw.get("workspace")))
    monkeypatch.setattr(E, "heads", lambda *a, **kw: None)
    assert decoders[0].step(None, None) is decoders[0].y
    assert len(seen) == 7 and all(w is decoders[0].workspace for w in seen)


def test_share_of_packed_sequences_without_frequencies():
    """Positions are needed where heads are rotated: no ends are one sequence, as
    for attention, and ends that do not ascend are refused there as ever."""
    from paper_2609_03905_amd.block import LlamaBlockShare

    make = lambda **kw: LlamaBlockShare(16, 256, 2, 128, 256, block=128, heads_kv=1, device="meta", **kw)
    freq = torch.ones(64)
    assert make(seq_ends=[]).positions is None and make(seq_ends=[], inv_freq=freq).positions is None
    assert make(seq_ends=[5, 3, 16]).seq_ends == [5, 3, 16]
    assert make(seq_ends=[4, 16], inv_freq=freq).positions.shape == (16,)
    for ends in ([5, 3, 16], [4, 4, 16], [0, 16], [4], [4, 17]):
        _raises(ARG, lambda: make(seq_ends=ends, inv_freq=freq))


def test_extend_refuses_counts_over_its_status():
    assert extend(add=A + (6 << 20)) == ARG and extend(add=A + (6 << 20) - 12) == ARG
    assert extend(add=A + (6 << 20) + 8, n=100) == CAPACITY


def _at(r):
    """The address that ``fake`` gave the newest relation, ``r``."""
    return _next[0] - (r.nbytes + 511) // 256 * 256


def test_arrays_and_workspaces_over_other_memory():
    """No output and no workspace lies over an array that a kernel reads."""
    # head rows
    q = fake([9, 256])
    at = _at(q)
    assert heads(q=q, freq=at) == ARG and heads(q=q, freq=at + 4 * 32 * 4, slots=at + 9 * 512 - 4) == ARG
    L, h = ea.lib(), lambda r: None if r is None else r._h
    x, k, v = fake([9, 512]), fake([9, 128]), fake([9, 128])
    run = lambda pos: L.ea_heads(h(x), None, None, h(q), h(k), h(v),
                                 ctypes.byref(E._HeadsParams(64, 0.0, 0, 0, None, pos, None)), None)
    assert run(at - 32) == ARG and run(at + 9 * 512 - 4) == ARG
    # their gradient
    dx = fake([9, 512])
    at = _at(dx)
    big = 1 << 30
    assert grad(dx=dx, ws=at, n=big) == ARG and grad(dx=dx, ws=at - 256, n=big) == ARG
    assert grad(ws=1 << 50, n=1000, dx=dx) == CAPACITY
    # attention over pages
    out = fake([8, 5, 128])
    at = _at(out)
    for name in ("lengths", "table", "start"):
        assert paged(out=out, ws=1 << 50, **{name: at}) == ARG
        assert paged(ws=1 << 50, **{name: (1 << 50) + 4096}) == ARG
    assert paged(out=out, ws=1 << 50, table=at - 5 * 4 * 4 + 4) == ARG
    for name in ("gs", "gk"):
        assert paged(out=out, ws=1 << 50, **{"n_group": 2, "gs": 1 << 45, "gk": 1 << 46, name: at}) == ARG
    assert paged(out=out, ws=at, lengths=1 << 45, table=1 << 46) == ARG
    q = fake([5, 1024])
    assert paged(q=q, ws=_at(q), lengths=1 << 45, table=1 << 46) == ARG
    # the page table
    c = cache(30, 2, 16, 64)
    at = _at(c)
    for bad in ("table", "lengths", "refs", "out_table", "out_refs", "status"):
        assert select([c], **{bad: at}) == ARG and compact([c], **{bad: at}) == ARG
    assert select([c], parent=at) == ARG and select([c], parent=at + c.nbytes - 4) == ARG
    for call in (select, compact):
        assert call([c], ws=at) == ARG
        for bad in (0, 1, 2, 3, 5, 6):
            assert call(ws=A + (bad << 20)) == ARG
    assert select(ws=A + (7 << 20)) == ARG
    for bad in (0, 1, 2, 5, 6, 7, 8):
        assert extend(ws=A + (bad << 20)) == ARG


def test_nothing_overlaps_an_empty_array():
    """No new tokens are asked for, or no element is rotated: where the empty
    array points does not matter."""
    s = state(out_table=A)
    run = lambda slots, pos: ea.lib().ea_pages_extend(ctypes.byref(s), A + (7 << 20), slots, pos, 0, 256, 100, None)
    assert run(A + 8, A + (6 << 20) + 4) == CAPACITY and run(A + (7 << 20) + 4, A + (7 << 20) + 4) == CAPACITY
    x, dq, dx = fake([9, 512]), fake([9, 256]), fake([9, 512])
    at = _at(dx) + 256
    prm = E._HeadsParams(64, 1e-6, 0, 0, at, None, None)
    w, dk = [fake([64], "f32") for _ in range(4)], [fake([9, 128]) for _ in range(2)]
    assert ea.lib().ea_heads_backward(x._h, w[0]._h, w[1]._h, dq._h, dk[0]._h, dk[1]._h, dx._h, w[2]._h, w[3]._h,
                                      ctypes.byref(prm), 1 << 50, 1000, None) == CAPACITY
