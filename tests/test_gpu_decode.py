"""The decoding operators together, as a program uses them: a prompt through
the block share into a paged cache, forked, continued token by token with the
prompt's keys shared, compacted on the way, against the same tokens in one
forward pass of the share."""
import numpy as np
import pytest
import torch

import decode_ref as R
from helpers import CHAIN_REL_FRO
from paper_2609_03905_amd import ea
from paper_2609_03905_amd.block import LlamaBlockDecode, LlamaBlockShare
from paper_2609_03905_amd.cache import KVCache

pytestmark = pytest.mark.gpu

HIDDEN, HEADS, HEADS_KV, FFN, PROMPT = 512, 4, 2, 640, 128


def _weights(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s, std=0.05: (torch.randn(s, generator=g, device="cuda") * std).to(torch.bfloat16)
    w = dict(n1=1 + n(HIDDEN, std=0.1), n2=1 + n(HIDDEN, std=0.1), wqkv=n(HIDDEN, (HEADS + 2 * HEADS_KV) * 128),
             wo=n(HEADS * 128, HIDDEN), wg=n(HIDDEN, FFN), wu=n(HIDDEN, FFN), wd=n(FFN, HIDDEN),
             qn=1 + n(128, std=0.1), kn=1 + n(128, std=0.1))
    return w, lambda t: torch.randn((t, HIDDEN), generator=g, device="cuda").to(torch.bfloat16)


def _share(t, w, x, **more):
    freq = (10000.0 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    s = LlamaBlockShare(t, HIDDEN, HEADS, 128, FFN, block=256, heads_kv=HEADS_KV, inv_freq=freq, qk_norm=True, **more)
    s.load({**w, "x": x})
    return s


def _set(rel, dense):
    ea.repartition(ea.Relation(rel.shape, "bf16", ea.whole_partition(rel.shape),
                               data=dense.contiguous().view(torch.uint8).reshape(-1)), rel)


def _close(got, ref):
    """Two chains of one computation, each within CHAIN_REL_FRO of the exact one
    (the block's end-to-end tolerance): twice that apart."""
    got, ref = got.double(), ref.double()
    assert torch.isfinite(got).all()
    assert (got - ref).norm() <= 2 * CHAIN_REL_FRO * ref.norm()


@pytest.mark.parametrize("page", [16, 20])
def test_forked_continuations(page):
    w, tokens = _weights(1)
    prompt = tokens(PROMPT)
    prefill = _share(PROMPT, w, prompt)
    first = R.unblocked(prefill.forward())
    n = 4  # sequences: three continuations, one place that stays empty at first
    cache = KVCache(2, 64, HEADS_KV, page, 128, n, 20)
    layer = 1
    for z in cache.k + cache.v:
        z.bytes().fill_(0xFF)  # NaN in every row that nothing is written to
    slots, positions = cache.extend(R.i32([PROMPT, 0, 0, 0]), PROMPT)
    assert cache.status.tolist()[0] == ea.PAGES_OK and torch.equal(positions.cpu(), torch.arange(PROMPT).int())
    prefill.store(cache, slots, layer)
    cache.select(R.i32([0, 0, -1, 0]))
    assert cache.lengths.tolist() == [PROMPT, PROMPT, 0, PROMPT]
    steps = [tokens(3) for _ in range(4)]
    rows = [0, 1, 3]  # the sequences that go on
    decode = LlamaBlockDecode(prefill, cache, 3, layer)
    shared = PROMPT // page * page
    # group 0: sequences 0 and 1, group 1: the empty one, group 2: sequence 3
    batch = dict(q_start=R.i32([0, 1, 2, 2, 3]), group_start=R.i32([0, 2, 3, 4]), group_shared=R.i32([shared, 0, 0]))
    outs = []
    for i, x in enumerate(steps):
        if i == 2:
            cache.select(R.i32([0, 1, -1, 3]))  # itself: nothing changes
            cache.compact()
            assert (cache.refs > 0).int().diff().max() <= 0  # used pages first
        sl, po = cache.extend(R.i32([1, 1, 0, 1]), 3)
        assert po.tolist() == [PROMPT + i] * 3
        _set(decode.x, x)
        outs.append(R.unblocked(decode.step(sl, po, **batch)).clone())
    # the same tokens, a sequence at a time in one forward pass
    for r in range(3):
        whole = torch.zeros((2 * PROMPT, HIDDEN), device="cuda", dtype=torch.bfloat16)
        whole[:PROMPT] = prompt
        for i, x in enumerate(steps):
            whole[PROMPT + i] = x[r]
        y = R.unblocked(_share(2 * PROMPT, w, whole).forward())
        _close(torch.stack([o[r] for o in outs]), y[PROMPT:PROMPT + len(steps)])
        _close(first, y[:PROMPT])
    # all freed: every page is free again
    cache.select(R.i32([-1] * n))
    assert cache.status.tolist() == [ea.PAGES_OK, 64] and not cache.refs.any()


def test_share_without_rotation_is_as_it_was():
    """No frequencies, no norms: the repartition, the same bits."""
    w, tokens = _weights(2)
    x = tokens(256)
    s = LlamaBlockShare(256, HIDDEN, HEADS, 128, FFN, block=256, heads_kv=HEADS_KV)
    s.load({**w, "x": x})
    s.forward()
    want = R.unblocked(s.qkv_heads).clone()
    assert torch.equal(want, R.unblocked(s.qkv))
    # and rotated by nothing, through ea.heads: the same rows
    t = LlamaBlockShare(256, HIDDEN, HEADS, 128, FFN, block=256, heads_kv=HEADS_KV,
                        inv_freq=torch.zeros(64, device="cuda"))
    t.load({**w, "x": x})
    t.forward()
    assert torch.equal(R.unblocked(t.qkv_heads), want) and torch.equal(R.unblocked(t.y), R.unblocked(s.y))


def test_packed_sequences_start_at_position_zero():
    w, tokens = _weights(3)
    x = tokens(384)
    both = R.unblocked(_share(384, w, x, seq_ends=[128, 384]).forward()).clone()
    _close(both[:128], R.unblocked(_share(128, w, x[:128]).forward()))
    _close(both[128:], R.unblocked(_share(256, w, x[128:]).forward()))


def test_two_caches_captured_grow_as_by_eager_calls():
    """Each cache has a workspace of its own: two graphs replayed on two streams
    give what eager calls give, every replay."""
    add = [R.i32([1, 3, 0]), R.i32([2, 0, 5])]
    make = lambda: [KVCache(1, 9000 + 100 * i, 1, 4, 64, 3, 40) for i in range(2)]
    caches, eager = make(), make()
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c, a in zip(caches, add):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.extend(a, 8))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(6):
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        want = [c.extend(a, 8) for c, a in zip(eager, add)]
        torch.cuda.synchronize()
        for c, e, o, w in zip(caches, eager, outs, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
            for x, y in ((c.table, e.table), (c.lengths, e.lengths), (c.refs, e.refs), (c.status, e.status)):
                assert torch.equal(x, y)
        assert caches[0].status.tolist()[0] == ea.PAGES_OK


def test_two_decoders_captured_step_as_by_eager_calls():
    """Steps captured one after the other on one stream, without a call before,
    and replayed on two: the same bits as eager steps of a third decoder."""
    w, tokens = _weights(4)
    share = _share(PROMPT, w, tokens(PROMPT))
    share.forward()
    n, long = 5, [300, 20, 170, 1, 64]
    caches, decoders, graphs, batches = [], [], [], []
    g = torch.Generator(device="cuda").manual_seed(5)
    for i in range(2):
        c = KVCache(1, 80, HEADS_KV, 16, 128, n, 24)
        c.k[0].bytes().view(torch.bfloat16).normal_(generator=g)
        c.v[0].bytes().view(torch.bfloat16).normal_(generator=g)
        slots, positions = c.extend(R.i32([x + 30 * i for x in long]), sum(long) + 30 * n * i)
        caches.append(c)
        # the second one's groups share nothing, but take the other walk
        batches.append({} if i == 0 else dict(group_start=R.i32([0, 2, 5]), group_shared=R.i32([0, 0])))
        decoders.append(LlamaBlockDecode(share, c, n))
    one = [c.extend(R.i32([1] * n), n) for c in caches]
    eager = [LlamaBlockDecode(share, c, n) for c in caches]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for d, (slots, positions), b in zip(decoders, one, batches):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            d.step(slots, positions, **b)
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(5):
        xs = [tokens(n) for _ in graphs]
        for d, e, x in zip(decoders, eager, xs):
            _set(d.x, x)
            _set(e.x, x)
            d.y.data.fill_(0xFF)
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for d, e, (slots, positions), b in zip(decoders, eager, one, batches):
            want = R.unblocked(e.step(slots, positions, **b))
            assert torch.isfinite(want.float()).all() and torch.equal(R.unblocked(d.y), want)
    assert not decoders[0].workspace[:ea.WS_COUNTER_BYTES].any()
