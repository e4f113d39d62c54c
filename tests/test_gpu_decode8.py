"""The operators of a cache in 8 bits together, as a program uses them: a prompt
through the block share into the cache, forked, continued token by token with the
prompt's keys shared, compacted on the way; pages that move take their scales
along; captured steps."""
import numpy as np
import pytest
import torch

import cache8_ref as C
import decode_ref as R
from paper_2609_03905_amd import ea
from paper_2609_03905_amd.block import LlamaBlockDecode
from paper_2609_03905_amd.cache import KVCache
from test_gpu_decode import HEADS, HEADS_KV, PROMPT, _set, _share, _weights

pytestmark = pytest.mark.gpu


def _codes(rel):
    """Codes [pages, heads, page, d] of a layer's K or V (its pages lie without gaps)."""
    assert int(np.prod(rel.shape[1:])) % 256 == 0
    return rel.bytes().view(C.TORCH[rel.dtype]).view(rel.shape)


def _values(cache, layer):
    """What a layer's K and V stand for, as bf16 (exact: four bits times a power of two)."""
    out = []
    for rel, scale in ((cache.k[layer], cache.k_scale[layer]), (cache.v[layer], cache.v_scale[layer])):
        s = scale.bytes().view(torch.float32).view(scale.shape).repeat_interleave(rel.shape[2] // scale.shape[2], 2)
        out.append((_codes(rel).float() * s[..., None]).bfloat16())
    return out


def _as_sixteen_bits(decode, batch):
    """The step's attention over the same keys in a bf16 cache."""
    c = decode.cache
    k, v = (R.pages_rel(x) for x in _values(c, decode.layer))
    out = ea.Relation(decode.attn.shape, "bf16", decode.attn.partition)
    ea.attention_paged(decode.q, k, v, out, scale=decode.share.scale, table=c.table, lengths=c.lengths, **batch)
    return R.unblocked(out).double()


@pytest.mark.parametrize("code,page,block", [("e4m3", 16, 8), ("e5m2", 20, None)])
def test_forked_continuations(code, page, block):
    w, tokens = _weights(1)
    prompt = tokens(PROMPT)
    prefill = _share(PROMPT, w, prompt)
    prefill.forward()
    n, layer = 4, 1
    cache = KVCache(2, 64, HEADS_KV, page, 128, n, 20, dtype=code, block=block)
    cache.data.bytes().fill_(0x7f)  # NaN in every row that nothing is written to
    cache.scales.bytes().fill_(0xff)
    cache.extend(R.i32([0, 0, 6 * page, 0]), 1)  # of a sequence that goes: holes for compact to fill
    cache.extend(R.i32([PROMPT, 0, 0, 0]), PROMPT)
    prefill.store(cache, None, layer, q_start=R.i32([0] + [PROMPT] * n))
    # what stands there is the prompt's keys and values, as the definition has them
    for rel, scale, x in ((cache.k[layer], cache.k_scale[layer], prefill.k), (cache.v[layer], cache.v_scale[layer], prefill.v)):
        codes = np.zeros(rel.shape)
        s = np.zeros(scale.shape)
        rows = R.f64(R.unblocked(x))[0].transpose(1, 0, 2)
        C.write(rows, codes, s, cache.table.cpu().numpy(), [PROMPT], [0, PROMPT], code)
        held = cache.table[0, :-(-PROMPT // page)].cpu().numpy()
        got, want = C.f64(_codes(rel))[held], codes[held]
        last = PROMPT - (len(held) - 1) * page  # rows of the last page
        C.same(got[:-1], want[:-1])
        C.same(got[-1, :, :last], want[-1, :, :last])
    back = [ea.Relation((PROMPT, HEADS_KV * 128), "f32", ea.whole_partition((PROMPT, HEADS_KV * 128))) for _ in range(2)]
    cache.read(layer, *back, R.i32([0] + [PROMPT] * n))
    for x, b in zip((prefill.k, prefill.v), back):
        rows = R.unblocked(x)[0].transpose(0, 1).reshape(PROMPT, -1).float()
        # half a step of the code, relative; below its normal range half the least step of the scale
        off = (R.unblocked(b).float() - rows).abs()
        assert (off <= rows.abs() * {"e4m3": 2 ** -4, "e5m2": 2 ** -3}[code] + rows.abs().max() * 2 ** -15).all()
    cache.select(R.i32([0, 0, -1, 0]))
    assert cache.status.tolist()[0] == ea.PAGES_OK and cache.lengths.tolist() == [PROMPT, PROMPT, 0, PROMPT]
    before = [x.clone() for x in _values(cache, layer)]
    decode = LlamaBlockDecode(prefill, cache, 3, layer)
    shared = PROMPT // page * page
    batch = dict(q_start=R.i32([0, 1, 2, 2, 3]), group_start=R.i32([0, 2, 3, 4]), group_shared=R.i32([shared, 0, 0]))
    for i in range(12):  # past the ends of blocks and pages
        if i == 5:
            cache.select(R.i32([3, 1, -1, 0]))  # two change places
            table = cache.table.clone()
            cache.compact()
            assert (cache.refs > 0).int().diff().max() <= 0 and not torch.equal(table, cache.table)
        slots, po = cache.extend(R.i32([1, 1, 0, 1]), 3)
        assert po.tolist() == [PROMPT + i] * 3
        _set(decode.x, tokens(3))
        y = R.unblocked(decode.step(slots, po, **batch))
        assert y.isfinite().all()
        # both off by at most half a bf16 step of the output, and a little
        got, want = R.unblocked(decode.attn).double(), _as_sixteen_bits(decode, batch)
        assert (got - want).norm() <= 2 ** -7 * 1.02 * want.norm()
        # the newest rows are the step's head rows, a code's half step off
        for x, vals in zip((decode.kr, decode.vr), _values(cache, layer)):
            rows = R.unblocked(x).view(3, HEADS_KV, 128).float()
            new = torch.stack([vals[s // page, :, s % page] for s in slots.tolist()]).float()
            step = {"e4m3": 2 ** -4, "e5m2": 2 ** -3}[code]
            assert ((new - rows).abs() <= rows.abs() * step + vals[vals.isfinite()].abs().max() * 2 ** -8).all()
    # the prompt's whole pages, shared and moved, hold what they held
    now = _values(cache, layer)
    for s in (0, 1, 3):
        for b, x in zip(before, now):
            first = cache.table[s, :shared // page].long()
            assert x[first].isfinite().all()
    cache.select(R.i32([-1] * n))
    assert cache.status.tolist() == [ea.PAGES_OK, 64] and not cache.refs.any()


@pytest.mark.parametrize("layers,heads,page,block,d", [(1, 2, 8, 4, 16), (3, 1, 6, 1, 32), (2, 3, 5, 5, 64)])
def test_pages_move_with_their_scales(layers, heads, page, block, d):
    """Random forks, growth and compaction: every sequence's rows stand for what
    they stood for, in every plane; scales of blocks without a row that moves stay."""
    rng = np.random.default_rng(layers)
    n = 9
    cache = KVCache(layers, 60, heads, page, d, n, 6, dtype="e4m3", block=block)
    assert cache.scales.shape == (2 * layers, 60, heads, page // block)
    whole = lambda: (cache.data.bytes().clone(), cache.scales.bytes().clone())
    cache.data.bytes().copy_(torch.randint(0, 120, cache.data.bytes().shape, dtype=torch.uint8, device="cuda"))
    for s in cache.k_scale + cache.v_scale:
        s.bytes().view(torch.float32).copy_(2.0 ** torch.randint(-9, 9, s.bytes().view(torch.float32).shape, device="cuda"))

    def rows():
        """{sequence: [planes][length] rows with their scales}"""
        out = []
        table, lens = cache.table.cpu().numpy(), cache.lengths.cpu().numpy()
        planes = [(C.f64(_rows_of(r)), s.bytes().view(torch.float32).view(s.shape).cpu().numpy())
                  for r, s in zip(cache.k + cache.v, cache.k_scale + cache.v_scale)]
        for s in range(n):
            at = np.arange(lens[s])
            pg, row = table[s][at // page], at % page
            out.append([(c[pg, :, row], z[pg, :, row // block]) for c, z in planes])
        return out

    def _rows_of(rel):
        pages = rel.shape[0]
        size = int(np.prod(rel.shape[1:]))
        pitch = -(-size // 256) * 256
        raw = rel.data.as_strided((pages, size), (pitch, 1), rel._byte_offset)
        return raw.contiguous().view(C.TORCH["e4m3"]).view(rel.shape)

    cache.extend(R.i32(rng.integers(0, 4 * page, n)), 1)
    assert cache.status.tolist()[0] == ea.PAGES_OK
    for i in range(12):
        was = rows()
        if i % 3 == 2:
            cache.compact()
            parent = np.arange(n)
        else:
            parent = rng.integers(-1, n, n)
            cache.select(R.i32(parent))
        if cache.status.tolist()[0] != ea.PAGES_OK:
            parent = np.arange(n)
        now = rows()
        for s in range(n):
            for (c, z), (c0, z0) in zip(now[s], was[parent[s]] if parent[s] >= 0 else now[s]):
                assert np.array_equal(c, c0, equal_nan=True) and np.array_equal(z, z0)
        cache.extend(R.i32(rng.integers(0, 3, n)), 1)


def test_scales_of_blocks_behind_a_copied_row_stay():
    """A fork copies 5 rows of a page of 8 in blocks of 2: three blocks' scales."""
    cache = KVCache(1, 4, 1, 8, 16, 2, 2, dtype="e5m2", block=2)
    cache.extend(R.i32([5, 0]), 5)
    z = cache.k_scale[0].bytes().view(torch.float32).view(4, 4)
    z.copy_(torch.arange(16, device="cuda").view(4, 4))
    cache.select(R.i32([0, 0]))
    assert cache.table[:, 0].tolist() == [0, 1]
    assert z.tolist() == [[0, 1, 2, 3], [0, 1, 2, 7], [8, 9, 10, 11], [12, 13, 14, 15]]


def test_a_step_that_has_no_places_leaves_the_cache():
    """extend finds too few free pages: the step that follows writes nothing, eager
    or captured; when pages are free again, the same calls are served."""
    w, tokens = _weights(6)
    share = _share(PROMPT, w, tokens(PROMPT))
    share.forward()
    cache = KVCache(1, 8, HEADS_KV, 16, 128, 3, 8, dtype="e4m3", block=4)
    cache.scales.bytes().view(torch.float32).fill_(0.25)
    cache.extend(R.i32([32, 80, 10]), 1)  # 2, 5 and 1 of 8 pages
    assert cache.status.tolist() == [ea.PAGES_OK, 0]
    decode, one, pos = LlamaBlockDecode(share, cache, 3), R.i32([1, 1, 1]), R.i32([32, 80, 10])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        slots, _ = cache.extend(one, 3)
        decode.step(slots, pos)
    _set(decode.x, tokens(3))
    whole = lambda: [x.bytes().clone() for x in (cache.data, cache.scales)]
    was, lens = whole(), cache.lengths.tolist()
    for run in (lambda: decode.step(cache.extend(one, 3)[0], pos), graph.replay):
        run()
        assert cache.status.tolist()[0] == ea.PAGES_NONE_FREE and cache.lengths.tolist() == lens
        assert all(torch.equal(a, b) for a, b in zip(was, whole()))
    rows = [ea.Relation((3, HEADS_KV * 128), "bf16", ea.whole_partition((3, HEADS_KV * 128))) for _ in range(2)]
    cache.read(0, *rows, slots=slots)  # no keys for them either
    assert not any(R.unblocked(x).any() for x in rows)
    for bad in (R.i32([0, 0]), slots.float(), slots.cpu()):
        with pytest.raises(ea.EAError):
            cache.write(0, *rows, slots=bad)
    cache.lengths.copy_(R.i32([32, 64, 10]))  # the second sequence gives its last page back
    cache.refs[cache.table[1, 4]] = 0
    decode.step(cache.extend(R.i32([0, 0, 1]), 3)[0], pos, q_start=R.i32([0, 0, 0, 1]))
    assert cache.status.tolist()[0] == ea.PAGES_OK and cache.lengths.tolist() == [32, 64, 11]
    assert not torch.equal(was[0], cache.data.bytes())


def test_captured_steps_as_eager_ones():
    """Two decoders over caches in 8 bits, captured and replayed on two streams:
    the bits of eager steps of a third, every replay."""
    w, tokens = _weights(4)
    share = _share(PROMPT, w, tokens(PROMPT))
    share.forward()
    n, long = 5, [300, 20, 170, 1, 64]
    sets = []
    for i, code in enumerate(("e4m3", "e5m2")):
        pair = []
        for _ in range(2):  # one for the graph, one for eager steps
            g = torch.Generator(device="cuda").manual_seed(5 + i)
            c = KVCache(1, 90, HEADS_KV, 16, 128, n, 24, dtype=code, block=[16, 4][i])
            for rel, s in zip(c.k + c.v, c.k_scale + c.v_scale):
                _codes(rel).view(torch.uint8).copy_(torch.randint(0, 96, rel.shape, generator=g, device="cuda").to(torch.uint8))
                s.bytes().view(torch.float32).fill_(0.25 if code == "e4m3" else 2.0 ** -9)
            c.extend(R.i32(long), sum(long))
            pair.append(LlamaBlockDecode(share, c, n))
        batch = {} if i == 0 else dict(group_start=R.i32([0, 2, 5]), group_shared=R.i32([0, 0]))
        sets.append((*pair, R.i32(long), R.i32([1] * n), batch))
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in sets]
    for (d, _, pos, one, batch), st in zip(sets, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            d.cache.extend(one, n)
            d.step(None, pos, **batch)
            pos.add_(1)
        graphs.append(graph)
    at = [[x for x in long] for _ in sets]
    for _ in range(6):
        xs = [tokens(n) for _ in sets]
        for (d, e, *_), x in zip(sets, xs):
            _set(d.x, x)
            _set(e.x, x)
        torch.cuda.synchronize()
        for st, graph in zip(streams, graphs):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for i, (d, e, pos, one, batch) in enumerate(sets):
            e.cache.extend(one, n)
            want = R.unblocked(e.step(None, R.i32(at[i]), **batch))
            at[i] = [x + 1 for x in at[i]]
            assert pos.tolist() == at[i] and e.cache.lengths.tolist() == at[i] == d.cache.lengths.tolist()
            assert want.isfinite().all() and torch.equal(R.unblocked(d.y), want)
            for a, b in zip(d.cache.k + d.cache.v + d.cache.k_scale + d.cache.v_scale,
                            e.cache.k + e.cache.v + e.cache.k_scale + e.cache.v_scale):
                assert torch.equal(a.bytes(), b.bytes())


@pytest.mark.parametrize("code,page,block", [("e4m3", 16, 8), ("e5m2", 20, None), ("e4m3", 20, 5)])
def test_a_forked_prompt_holds_what_it_held(code, page, block):
    """Continuations forked off a prompt, reordered and compacted on the way: the
    codes and scales of every sequence's prompt, in blocks that no later token goes
    to, are those of before, in the layer that is written and in the other one."""
    w, tokens = _weights(9)
    prefill = _share(PROMPT, w, tokens(PROMPT))
    prefill.forward()
    n, layer = 4, 1
    cache = KVCache(2, 64, HEADS_KV, page, 128, n, 20, dtype=code, block=block)
    g = torch.Generator(device="cuda").manual_seed(10)
    cache.data.bytes().copy_(torch.randint(0, 112, cache.data.bytes().shape, generator=g, device="cuda"))
    cache.scales.bytes().view(torch.int32).copy_(
        torch.randint(100, 140, (cache.scales.nbytes // 4,), generator=g, device="cuda") << 23)
    cache.extend(R.i32([0, 0, 6 * page, 0]), 1)  # of a sequence that goes: holes for compact to fill
    cache.extend(R.i32([PROMPT, 0, 0, 0]), PROMPT)
    prefill.store(cache, None, layer, q_start=R.i32([0] + [PROMPT] * n))
    b = block or page
    whole = torch.arange(PROMPT // b * b, device="cuda")

    def prompt(s):
        out = []
        for rel, scale in zip(cache.k + cache.v, cache.k_scale + cache.v_scale):
            pg = cache.table[s][whole // page].long()
            z = scale.bytes().view(torch.float32).view(scale.shape)
            out += [_codes(rel).view(torch.uint8)[pg, :, whole % page], z[pg, :, whole % page // b]]
        return out

    held = prompt(0)
    cache.select(R.i32([0, 0, -1, 0]))
    decode = LlamaBlockDecode(prefill, cache, 3, layer)
    shared = PROMPT // page * page
    batch = dict(q_start=R.i32([0, 1, 2, 2, 3]), group_start=R.i32([0, 2, 3, 4]), group_shared=R.i32([shared, 0, 0]))
    for i in range(12):
        if i == 5:
            cache.select(R.i32([3, 1, -1, 0]))
            table = cache.table.clone()
            cache.compact()
            assert not torch.equal(table, cache.table)
        slots, po = cache.extend(R.i32([1, 1, 0, 1]), 3)
        _set(decode.x, tokens(3))
        decode.step(slots, po, **batch)
        for s in (0, 1, 3):
            assert all(torch.equal(x, y) for x, y in zip(prompt(s), held)), (i, s)
