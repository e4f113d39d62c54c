"""The page table's calls against their definition, page by page: exact, over
random walks of extend, select and compact, and where they have to do nothing."""
import numpy as np
import pytest
import torch

import decode_ref as R
from paper_2609_03905_amd import ea

pytestmark = pytest.mark.gpu


class Device:
    """The same state on the device, and the calls."""

    def __init__(self, ref: R.Pages, caches=()):
        self.page = ref.page
        self.table, self.len, self.refs = R.i32(ref.table), R.i32(ref.len), R.i32(ref.refs)
        self.status = R.i32([9, 9])
        self.caches = list(caches)

    def extend(self, add, n_tokens, in_place=True):
        slots, pos = R.i32([7] * n_tokens), R.i32([7] * n_tokens)
        ol, orf = (self.len, self.refs) if in_place else (torch.empty_like(self.len), torch.empty_like(self.refs))
        before = self.len.clone(), self.refs.clone()
        ea.pages_extend(self.table, self.len, self.refs, R.i32(add), page_size=self.page, out_lengths=ol,
                        out_refs=orf, status=self.status, slots=slots, positions=pos)
        if not in_place:
            assert torch.equal(self.len, before[0]) and torch.equal(self.refs, before[1])
        self.len, self.refs = ol, orf
        return tuple(self.status.tolist()), slots.cpu().numpy(), pos.cpu().numpy()

    def select(self, parent):
        new = [torch.full_like(z, 5) for z in (self.table, self.len, self.refs)]
        ea.pages_select(self.caches, R.i32(parent), self.table, self.len, self.refs, out_table=new[0],
                        out_lengths=new[1], out_refs=new[2], status=self.status, page_size=self.page)
        self.table, self.len, self.refs = new
        return tuple(self.status.tolist())

    def compact(self, in_place=True):
        t, r = (self.table, self.refs) if in_place else (torch.full_like(self.table, 5), torch.full_like(self.refs, 5))
        ea.pages_compact(self.caches, self.table, self.len, self.refs, out_table=t, out_refs=r, status=self.status,
                         page_size=self.page)
        self.table, self.refs = t, r
        return tuple(self.status.tolist())

    def same(self, ref: R.Pages):
        assert np.array_equal(self.len.cpu().numpy(), ref.len)
        assert np.array_equal(self.refs.cpu().numpy(), ref.refs)
        t = self.table.cpu().numpy()
        for s, n in enumerate(ref.len):
            k = min(ref.held(max(n, 0)), ref.stride)
            assert np.array_equal(t[s, :k], ref.table[s, :k]), s


@pytest.mark.parametrize("n_seq,stride,n_pages,page,seed", [(1, 3, 4, 1, 0), (1, 1, 1, 16, 1), (5, 6, 17, 4, 2),
                                                            (40, 9, 300, 7, 3), (300, 5, 1025, 16, 4),
                                                            (7, 40, 5000, 3, 5),
                                                            (200, 60, 9000, 2, 6), (4, 5000, 3000, 2, 7)])
def test_random_walk(n_seq, stride, n_pages, page, seed):
    rng = np.random.default_rng(seed)
    planes = rng.integers(-30000, 30000, (2, n_pages, 2, page, 64)).astype(np.int16)
    data = torch.from_numpy(planes.copy()).cuda().view(torch.bfloat16)
    ref = R.Pages(n_seq, stride, n_pages, page, planes)
    # two caches of one plane each, or one of two
    if seed % 2:
        dev = Device(ref, [R.pages_rel(data)])
    else:
        a, b = data[0].clone(), data[1].clone()
        dev = Device(ref, [R.pages_rel(a), R.pages_rel(b)])
    seen = set()
    for step in range(24):
        op = rng.choice(["extend", "extend", "select", "compact"])
        if op == "extend":
            add = rng.integers(-1, max(2, stride * page // 3), n_seq)
            if rng.random() < 0.3:
                add = rng.integers(0, 2, n_seq)
            n_tokens = int(max(0, int(np.maximum(add, 0).sum()) + rng.integers(-2, 4)))
            want, got = ref.extend(add, n_tokens), dev.extend(add, n_tokens, in_place=step % 2 == 0)
            assert got[0] == want[0]
            assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
            code = want[0]
        elif op == "select":
            parent = rng.integers(-1, n_seq + 1, n_seq)
            if rng.random() < 0.3:
                parent = rng.permutation(n_seq)
            code = ref.select(parent)
            assert dev.select(parent) == code
        else:
            code = ref.compact()
            assert dev.compact(in_place=step % 2 == 0) == code
        seen.add((op, code[0]))
        dev.same(ref)
        # the held rows of every sequence, in every plane
        got = data.view(torch.int16).cpu().numpy() if seed % 2 else \
            np.stack([a.view(torch.int16).cpu().numpy(), b.view(torch.int16).cpu().numpy()])
        assert np.array_equal(got, ref.planes), op
    assert len(seen) > 1


def test_nothing_is_done_without_pages():
    """One page short: the state goes through as it came, in every output."""
    ref = R.Pages(3, 4, 6, 8)
    dev = Device(ref)
    assert dev.extend([8, 9, 17], 34)[0] == ref.extend([8, 9, 17], 34)[0] == (ea.PAGES_OK, 0)
    for add in ([0, 8, 0], [8, 7, 7]):
        want, got = ref.extend(add, 4), dev.extend(add, 4, in_place=False)
        assert got[0] == want[0] == (ea.PAGES_NONE_FREE, 0)
        assert (got[1] == -1).all() and (got[2] == 0).all()
        dev.same(ref)
    assert dev.select([1, 1, 2]) == ref.select([1, 1, 2]) == (ea.PAGES_OK, 0)  # the freed page serves the copy
    dev.same(ref)
    assert dev.select([2, 2, 2]) == ref.select([2, 2, 2])
    dev.same(ref)


@pytest.mark.parametrize("in_place", [True, False])
def test_more_pages_than_one_round_hands_out(in_place):
    """9000 new pages in one call, the cache a third full of holes, page counts
    that no four divides."""
    n, stride, n_pages, page = 3, 4000, 13001, 2
    ref = R.Pages(n, stride, n_pages, page)
    ref.refs[1::3] = 1  # held by somebody else
    ref.len[1], ref.table[1, 0], ref.refs[5] = 1, 5, 1
    dev = Device(ref)
    for add in ([6000, 3999, 3001], [0, 0, 4300], [1, 1, 1]):
        want, got = ref.extend(add, sum(add) + 5), dev.extend(add, sum(add) + 5, in_place)
        assert got[0] == want[0] and np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
        dev.same(ref)


@pytest.mark.parametrize("n_pages", [4096, 16384, 16385, 40000])
def test_few_free_places_of_many(n_pages):
    """Free pages at the ends of blocks of pages, and one short of enough."""
    ref = R.Pages(5, 20, n_pages, 3)
    ref.refs[:] = 1
    places = sorted({0, 4095, n_pages // 2, n_pages - 4, n_pages - 1} | ({4096, 8191, 8192, 16383} if n_pages > 16384
                                                                       else set()))
    ref.refs[places] = 0
    dev = Device(ref)
    for add in ([0, 3, 1, 0, 0], [1, 0, 0, 0, 4], [60, 0, 0, 0, 0], [3] * 5):
        want, got = ref.extend(add, sum(add)), dev.extend(add, sum(add), in_place=n_pages % 2 == 0)
        assert got[0] == want[0] and np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
        dev.same(ref)


def test_a_fork_over_a_large_table_that_fits_nowhere():
    ref = R.Pages(4, 5000, 100, 4)
    dev = Device(ref)
    assert dev.extend([200, 99, 99, 0], 0)[0] == ref.extend([200, 99, 99, 0], 0)[0] == (ea.PAGES_OK, 0)
    assert dev.select([0, 1, 2, 1]) == ref.select([0, 1, 2, 1]) == (ea.PAGES_NONE_FREE, 0)
    dev.same(ref)
    assert dev.select([0, 1, 0, 1]) == ref.select([0, 1, 0, 1]) == (ea.PAGES_OK, 24)
    dev.same(ref)


def test_a_fork_that_fits_nowhere_does_nothing():
    ref = R.Pages(2, 3, 2, 4)
    dev = Device(ref)
    for add in ([3, 0], [0, 3]):
        assert dev.extend(add, 0)[0] == ref.extend(add, 0)[0]
    ref2 = R.Pages(3, 3, 2, 4)
    ref2.table[:2], ref2.len[:2], ref2.refs[:] = ref.table, ref.len, ref.refs
    dev2 = Device(ref2)
    assert dev2.select([0, 1, 1]) == ref2.select([0, 1, 1]) == (ea.PAGES_NONE_FREE, 0)
    dev2.same(ref2)


def test_lengths_that_no_row_holds():
    ref = R.Pages(2, 2, 8, 4)
    ref.len[:] = [9, 3]
    ref.table[1, 0], ref.refs[0] = 0, 1
    dev = Device(ref)
    assert dev.extend([0, 1], 1)[0] == ref.extend([0, 1], 1)[0] == (ea.PAGES_TOO_LONG, 7)
    assert dev.select([1, 0]) == ref.select([1, 0]) == (ea.PAGES_TOO_LONG, 7)
    dev.same(ref)
    ref.len[:] = dev_len = np.asarray([-1, 3], np.int32)
    dev.len = R.i32(dev_len)
    assert dev.extend([1, 1], 1)[0] == ref.extend([1, 1], 1)[0] == (ea.PAGES_TOO_LONG, 7)
    dev.same(ref)


def test_entries_outside_the_cache():
    """A table entry that names no page counts none, copies none and is kept."""
    ref = R.Pages(3, 3, 9, 4, np.arange(9 * 4 * 32, dtype=np.int16).reshape(1, 9, 1, 4, 32))
    ref.len[:] = [7, 4, 2]
    ref.table[0, :2], ref.table[1, :1], ref.table[2, :1] = [-4, 100], [8], [2 ** 30]
    ref.refs[8] = 1
    data = torch.from_numpy(ref.planes.copy()).cuda().view(torch.bfloat16)
    dev = Device(ref, [R.pages_rel(data)])
    assert dev.extend([1, 0, 1], 2)[0] == ref.extend([1, 0, 1], 2)[0]
    assert dev.select([0, 0, 2]) == ref.select([0, 0, 2])
    dev.same(ref)
    assert dev.compact() == ref.compact()
    dev.same(ref)
    assert np.array_equal(data.view(torch.int16).cpu().numpy(), ref.planes)


def test_pages_with_padding_between_them():
    """Pages of 48 and 80 bytes, each at a 256-byte multiple."""
    for d, heads in ((8, 1), (40, 1)):
        planes = np.random.default_rng(d).integers(0, 30000, (3, 11, heads, 3, d)).astype(np.int16)
        ref = R.Pages(4, 4, 11, 3, planes)
        cache = R.pages_rel(torch.from_numpy(planes.copy()).cuda().view(torch.bfloat16))
        dev = Device(ref, [cache])
        assert dev.extend([4, 2, 7, 1], 14)[0] == ref.extend([4, 2, 7, 1], 14)[0]
        assert dev.select([0, 0, 2, -1]) == ref.select([0, 0, 2, -1])
        assert dev.select([-1, 1, 0, 1]) == ref.select([-1, 1, 0, 1])
        assert dev.compact() == ref.compact()
        dev.same(ref)
        assert np.array_equal(R.unblocked(cache).view(torch.int16).cpu().numpy(), ref.planes)


def test_captured_step():
    """extend and select captured into one graph and replayed: every replay is
    the definition's."""
    n, stride, n_pages, page = 6, 8, 60, 4
    ref = R.Pages(n, stride, n_pages, page)
    table, ln, refs = R.i32(ref.table), R.i32(ref.len), R.i32(ref.refs)
    t2, l2, r2 = torch.empty_like(table), torch.empty_like(ln), torch.empty_like(refs)
    add, parent = R.i32([1, 2, 3, 0, 1, 5]), R.i32([0, 0, 2, 3, -1, 5])
    st, ws = R.i32([0, 0]), ea.new_workspace(1 << 20)

    def step():
        ea.pages_extend(table, ln, refs, add, page_size=page, status=st, workspace=ws)
        ea.pages_select([], parent, table, ln, refs, out_table=t2, out_lengths=l2, out_refs=r2, status=st,
                        page_size=page, workspace=ws)
        table.copy_(t2), ln.copy_(l2), refs.copy_(r2)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        ref.extend(add.tolist(), 0)
        code = ref.select(parent.tolist())
        assert tuple(st.tolist()) == code
        assert np.array_equal(table.cpu().numpy(), ref.table) and np.array_equal(refs.cpu().numpy(), ref.refs)
        assert torch.equal(ln.cpu(), torch.from_numpy(ref.len))


def test_pages_past_4_gib():
    """Copies and moves between pages whose byte offsets pass 2^32, in two
    planes; a page of several pieces."""
    heads, page, d, n_pages = 8, 100, 128, 12000
    cache = torch.empty((2, n_pages, heads, page, d), device="cuda", dtype=torch.bfloat16)
    assert cache[0].numel() * 2 > 2 << 30 and cache.numel() * 2 > 1 << 32
    rel = R.pages_rel(cache)
    table, ln = R.i32([[n_pages - 1, n_pages - 2], [-1, -1]]), R.i32([page + 37, 0])
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    refs[n_pages - 7] = 0  # the only free place
    cache[:, n_pages - 2:] = torch.randn((2, 2, heads, page, d), device="cuda").to(torch.bfloat16)
    cache[:, n_pages - 7] = 5.0
    want = cache[:, n_pages - 2, :, :37].clone()
    t2, l2, r2, st = torch.empty_like(table), torch.empty_like(ln), torch.empty_like(refs), R.i32([9, 9])
    ea.pages_select([rel], R.i32([0, 0]), table, ln, refs, out_table=t2, out_lengths=l2, out_refs=r2, status=st)
    assert st.tolist() == [ea.PAGES_OK, 0]
    assert t2.tolist() == [[n_pages - 1, n_pages - 2], [n_pages - 1, n_pages - 7]] and l2.tolist() == [page + 37] * 2
    assert torch.equal(cache[:, n_pages - 7, :, :37], want) and (cache[:, n_pages - 7, :, 37:] == 5.0).all()
    assert r2[n_pages - 1] == 2 and r2[n_pages - 7] == 1
    # three places of the first pages become free: the last three used pages move there
    r2[[2, 9, 11]] = 0
    last = cache[:, n_pages - 3:].clone()
    ea.pages_compact([rel], t2, l2, r2, status=st)
    assert st.tolist() == [ea.PAGES_OK, 3] and t2.tolist() == [[11, 9], [11, n_pages - 7]]
    assert all(torch.equal(cache[:, p], last[:, i]) for i, p in enumerate((2, 9, 11)))
    assert r2[:n_pages - 3].min() == 1 and r2[11] == 2 and not r2[n_pages - 3:].any()


def test_positions_alone_and_nothing_wanted():
    ref = R.Pages(3, 4, 9, 4)
    t, ln, rf, st = R.i32(ref.table), R.i32(ref.len), R.i32(ref.refs), R.i32([9, 9])
    pos = R.i32([7] * 6)
    ea.pages_extend(t, ln, rf, R.i32([2, 0, 3]), page_size=4, status=st, positions=pos)
    assert pos.tolist() == [0, 1, 0, 1, 2, 0] and st.tolist() == [ea.PAGES_OK, 7]
    ea.pages_extend(t, ln, rf, R.i32([3, 1, 0]), page_size=4, status=st)
    assert ln.tolist() == [5, 1, 3] and t[0, :2].tolist() == [0, 2] and t[1, 0] == 3 and st.tolist() == [0, 5]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("length", [-1, -2 ** 31, 3 * 4 + 1, 2 ** 31 - 1, 2 ** 31 - 4])
def test_compact_of_lengths_that_no_row_holds(length, in_place):
    """Nothing is done: table, counts and pages stay as they came, entries behind
    the sequences' pages too."""
    data = torch.randn((2, 9, 1, 4, 32), device="cuda").to(torch.bfloat16)
    table = R.i32([[7, 8, 5], [6, 3, 11]])
    lengths, refs, status = R.i32([9, length]), R.i32([0, 0, 0, 1, 0, 1, 1, 1, 1]), R.i32([9, 9])
    kept = [z.clone() for z in (data, table, lengths, refs)]
    t, r = (table, refs) if in_place else (torch.full_like(table, 5), torch.full_like(refs, 5))
    ea.pages_compact([R.pages_rel(data)], table, lengths, refs, out_table=t, out_refs=r, status=status)
    assert status.tolist() == [ea.PAGES_TOO_LONG, 4]
    for got, want in zip((data, table, lengths, refs), kept):
        assert torch.equal(got.view(torch.uint8) if got.dtype == torch.bfloat16 else got,
                           want.view(torch.uint8) if want.dtype == torch.bfloat16 else want)
    assert torch.equal(t, kept[1]) and torch.equal(r, kept[3])
    # with a length that the row holds, the same call moves the pages together
    lengths[1] = 8
    ea.pages_compact([R.pages_rel(data)], table, lengths, refs, out_table=t, out_refs=r, status=status)
    assert status.tolist() == [ea.PAGES_OK, 4] and r.tolist() == [1] * 5 + [0] * 4
    assert t.tolist() == [[2, 4, 0], [1, 3, -1]]  # pages 5, 6, 7, 8 to 0, 1, 2, 4
