"""Relations of one byte an element are repartitioned byte by byte: odd extents,
blocks that begin at any byte of a row, rows that no wide copy fits."""
import numpy as np
import pytest
import torch

import cache8_ref as C
from paper_2609_03905_amd import ea

pytestmark = pytest.mark.gpu

FILL = 0xAA


def _cuts(n, at):
    return [0] + sorted({x for x in at if 0 < x < n}) + [n]


def _filled(shape, code, part):
    r = ea.Relation(shape, code, part)
    r.bytes().fill_(FILL)
    return r


def _expected(x, rel):
    """The relation's bytes: every block row-major at its offset, the rest as it was."""
    out = np.full(rel.nbytes, FILL, np.uint8)
    for b in range(rel.num_blocks()):
        lo, hi, at = rel.block(b)
        block = x[tuple(slice(i, j) for i, j in zip(lo, hi))]
        out[at:at + block.size] = block.reshape(-1)
    return out


CASES = [
    ((1,), [[0, 1]], [[0, 1]]),
    ((1000,), [_cuts(1000, [1, 2, 5, 333])], [_cuts(1000, [7, 512, 999])]),
    ((7, 13), [[0, 7], [0, 13]], [_cuts(7, range(7)), _cuts(13, [1, 4, 9])]),
    ((65, 131), [_cuts(65, [16, 33]), _cuts(131, [64, 127])], [_cuts(65, [1, 64]), _cuts(131, [3, 66, 130])]),
    ((3, 40001), [_cuts(3, [1]), [0, 40001]], [[0, 3], _cuts(40001, [1, 16385, 32768])]),
    ((5, 6, 17), [_cuts(5, [2]), _cuts(6, [1, 3]), [0, 17]], [[0, 5], _cuts(6, [2]), _cuts(17, [5, 16])]),
    ((9, 3, 20, 96), [list(range(10)), [0, 3], [0, 20], [0, 96]], [[0, 9], _cuts(3, [1]), _cuts(20, [7]), [0, 96]]),
    ((9, 3, 20, 96), [[0, 9], [0, 3], [0, 20], [0, 96]], [list(range(10)), [0, 3], [0, 20], [0, 96]]),
    ((2, 3, 5, 7, 11), [[0, 2], [0, 3], _cuts(5, [1, 2]), [0, 7], [0, 11]],
     [_cuts(2, [1]), [0, 3], [0, 5], _cuts(7, [3]), _cuts(11, [10])]),
]


@pytest.mark.parametrize("code", ["e4m3", "e5m2"])
@pytest.mark.parametrize("shape,a,b", CASES, ids=["x".join(map(str, c[0])) + f"_{i}" for i, c in enumerate(CASES)])
def test_blocks_of_one_byte_elements(shape, a, b, code):
    x = np.random.default_rng(1).integers(0, 256, shape, np.uint8)
    dense = torch.from_numpy(x).cuda()
    src = _filled(shape, code, a)
    ea.repartition(ea.Relation(shape, code, ea.whole_partition(shape), data=dense.reshape(-1)), src)
    assert np.array_equal(src.bytes().cpu().numpy(), _expected(x, src))
    for store in (0, 1):  # cached and streamed stores
        dst = _filled(shape, code, b)
        ea.repartition(src, dst, store=store)
        assert np.array_equal(dst.bytes().cpu().numpy(), _expected(x, dst))
    rel = ea.from_dense(dense.view(C.TORCH[code]), code, b)
    assert np.array_equal(ea.to_dense(rel).cpu().numpy(), x.reshape(-1))


def test_large_blocks_of_one_byte_elements():
    """Many tasks of boxes that no wide copy fits, and of ones that it does."""
    for shape, a, b in [((4099, 4097), [[0, 4099], [0, 4097]], [_cuts(4099, [2048]), _cuts(4097, [1, 2050])]),
                        ((4096, 4352), [[0, 4096], _cuts(4352, [256])], [_cuts(4096, [1000]), _cuts(4352, [4096])])]:
        x = torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda")
        src = ea.from_dense(x, "e4m3", a)
        dst = ea.Relation(shape, "e4m3", b)
        ea.repartition(src, dst)
        assert torch.equal(ea.to_dense(dst).view(shape), x)


def test_captured_with_one_byte_elements():
    shape, a, b = (33, 3, 20, 96), [list(range(34)), [0, 3], [0, 20], [0, 96]], [[0, 33], _cuts(3, [1]), [0, 20], _cuts(96, [5])]
    src, dst = _filled(shape, "e5m2", a), _filled(shape, "e5m2", b)
    ea.repartition(src, dst)  # planned
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ea.repartition(src, dst)
    for _ in range(3):
        x = torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda")
        ea.repartition(ea.Relation(shape, "e5m2", ea.whole_partition(shape), data=x.view(-1)), src)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ea.to_dense(dst).view(shape), x)


@pytest.mark.parametrize("dtype,n", [("e4m3", 2 ** 31 - 1), ("bf16", 2 ** 30 - 8), ("f32", 2 ** 29 - 4)])
def test_a_box_of_all_bytes_that_31_bits_count(dtype, n):
    """The last task of a box of almost 2^31 bytes, of bytes and of 16 at a time: no
    thread goes on behind it."""
    src, dst = (ea.Relation((n,), dtype, [[0, n]]) for _ in range(2))
    assert src.nbytes > 2 ** 31 - 2 ** 14
    g = torch.Generator(device="cuda").manual_seed(3)
    for at in range(0, src.nbytes, 2 ** 28):
        src.bytes()[at:at + 2 ** 28].random_(0, 256, generator=g)
    dst.bytes().fill_(FILL)
    ea.repartition(src, dst)
    assert torch.equal(src.bytes(), dst.bytes())
