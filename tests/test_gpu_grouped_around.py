"""What lies between the rows of the grouped products' tensors: outputs leave it as it was, whatever their rows' length and distance, and what inputs have there (NaN) takes no part."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def whole(seed, shape, ld, dtype, around, offset=0):
    """Small whole numbers in rows ld apart (matrices one behind the other), `around` between them; the view and all of its memory"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = math.prod(shape[:-1])
    flat = torch.full((offset + rows * ld + 64,), around, dtype=dtype, device="cuda")
    view = flat[offset:offset + rows * ld].view(*shape[:-1], ld)[..., :shape[-1]]
    view.copy_(torch.randint(-2, 3, shape, generator=g, device="cuda"))
    return view, flat


# rows whose length is no multiple of 16 bytes, a distance apart that is: single blocks and pairs, slices, empty groups, rows of no group
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("sizes,width,out", [([20, 0, 131], 7, 5), ([20, 0, 131], 77, 330), ([3, 3], 4097, 331), ([0, 2000, 1500, 1], 509, 771), ([9000], 68, 141), ([1, 0, 1], 66, 3317),
                                             ([17] * 300, 15, 9), ([300], 33001, 60)], ids=str)
@pytest.mark.parametrize("offset", [0, 8])
def test_between_the_rows(ops, sizes, width, out, dtype, offset):
    first, groups = 5, len(sizes)
    ends = [first]
    for n in sizes:
        ends.append(ends[-1] + n)
    rows, to8 = ends[-1] + 21, lambda n: (n + 8) // 8 * 8
    x, dy, w = (whole(i, s, to8(s[-1]), dtype, math.nan, offset)[0] for i, s in enumerate([(rows, width), (rows, out), (groups, out, width)]))
    off = torch.tensor(ends, device="cuda")
    (y, fy), (dx, fdx) = (whole(3, s, to8(s[-1]), dtype, 7.0, offset) for s in ((rows, out), (rows, width)))
    y.fill_(7.0)
    dx.fill_(7.0)
    ops.grouped_linear(x, w, off, out=y)
    for t in (dtype, torch.float32):
        dw, fdw = whole(4, (groups, out, width), to8(width), t, 7.0, offset)
        dx.fill_(7.0)
        ops.grouped_linear_backward(dy, x, w, off, dx=dx, dweight=dw)
        ops.sync()
        for g in range(groups):
            p = slice(ends[g], ends[g + 1])
            a, m, d = x[p].double(), w[g].double(), dy[p].double()
            assert torch.equal(dw[g], (d.T @ a).float().to(t)), f"dweight of group {g}"
            assert torch.equal(dx[p], (d @ m).float().to(dtype)), f"dx of group {g}"
            assert torch.equal(y[p], (a @ m.T).float().to(dtype)), f"y of group {g}"
        dw.fill_(7.0)
        assert bool((fdw == 7).all()), "around dweight"
        dx[first:ends[-1]] = 7.0
        assert bool((fdx == 7).all()), "around dx"
    y[first:ends[-1]] = 7.0
    assert bool((fy == 7).all()), "around y"


@pytest.mark.parametrize("dtype", HALF, ids=str)
def test_columns_of_one_array(ops, dtype):
    """Two outputs beside one another in the rows of one array: each call writes its own columns."""
    off = torch.tensor([0, 40, 100], device="cuda")
    x = whole(1, (100, 64), 64, dtype, 0.0)[0]
    ws = [whole(2 + i, (2, n, 64), 64, dtype, 0.0)[0] for i, n in enumerate((20, 28))]
    both = torch.zeros(100, 48, dtype=dtype, device="cuda")
    for _ in range(2):                                               # either one last
        for at, w in ((0, ws[0]), (20, ws[1])):
            ops.grouped_linear(x, w, off, out=both[:, at:at + w.shape[1]])
        assert torch.equal(both[:, :20], ops.grouped_linear(x, ws[0], off)) and torch.equal(both[:, 20:], ops.grouped_linear(x, ws[1], off))
        ops.grouped_linear(x, ws[0], off, out=both[:, :20])
        assert torch.equal(both[:, 20:], ops.grouped_linear(x, ws[1], off))
