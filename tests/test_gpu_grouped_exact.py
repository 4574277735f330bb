"""Products grouped by expert of small whole numbers, whose sums 32 bits hold exactly however they are split: every row counts once, whatever the length of the sum, so a row lost or
taken twice where slices, stages or groups meet shows, which a bound that grows with the length would let pass.

No tolerance: magnitudes are at most 2, so that sums of 2^21 products stay below 2^24, and the outputs are those sums rounded once, to nearest.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def whole(seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(dtype)


def check(ops, sizes, first, behind, width, out, dtype):
    ends = [first]
    for n in sizes:
        ends.append(ends[-1] + n)
    rows, groups = ends[-1] + behind, len(sizes)
    x, w, dy = whole(1, rows, width, dtype=dtype), whole(2, groups, out, width, dtype=dtype), whole(3, rows, out, dtype=dtype)
    x[:, 0] = 2.0                                                    # a column of one sign: every row of dy adds to it
    off = torch.tensor(ends, device="cuda")
    wide = torch.full(w.shape, 7.0, device="cuda")
    y = ops.grouped_linear(x, w, off)
    dx, dw = ops.grouped_linear_backward(dy, x, w, off)
    _, wide = ops.grouped_linear_backward(dy, x, w, off, dx=False, dweight=wide)
    ops.sync()
    for g in range(groups):
        p = slice(ends[g], ends[g + 1])
        xd, wd, dd = x[p].double(), w[g].double(), dy[p].double()
        assert torch.equal(y[p], (xd @ wd.T).float().to(dtype)), f"y of group {g}"
        assert torch.equal(dx[p], (dd @ wd).float().to(dtype)), f"dx of group {g}"
        want = (dd.T @ xd).float()
        assert torch.equal(wide[g], want) and torch.equal(dw[g], want.to(dtype)), f"dweight of group {g}"


# groups cut into slices of rows, at borders of stages, beside them and far from them
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("sizes", [[1025], [6000], [5000, 0, 130, 2000], [64, 4097, 1, 63, 65, 0], [3000] * 5, [1030] + [7] * 40, [21000] + [7] * 40, [33333, 1, 20011]], ids=str)
@pytest.mark.parametrize("width,out", [(64, 200), (300, 260), (333, 40), (768, 512)])
def test_slices_of_rows(ops, sizes, width, out, dtype):
    check(ops, sizes, 5, 70, width, out, dtype)


# K cut into slices
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("sizes", [[1], [5, 0, 2], [0, 17, 33, 0], [300]], ids=str)
@pytest.mark.parametrize("width,out", [(4096, 200), (200, 4096), (3413, 77), (77, 3413), (2050, 1024), (1087, 1025), (9001, 65)])
def test_slices_of_k(ops, sizes, width, out, dtype):
    check(ops, sizes, 3, 4, width, out, dtype)


# whole sums, outputs through the workspace, many groups, parts
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("sizes,width,out", [([700, 0, 33, 0, 1, 1500, 0], 1001, 1333), ([513, 511, 90, 1, 0, 64], 512, 768), ([i * 7 % 5 for i in range(2048)], 64, 40),
                                             ([i * 37 % 301 for i in range(300)], 72, 136), ([140_000, 3], 64, 2100), ([0, 200_001, 77] + [1] * 290, 136, 64), ([130], 33000, 600),
                                             ([40, 90], 140_000, 5000), ([900, 0, 333], 33_001, 2101), ([1100], 131_075, 2101)], ids=lambda v: str(v)[:40])
def test_whole_sums(ops, sizes, width, out, dtype):
    check(ops, sizes, 11, 30, width, out, dtype)
