"""Products grouped by expert against plain ones in 64 bits, and the order that they take.

Tolerances before any run: u is half a step of the output's type; 32-bit sums of K products on the tensor cores, which may truncate instead of rounding,
are off by at most 2 (K + 4) 2^-24 times the sum of the magnitudes.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def randn(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def within(got, want, bound, what):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    over = ((got - want).abs() - bound).nan_to_num(0.0, posinf=math.inf, neginf=-math.inf)
    assert float(over.max() if over.numel() else 0.0) <= 0.0, (what, float(over.max()))


def product(a, b, dtype):
    """a b^T in 64 bits and what it may be off by"""
    a, b = a.double(), b.double()
    want = a @ b.T
    e = 2 * (a.shape[1] + 4) * 2.0 ** -24 * (a.abs() @ b.abs().T)
    return want, e + U[dtype] * (want.abs() + e) + TINY[dtype]


def ends(sizes, first=0):
    out = [first]
    for s in sizes:
        out.append(out[-1] + s)
    return out


def offsets_of(e):
    return torch.tensor(e, dtype=torch.int64, device="cuda")


def check(ops, e, rows, width, out, dtype, x=None, w=None, dy=None, dweight_type=None):
    groups = len(e) - 1
    x = randn(1, rows, width, dtype=dtype) if x is None else x
    w = randn(2, groups, out, width, dtype=dtype) if w is None else w
    dy = randn(3, rows, out, dtype=dtype) if dy is None else dy
    off = offsets_of(e)
    y = ops.grouped_linear(x, w, off)
    given = torch.full(w.shape, math.nan, dtype=dweight_type, device="cuda") if dweight_type else None
    dx, dw = ops.grouped_linear_backward(dy, x, w, off, dweight=given)
    ops.sync()
    assert y.shape == (rows, out) and y.dtype == dtype and dx.shape == x.shape and dw.shape == w.shape
    for g in range(groups):
        p = slice(e[g], e[g + 1])
        within(y[p], *product(x[p], w[g], dtype), f"y of group {g}")
        within(dx[p], *product(dy[p], w[g].T, dtype), f"dx of group {g}")
        within(dw[g], *product(dy[p].T, x[p].T, dw.dtype), f"dweight of group {g}")
    outside = torch.ones(rows, dtype=torch.bool, device="cuda")
    outside[e[0]:e[-1]] = False
    assert not y[outside].any() and not dx[outside].any()
    return y, dx, dw


# group sizes beside every border of the tiles (8, 16, 32, 64, 128, 256) and of a stage of K, empty ones at both ends and between
SIZES = [[1], [0, 1, 0], [5, 0, 0, 3], [16, 17, 15], [31, 32, 33, 0], [63, 64, 65], [127, 128, 129], [255, 256, 257], [300, 1, 0, 700, 2], [513, 511, 90], [1000], [8] * 40]


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("width,out", [(64, 64), (72, 136), (768, 256), (8, 520)])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_group_sizes(ops, sizes, width, out, dtype):
    e = ends(sizes)
    check(ops, e, e[-1], width, out, dtype)


# rows TMA cannot address, extents that end inside every tile and instruction
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("width,out", [(1, 1), (1, 77), (77, 1), (63, 65), (65, 63), (130, 129), (17, 400), (257, 255), (1001, 333)])
def test_odd_extents(ops, width, out, dtype):
    e = ends([3, 0, 70, 131])
    check(ops, e, e[-1], width, out, dtype)


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("first,behind", [(0, 9), (5, 0), (3, 300), (70, 1)])
def test_rows_of_no_group(ops, first, behind, dtype):
    e = ends([40, 0, 33], first)
    rows = e[-1] + behind
    x, dy = randn(1, rows, 96, dtype=dtype), randn(3, rows, 200, dtype=dtype)
    outside = torch.ones(rows, dtype=torch.bool, device="cuda")
    outside[e[0]:e[-1]] = False
    x[outside], dy[outside] = math.nan, math.inf                     # they may hold anything
    y, dx, dw = check(ops, e, rows, 96, 200, dtype, x=x, dy=dy)
    # given outputs keep what they had there
    w, off = randn(2, 3, 200, 96, dtype=dtype), offsets_of(e)
    oy, ox = torch.full_like(y, 7.0), torch.full_like(dx, 5.0)
    assert ops.grouped_linear(x, w, off, out=oy) is oy
    got = ops.grouped_linear_backward(dy, x, w, off, dx=ox, dweight=False)
    assert got[0] is ox and got[1] is None
    assert bool((oy[outside] == 7).all()) and bool((ox[outside] == 5).all())
    assert torch.equal(oy[~outside], y[~outside]) and torch.equal(ox[~outside], dx[~outside])


def test_no_group_has_a_row(ops):
    x, dy = randn(1, 50, 64, dtype=torch.bfloat16), randn(3, 50, 72, dtype=torch.bfloat16)
    for e in ([0, 0, 0], [50, 50, 50], [20, 20, 20]):
        check(ops, e, 50, 64, 72, torch.bfloat16, x=x, dy=dy)


@pytest.mark.parametrize("dtype", HALF, ids=str)
def test_no_rows(ops, dtype):
    x, dy, w = torch.empty(0, 64, dtype=dtype, device="cuda"), torch.empty(0, 40, dtype=dtype, device="cuda"), randn(1, 3, 40, 64, dtype=dtype)
    off = offsets_of([0, 0, 0, 0])
    assert ops.grouped_linear(x, w, off).shape == (0, 40)
    dx, dw = ops.grouped_linear_backward(dy, x, w, off)
    assert dx.shape == (0, 64) and not dw.any()
    wide = torch.full((3, 40, 100), 3.0, dtype=torch.float32, device="cuda")
    ops.grouped_linear_backward(dy, x, w, off, dweight=wide[:, :, 10:74])
    assert not wide[:, :, 10:74].any() and bool((wide[:, :, :10] == 3).all()) and bool((wide[:, :, 74:] == 3).all())


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("width,out", [(64, 128), (200, 300), (1001, 130)])
def test_what_a_neighbouring_group_holds_does_not_matter(ops, width, out, dtype):
    """Infinities and NaN in one group's rows and matrix reach nothing of the others."""
    e = ends([37, 50, 3, 129])
    x, w, dy, off = randn(1, e[-1], width, dtype=dtype), randn(2, 4, out, width, dtype=dtype), randn(3, e[-1], out, dtype=dtype), offsets_of(e)
    want = [ops.grouped_linear(x, w, off), *ops.grouped_linear_backward(dy, x, w, off)]
    for bad in range(4):
        x2, w2, dy2 = x.clone(), w.clone(), dy.clone()
        p = slice(e[bad], e[bad + 1])
        x2[p], dy2[p], w2[bad] = math.nan, math.inf, math.nan
        y, dx, dw = ops.grouped_linear(x2, w2, off), *ops.grouped_linear_backward(dy2, x2, w2, off)
        others = torch.ones(e[-1], dtype=torch.bool, device="cuda")
        others[p] = False
        assert torch.equal(y[others], want[0][others]) and torch.equal(dx[others], want[1][others])
        for g in range(4):
            assert g == bad or torch.equal(dw[g], want[2][g])
        assert bool(torch.isnan(y[p]).all()) and bool(torch.isnan(dw[bad]).all())


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("width,out", [(64, 96), (136, 250), (33, 77)])
def test_gradients_of_the_matrices_in_32_bits(ops, width, out, dtype):
    check(ops, ends([0, 5, 200, 64, 1100]), 1369, width, out, dtype, dweight_type=torch.float32)


@pytest.mark.parametrize("dtype", HALF, ids=str)
def test_long_groups_in_32_bits(ops, dtype):
    """Sums over many rows of one sign: parts of 1024 rows are added with rounding, so that the truncation stays that of a part:
    2^-24 for each of 64 additions of 16 products, and rounding of the sum of the parts."""
    rows, width, out = 20000, 64, 128
    x, dy = randn(1, rows, width, dtype=dtype).abs(), randn(3, rows, out, dtype=dtype).abs()
    w, off = randn(2, 1, out, width, dtype=dtype), offsets_of([0, rows])
    dw = torch.empty(1, out, width, device="cuda")
    ops.grouped_linear_backward(dy, x, w, off, dx=False, dweight=dw)
    want = dy.double().T @ x.double()
    # fp16 products and their alignment lose up to 4 times what bf16's do
    bound = (2 * 64 * (4 if dtype == torch.float16 else 1) + 20) * 2.0 ** -24
    assert float(((dw[0].double() - want).abs() / want).max()) <= bound


# few tiles and many rows: a group's rows are shared out among several blocks and the sums joined
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("sizes", [[1025], [6000], [5000, 0, 130, 2000], [64, 4097, 1, 63, 65, 0], [3000] * 5, [1030] + [7] * 40, [21000] + [7] * 40], ids=str)
@pytest.mark.parametrize("width,out", [(64, 200), (300, 260), (333, 40), (768, 512)])
def test_long_groups_of_small_matrices(ops, sizes, width, out, dtype):
    e = ends(sizes, 5)
    check(ops, e, e[-1] + 70, width, out, dtype)
    check(ops, e, e[-1] + 70, width, out, dtype, dweight_type=torch.float32)


# few rows and long sums: K in slices
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("sizes", [[1], [5, 0, 2], [0, 17, 33, 0], [128, 1], [300]], ids=str)
@pytest.mark.parametrize("width,out", [(4096, 200), (200, 4096), (3413, 77), (77, 3413), (2050, 1024), (1087, 1025)])
def test_few_rows_and_long_sums(ops, sizes, width, out, dtype):
    e = ends(sizes, 3)
    rows = e[-1] + 4
    x, dy = randn(1, rows, width, dtype=dtype), randn(3, rows, out, dtype=dtype)
    y, dx, _ = check(ops, e, rows, width, out, dtype, x=x, dy=dy)
    w, off = randn(2, len(sizes), out, width, dtype=dtype), offsets_of(e)
    oy, ox = torch.full_like(y, 7.0), torch.full_like(dx, 5.0)
    ops.grouped_linear(x, w, off, out=oy)
    ops.grouped_linear_backward(dy, x, w, off, dx=ox, dweight=False)
    for o, t, v in ((oy, y, 7), (ox, dx, 5)):
        assert torch.equal(o[e[0]:e[-1]], t[e[0]:e[-1]]) and bool((o[:e[0]] == v).all()) and bool((o[e[-1]:] == v).all())


# outputs of some megabytes whose rows the copy engine cannot write, or that begin off its boundaries
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("width,out", [(1001, 1333), (1002, 1334), (1004, 1340), (2049, 515), (75, 3001), (1400, 1416)])
def test_large_outputs_of_odd_rows(ops, width, out, dtype):
    e = ends([700, 0, 33, 0, 1, 1500, 0], 11)
    y, dx, dw = check(ops, e, e[-1] + 300, width, out, dtype)
    check(ops, e, e[-1] + 300, width, out, dtype, dweight_type=torch.float32)
    x, w, dy, off = randn(1, e[-1] + 300, width, dtype=dtype), randn(2, 7, out, width, dtype=dtype), randn(3, e[-1] + 300, out, dtype=dtype), offsets_of(e)
    outside = torch.ones(len(x), dtype=torch.bool, device="cuda")
    outside[e[0]:e[-1]] = False
    for at in (0, 1, 3, 8):                                          # given, from another boundary, with something around them that stays
        flat = [torch.full((at + t.numel() + 40,), 6.0, dtype=dtype, device="cuda") for t in (y, dx, dw)]
        oy, ox, ow = (f[at:at + t.numel()].view(t.shape) for f, t in zip(flat, (y, dx, dw)))
        ops.grouped_linear(x, w, off, out=oy)
        ops.grouped_linear_backward(dy, x, w, off, dx=ox, dweight=ow)
        assert torch.equal(oy[~outside], y[~outside]) and torch.equal(ox[~outside], dx[~outside]) and torch.equal(ow, dw)
        assert bool((oy[outside] == 6).all()) and bool((ox[outside] == 6).all())
        assert all(bool((f[:at] == 6).all()) and bool((f[-40:] == 6).all()) for f in flat)
    ops.sync()


@pytest.mark.parametrize("dtype", HALF, ids=str)
def test_large_gradients_of_few_groups_with_odd_rows(ops, dtype):
    """K split, the sums joined and the rows put together."""
    for dweight_type in (None, torch.float32):
        check(ops, ends([9000]), 9000, 1501, 1777, dtype, dweight_type=dweight_type)
        check(ops, ends([5000, 0, 100]), 5100, 777, 1503, dtype, dweight_type=dweight_type)


def views(dtype, rows, cols, pad, offset, seed):
    """A matrix whose rows are cols + pad apart and begin off any boundary, and the same numbers alone"""
    whole = randn(seed, rows * (cols + pad) + offset, dtype=dtype)
    v = whole[offset:].view(rows, cols + pad)[:, :cols]
    return v


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("pad,offset", [(8, 0), (3, 0), (0, 1), (24, 8), (5, 3)])
def test_strides_and_offsets(ops, pad, offset, dtype):
    e = ends([20, 0, 131])
    rows, width, out, off = 151, 104, 72, offsets_of(e)
    x, dy = views(dtype, rows, width, pad, offset, 1), views(dtype, rows, out, pad, offset, 2)
    w = views(dtype, 3 * out, width, pad, offset, 3)
    w = w.as_strided((3, out, width), (out * w.stride(0), w.stride(0), 1))
    want = [ops.grouped_linear(x.contiguous(), w.contiguous(), off), *ops.grouped_linear_backward(dy.contiguous(), x.contiguous(), w.contiguous(), off)]
    y, dx = views(dtype, rows, out, pad, offset, 4).zero_(), views(dtype, rows, width, pad, offset, 5).zero_()
    dw = views(dtype, 3 * out, width, pad, offset, 6)
    dw = dw.as_strided((3, out, width), (out * dw.stride(0), dw.stride(0), 1))
    ops.grouped_linear(x, w, off, out=y)
    ops.grouped_linear_backward(dy, x, w, off, dx=dx, dweight=dw)
    assert torch.equal(y, want[0]) and torch.equal(dx, want[1]) and torch.equal(dw, want[2])
    ops.sync()


def test_one_matrix_for_all_groups(ops):
    """A broadcast matrix is read as one (its gradients are of the groups' own)."""
    e = ends([20, 30])
    x, one = randn(1, 50, 64, dtype=torch.bfloat16), randn(2, 1, 72, 64, dtype=torch.bfloat16)
    got = ops.grouped_linear(x, one.expand(2, 72, 64), offsets_of(e))
    assert torch.equal(got, ops.grouped_linear(x, one, offsets_of([0, 50])))


def test_offsets_that_are_no_offsets_reach_nothing(ops):
    """Bad offsets give bad results, but nothing outside the tensors is read or written: rows are taken as the nearest that exist."""
    x, w, dy = (randn(i, *s, dtype=torch.bfloat16) for i, s in enumerate([(100, 64), (3, 72, 64), (100, 72)]))
    ahead = torch.full((300, 72), 9.0, dtype=torch.bfloat16, device="cuda")
    for e in ([-5, 40, 200, 1 << 40], [90, 50, 20, 100], [-(1 << 62), -1, 0, 1 << 62], [100, 0, 100, 0]):
        off = offsets_of(e)
        ops.grouped_linear(x, w, off, out=ahead[100:200])
        ops.grouped_linear(x, w, off)
        ops.grouped_linear_backward(dy, x, w, off)
        ops.sync()
        assert bool((ahead[:100] == 9).all()) and bool((ahead[200:] == 9).all())
    got = ops.grouped_linear(x, w, offsets_of([-5, 40, 60, 1000]))
    assert torch.equal(got, ops.grouped_linear(x, w, offsets_of([0, 40, 60, 100])))


@pytest.mark.parametrize("groups", [1, 30, 31, 63, 500, 2048])
def test_many_groups(ops, groups):
    sizes = [(i * 7) % 5 for i in range(groups)]
    e = ends(sizes, 2)
    check(ops, e, e[-1] + 3, 64, 40, torch.bfloat16)


def test_several_tiles_a_block(ops):
    """More tiles than blocks, of unlike lengths: accumulators and stages go round, empty groups between."""
    sizes = [700, 0, 3, 0, 0, 1500, 260, 17, 0, 900, 4, 4, 4, 2000]
    for width, out in ((512, 1024), (1000, 776)):
        e = ends(sizes, 9)
        check(ops, e, e[-1] + 77, width, out, torch.bfloat16)
        check(ops, e, e[-1] + 77, width, out, torch.float16)


def test_rows_beyond_32_bits(ops):
    """Outputs and operands whose elements have numbers above 2^31."""
    rows, width, out = 700_000, 8, 4096
    e = ends([699_000, 900], 50)
    off = offsets_of(e)
    x, w = randn(1, rows, width, dtype=torch.bfloat16), randn(2, 2, out, width, dtype=torch.bfloat16)
    y = ops.grouped_linear(x, w, off)
    for p, g in ((slice(60, 100), 0), (slice(698_900, 699_050), 0), (slice(699_050, 699_950), 1)):
        within(y[p], *product(x[p], w[g], torch.bfloat16), "y")
    assert not y[:50].any() and not y[699_950:].any()
    dy = y
    dx, dw = ops.grouped_linear_backward(dy, x, w, off)
    within(dx[699_050:699_950], *product(dy[699_050:699_950], w[1].T, torch.bfloat16), "dx")
    within(dw[1], *product(dy[699_050:699_950].T, x[699_050:699_950].T, torch.bfloat16), "dweight")
    ops.sync()


def test_gradients_against_differences(ops):
    e = ends([20, 0, 33])
    off, dtype = offsets_of(e), torch.float16
    x, w, c = randn(1, 53, 40, dtype=dtype), randn(2, 3, 24, 40, dtype=dtype), randn(3, 53, 24, dtype=dtype)
    dw = torch.empty(3, 24, 40, device="cuda")
    dx, _ = ops.grouped_linear_backward(c, x, w, off, dweight=dw)

    def f(x, w):
        y = torch.cat([x[a:b] @ w[g].T for g, (a, b) in enumerate(zip(e, e[1:]))])
        return float((c.double() * y).sum())

    for grad, at in ((dx, 0), (dw, 1)):
        way = randn(20 + at, *grad.shape).double()
        args = [x.double(), w.double()]
        ahead, back = list(args), list(args)
        ahead[at], back[at] = args[at] + 1e-3 * way, args[at] - 1e-3 * way
        slope = (f(*ahead) - f(*back)) / 2e-3                         # linear in each: exact but for the rounding of the sums
        assert abs(float((grad.double() * way).sum()) - slope) <= (2.0 ** -11 + 1e-6) * float((grad.double() * way).abs().sum())


def test_same_bits_every_time(ops):
    e = ends([700, 3, 1200])
    off = offsets_of(e)
    x, w, dy = randn(1, e[-1], 300, dtype=torch.float16), randn(2, 3, 200, 300, dtype=torch.float16), randn(3, e[-1], 200, dtype=torch.float16)
    first = [ops.grouped_linear(x, w, off), *ops.grouped_linear_backward(dy, x, w, off)]
    for _ in range(5):
        again = [ops.grouped_linear(x, w, off), *ops.grouped_linear_backward(dy, x, w, off)]
        assert all(torch.equal(a, b) for a, b in zip(first, again))


# ---- the order -----------------------------------------------------------------------------------------------------------
def sorted_plainly(experts, groups):
    e = experts.flatten().tolist()
    key = [v if 0 <= v < groups else groups for v in e]
    order = sorted(range(len(e)), key=lambda i: key[i])
    places = [0] * len(e)
    for j, i in enumerate(order):
        places[i] = j
    counts = [0] * (groups + 1)
    for k in key:
        counts[k] += 1
    return order, places, ends(counts[:-1])


@pytest.mark.parametrize("dtype", [torch.int64, torch.int32], ids=str)
@pytest.mark.parametrize("n,groups", [(1, 1), (5, 3), (31, 2), (32, 8), (33, 8), (1000, 1), (1024, 64), (1025, 1023), (5000, 1024), (8192, 1500), (8193, 7), (9000, 2048),
                                      (50_001, 256), (400_000, 33)])
def test_sort_by_expert(ops, n, groups, dtype):
    g = torch.Generator(device="cuda").manual_seed(n)
    experts = torch.randint(-2, groups + 2, (n,), generator=g, device="cuda").to(dtype)
    order, places, offsets = ops.sort_by_expert(experts, groups)
    want = sorted_plainly(experts, groups)
    assert [t.dtype for t in (order, places, offsets)] == [torch.int64] * 3
    assert order.tolist() == want[0] and places.tolist() == want[1] and offsets.tolist() == want[2]


@pytest.mark.parametrize("n", [40, 70_000])
def test_sort_by_expert_one_sided(ops, n):
    for experts, groups in ((torch.zeros(n), 5), (torch.full((n,), 4), 5), (torch.full((n,), -1), 5), (torch.full((n,), 1 << 40), 5),
                            (torch.arange(n) % 3, 1000), ((torch.arange(n) < n // 2).long(), 2)):
        experts = experts.to(torch.int64).cuda()
        got = ops.sort_by_expert(experts, groups)
        assert [t.tolist() for t in got] == [list(w) for w in sorted_plainly(experts, groups)]


def test_sort_by_expert_shapes(ops):
    experts = torch.randint(0, 6, (100, 2), device="cuda")
    order, places, offsets = ops.sort_by_expert(experts, 6)
    assert places.shape == (100, 2) and torch.equal(order[places.flatten()], torch.arange(200, device="cuda"))
    order, places, offsets = ops.sort_by_expert(torch.empty(0, dtype=torch.int64, device="cuda"), 3)
    assert order.numel() == places.numel() == 0 and offsets.tolist() == [0, 0, 0, 0]
