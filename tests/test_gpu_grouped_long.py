"""Products grouped by expert whose sums are long: what the tensor cores truncate stays below the outputs' own rounding whatever the length.

Tolerances before any run: u is half a step of the output's type. A part of 1024 products of one sign comes out at most 2 (64 + 4) 2^-24 too small for bf16 operands (64 additions
of 16 products, each with the alignment of its operands), up to four times as much for fp16; parts are joined with a rounding each, 2^-24.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def positive(seed, *shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.rand(shape, generator=g, device="cuda") + 0.5).mul_(scale).to(dtype)


def part_error(length, dtype):
    return (2 * 68 * (4 if dtype == torch.float16 else 1) + length / 1024 + 4) * 2.0 ** -24


def product(a, b):
    """a^T b in 64 bits, some rows at a time"""
    return sum(a[i:i + (1 << 18)].double().T @ b[i:i + (1 << 18)].double() for i in range(0, len(a), 1 << 18))


# a group of so many rows that its sums pass the rounding of 16 bits, among so many groups that none is cut into slices
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("rows,width,out", [(3 << 20, 64, 64), (1_500_077, 256, 240)])
def test_matrices_gradients_of_a_group_of_millions_of_rows(ops, rows, width, out, dtype):
    groups, before = 300, 700
    total = before + rows + 50
    # fp16's largest number is 65504
    x, dy = positive(1, total, width, dtype=dtype), positive(2, total, out, dtype=dtype, scale=2.0 ** -10 if dtype == torch.float16 else 1.0)
    offsets = torch.full((groups + 1,), before + rows, device="cuda")
    offsets[0], offsets[1:8] = 0, before
    offsets[-1] = total
    w = torch.zeros(groups, out, width, dtype=dtype, device="cuda")
    _, dw = ops.grouped_linear_backward(dy, x, w, offsets, dx=False)
    ops.sync()
    for g, part in ((7, slice(before, before + rows)), (0, slice(0, before)), (groups - 1, slice(before + rows, total))):
        want = product(dy[part], x[part])
        assert float(((dw[g].double() - want).abs() / want).max()) <= U[dtype] * (1 + 1e-3) + part_error(rows, dtype), g
    assert not dw[1:7].any() and not dw[8:groups - 1].any()


# K of a million values: so many groups that each block has a tile of its own, or so few rows that K is cut into slices
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("sizes,K,other", [([1] * 70 + [0, 17, 3], 1 << 20, 8), ([2, 0, 40], (1 << 20) - 5, 9), ([1] * 80, 131073, 40), ([300, 129], 140001, 2000)],
                         ids=["tiles", "slices", "just beyond", "tiles of many columns"])
@pytest.mark.parametrize("way", ["y", "dx"])
def test_long_rows(ops, way, sizes, K, other, dtype):
    first, groups = 3, len(sizes)
    ends = [first]
    for n in sizes:
        ends.append(ends[-1] + n)
    rows = ends[-1] + 40
    # fp16's largest number is 65504
    x = positive(1, rows, K, dtype=dtype, scale=2.0 ** -10 if dtype == torch.float16 else 1.0)
    w = positive(2, groups, *((other, K) if way == "y" else (K, other)), dtype=dtype)
    x[:first], x[ends[-1]:] = float("nan"), float("inf")
    offsets = torch.tensor(ends, device="cuda")

    def call(out=None):
        if way == "y":
            return ops.grouped_linear(x, w, offsets, out=out)
        like = torch.zeros(rows, other, dtype=dtype, device="cuda")           # x of the forward pass, which dx does not need
        return ops.grouped_linear_backward(x, like, w, offsets, dx=out, dweight=False)[0]

    got = call()
    ops.sync()
    assert not got[:first].any() and not got[ends[-1]:].any()
    bound = U[dtype] * (1 + 1e-3) + part_error(K, dtype)
    for g in range(groups):
        a, b = ends[g], ends[g + 1]
        m = w[g].double()
        want = x[a:b].double() @ (m.T if way == "y" else m)
        assert a == b or float(((got[a:b].double() - want).abs() / want).max()) <= bound, g
    flat = torch.full((rows * (other + 3) + 1,), 7.0, dtype=dtype, device="cuda")           # into rows that begin anywhere; what lies around them stays
    out = flat[1:].view(rows, other + 3)[:, :other]
    assert call(out) is out and torch.equal(out[first:ends[-1]], got[first:ends[-1]])
    out[first:ends[-1]] = 7.0
    assert bool((flat == 7).all())


@pytest.mark.parametrize("dtype,K", [(torch.bfloat16, 131072), (torch.float16, 32768)], ids=str)
@pytest.mark.parametrize("way", ["y", "dx"])
def test_the_longest_rows_in_one_accumulation(ops, way, K, dtype):
    """What is truncated stays below half a step, which the output's own rounding may add."""
    groups, other = 90, 16
    for draw in (positive, lambda seed, *shape, dtype, scale=1.0: torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").abs().mul_(scale).to(dtype)):
        x = draw(1, 2 * groups, K, dtype=dtype, scale=2.0 ** -6 if dtype == torch.float16 else 1.0)
        w = draw(2, groups, *((other, K) if way == "y" else (K, other)), dtype=dtype)
        offsets = torch.arange(groups + 1, device="cuda") * 2
        got = ops.grouped_linear(x, w, offsets) if way == "y" else ops.grouped_linear_backward(x, x[:, :other].contiguous(), w, offsets, dweight=False)[0]
        for g in range(groups):
            m = w[g].double()
            want = x[2 * g:2 * g + 2].double() @ (m.T if way == "y" else m)
            assert float(((got[2 * g:2 * g + 2].double() - want).abs() / want).max()) <= 2 * U[dtype], g
