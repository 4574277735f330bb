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
