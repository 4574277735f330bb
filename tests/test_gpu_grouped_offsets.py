"""Offsets of groups that are none, on every path of the grouped products: K in slices, weight gradients' rows in slices, outputs that go through the workspace, and plain tiles.

What lies outside the rows is taken as the nearest that does not. Offsets that decrease give unspecified results; nothing around the tensors is read or written for them.
"""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# rows, width, out
PATHS = {"plain tiles": (900, 136, 264), "K in slices": (100, 4096, 200), "rows in slices": (7000, 64, 200), "through the workspace": (2600, 1001, 1333),
         "both": (9000, 777, 1503), "copied operands": (300, 77, 131)}
FAR = 1 << 62


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def randn(seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def offsets_of(e):
    return torch.tensor(e, dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("dweight_type", [None, torch.float32], ids=str)
@pytest.mark.parametrize("path", PATHS)
def test_offsets_outside_the_rows(ops, path, dweight_type):
    rows, width, out = PATHS[path]
    dtype = torch.bfloat16
    x, w, dy = randn(1, rows, width, dtype=dtype), randn(2, 3, out, width, dtype=dtype), randn(3, rows, out, dtype=dtype)

    def call(e):
        given = torch.full(w.shape, 5.0, dtype=dweight_type, device="cuda") if dweight_type else None
        off = offsets_of(e)
        return [ops.grouped_linear(x, w, off), *ops.grouped_linear_backward(dy, x, w, off, dweight=given)]

    a, b = rows * 2 // 5, rows * 3 // 5
    for bad, good in (([-5, a, b, rows + 1000], [0, a, b, rows]), ([-FAR, -1, a, FAR], [0, 0, a, rows]), ([a, b, rows + 1, 1 << 40], [a, b, rows, rows]),
                      ([rows + 5, rows + 6, FAR, FAR], [rows] * 4), ([-9, -8, -7, -6], [0] * 4)):
        assert all(torch.equal(s, t) for s, t in zip(call(bad), call(good))), bad
    ops.sync()


@pytest.mark.parametrize("path", PATHS)
def test_offsets_that_decrease_reach_nothing_around_the_tensors(ops, path):
    rows, width, out = PATHS[path]
    dtype = torch.bfloat16
    x, w, dy = randn(1, rows, width, dtype=dtype), randn(2, 3, out, width, dtype=dtype), randn(3, rows, out, dtype=dtype)
    guard = 4096
    flat = [torch.full((n + 2 * guard,), 9.0, dtype=t, device="cuda") for n, t in ((rows * out, dtype), (rows * width, dtype), (w.numel(), dtype), (w.numel(), torch.float32))]
    y, dx, dw, dw32 = (f[guard:-guard].view(s) for f, s in zip(flat, (dy.shape, x.shape, w.shape, w.shape)))
    for e in ([rows, rows // 2, rows // 5, rows], [rows, 0, rows, 0], [0, rows * 3 // 5, rows // 5, rows], [0, rows * 3 // 5, rows * 2 // 5, rows * 2 // 5], [FAR, -FAR, FAR, -FAR]):
        off = offsets_of(e)
        ops.grouped_linear(x, w, off, out=y)
        ops.grouped_linear(x, w, off)
        ops.grouped_linear_backward(dy, x, w, off, dx=dx, dweight=dw)
        ops.grouped_linear_backward(dy, x, w, off, dweight=dw32)
        ops.sync()
        assert all(bool((f[:guard] == 9).all()) and bool((f[-guard:] == 9).all()) for f in flat), e
    off = offsets_of([0, 5, 50, rows])                               # and the next call is whole again
    want = ops.grouped_linear(x, w, off)
    ops.grouped_linear(x, w, off, out=y)
    assert torch.equal(y, want)
