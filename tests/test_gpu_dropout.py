"""Dropout from a counter: the mask against the generator in whole numbers of Python, values against 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
TYPES = list(U)
MASK = (1 << 64) - 1


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def output(start, number):
    """Output `number` of splitmix64 (Steele, Lea, Flood 2014) started at `start`"""
    z = (start + number * 0x9E3779B97F4A7C15) & MASK
    z = (z ^ z >> 30) * 0xBF58476D1CE4E5B9 & MASK
    z = (z ^ z >> 27) * 0x94D049BB133111EB & MASK
    return z ^ z >> 31


def fields(seed, first, n):
    key = output(seed & MASK, 1)
    return torch.tensor([output(key, i // 4 + 1) >> 16 * (i % 4) & 0xFFFF for i in range(first, first + n)])


def randn(seed, *shape, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def check(got, x, residual, p, seed):
    below = round(p * 65536)
    keep = (fields(seed, 0, x.numel()) >= below).view(x.shape).cuda()
    kept = torch.where(keep, x.double() * (65536 / (65536 - below) if below < 65536 else 0.0), 0.0)
    want = kept + (residual.double() if residual is not None else 0.0)
    u = U[x.dtype]
    # the factor is rounded to 32 bits, the sum or product once in 32 bits and once to the type
    e = 2.0 ** -24 * kept.abs() + 2.0 ** -24 * want.abs()
    bound = e + u * (want.abs() + e) + TINY[x.dtype]
    assert float(((got.double() - want).abs() - bound).max()) <= 0
    if residual is None:
        assert not got[~keep].any()
    else:
        assert torch.equal(got[~keep], residual[~keep])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", [(1,), (3,), (8,), (9,), (1, 1), (7, 13), (16, 768), (5, 1001), (3, 4, 33), (4096,), (4099,)], ids=str)
@pytest.mark.parametrize("with_residual", [False, True])
def test_dropout(ops, shape, dtype, with_residual):
    x, r = randn(1, *shape, dtype=dtype), randn(2, *shape, dtype=dtype) if with_residual else None
    for p, seed in ((0.1, 7), (0.5, -3), (0.9, (1 << 64) - 1)):
        check(ops.dropout(x, p, seed, residual=r), x, r, p, seed)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_the_ends_of_p(ops, dtype):
    x, r = randn(1, 300, 5, dtype=dtype), randn(2, 300, 5, dtype=dtype)
    assert torch.equal(ops.dropout(x, 0.0, 5), x)
    assert not ops.dropout(x, 1.0, 5).any() and torch.equal(ops.dropout(x, 1.0, 5, residual=r), r)
    check(ops.dropout(x, 65535 / 65536, 5), x, None, 65535 / 65536, 5)
    check(ops.dropout(x, 2.0 ** -16, 5), x, None, 2.0 ** -16, 5)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_what_is_dropped_may_hold_anything(ops, dtype):
    x, r = randn(1, 40, 50, dtype=dtype), randn(2, 40, 50, dtype=dtype)
    dropped = (fields(9, 0, 2000) < round(0.3 * 65536)).view(40, 50).cuda()
    bad = x.clone()
    bad[dropped] = math.nan
    assert torch.equal(ops.dropout(bad, 0.3, 9), ops.dropout(x, 0.3, 9))
    bad[dropped] = math.inf
    assert torch.equal(ops.dropout(bad, 0.3, 9, residual=r), ops.dropout(x, 0.3, 9, residual=r))


# row lengths and distances that are and are not whole accesses; the mask goes by the value's number, not by its address
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("cols,pad,offset", [(64, 8, 0), (64, 16, 8), (64, 4, 4), (4096, 4096, 0), (64, 8, 1), (65, 0, 1), (40, 3, 0), (7, 1, 2), (1, 4, 3), (1000, 24, 8)])
def test_strides(ops, cols, pad, offset, dtype):
    rows = 37

    def view(seed):
        return randn(seed, rows * (cols + pad) + offset, dtype=dtype)[offset:].view(rows, cols + pad)[:, :cols]

    x, r, out = view(1), view(2), view(3)
    whole = out._base if out._base is not None else out
    before = whole.clone()
    assert ops.dropout(x, 0.4, 11, residual=r, out=out) is out
    assert torch.equal(out, ops.dropout(x.contiguous(), 0.4, 11, residual=r.contiguous()))
    inside = torch.zeros(whole.shape, dtype=torch.bool, device="cuda")
    inside.as_strided(out.shape, out.stride(), out.storage_offset()).fill_(True)
    assert torch.equal(whole[~inside], before[~inside])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("shape", [(33, 100), (33, 101)])
def test_in_place(ops, shape, dtype):
    x, r = randn(1, *shape, dtype=dtype), randn(2, *shape, dtype=dtype)
    want = ops.dropout(x, 0.2, 3, residual=r)
    for over in (0, 1):
        pair = [x.clone(), r.clone()]
        assert torch.equal(ops.dropout(pair[0], 0.2, 3, residual=pair[1], out=pair[over]), want)
    same = x.clone()
    assert torch.equal(ops.dropout(same, 0.2, 3, residual=same), ops.dropout(x, 0.2, 3, residual=x))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_backward_is_the_gradient(ops, dtype):
    """Linear in x: the forward pass on the gradient's direction gives the same inner product."""
    dy = randn(3, 60, 70, dtype=dtype)
    dx = ops.dropout_backward(dy, 0.3, 21)
    check(dx, dy, None, 0.3, 21)
    over = dy.clone()
    assert ops.dropout_backward(over, 0.3, 21, dx=over) is over and torch.equal(over, dx)
    x, step = randn(4, 60, 70), 0.5
    ahead, back = ops.dropout(x + step * dy.float(), 0.3, 21), ops.dropout(x - step * dy.float(), 0.3, 21)
    way = dy.double()
    slope = float((way * (ahead.double() - back.double())).sum()) / (2 * step)
    # differences of 32-bit numbers of up to about 10, and the rounding of dx
    assert abs(float((dx.double() * way).sum()) - slope) <= (U[dtype] + 1e-5) * float((way * way).sum()) * 2


def test_seed_on_the_device(ops):
    x, seed = randn(1, 100, 9), torch.tensor([-12345], dtype=torch.int64, device="cuda")
    assert torch.equal(ops.dropout(x, 0.3, seed), ops.dropout(x, 0.3, -12345))
    ops.dropout(x, 0.3, seed)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ops.dropout(x, 0.3, seed)
        dx = ops.dropout_backward(x, 0.3, seed)
    for s in (5, 1 << 60):
        seed.fill_(s)
        graph.replay()
        assert torch.equal(y, ops.dropout(x, 0.3, s)) and torch.equal(dx, y)


def test_shares_and_independence(ops):
    """The kept share, and that of pairs of neighbours, of the same place under two seeds, and of columns a step apart: within six standard
    deviations of a fair generator's, over a few million values."""
    n, p = 1 << 22, 0.25
    x = torch.ones(n, device="cuda")
    a, b = (ops.dropout(x, p, s) != 0 for s in (1, 2))
    for event, q in ((a, 1 - p), (a[1:] & a[:-1], (1 - p) ** 2), (a[4:] & a[:-4], (1 - p) ** 2), (a & b, (1 - p) ** 2), (a[1024:] & a[:-1024], (1 - p) ** 2)):
        assert abs(float(event.double().mean()) - q) <= 6 * math.sqrt(2 * q * (1 - q) / n)


def test_values_beyond_32_bits(ops):
    n = (1 << 32) + 1000
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = ops.dropout(x, 0.5, 77, out=x)
    first = n - 3000
    keep = fields(77, first, 3000) >= 32768
    assert torch.equal((y[first:] != 0).cpu(), keep)
    first = (1 << 31) - 1000
    assert torch.equal((y[first:first + 2000] != 0).cpu(), fields(77, first, 2000) >= 32768)
