"""The language-model operators against plain implementations in 64 bits.

Tolerances are bounds derived from the number formats, before any run: u is the unit roundoff of the output's (or an
operand's) type, 2^-24 that of 32-bit sums, whose error is at most (number of terms) * 2^-24 * (sum of magnitudes) in any order.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}    # smallest steps
TYPES = list(U)
HALF = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(seed, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen(seed), device="cuda") * scale).to(dtype)


def within(got, want, bound, what):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    over = ((got - want).abs() - bound).nan_to_num(0.0, posinf=math.inf, neginf=-math.inf)
    assert float(over.max() if over.numel() else 0.0) <= 0.0, (what, float(over.max()))


# ---- layer norm ----------------------------------------------------------------------------------------------------------
def norm_ref(x, w, b, eps):
    x = x.double()
    mean = x.mean(-1)
    c = x - mean[..., None]
    rstd = 1.0 / torch.sqrt((c * c).mean(-1) + eps)
    h = c * rstd[..., None]
    y = h * (w.double() if w is not None else 1.0) + (b.double() if b is not None else 0.0)
    return y, mean, rstd, h


# every row length of the list sits beside a border of the kernels (256, 1024, 4096, 16384 / 256, 1024, 2048, 8192)
COLS = [1, 2, 17, 64, 255, 256, 257, 768, 1000, 1024, 1025, 2048, 2056, 4096, 4097, 8192, 8200, 16384, 16400, 20001]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("cols", COLS)
def test_layer_norm(ops, cols, dtype):
    rows = 5
    x = randn(1, rows, cols, dtype=dtype, scale=1.5) + randn(2, rows, 1, dtype=dtype)
    w, b = 1 + randn(3, cols, scale=0.1), randn(4, cols, scale=0.1)
    y, mean, rstd = ops.layer_norm(x, w, b, eps=1e-5)
    want, m, r, h = norm_ref(x, w, b, 1e-5)
    # mean: a sum of cols terms; it enters the centred values, relative to their spread 1/r
    em = (cols + 2) * 2.0 ** -24 * x.double().abs().mean(-1)
    er = r * ((cols + 8) * 2.0 ** -24 + 2 * em * r)
    within(mean, m, em + 2.0 ** -24 * m.abs(), "mean")
    within(rstd, r, er + 2.0 ** -22 * r, "rstd")
    eh = ((em * r)[:, None] + h.abs() * (er / r)[:, None] + 4 * 2.0 ** -24 * (h.abs() + (m.abs() * r)[:, None])) * w.double().abs()
    within(y, want, U[dtype] * (want.abs() + eh) + eh + 2.0 ** -23 * want.abs() + TINY[dtype], "y")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 64), (3, 17), (9, 256), (33, 257), (700, 768), (2500, 96), (5, 1025), (301, 2048), (7, 2049), (5, 8192), (256, 300), (257, 300), (200, 1001), (260, 500),
                                       (3, 8200), (700, 9000)])
def test_layer_norm_backward(ops, rows, cols, dtype):
    backward_close(ops, rows, cols, dtype)


# few rows of nearly the most columns that a block's threads hold, off the 16-byte boundary
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(3, 8185), (40, 8190), (256, 8191), (5, 8184), (2, 8180)])
def test_layer_norm_backward_nearly_long_rows(ops, rows, cols, dtype):
    backward_close(ops, rows, cols, dtype)


# the rows' number at which the weights' gradients are formed another way, with whole 16-byte accesses
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(64, 8), (65, 24), (256, 8192), (257, 768), (300, 8184), (1000, 40), (1023, 1008), (1024, 4096), (1024, 4104), (1025, 256)])
def test_layer_norm_backward_some_hundred_rows(ops, rows, cols, dtype):
    backward_close(ops, rows, cols, dtype)


def backward_close(ops, rows, cols, dtype):
    x = randn(1, rows, cols, dtype=dtype, scale=1.5)
    dy = randn(2, rows, cols, dtype=dtype)
    w = 1 + randn(3, cols, scale=0.1)
    _, mean, rstd = ops.layer_norm(x, w, None)
    dx, dw, db = ops.layer_norm_backward(dy, x, w, mean, rstd)
    r = rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r                  # the formulas on the statistics that were passed
    g = dy.double() * w.double()
    m2 = (g * h).mean(1, keepdim=True)
    want = r * (g - g.mean(1, keepdim=True) - h * m2)
    e = 2.0 ** -24
    eh = 2 * e * ((x.double().abs() + mean.double().abs()[:, None]) * r)            # difference and product of h
    em = (cols + 4) * e * ((g.abs()).mean(1, keepdim=True) + h.abs() * (g * h).abs().mean(1, keepdim=True))
    ex = r * (em + eh * (m2.abs() + g.abs().mean(1, keepdim=True) * h.abs()) + h.abs() * (g.abs() * eh).mean(1, keepdim=True)
              + 6 * e * (g.abs() + g.abs().mean(1, keepdim=True) + (h * m2).abs()))
    within(dx, want, U[dtype] * (want.abs() + ex) + ex + TINY[dtype], "dx")
    d = dy.double()
    within(dw, (d * h).sum(0), (rows + 4) * e * (d * h).abs().sum(0) + (d.abs() * eh).sum(0), "dw")
    within(db, d.sum(0), (rows + 4) * e * d.abs().sum(0), "db")


# y over x, and dx over dy or x: the same bits as apart, also where extra blocks read the inputs a second time
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", [(1, 8), (16, 768), (200, 4096), (256, 1001), (256, 8184), (700, 512), (1024, 4096), (1500, 768), (3000, 333), (40, 9000)])
def test_layer_norm_in_place(ops, rows, cols, dtype):
    x, dy, w = randn(1, rows, cols, dtype=dtype), randn(2, rows, cols, dtype=dtype), 1 + randn(3, cols, scale=0.1)
    y, mean, rstd = ops.layer_norm(x, w, None)
    same = x.clone()
    assert ops.layer_norm(same, w, None, out=same)[0] is same and torch.equal(same, y)
    want = ops.layer_norm_backward(dy, x, w, mean, rstd)
    for over in (0, 1):
        for _ in range(3):
            pair = [dy.clone(), x.clone()]
            got = ops.layer_norm_backward(*pair, w, mean, rstd, dx=pair[over])
            assert got[0] is pair[over] and all(torch.equal(g, t) for g, t in zip(got, want))
    only = ops.layer_norm_backward(dy, x, w, mean, rstd, dx=False)
    assert only[0] is None and torch.equal(only[1], want[1]) and torch.equal(only[2], want[2])
    ops.sync()


def test_layer_norm_gradient_against_differences(ops):
    x, dy, w, b = randn(1, 6, 40), randn(2, 6, 40), 1 + randn(3, 40, scale=0.1), randn(4, 40)
    _, mean, rstd = ops.layer_norm(x, w, b)
    dx, dw, db = ops.layer_norm_backward(dy, x, w, mean, rstd)
    t = 1e-4                                                        # central differences: error of order t^2
    for seed, (grad, at) in enumerate(((dx, 0), (dw, 1), (db, 2))):
        way = randn(10 + seed, *grad.shape).double()
        f = []
        for s in (t, -t):
            args = [x.double(), w.double(), b.double()]
            args[at] = args[at] + s * way
            f.append(float((dy.double() * norm_ref(*args, 1e-5)[0]).sum()))
        slope = (f[0] - f[1]) / (2 * t)
        assert abs(float((grad.double() * way).sum()) - slope) <= 1e-5 * float((grad.double() * way).abs().sum())


def test_layer_norm_layouts(ops):
    """Rows apart from each other, a start off the vector boundary, leading axes, no weight, 16-bit weights, no rows."""
    big = randn(1, 12, 300, dtype=torch.bfloat16)
    for x in (big[:, :256], big[:, 1:257], big[::2, 3:260], big[0], big.view(3, 4, 300)):
        w, b = randn(2, x.shape[-1], dtype=torch.bfloat16), randn(3, x.shape[-1], dtype=torch.bfloat16)
        for ww, bb in ((w, b), (None, None), (w, None), (None, b)):
            y, mean, rstd = ops.layer_norm(x, ww, bb)
            want, m, r, _ = norm_ref(x, ww, bb, 1e-5)
            assert y.shape == x.shape and mean.shape == x.shape[:-1]
            within(y, want, 2.0 ** -8 * want.abs() + 1e-4, "y")
        dy = randn(4, 24, 300, dtype=torch.bfloat16).flatten()[5:5 + x.numel()].view(x.shape)
        dx, dw, db = ops.layer_norm_backward(dy, x, w, mean, rstd)
        assert dw.dtype == torch.bfloat16
        h = (x.double() - m[..., None]) * r[..., None]
        within(dw, (dy.double() * h).reshape(-1, x.shape[-1]).sum(0), 2.0 ** -8 * (dy.double() * h).reshape(-1, x.shape[-1]).sum(0).abs() + 1e-4, "dw")
    out = torch.zeros(12, 300, dtype=torch.bfloat16, device="cuda")
    ops.layer_norm(big[:, 1:257], out=out[:, 2:258])
    assert not out[:, :2].any() and not out[:, 258:].any() and bool(out[:, 2:258].any())
    none = torch.empty(0, 64, device="cuda")
    assert ops.layer_norm(none)[0].shape == (0, 64)
    _, dw, db = ops.layer_norm_backward(none, none, torch.ones(64, device="cuda"), none[:, 0], none[:, 0])
    assert not dw.any() and not db.any()


def test_layer_norm_parts_of_the_gradient(ops):
    x, dy, w = randn(1, 50, 96), randn(2, 50, 96), randn(3, 96)
    _, mean, rstd = ops.layer_norm(x, w)
    full = ops.layer_norm_backward(dy, x, w, mean, rstd)
    for leave in range(1, 8):
        kw = {n: False for i, n in enumerate(("dx", "dweight", "dbias")) if leave >> i & 1}
        got = ops.layer_norm_backward(dy, x, w, mean, rstd, **kw)
        for i, (a, b) in enumerate(zip(got, full)):
            assert (a is None) == bool(leave >> i & 1)
            assert a is None or torch.equal(a, b)
    row = torch.zeros(1000, device="cuda")                           # a worker's row of the gradient array, any offset
    ops.layer_norm_backward(dy, x, w, mean, rstd, dweight=row[7:103], dbias=row[103:199])
    assert torch.equal(row[7:103], full[1]) and torch.equal(row[103:199], full[2]) and not row[:7].any() and not row[199:].any()


def test_layer_norm_rows_with_infinities_keep_to_themselves(ops):
    x = randn(1, 6, 768, dtype=torch.bfloat16)
    clean = ops.layer_norm(x)[0]
    x[2, 5] = math.inf
    x[4, 7] = math.nan
    y, _, _ = ops.layer_norm(x)
    for r in range(6):
        assert bool(torch.isnan(y[r]).all()) if r in (2, 4) else torch.equal(y[r], clean[r])
    zero = torch.zeros(2, 768, device="cuda")                        # a constant row: variance 0
    assert torch.equal(ops.layer_norm(zero)[0], zero)


# ---- linear cross entropy --------------------------------------------------------------------------------------------------
def head_inputs(tokens, vocab, width, dtype, seed=0):
    w = randn(seed + 1, vocab, width, dtype=dtype, scale=2 / math.sqrt(width))
    t = torch.randint(0, vocab, (tokens,), generator=gen(seed + 2), device="cuda")
    h = randn(seed + 3, tokens, width, dtype=dtype)
    if tokens > 2:
        t[1] = -100
        h[2] = 3 * w[t[2]]                                           # a confident one
    return h, w, t


def head_ref(h, w, t):
    z = h.double() @ w.double().T
    lse = torch.logsumexp(z, 1)
    loss = torch.where(t >= 0, lse - z.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    # 32-bit sums of width products (tensor cores may truncate instead of rounding: twice 2^-24)
    ez = 2 * (width_of(h) + 4) * 2.0 ** -24 * (h.double().abs() @ w.double().abs().T)
    return z, lse, loss, ez


def width_of(h):
    return h.shape[1]


SIZES = [(1, 1, 1), (1, 50, 8), (2, 257, 63), (5, 1000, 64), (128, 128, 64), (129, 300, 72), (256, 512, 128), (300, 1001, 100), (513, 2050, 65), (77, 4000, 770)]


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
def test_linear_cross_entropy(ops, tokens, vocab, width, dtype):
    h, w, t = head_inputs(tokens, vocab, width, dtype)
    loss, lse = ops.linear_cross_entropy(h, w, t)
    z, want_lse, want_loss, ez = head_ref(h, w, t)
    # the largest logit error, the exponentials' and their sum's (2^-21 with the rounding of z in units of log 2), the logarithm's
    e = ez.amax(1) + 2.0 ** -20 * (1 + z.abs().amax(1))
    within(lse, want_lse, e, "lse")
    within(loss, want_loss, 2 * e, "loss")
    ops.sync()


def head_backward_ref(dloss, h, w, t, lse):
    p = torch.exp(h.double() @ w.double().T - lse.double()[:, None])
    live = (t >= 0) & (t < w.shape[0])
    one = torch.zeros_like(p)
    one[live, t[live]] = 1.0
    scale = torch.where(live, dloss.double(), 0.0)[:, None]
    return (p - one) * scale, p * scale.abs()


@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("tokens,vocab,width", SIZES)
def test_linear_cross_entropy_backward(ops, tokens, vocab, width, dtype):
    h, w, t = head_inputs(tokens, vocab, width, dtype)
    _, lse, _, ez = head_ref(h, w, t)
    lse = lse.float()
    dloss = randn(9, tokens) / tokens
    dh, dw = ops.linear_cross_entropy_backward(dloss, h, w, t, lse)
    g, p = head_backward_ref(dloss, h, w, t, lse)
    # G is rounded to the operands' type; its probabilities carry the logits' error
    eg = U[dtype] * g.abs() + (1 + U[dtype]) * p * (ez + 2.0 ** -20 * (1 + (h.double() @ w.double().T).abs()))
    if dtype == torch.float16:
        eg = eg + 2.0 ** -37 * float(dloss.abs().max())              # below fp16's range, after the scaling
    for got, a, ea, b, what in ((dh, g, eg, w.double(), "dh"), (dw, g.T, eg.T, h.double(), "dw")):
        want = a @ b
        e = ea @ b.abs() + 2 * (a.shape[1] + 4) * 2.0 ** -24 * (a.abs() @ b.abs())
        within(got, want, e + U[dtype] * (want.abs() + e) + TINY[dtype], what)
    fh, fw = torch.empty_like(h, dtype=torch.float32), torch.empty_like(w, dtype=torch.float32)
    ops.linear_cross_entropy_backward(dloss, h, w, t, lse, dhidden=fh, dweight=fw)
    assert torch.equal(fh.to(dtype), dh) and torch.equal(fw.to(dtype), dw)       # the same sums, unrounded
    ops.sync()


def test_linear_cross_entropy_gradient_against_differences(ops):
    h, w, t = head_inputs(40, 130, 32, torch.float16)
    c = randn(5, 40)
    loss, lse = ops.linear_cross_entropy(h, w, t)
    fh, fw = torch.empty_like(h, dtype=torch.float32), torch.empty_like(w, dtype=torch.float32)
    ops.linear_cross_entropy_backward(c, h, w, t, lse, dhidden=fh, dweight=fw)
    step = 1e-4
    for grad, at in ((fh, 0), (fw, 1)):
        way = randn(20 + at, *grad.shape).double()
        f = []
        for s in (step, -step):
            args = [h.double(), w.double()]
            args[at] = args[at] + s * way
            z = args[0] @ args[1].T
            l = torch.logsumexp(z, 1) - z.gather(1, t.clamp(min=0)[:, None])[:, 0]
            f.append(float((c.double() * torch.where(t >= 0, l, 0.0)).sum()))
        slope = (f[0] - f[1]) / (2 * step)
        # G rounded to fp16 (2^-11), and the third derivative times step^2
        assert abs(float((grad.double() * way).sum()) - slope) <= (2.0 ** -11 + 1e-5) * float((grad.double() * way).abs().sum())


def test_linear_cross_entropy_pieces_of_the_vocabulary(ops):
    """More than one piece: G's half GiB ends inside the vocabulary, and the last piece is ragged."""
    tokens, vocab, width = 2048, 140_003, 40
    h, w, t = head_inputs(tokens, vocab, width, torch.bfloat16)
    loss, lse = ops.linear_cross_entropy(h, w, t)
    dloss = torch.full((tokens,), 1.0 / tokens, device="cuda")
    dh, dw = ops.linear_cross_entropy_backward(dloss, h, w, t, lse)
    g, p = head_backward_ref(dloss, h, w, t, lse)
    u = 2.0 ** -8
    eg = u * g.abs() + 1e-4 * p
    for got, a, ea, b, what in ((dh, g, eg, w.double(), "dh"), (dw, g.T, eg.T, h.double(), "dw")):
        want = a @ b
        e = ea @ b.abs() + 2 * (a.shape[1] + 4) * 2.0 ** -24 * (a.abs() @ b.abs())
        within(got, want, e + u * (want.abs() + e), what)


def test_linear_cross_entropy_masked_rows(ops):
    h, w, t = head_inputs(200, 300, 64, torch.bfloat16)
    t[:] = -1                                                        # nothing takes part
    loss, lse = ops.linear_cross_entropy(h, w, t)
    dh, dw = ops.linear_cross_entropy_backward(torch.ones(200, device="cuda"), h, w, t, lse)
    assert not loss.any() and not dh.any() and not dw.any()
    h, w, t = head_inputs(200, 300, 64, torch.bfloat16)
    one = torch.ones(200, device="cuda")
    t[7], t[150] = -100, -5
    loss, lse = ops.linear_cross_entropy(h, w, t)
    dh, dw = ops.linear_cross_entropy_backward(one, h, w, t, lse)
    bad = h.clone()                                                  # padding may hold anything
    bad[7], bad[150] = math.nan, math.inf
    loss2, lse2 = ops.linear_cross_entropy(bad, w, t)
    assert torch.equal(loss, loss2)
    one2 = one.clone()
    one2[7] = math.nan
    dh2, dw2 = ops.linear_cross_entropy_backward(one2, bad, w, t, lse2)
    assert torch.equal(dh, dh2) and torch.equal(dw, dw2)
    t[9] = 300                                                       # outside the vocabulary
    loss3, lse3 = ops.linear_cross_entropy(h, w, t)
    assert math.isnan(float(loss3[9])) and int(torch.isnan(loss3).sum()) == 1
    dh3, _ = ops.linear_cross_entropy_backward(one, h, w, t, lse3)
    assert not dh3[9].any() and torch.equal(dh3[10:], dh[10:])


def test_linear_cross_entropy_extreme_logits(ops):
    """Logits of the type's largest magnitudes: the maximum is taken out before the exponentials."""
    h = torch.zeros(4, 8, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(300, 8, dtype=torch.bfloat16, device="cuda")
    h[:, 0] = torch.tensor([1.0, -1.0, 1e18, 3e38], device="cuda")
    w[:, 0] = torch.linspace(-50, 50, 300, device="cuda")
    w[17, 0] = -3e38 / 1e19
    t = torch.tensor([3, 3, 299, 299], device="cuda")
    loss, lse = ops.linear_cross_entropy(h, w, t)
    z = h.double() @ w.double().T
    want = torch.logsumexp(z, 1)
    assert bool(torch.isfinite(lse[:3]).all())
    within(lse[:3], want[:3], 2.0 ** -20 * (1 + want[:3].abs()), "lse")
    hi = h.clone()
    hi[1, 0] = math.inf                                              # one row's infinity is that row's own
    l2, _ = ops.linear_cross_entropy(hi, w, t)
    assert math.isnan(float(l2[1])) and float(l2[0]) == float(loss[0])


def test_linear_cross_entropy_layouts(ops):
    """Rows apart from each other and starts off TMA's boundary give what contiguous inputs give; outputs into slices."""
    big_h, big_w = randn(1, 130, 200, dtype=torch.bfloat16), randn(2, 500, 200, dtype=torch.bfloat16, scale=0.1)
    t = torch.randint(0, 500, (130,), generator=gen(3), device="cuda")
    d = torch.full((130,), 1 / 130, device="cuda")
    for cut in (slice(0, 128), slice(8, 136), slice(3, 131), slice(1, 102)):
        h, w = big_h[:, cut], big_w[:, cut]
        loss, lse = ops.linear_cross_entropy(h.contiguous(), w.contiguous(), t)
        l2, s2 = ops.linear_cross_entropy(h, w, t)
        assert torch.equal(loss, l2) and torch.equal(lse, s2)
        dh, dw = ops.linear_cross_entropy_backward(d, h.contiguous(), w.contiguous(), t, lse)
        n = w.numel()
        grads = torch.zeros(n + 40, dtype=torch.bfloat16, device="cuda")         # a worker's gradients in one row
        view = grads[13:13 + n].view(500, -1)
        wide = torch.zeros(130, 300, dtype=torch.float32, device="cuda")
        ops.linear_cross_entropy_backward(d, h, w, t, lse, dhidden=wide[:, 5:5 + h.shape[1]], dweight=view)
        assert torch.equal(view, dw) and not grads[:13].any() and not grads[13 + n:].any()
        assert torch.equal(wide[:, 5:5 + h.shape[1]].to(torch.bfloat16), dh) and not wide[:, :5].any() and not wide[:, 5 + h.shape[1]:].any()
        assert ops.linear_cross_entropy_backward(d, h, w, t, lse, dweight=False)[1] is None
        only = ops.linear_cross_entropy_backward(d, h, w, t, lse, dhidden=False)
        assert only[0] is None and torch.equal(only[1], dw)


def test_linear_cross_entropy_no_tokens(ops):
    h, w = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), randn(1, 100, 64, dtype=torch.bfloat16)
    t = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = ops.linear_cross_entropy(h, w, t)
    dh, dw = ops.linear_cross_entropy_backward(loss, h, w, t, lse)
    assert loss.shape == (0,) and dh.shape == (0, 64) and not dw.any()


# ---- orthogonalised updates ------------------------------------------------------------------------------------------------
COEF = (3.4445, -4.7750, 2.0315)


def ortho_ref(u, steps=5, coef=COEF, eps=1e-7):
    x = u.double()
    x = x / (torch.linalg.matrix_norm(x)[..., None, None] + eps)
    flip = x.shape[-2] > x.shape[-1]
    x = x.mT if flip else x
    for _ in range(steps):
        a = x @ x.mT
        x = coef[0] * x + (coef[1] * a + coef[2] * a @ a) @ x
    return x.mT if flip else x


# The scheme modelled in 64 bits with fp16 roundings of the same places gave at most 1.6e-3 (2-norm) over gaussian, low-rank
# and power-law spectra at 5 steps; half as much again, plus the output's rounding (rms 0.42 u)
ORTHO = {torch.bfloat16: 2.5e-3 + 0.5 * 2.0 ** -8, torch.float16: 2.5e-3 + 0.5 * 2.0 ** -11}


def ortho_close(got, want):
    err = torch.linalg.matrix_norm(got.double() - want) / torch.linalg.matrix_norm(want)
    assert float(err.max()) <= ORTHO[got.dtype], float(err.max())


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (1, 1, 70), (1, 70, 1), (2, 16, 16), (3, 33, 65), (1, 65, 33), (1, 128, 128), (2, 127, 300), (1, 300, 129),
                                             (1, 256, 256), (1, 257, 255), (5, 64, 512), (1, 640, 384), (2, 1100, 1300), (2, 100, 2100), (1, 4096, 128), (1, 60, 4100), (1, 2304, 2100)])
def test_orthogonalize(ops, batch, rows, cols, dtype):
    u = randn(1, batch, rows, 4) @ randn(2, batch, 4, cols) + randn(3, batch, rows, cols, scale=0.3)
    u = (u * 1e-3).to(dtype)
    out = ops.orthogonalize(u)
    assert out.dtype == (torch.float16 if dtype == torch.float16 else torch.bfloat16) and out.shape == u.shape
    ortho_close(out, ortho_ref(u))
    ops.sync()


# few tiles and a long side: the gram product's sums in slices, of both tile sizes, ragged ones and several matrices
@pytest.mark.parametrize("batch,rows,cols", [(1, 200, 2100), (1, 2688, 256), (2, 333, 4001), (1, 1000, 4096), (1, 2500, 640), (6, 130, 4100)])
def test_orthogonalize_long_side(ops, batch, rows, cols):
    u = randn(1, batch, rows, 4) @ randn(2, batch, 4, cols) + randn(3, batch, rows, cols, scale=0.3)
    for dtype in (torch.float32, torch.bfloat16):
        out = ops.orthogonalize(u.to(dtype))
        ortho_close(out, ortho_ref(u.to(dtype)))
        for _ in range(3):
            assert torch.equal(ops.orthogonalize(u.to(dtype)), out)
    ops.sync()


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
def test_orthogonalize_steps_and_coefficients(ops, steps):
    u = randn(1, 200, 264)
    for coef in (COEF, (1.875, -1.25, 0.375)):
        ortho_close(ops.orthogonalize(u, steps=steps, coefficients=coef), ortho_ref(u, steps, coef))


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_orthogonalize_momentum(ops, dtype, nesterov):
    m = randn(1, 3, 90, 130)
    g = randn(2, 3, 90, 130, dtype=dtype)
    want_m = 0.9 * m.double() + g.double()
    want_u = g.double() + 0.9 * want_m if nesterov else want_m
    out = ops.orthogonalize(g, momentum=m, beta=0.9, nesterov=nesterov)
    within(m, want_m, 2.0 ** -23 * (want_m.abs() + 1), "momentum")      # beta is rounded to 32 bits too
    ortho_close(out, ortho_ref(want_u))


@pytest.mark.parametrize("spectrum", ["power", "strong", "scaled"])
def test_orthogonalize_ill_conditioned(ops, spectrum):
    """What real gradients look like: the weak directions must not drown in the rounding of the strong ones."""
    u = randn(1, 384, 512)
    if spectrum == "power":
        a, s, b = torch.linalg.svd(u.double(), full_matrices=False)
        u = (a * torch.arange(1, 385, device="cuda").double() ** -1.0) @ b
    elif spectrum == "strong":
        u = randn(2, 384, 8) @ randn(3, 8, 512) + 0.1 * u
    else:
        u = u * torch.logspace(-2, 0, 384, device="cuda")[:, None]
    u = u.float()
    ortho_close(ops.orthogonalize(u), ortho_ref(u))


def test_orthogonalize_values_and_layouts(ops):
    u = randn(1, 2, 100, 140)
    base = ops.orthogonalize(u)
    assert torch.equal(ops.orthogonalize(u[1]), base[1])                 # a matrix alone and in a batch
    for scale in (2.0 ** -60, 2.0 ** 60, 2.0 ** 100):                    # squares beyond 32 bits
        ortho_close(ops.orthogonalize(u * scale, eps=0.0), ortho_ref(u))
    assert not ops.orthogonalize(torch.zeros(3, 20, 30, device="cuda")).any()
    bad = u.clone()
    bad[0, 3, 4] = math.nan
    got = ops.orthogonalize(bad)
    assert bool(torch.isnan(got[0]).any()) and torch.equal(got[1], base[1])
    big = torch.zeros(2, 120, 200, device="cuda")
    big[:, 5:105, 7:147] = u
    out = torch.zeros(2, 110, 160, dtype=torch.bfloat16, device="cuda")
    ops.orthogonalize(big[:, 5:105, 7:147], out=out[:, 2:102, 3:143])
    assert torch.equal(out[:, 2:102, 3:143], base)
    out[:, 2:102, 3:143] = 0
    assert not out.any()
    half = torch.empty(2, 100, 140, dtype=torch.float16, device="cuda")
    ortho_close(ops.orthogonalize(u, out=half), ortho_ref(u))
    assert ops.orthogonalize(torch.empty(0, 4, 5, device="cuda")).shape == (0, 4, 5)
    assert ops.orthogonalize(torch.empty(4, 0, device="cuda")).shape == (4, 0)


# ---- how they are called ---------------------------------------------------------------------------------------------------
def test_operators_on_another_stream(ops):
    h, w, t = head_inputs(300, 900, 96, torch.bfloat16)
    want = ops.linear_cross_entropy(h, w, t)
    u = randn(4, 150, 90)
    want_u = ops.orthogonalize(u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.linear_cross_entropy(h, w, t, stream=side)
    with torch.cuda.stream(side):
        got_u = ops.orthogonalize(u)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got_u, want_u)
    ops.sync(side)


def test_operators_give_the_same_bits_every_time(ops):
    h, w, t = head_inputs(700, 3000, 200, torch.bfloat16)
    x, dy, wn = randn(1, 3000, 300), randn(2, 3000, 300), randn(3, 300)
    _, mean, rstd = ops.layer_norm(x, wn)
    u = randn(4, 2, 500, 700)
    runs = []
    for _ in range(3):
        loss, lse = ops.linear_cross_entropy(h, w, t)
        runs.append([loss, lse, *ops.linear_cross_entropy_backward(loss, h, w, t, lse), *ops.layer_norm_backward(dy, x, wn, mean, rstd), ops.orthogonalize(u)])
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], r))


def test_operators_refuse(ops):
    from paper_2210_07454_b200.binding import SkError
    x, w = randn(1, 8, 64), randn(2, 64)
    h, wv, t = head_inputs(8, 100, 64, torch.bfloat16)
    d = torch.ones(8, device="cuda")
    _, mean, rstd = ops.layer_norm(x, w)
    bad = [
        lambda: ops.layer_norm(x.cpu()),
        lambda: ops.layer_norm(x.double()),
        lambda: ops.layer_norm(x, w[:63]),
        lambda: ops.layer_norm(x, w, w.half()),
        lambda: ops.layer_norm(x, eps=-1.0),
        lambda: ops.layer_norm(x, eps=math.nan),
        lambda: ops.layer_norm(x.T),
        lambda: ops.layer_norm(x, out=x.half()),
        lambda: ops.layer_norm(torch.empty(3, 0, device="cuda")),
        lambda: ops.layer_norm(x, out=x[:4]),
        lambda: ops.layer_norm(x[:1].expand(8, 64), out=x[:1].expand(8, 64)),
        lambda: ops.layer_norm_backward(x[:4], x, w, mean, rstd),
        lambda: ops.layer_norm_backward(x, x, w, mean[:4], rstd),
        lambda: ops.layer_norm_backward(x, x, w, mean, rstd.half()),
        lambda: ops.layer_norm_backward(x, x, w, mean, rstd, dweight=w[:3]),
        lambda: ops.linear_cross_entropy(h.float(), wv.float(), t),
        lambda: ops.linear_cross_entropy(h, wv.half(), t),
        lambda: ops.linear_cross_entropy(h, wv[:, :32], t),
        lambda: ops.linear_cross_entropy(h, wv, t.int()),
        lambda: ops.linear_cross_entropy(h, wv, t[:4]),
        lambda: ops.linear_cross_entropy(h, wv[:0], t),
        lambda: ops.linear_cross_entropy(h.T, wv, t),
        lambda: ops.linear_cross_entropy_backward(d[:4], h, wv, t, d),
        lambda: ops.linear_cross_entropy_backward(d, h, wv, t, d, dweight=torch.empty(100, 64, dtype=torch.float16, device="cuda")),
        lambda: ops.linear_cross_entropy_backward(d, h, wv, t, d, dhidden=torch.empty(8, 63, dtype=torch.bfloat16, device="cuda")),
        lambda: ops.orthogonalize(x[0]),
        lambda: ops.orthogonalize(x, steps=0),
        lambda: ops.orthogonalize(x, steps=33),
        lambda: ops.orthogonalize(x, coefficients=(20.0, 0.0, 0.0)),
        lambda: ops.orthogonalize(x, coefficients=(math.nan, 0.0, 0.0)),
        lambda: ops.orthogonalize(x, coefficients=(1.0, 2.0)),
        lambda: ops.orthogonalize(x, out=torch.empty_like(x)),
        lambda: ops.orthogonalize(x, momentum=x.half()),
        lambda: ops.orthogonalize(x, momentum=x[:4]),
        lambda: ops.orthogonalize(x.unsqueeze(0).expand(2, 8, 64), out=torch.empty(8, 64, dtype=torch.bfloat16, device="cuda").expand(2, 8, 64)),
        lambda: ops.orthogonalize(x, eps=-1.0),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(SkError):
            f()
            pytest.fail(f"call {i} was not refused")
    ops.sync()


def test_workspaces_are_checked():
    import ctypes
    from paper_2210_07454_b200 import binding
    L = binding.lib()
    n = 160
    u = randn(1, n, n)
    out = torch.empty(n, n, dtype=torch.bfloat16, device="cuda")
    need = L.sk_orthogonalize_workspace(1, n, n)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    coef = (ctypes.c_float * 3)(*COEF)

    def call(ptr, size):
        return L.sk_orthogonalize(u.data_ptr(), n, n * n, 0, None, 0, 0, 0.0, 0, out.data_ptr(), n, n * n, 1, 1, n, n, 5, coef, 1e-7, ptr, size, None)

    assert call(ws.data_ptr(), need) == 0
    assert call(ws.data_ptr(), need - 1) == -1 and b"workspace" in L.sk_last_error()
    assert call(None, need) == -1
    assert call(ws.data_ptr() + 16, need) == -1 and b"aligned" in L.sk_last_error()
    assert L.sk_layer_norm(u.data_ptr(), 63, u.data_ptr(), 64, 0, 64, 64, None, None, 0, 1e-5, None, None, None) == -1
    assert L.sk_layer_norm(u.data_ptr() + 2, 64, u.data_ptr(), 64, 0, 4, 64, None, None, 0, 1e-5, None, None, None) == -1
    assert L.sk_layer_norm(None, 64, u.data_ptr(), 64, 0, 4, 64, None, None, 0, 1e-5, None, None, None) == -1
    torch.cuda.synchronize()


def test_offsets_beyond_32_bits(ops):
    """Rows 2^21 elements apart: the last ones start beyond 2^32 elements."""
    gap, rows = 2 ** 21, 2100
    big = torch.empty(gap * rows, dtype=torch.bfloat16, device="cuda").view(rows, gap)
    for cols in (200, 333):
        x = big[:, 5:5 + cols]
        x.copy_(randn(1, rows, cols))
        w, b = randn(2, cols), randn(3, cols)
        want = ops.layer_norm(x.contiguous(), w, b)
        got = ops.layer_norm(x, w, b, out=big[:, 1000:1000 + cols])
        # not the same grouping of the columns, so not the same bits: some ulp of the output, and of the statistics
        within(got[0], want[0].double(), 2.0 ** -6 * want[0].double().abs() + 1e-4, "y")
        within(got[1], want[1].double(), 1e-5 + 1e-5 * want[1].double().abs(), "mean")
        dy = randn(4, rows, cols, dtype=torch.bfloat16)
        a = ops.layer_norm_backward(dy, x, w, want[1], want[2], dx=big[:, 1000:1000 + cols])
        c = ops.layer_norm_backward(dy, x.contiguous(), w, want[1], want[2])
        within(a[0], c[0].double(), 2.0 ** -6 * c[0].double().abs() + 1e-4, "dx")
        within(a[1], c[1].double(), 1e-3 + 1e-5 * c[1].double().abs(), "dw")
        t = torch.randint(0, rows, (300,), generator=gen(5), device="cuda")
        h = randn(6, 300, cols, dtype=torch.bfloat16)
        loss, lse = ops.linear_cross_entropy(h, x.contiguous(), t)
        l2, s2 = ops.linear_cross_entropy(h, x, t)
        assert torch.equal(loss, l2) and torch.equal(lse, s2)
        dw = ops.linear_cross_entropy_backward(loss, h, x.contiguous(), t, lse)[1]
        ops.linear_cross_entropy_backward(loss, h, x, t, lse, dhidden=False, dweight=big[:, 1000:1000 + cols])
        assert torch.equal(big[:, 1000:1000 + cols], dw)
        for part in (x, x[:, :100]):
            out = ops.orthogonalize(part.contiguous())
            assert torch.equal(ops.orthogonalize(part, out=big[:, 1000:1000 + part.shape[1]]), out)
    ops.sync()


# ---- together ----------------------------------------------------------------------------------------------------------------
def test_the_example_learns():
    """The example trains with every operator and the compressed step; the loss falls well below that of a uniform guess."""
    import importlib.util
    import os
    from conftest import ROOT
    spec = importlib.util.spec_from_file_location("language_model", os.path.join(ROOT, "examples", "language_model.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(steps=80)
    assert all(math.isfinite(v) for v in losses)
    assert losses[-1] < min(losses[0], math.log(1024)) - 1.0
