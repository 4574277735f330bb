"""The operators where a thread has several rows and a unit several tiles, against plain implementations in 64 bits.

Bounds as beside the smaller sizes (test_gpu_operators.py), with what longer sums add: they are stated before any run.
"""
import math

import pytest

from test_gpu_operators import HALF, TINY, TYPES, U, backward_close, gen, head_inputs, head_ref, norm_ref, randn, within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def forward_close(ops, x, w, b):
    """y, mean and rstd of every row; x may have any layout."""
    cols, dtype = x.shape[-1], x.dtype
    y, mean, rstd = ops.layer_norm(x, w, b, eps=1e-5)
    for part in torch.arange(x.shape[0], device="cuda").split(4096):              # 64-bit copies of some rows at a time
        want, m, r, h = norm_ref(x[part], w, b, 1e-5)
        em = (cols + 2) * 2.0 ** -24 * x[part].double().abs().mean(-1)
        er = r * ((cols + 8) * 2.0 ** -24 + 2 * em * r)
        within(mean[part], m, em + 2.0 ** -24 * m.abs(), "mean")
        within(rstd[part], r, er + 2.0 ** -22 * r, "rstd")
        eh = ((em * r)[:, None] + h.abs() * (er / r)[:, None] + 4 * 2.0 ** -24 * (h.abs() + (m.abs() * r)[:, None])) * w.double().abs()
        within(y[part], want, U[dtype] * (want.abs() + eh) + eh + 2.0 ** -23 * want.abs() + TINY[dtype], "y")


# several rows a thread (the ring goes round more than once) for every division of rows over threads; widths on and off the 16-byte boundary,
# where the rows' starts differ, and rows beyond the register kernels
MANY = [(80001, 61), (80000, 64), (30003, 200), (30000, 256), (30001, 333), (20000, 512), (12001, 768), (12000, 770), (9000, 1001), (5000, 1024),
        (6001, 1027), (4000, 2048), (3001, 4096), (3000, 4097), (2003, 8191), (2500, 8192), (1500, 12288), (1300, 16384), (1300, 16385)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", MANY)
def test_layer_norm_of_many_rows(ops, rows, cols, dtype):
    x = randn(1, rows, cols, dtype=dtype, scale=1.5) + randn(2, rows, 1, dtype=dtype)
    forward_close(ops, x, 1 + randn(3, cols, scale=0.1), randn(4, cols, scale=0.1))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols", MANY)
def test_layer_norm_backward_of_many_rows(ops, rows, cols, dtype):
    backward_close(ops, rows, cols, dtype)


# rows that start off the boundary though their distance is a multiple of 16 bytes, rows whose distance is not, and y, dy and dx that lie
# otherwise than x
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows,cols,ld,start", [(9000, 1001, 1008, 3), (9000, 1001, 1013, 5), (9000, 1000, 1016, 1), (5000, 2049, 2057, 7), (12000, 300, 303, 2)])
def test_layer_norm_of_many_rows_apart(ops, rows, cols, ld, start, dtype):
    def apart(seed, ld, start):
        return randn(seed, rows * ld + start + 8, dtype=dtype)[start:start + rows * ld].view(rows, ld)[:, :cols]

    x, w, b = apart(1, ld, start), 1 + randn(3, cols, scale=0.1), randn(4, cols, scale=0.1)
    forward_close(ops, x, w, b)
    want, mean, rstd = ops.layer_norm(x.contiguous(), w, b)
    for out_ld, out_start in ((ld, start), (ld + 1, 0)):
        room = torch.zeros(rows * out_ld + out_start + 8, dtype=dtype, device="cuda")
        out = room[out_start:out_start + rows * out_ld].view(rows, out_ld)[:, :cols]
        ops.layer_norm(x, w, b, out=out)
        # two groupings of the columns: each within its bound, so at most two roundings and some units of 2^-24 times cols apart
        within(out, want.double(), 2 * U[dtype] * want.double().abs() + 2.0 ** -20 * (1 + want.double().abs()) + TINY[dtype], "y")
        out.zero_()
        assert not room.any()                                        # nothing beside the rows
    dy = apart(5, ld + 2, 1)
    plain = ops.layer_norm_backward(dy.contiguous(), x.contiguous(), w, mean, rstd)
    room = torch.zeros(rows * ld + start + 8, dtype=dtype, device="cuda")
    dx = room[start:start + rows * ld].view(rows, ld)[:, :cols]
    for d in (dy, apart(5, ld, start)):
        if d is not dy:
            plain = ops.layer_norm_backward(d.contiguous(), x.contiguous(), w, mean, rstd)
        got = ops.layer_norm_backward(d, x, w, mean, rstd, dx=dx)
        scale = rstd.double()[:, None] * (d.double() * w.double()).abs().amax(1, keepdim=True)
        within(got[0], plain[0].double(), 2 * U[dtype] * plain[0].double().abs() + (cols + 16) * 2.0 ** -24 * 2 * scale + TINY[dtype], "dx")
        h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        bound = 2 * (rows + 8) * 2.0 ** -24 * (d.double() * h).abs().sum(0)
        within(got[1], plain[1].double(), bound, "dw")
        within(got[2], plain[2].double(), 2 * (rows + 4) * 2.0 ** -24 * d.double().abs().sum(0), "db")
        dx.zero_()
        assert not room.any()


# tiles of both sizes with several tiles a unit: accumulators take turns, the ring is carried from tile to tile
@pytest.mark.parametrize("dtype", HALF, ids=str)
@pytest.mark.parametrize("tokens,vocab,width", [(2048, 20000, 256), (1500, 33001, 320), (300, 20001, 100), (9, 60000, 64), (4097, 9999, 65), (1000, 32003, 1000)])
def test_linear_cross_entropy_of_many_tiles(ops, tokens, vocab, width, dtype):
    h, w, t = head_inputs(tokens, vocab, width, dtype)
    loss, lse = ops.linear_cross_entropy(h, w, t)
    z, want_lse, want_loss, ez = head_ref(h, w, t)
    # beside the logits' errors: 17 additions in a chunk of 32 columns, four chunks with a rescaling each, the pieces of 64 columns dealt over 64
    # threads, and 18 additions over those
    adds = 17 + 8 + (2 * ((vocab + 127) // 128) + 63) // 64 + 18
    e = ez.amax(1) + 2.0 ** -20 * (1 + z.abs().amax(1)) + adds * 2.0 ** -24
    within(lse, want_lse, e, "lse")
    within(loss, want_loss, 2 * e, "loss")
    ops.sync()


# beyond one piece of the vocabulary, in both types: the loss, and the gradients on the definition's lse
@pytest.mark.parametrize("dtype", HALF, ids=str)
def test_linear_cross_entropy_of_several_pieces(ops, dtype):
    tokens, vocab, width = 2048, 140_003, 40
    h, w, t = head_inputs(tokens, vocab, width, dtype)
    loss, lse = ops.linear_cross_entropy(h, w, t)
    want, norm = torch.empty(tokens, dtype=torch.float64, device="cuda"), torch.empty(tokens, dtype=torch.float64, device="cuda")
    bound = torch.empty_like(want)
    for part in torch.arange(tokens, device="cuda").split(512):
        z, norm[part], want[part], ez = head_ref(h[part], w, t[part])
        bound[part] = ez.amax(1) + 2.0 ** -20 * (1 + z.abs().amax(1)) + (17 + 8 + 35 + 18) * 2.0 ** -24
    within(lse, norm, bound, "lse")
    within(loss, want, 2 * bound, "loss")
    dloss = torch.rand(tokens, generator=gen(7), device="cuda") / tokens
    dh, dw = ops.linear_cross_entropy_backward(dloss, h, w, t, norm.float())
    scale = torch.where(t >= 0, dloss.double(), 0.0)
    sums, sums_bound = torch.zeros(vocab, width, dtype=torch.float64, device="cuda"), torch.zeros(vocab, width, dtype=torch.float64, device="cuda")
    for part in torch.arange(tokens, device="cuda").split(512):
        z = h[part].double() @ w.double().T
        p = torch.exp(z - norm[part].float().double()[:, None]) * scale[part][:, None]
        g = p.clone()
        g[torch.arange(len(part), device="cuda"), t[part].clamp(min=0)] -= scale[part]
        eg = U[dtype] * g.abs() + (1 + U[dtype]) * p * (bound[part].amax() + 2.0 ** -20 * (1 + z.abs()))
        if dtype == torch.float16:
            eg = eg + 2.0 ** -37 * float(dloss.max())
        ref = g @ w.double()
        e = eg @ w.double().abs() + 2 * (vocab + 4) * 2.0 ** -24 * (g.abs() @ w.double().abs())
        within(dh[part], ref, e + U[dtype] * (ref.abs() + e) + TINY[dtype], "dh")
        sums += g.T @ h[part].double()
        sums_bound += eg.T @ h[part].double().abs() + 2 * (tokens + 4) * 2.0 ** -24 * (g.abs().T @ h[part].double().abs())
    within(dw, sums, sums_bound + U[dtype] * (sums.abs() + sums_bound) + TINY[dtype], "dw")
    ops.sync()
