"""Outputs that hold more bits than the formats inside might keep: the error against 64 bits is little more than the output's own rounding."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def newton_schulz(u, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    x = u.double()
    x = x / (torch.linalg.matrix_norm(x)[..., None, None] + eps)
    flip = x.shape[-2] > x.shape[-1]
    x = x.mT if flip else x
    a, b, c = coefficients
    for _ in range(steps):
        g = x @ x.mT
        x = a * x + (b * g + c * g @ g) @ x
    return x.mT if flip else x


# fp16's rounding has an rms of at most 0.42 u, u = 2^-11: half a u.  Inside, pairs of fp16 (22 bits, errors of 1e-6 when modelled in 64 bits) and 32-bit
# sums that the tensor cores truncate: about 1e-6 of a sum of 2500 products, in each of fifteen products, three times amplified: 5e-5.
FP16 = 0.5 * 2.0 ** -11 + 5e-5


def error(got, want):
    return float((torch.linalg.matrix_norm(got.double() - want) / torch.linalg.matrix_norm(want)).max())


# the cluster's kernel with one block and with several, tiles of both sizes, sums in slices, wide and tall, ragged
@pytest.mark.parametrize("batch,rows,cols", [(12, 25, 70), (2, 128, 40), (1, 1, 70), (1, 65, 33), (2, 320, 64), (2, 59, 832), (1, 1638, 32), (1, 100, 4000), (2, 33, 4096),
                                             (3, 142, 229), (2, 300, 129), (1, 257, 255), (12, 256, 256), (4, 640, 512), (1, 2688, 256), (1, 200, 2100),
                                             (1, 1000, 4096), (2, 1664, 931), (1, 2304, 2100), (2, 130, 5000)])
def test_orthogonalize_keeps_fp16s_bits(batch, rows, cols):
    from paper_2210_07454_b200 import operators as ops
    u = (randn(1, batch, rows, 16) @ randn(2, batch, 16, cols) / 4 + 0.25 * randn(3, batch, rows, cols)) * 1e-3
    half = torch.empty(batch, rows, cols, dtype=torch.float16, device="cuda")
    for update in (u.half(), u, u.bfloat16()):
        got = ops.orthogonalize(update, out=half)
        assert error(got, newton_schulz(update)) <= FP16, update.dtype
        again = ops.orthogonalize(update, out=torch.empty_like(half))
        assert torch.equal(got, again)
    m = (randn(4, batch, rows, 16) @ randn(5, batch, 16, cols) / 4 + 0.1 * randn(6, batch, rows, cols)) * 5e-3
    want_m = 0.95 * m.double() + u.half().double()
    got = ops.orthogonalize(u.half(), momentum=m)
    assert got.dtype == torch.float16 and error(got, newton_schulz(u.half().double() + 0.95 * want_m)) <= FP16
    ops.sync()


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 7])
@pytest.mark.parametrize("rows,cols", [(90, 130), (300, 260)])
def test_orthogonalize_keeps_fp16s_bits_whatever_the_steps(rows, cols, steps):
    from paper_2210_07454_b200 import operators as ops
    u = randn(7, rows, cols).half()
    for coefficients in ((3.4445, -4.7750, 2.0315), (1.875, -1.25, 0.375)):
        got = ops.orthogonalize(u, steps=steps, coefficients=coefficients)
        # after few steps some entries are in fp16's subnormal range: half a step of 2^-24 each
        want = newton_schulz(u, steps, coefficients)
        small = 2.0 ** -25 * math.sqrt(rows * cols) / float(torch.linalg.matrix_norm(want))
        assert error(got, want) <= FP16 + small


# Beside the output's own rounding, which is that of the definition's value: the logits' errors (1e-6 of values about ten, in the exponent), the
# exponentials', 32-bit sums, and the gradient of the logits as a pair of 16-bit values (2^-17): 4e-5.
HEAD = 4e-5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("tokens,vocab,width", [(1, 3941, 1024), (1, 300, 64), (2, 7374, 2113), (4, 2048, 204), (5, 50257, 768), (10, 5332, 114), (17, 4288, 1127),
                                                (31, 1001, 65), (32, 130, 96), (33, 9000, 200), (48, 20001, 100), (63, 4000, 770), (64, 32003, 320)])
def test_linear_cross_entropy_backward_of_few_tokens_keeps_the_types_bits(tokens, vocab, width, dtype):
    """Few gradients of logits are large (those of the targets): what rounding them would cost is not averaged away over few tokens."""
    from paper_2210_07454_b200 import operators as ops
    w = (randn(1, vocab, width) * (2 / math.sqrt(width))).to(dtype)
    t = torch.randint(0, vocab, (tokens,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    sure = torch.arange(tokens, device="cuda") % 2 == 1
    h = (randn(3, tokens, width) + 2.5 * sure[:, None] * w[t].float()).to(dtype)
    if tokens > 4:
        t[3] = -100
    z = h.double() @ w.double().T
    lse = torch.logsumexp(z, 1).float()
    dloss = (0.5 + torch.rand(tokens, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")) / tokens
    dh, dw = ops.linear_cross_entropy_backward(dloss, h, w, t, lse)
    g = torch.exp(z - lse.double()[:, None])
    g[torch.arange(tokens, device="cuda"), t.clamp(min=0)] -= 1.0
    g *= torch.where(t >= 0, dloss.double(), 0.0)[:, None]
    for got, want in ((dh, g @ w.double()), (dw, g.T @ h.double())):
        rounding = float((want.to(dtype).double() - want).norm())
        assert float((got.double() - want).norm()) <= rounding + HEAD * float(want.norm())
    fh, fw = torch.empty_like(h, dtype=torch.float32), torch.empty_like(w, dtype=torch.float32)
    ops.linear_cross_entropy_backward(dloss, h, w, t, lse, dhidden=fh, dweight=fw)
    assert torch.equal(fh.to(dtype), dh) and torch.equal(fw.to(dtype), dw)
    for got, want in ((fh, g @ w.double()), (fw, g.T @ h.double())):
        assert float((got.double() - want).norm()) <= HEAD * float(want.norm())
    one = ops.linear_cross_entropy_backward(dloss, h, w, t, lse, dweight=False)[0], ops.linear_cross_entropy_backward(dloss, h, w, t, lse, dhidden=False)[1]
    assert torch.equal(one[0], dh) and torch.equal(one[1], dw)
    ops.sync()


@pytest.mark.parametrize("dtype,bits", [(torch.bfloat16, 8), (torch.float16, 11)], ids=["bfloat16", "float16"])
@pytest.mark.parametrize("tokens,vocab,width", [(300, 5000, 64), (1100, 20000, 96), (65, 3000, 100)])
def test_linear_cross_entropy_backward_of_a_mean(tokens, vocab, width, dtype, bits):
    """The gradient of a mean: every token has the same dloss, here one that the type rounds by half a unit.  The targets' entries of the
    logits' gradient are all about -dloss: an error that they have in common would scale the gradients as a whole."""
    from paper_2210_07454_b200 import operators as ops
    w = (randn(1, vocab, width) * (0.2 / math.sqrt(width))).to(dtype)
    t = torch.randint(0, vocab, (tokens,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    h = randn(3, tokens, width).to(dtype)
    z = h.double() @ w.double().T
    lse = torch.logsumexp(z, 1).float()
    rows = torch.arange(tokens, device="cuda")
    for c in ((1 + 2.0 ** -bits) * 2.0 ** -9, 1.0 / tokens):
        dloss = torch.full((tokens,), c, device="cuda")
        fh, fw = torch.empty_like(h, dtype=torch.float32), torch.empty_like(w, dtype=torch.float32)
        ops.linear_cross_entropy_backward(dloss, h, w, t, lse, dhidden=fh, dweight=fw)
        p = torch.exp(z - lse.double()[:, None])
        g = p.clone()
        g[rows, t] -= 1.0
        # -1 is exact: p - 1 is off by at most p, the other entries by half a unit (and by half of 2^-38 of -1 below fp16's range)
        off = p * 2.0 ** -bits + (2.0 ** -39 if dtype == torch.float16 else 0.0)
        off[rows, t] = p[rows, t]
        for got, want, norm in ((fh, g @ w.double(), torch.linalg.matrix_norm(w.double(), 2)), (fw, g.T @ h.double(), torch.linalg.matrix_norm(h.double(), 2))):
            want = want * float(dloss[0])
            assert float((got.double() - want).norm()) <= float(off.norm() * norm) * c + HEAD * float(want.norm()), c
    ops.sync()


# The tensor cores add sixteen products and the accumulator a step, each truncated to at least 24 bits of the largest: 17 times 2^-24 of what has been added up
# so far, at most.  For few tokens the accumulator is emptied after 256 values and the parts are added with rounding: of a sum of values of one sign,
# (s + 1) / 2 steps' errors for the s steps of a part and (n + 1) / 2 half ulps for n parts.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("width", [16, 64, 100, 256, 257, 300, 768, 1000, 2048, 2500, 4096, 8192])
def test_logits_of_few_tokens_are_sums_of_32_bits(width, dtype):
    """With a vocabulary of one word, lse is the logit.  (One accumulation of 2500 fp16 values came out 1.6e-5 too small, one of 4096 2.7e-5.)"""
    from paper_2210_07454_b200 import operators as ops
    bound = 17 * 2.0 ** -24 * (min(width, 256) / 16 + 1) / 2 + 2.0 ** -24 * (math.ceil(width / 256) + 1) / 2
    for tokens in (1, 5, 100):
        h, w = randn(1, tokens, width).abs().to(dtype), randn(2, 1, width).abs().to(dtype)
        z = (h.double() @ w.double().T)[:, 0]
        lse = ops.linear_cross_entropy(h, w, torch.zeros(tokens, dtype=torch.int64, device="cuda"))[1]
        assert float(((lse.double() - z) / z).abs().max()) <= bound
    ops.sync()


def test_the_loss_of_confident_tokens():
    """Two words, whose logits are exact, large, and apart by d: the loss is log(1 + exp(-d)).  It comes from their difference, which is exact, and the
    logarithm of a sum just above 1 (half an ulp of it, an ulp of the logarithm), with exp(-d) off by d 2^-23 (its argument's two roundings) and 2^-22.  Formed
    from a logarithm of sums of 1000 it would be off by half an ulp of that, 3e-5."""
    from paper_2210_07454_b200 import operators as ops
    d = torch.arange(0.25, 12.25, 0.25, device="cuda")
    h = torch.zeros(len(d), 64, dtype=torch.float16, device="cuda")
    h[:, 0], h[:, 1] = 1000.0, d
    w = torch.zeros(2, 64, dtype=torch.float16, device="cuda")
    w[:, 0], w[1, 1] = 1.0, -1.0
    loss, lse = ops.linear_cross_entropy(h, w, torch.zeros(len(d), dtype=torch.int64, device="cuda"))
    d = d.double()
    want = torch.log1p(torch.exp(-d))
    assert bool(((loss.double() - want).abs() <= 2.0 ** -23 + 2.0 ** -23 + torch.exp(-d) * (d * 2.0 ** -23 + 2.0 ** -22)).all())
    assert float((lse.double() - 1000 - want).abs().max()) <= 2.0 ** -14
    second = ops.linear_cross_entropy(h, w, torch.ones(len(d), dtype=torch.int64, device="cuda"))[0]
    assert bool(((second.double() - want - d).abs() <= 2.0 ** -22 + torch.exp(-d) * (d * 2.0 ** -23 + 2.0 ** -22) + 2.0 ** -24 * (d + want)).all())
    ops.sync()
