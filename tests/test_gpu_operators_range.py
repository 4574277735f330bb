"""The operators at the ends of the range that they accept, where an index or a product of sizes may not fit its type."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_linear_cross_entropy_backward_of_a_row_beyond_4_gib():
    """fp32 gradients of one row whose bytes do not fit 32 bits.  Hidden state and weight have no column in common, so the logit is 0;
    with lse = -log 2 the logit's gradient is exactly 1 in bf16, and the gradients are the inputs."""
    from paper_2210_07454_b200 import operators as ops
    width = 2 ** 30 + 8
    values = torch.arange(width, dtype=torch.int32, device="cuda").remainder_(251).to(torch.bfloat16).view(1, -1)
    h, w = values.clone(), values
    h[:, 1::2] = 0
    w[:, ::2] = 0
    one = torch.ones(1, device="cuda")
    dh, dw = torch.full((1, width), -1.0, device="cuda"), torch.full((1, width), -1.0, device="cuda")
    ops.linear_cross_entropy_backward(one, h, w, torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), -math.log(2.0), device="cuda"),
                                      dhidden=dh, dweight=dw)
    ops.sync()
    assert torch.equal(dw, h.float()) and torch.equal(dh, w.float())


def newton_schulz(u, steps=5, coefficients=(3.4445, -4.7750, 2.0315)):
    x = u.double()
    x = x / torch.linalg.matrix_norm(x)[..., None, None]
    flip = x.shape[-2] > x.shape[-1]
    x = x.mT if flip else x
    a, b, c = coefficients
    for _ in range(steps):
        g = x @ x.mT
        x = a * x + (b * g + c * g @ g) @ x
    return x.mT if flip else x


# 2-norm error of the iteration in its formats (see test_gpu_operators.py) plus half a unit of the output's rounding
BOUND = {torch.bfloat16: 2.5e-3 + 0.5 * 2.0 ** -8, torch.float16: 2.5e-3 + 0.5 * 2.0 ** -11}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("shape", [(100, 140), (2, 250, 180), (1, 2100, 200)], ids=str)
def test_orthogonalize_whatever_the_norm(shape, dtype):
    """The normalised matrix does not depend on a power of two in the update, from where its values are subnormal to the type's largest: a few
    strong directions over weak ones, which a format too small inside would drown."""
    from paper_2210_07454_b200 import operators as ops
    gen = torch.Generator(device="cuda").manual_seed(5)
    strong = torch.randn(*shape[:-1], 8, generator=gen, device="cuda") @ torch.randn(*shape[:-2], 8, shape[-1], generator=gen, device="cuda")
    u = (strong + 0.1 * torch.randn(shape, generator=gen, device="cuda")).to(dtype)
    for power in (-126, -121, -110, -90, -40, 0, 40, 90, 110, 116):      # |u| <= 2^5, norms up to 2^11
        scaled = (u.double() * 2.0 ** power).to(dtype)
        got, want = ops.orthogonalize(scaled, eps=0.0), newton_schulz(scaled)
        err = torch.linalg.matrix_norm(got.double() - want) / torch.linalg.matrix_norm(want)
        assert float(err.max()) <= BOUND[got.dtype], (power, float(err.max()))
    ops.sync()


@pytest.mark.parametrize("rows,cols", [(20, 600), (600, 20), (128, 1100), (1100, 127), (1, 2100), (3, 2500), (65, 4090)])
def test_orthogonalize_in_a_cluster_with_blocks_that_hold_nothing(rows, cols):
    """A cluster has a power of two of blocks of 256 columns each: the last ones may have none."""
    from paper_2210_07454_b200 import operators as ops
    u = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda")
    got, want = ops.orthogonalize(u, out=torch.empty(rows, cols, dtype=torch.float16, device="cuda")), newton_schulz(u)
    assert float(torch.linalg.matrix_norm(got.double() - want) / torch.linalg.matrix_norm(want)) <= BOUND[torch.float16]
    m = torch.zeros_like(u)
    ops.orthogonalize(u, momentum=m, beta=0.5, nesterov=False, out=got)
    assert torch.equal(m, u)
    assert float(torch.linalg.matrix_norm(got.double() - want) / torch.linalg.matrix_norm(want)) <= BOUND[torch.float16]
    ops.sync()
