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
