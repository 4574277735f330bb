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
