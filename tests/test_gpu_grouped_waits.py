"""Waits inside the grouped products' kernels that run out: no operands are copied, the kernels end by themselves soon after the limit, the host reads an error, and the next call is
whole again."""
import time

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# single blocks, pairs, K in slices, rows in slices, sums in parts, outputs through the workspace, groups without rows
SIZES = [([1, 0, 3], 64, 72), ([900, 0, 1500, 260], 512, 768), ([5, 0, 2], 4096, 200), ([5000, 0, 130, 2000], 64, 200), ([130, 40], 33000, 2000), ([700, 0, 33, 1500], 1001, 1333)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("sizes,width,out", SIZES, ids=str)
def test_operands_that_do_not_come_end_in_an_error(sizes, width, out, dtype):
    from paper_2210_07454_b200 import binding, operators as ops
    gen = torch.Generator(device="cuda").manual_seed(width)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)
    ends = torch.tensor([0] + sizes, device="cuda").cumsum(0)
    rows = sum(sizes) + 9
    x, w, dy, wide = randn(rows, width), randn(len(sizes), out, width), randn(rows, out), torch.zeros(len(sizes), out, width, device="cuda")
    calls = [lambda: (ops.grouped_linear(x, w, ends),), lambda: ops.grouped_linear_backward(dy, x, w, ends), lambda: ops.grouped_linear_backward(dy, x, w, ends, dx=False, dweight=wide)[1:]]
    for call in calls:
        want = [t.clone() for t in call()]
        ops.sync()
        binding._check(binding.lib().sk_test_operators_wait(50))
        start = time.monotonic()
        call()
        with pytest.raises(binding.SkError, match="ran out"):
            ops.sync()
        assert 0.05 <= time.monotonic() - start < 2.0                # a limit or two for each of a call's products, not the thirty seconds that a call has otherwise
        ops.sync()                                                   # reported once
        assert all(torch.equal(a, b) for a, b in zip(call(), want))
        ops.sync()
