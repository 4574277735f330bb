"""Waits inside the operators' kernels that run out: a signal is withheld, the kernel ends by itself soon after the limit, the host
reads an error, and the next call is whole again."""
import time

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# tiles of both sizes, with the gram product's sums in slices and without
SIZES = [(1, 300, 300), (12, 768, 768), (1, 2688, 256), (1, 1000, 4096), (1, 2304, 2100)]


@pytest.mark.parametrize("batch,rows,cols", SIZES)
def test_a_withheld_signal_ends_in_an_error(batch, rows, cols):
    from paper_2210_07454_b200 import binding, operators as ops
    gen = torch.Generator(device="cuda").manual_seed(rows)
    u = torch.randn(batch, rows, cols, generator=gen, device="cuda")
    want = ops.orthogonalize(u)
    ops.sync()
    binding._check(binding.lib().sk_test_operators_wait(100))
    start = time.monotonic()
    ops.orthogonalize(u)
    with pytest.raises(binding.SkError, match="wait"):
        ops.sync()
    assert 0.1 <= time.monotonic() - start < 2.0     # one limit and what follows from it; not the thirty seconds that a call has otherwise
    ops.sync()                                       # reported once
    assert torch.equal(ops.orthogonalize(u), want)
    ops.sync()


def test_the_limit_is_checked():
    from paper_2210_07454_b200 import binding
    for bad in (0, 1001):
        assert binding.lib().sk_test_operators_wait(bad) == -1


def test_every_wait_is_reported_once_whatever_the_stream():
    """Waits that run out in one stream while another's are being reported: none is lost, none reported twice."""
    from paper_2210_07454_b200 import binding, operators as ops
    u = torch.randn(1, 300, 300, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    ops.orthogonalize(u)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for sync_on in (None, side):
        for _ in range(2):
            binding._check(binding.lib().sk_test_operators_wait(20))
            ops.orthogonalize(u, stream=side)
        side.synchronize()
        with pytest.raises(binding.SkError, match="ran out"):
            ops.sync(sync_on)                        # the whole device's, from any stream
        ops.sync()
        ops.sync(side)
        binding._check(binding.lib().sk_test_operators_wait(20))
        ops.orthogonalize(u)                         # after a report another
        with pytest.raises(binding.SkError, match="ran out"):
            ops.sync()
        ops.sync(side)


@pytest.mark.parametrize("batch,rows,cols", SIZES)
def test_a_withheld_signal_ends_in_an_error_where_every_matrix_is_a_pair(batch, rows, cols):
    """fp16 outputs have kernels of their own."""
    from paper_2210_07454_b200 import binding, operators as ops
    u = torch.randn(batch, rows, cols, generator=torch.Generator(device="cuda").manual_seed(cols), device="cuda").half()
    want = ops.orthogonalize(u)
    ops.sync()
    binding._check(binding.lib().sk_test_operators_wait(100))
    start = time.monotonic()
    ops.orthogonalize(u)
    with pytest.raises(binding.SkError, match="ran out"):
        ops.sync()
    assert 0.1 <= time.monotonic() - start < 2.0
    assert torch.equal(ops.orthogonalize(u), want)
    ops.sync()
