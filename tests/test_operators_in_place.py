"""Outputs that are one of the inputs: what the kernels cannot do in place is refused before anything is launched (no device needed)."""
import pytest

pytest.importorskip("torch")

P, Q = 4096, 1 << 20                                               # aligned addresses that are never read


@pytest.fixture
def refused():
    from paper_2210_07454_b200 import binding
    L = binding.lib()

    def check(name, *args):
        return getattr(L, name)(*args) == -1 and b"in place" in L.sk_last_error()
    return check


def test_layer_norm_over_its_input_needs_the_same_rows(refused):
    def norm(y, ld_y):
        return refused("sk_layer_norm", P, 16, y, ld_y, 0, 4, 8, None, None, 0, 1e-5, None, None, None)

    assert norm(P, 8) and norm(P, 24)
    assert not norm(P, 16) and not norm(Q, 8)                      # these get as far as the device

    def backward(dx, ld_dx):
        return refused("sk_layer_norm_backward", P, 16, Q, 24, dx, ld_dx, 0, 4, 8, None, 0, P, P, None, None, 0, None, 0, None)

    assert backward(P, 24) and backward(Q, 16)
    assert not backward(P, 16) and not backward(Q, 24) and not backward(2 * Q, 8)


def test_the_heads_weight_gradient_is_not_written_over_the_weight(refused):
    """The weight is read again while its gradient is written."""
    def backward(dhidden, dweight):
        return refused("sk_linear_cross_entropy_backward", P, P, 8, Q, 8, 1, 4, 10, 8, P, P, dhidden, 8, 1, dweight, 8, 1, None, 0, None)

    assert backward(None, Q) and backward(2 * Q, Q) and backward(Q, None)
    assert not backward(P, 2 * Q)                                  # dhidden over hidden is fine: hidden is copied first
