"""Outputs that are one of the inputs: what the kernels cannot do in place is refused before anything is launched."""
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


# Every call below ends in a refusal, also where there is a device: no kernel may ever see these addresses.
def test_layer_norm_over_its_input_needs_the_same_rows(refused):
    def norm(y, ld_y):
        return refused("sk_layer_norm", P, 16, y, ld_y, 0, 4, 8, None, None, 0, 1e-5, None, None, None)

    assert norm(P, 8) and norm(P, 24)

    def backward(dx, ld_dx):
        return refused("sk_layer_norm_backward", P, 16, Q, 24, dx, ld_dx, 0, 4, 8, None, 0, P, P, None, None, 0, None, 0, None)

    assert backward(P, 24) and backward(Q, 16)


def test_the_heads_weight_gradient_is_not_written_over_the_weight(refused):
    """The weight is read again while its gradient is written."""
    def backward(dhidden, dweight):
        return refused("sk_linear_cross_entropy_backward", P, P, 8, Q, 8, 1, 4, 10, 8, P, P, dhidden, 8, 1, dweight, 8, 1, None, 0, None)

    assert backward(None, Q) and backward(2 * Q, Q) and backward(Q, None)
    assert not backward(P, 2 * Q)                                  # dhidden over hidden is fine, as hidden is copied first: refused for its workspace


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,vocab,width", [(5, 300, 64), (200, 1000, 72), (2048, 140_003, 40)])
def test_the_hidden_states_gradient_over_the_hidden_states(tokens, vocab, width):
    import torch
    from paper_2210_07454_b200 import operators as ops
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    h, w = (torch.randn(n, width, generator=gen, device="cuda").bfloat16() for n in (tokens, vocab))
    t = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    loss, lse = ops.linear_cross_entropy(h, w, t)
    dh, dw = ops.linear_cross_entropy_backward(loss, h, w, t, lse)
    over = h.clone()
    got = ops.linear_cross_entropy_backward(loss, over, w, t, lse, dhidden=over)
    assert got[0] is over and torch.equal(over, dh) and torch.equal(got[1], dw)
