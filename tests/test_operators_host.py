"""The operators' host side without a device: what is refused before anything is launched, and the example's plain parts."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


def test_operators_refuse_host_tensors():
    from paper_2210_07454_b200 import binding, operators
    x = torch.zeros(4, 8)
    t = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: operators.layer_norm(x), lambda: operators.layer_norm_backward(x, x, None, x[:, 0], x[:, 0]),
                 lambda: operators.linear_cross_entropy(x, x, t), lambda: operators.linear_cross_entropy_backward(x[:, 0], x, x, t, x[:, 0]),
                 lambda: operators.orthogonalize(x)):
        with pytest.raises(binding.SkError):
            call()


def test_c_entries_check_before_they_launch():
    """Arguments are checked before the device is touched, so the refusals need none; sizes of workspaces are host arithmetic."""
    from paper_2210_07454_b200 import binding
    L = binding.lib()
    coef = (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315)
    p = 4096                                                       # an aligned address that is never read

    def ortho(batch=1, rows=200, cols=200, steps=5, c=coef, ld=200, out_type=1, eps=1e-7, ws=0):
        return L.sk_orthogonalize(p, ld, 64, 0, None, 0, 0, 0.0, 0, p, ld, 64, out_type, batch, rows, cols, steps, c, eps, None, ws, None)

    assert ortho(rows=0) == 0 and ortho(cols=0) == 0 and ortho(batch=0) == 0
    for kw, word in ((dict(steps=0), b"steps"), (dict(c=None), b"coefficients"), (dict(ld=199), b"leading"), (dict(out_type=0), b"out_type"),
                     (dict(rows=70000), b"rows"), (dict(eps=-1.0), b"eps"), ({}, b"workspace")):
        assert ortho(**kw) == -1 and word in L.sk_last_error(), kw

    def head(vocab=10, width=8, ld=8, type_=1, tokens=4):
        return L.sk_linear_cross_entropy(p, ld, p, ld, type_, tokens, vocab, width, p, p, p, None, 0, None)

    assert head(tokens=0) == 0
    for kw, word in ((dict(vocab=0), b"vocab"), (dict(ld=7), b"leading"), (dict(type_=0), b"type"), ({}, b"workspace")):
        assert head(**kw) == -1 and word in L.sk_last_error(), kw
    assert L.sk_layer_norm(p, 8, p, 8, 9, 4, 8, None, None, 0, 1e-5, None, None, None) == -1
    assert L.sk_layer_norm(p, 8, p, 8, 0, 0, 8, None, None, 0, 1e-5, None, None, None) == 0
    small, large = (L.sk_linear_cross_entropy_backward_workspace(p, 64, p, 64, t, 50257, 64) for t in (1, 8192))
    assert 0 < small < large < (600 << 20)                         # a piece of the gradient of the logits, not all of it
    assert L.sk_orthogonalize_workspace(1, 70000, 8) == 0
