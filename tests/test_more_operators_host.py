"""The host side of the products grouped by expert, of the order they take, of dropout and of the policy loss without a device: what is refused before
anything is launched."""
import math

import pytest

torch = pytest.importorskip("torch")

P, Q, R = 4096, 1 << 20, 1 << 24                                   # aligned addresses that are never read


@pytest.fixture(scope="module")
def L():
    from paper_2210_07454_b200 import binding
    return binding.lib()


def refused(L, code, word):
    return code == -1 and word in L.sk_last_error()


def test_host_tensors_are_refused():
    from paper_2210_07454_b200 import binding, operators as o
    x, w, i = torch.zeros(4, 8), torch.zeros(2, 8, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: o.grouped_linear(x, w, i), lambda: o.grouped_linear_backward(x, x, w, i), lambda: o.sort_by_expert(i, 2), lambda: o.dropout(x, 0.1, 1),
                 lambda: o.dropout_backward(x, 0.1, 1), lambda: o.policy_loss(x[:, 0], x[:, 0], x[:, 0]),
                 lambda: o.policy_loss_backward(None, x[:, 0], x[:, 0], x[:, 0], x[:, 0])):
        with pytest.raises(binding.SkError):
            call()


def test_grouped_linear_checks(L):
    def call(x=P, ld_x=8, w=Q, ld_w=8, s_w=64, type_=1, rows=4, groups=2, width=8, out=8, off=P, y=R, ld_y=8, ws=None, need=0):
        return L.sk_grouped_linear(x, ld_x, w, ld_w, s_w, type_, rows, groups, width, out, off, y, ld_y, 1, ws, need, None)

    assert call(rows=0) == 0
    for kw, word in ((dict(type_=0), b"type"), (dict(type_=7), b"type"), (dict(groups=0), b"groups"), (dict(groups=2049), b"groups"), (dict(width=0), b"width"),
                     (dict(out=0), b"width"), (dict(rows=1 << 31), b"rows"), (dict(x=None), b"null"), (dict(w=None), b"null"), (dict(off=None), b"null"),
                     (dict(y=None), b"null"), (dict(ld_x=7), b"leading"), (dict(ld_w=7), b"leading"), (dict(ld_y=7), b"leading"), (dict(x=P + 1), b"aligned"),
                     (dict(w=Q + 1), b"aligned"), (dict(off=P + 4), b"aligned"), (dict(y=R + 1), b"aligned"), (dict(y=P), b"in place"), (dict(y=Q), b"in place"),
                     (dict(rows=1 << 30, out=1 << 20, ld_y=1 << 20), b"large"), (dict(x=P + 2), b"workspace"), (dict(ld_x=9), b"workspace"),
                     (dict(w=Q + 2), b"workspace"), (dict(s_w=65), b"workspace"), (dict(x=P + 2, ws=Q + 16, need=1 << 20), b"workspace")):
        assert refused(L, call(**kw), word), kw
    assert L.sk_grouped_linear_workspace(P, 8, Q, 8, 64, 4, 2, 8, 8, R, 8) == 0
    assert L.sk_grouped_linear_workspace(P + 2, 8, Q, 8, 64, 4, 2, 8, 8, R, 8) > 0


def test_grouped_linear_backward_checks(L):
    def call(dy=P, ld_dy=8, x=2 * P, ld_x=8, w=Q, ld_w=8, s_w=64, type_=1, rows=4, groups=2, width=8, out=8, off=P, dx=R, ld_dx=8, dw=2 * R, ld_dw=8, s_dw=64,
             dw_type=1):
        return L.sk_grouped_linear_backward(dy, ld_dy, x, ld_x, w, ld_w, s_w, type_, rows, groups, width, out, off, dx, ld_dx, 1, dw, ld_dw, s_dw, dw_type, None, 0,
                                            None)

    assert call(dx=None, dw=None) == 0 and call(rows=0, dw=None) == 0
    for kw, word in ((dict(type_=0), b"type"), (dict(dw_type=2), b"type"), (dict(dy=None), b"null"), (dict(x=None), b"null"), (dict(ld_dy=7), b"leading"),
                     (dict(ld_dx=7), b"leading"), (dict(ld_dw=7), b"leading"), (dict(s_dw=63), b"overlap"), (dict(dx=R + 1), b"aligned"),
                     (dict(dw=R + 2, dw_type=0), b"aligned"), (dict(dx=P), b"in place"), (dict(dx=2 * P), b"in place"), (dict(dx=Q), b"in place"),
                     (dict(dw=Q), b"in place"), (dict(dw=P), b"in place"), (dict(dy=P + 2), b"workspace")):
        assert refused(L, call(**kw), word), kw


def test_sizes_of_nothing(L):
    """Questions about empty extents are answered, whatever the call itself would say."""
    for rows, groups, width, out in ((0, 2, 8, 8), (4, 0, 8, 8), (4, 2, 0, 8), (4, 2, 8, 0)):
        assert L.sk_grouped_linear_workspace(P + 2, 9, Q, 9, 64, rows, groups, width, out, R, 9) == 0
        assert L.sk_grouped_linear_backward_workspace(P + 2, 9, P, 9, Q, 9, 64, rows, groups, width, out, R, 9, 2 * R, 9, 72, 1) == 0
    assert L.sk_sort_by_expert_workspace(0, 4) == 0 and L.sk_sort_by_expert_workspace(10, 0) == 0 and L.sk_sort_by_expert_workspace(10, 5000) == 0
    # few tiles and many rows: the sums of the slices, below 80 MB whatever the sizes
    for width, out, groups in ((64, 200, 2), (768, 2048, 1), (256, 64, 30)):
        assert 0 < L.sk_grouped_linear_backward_workspace(P, out, P, width, Q, width, out * width, 30000, groups, width, out, R, width, 2 * R, width, out * width, 1) < (80 << 20)


def test_sort_by_expert_checks(L):
    def call(e=P, bits=64, n=10, groups=4, order=Q, places=R, off=2 * R):
        return L.sk_sort_by_expert(e, bits, n, groups, order, places, off, None, 0, None)

    for kw, word in ((dict(bits=16), b"bits"), (dict(groups=0), b"groups"), (dict(groups=2049), b"groups"), (dict(n=1 << 31), b"2^31"), (dict(e=None), b"null"),
                     (dict(off=None), b"null"), (dict(e=P + 4), b"aligned"), (dict(e=P + 2, bits=32), b"aligned"), (dict(order=Q + 4), b"aligned"),
                     (dict(order=P), b"in place"), (dict(places=P), b"in place"), (dict(off=P), b"in place")):
        assert refused(L, call(**kw), word), kw


def test_dropout_checks(L):
    def call(x=P, ld_x=8, r=None, ld_r=0, y=Q, ld_y=8, type_=0, rows=4, cols=8, p=0.1, at=None):
        return L.sk_dropout(x, ld_x, r, ld_r, y, ld_y, type_, rows, cols, p, 1, at, None)

    assert call(rows=0) == 0 and call(cols=0) == 0
    for kw, word in ((dict(type_=3), b"type"), (dict(p=-0.1), b"p must"), (dict(p=1.1), b"p must"), (dict(p=math.nan), b"p must"), (dict(x=None), b"null"),
                     (dict(y=None), b"null"), (dict(ld_x=7), b"leading"), (dict(ld_y=7), b"leading"), (dict(r=R, ld_r=7), b"leading"), (dict(x=P + 2), b"aligned"),
                     (dict(y=P, ld_y=9), b"in place"), (dict(r=Q, ld_r=16), b"in place"), (dict(at=P + 4), b"aligned"), (dict(rows=1 << 39, cols=1 << 39, ld_x=1 << 39, ld_y=1 << 39), b"many")):
        assert refused(L, call(**kw), word), kw


def test_policy_loss_checks(L):
    def call(nll=P, old=P, a=P, of=0, t=None, off=P, s=2, ref=P, n=10, low=0.2, high=0.2, kl=0.1, result=Q, norm=R):
        return L.sk_policy_loss(nll, old, a, of, t, off, s, ref, n, low, high, kl, 0, result, norm, None, 0, None)

    def back(nll=P, old=P, a=P, of=0, t=None, off=P, s=2, ref=P, n=10, low=0.2, high=0.2, kl=0.1, norm=Q, dnll=R, dloss=None):
        return L.sk_policy_loss_backward(dloss, nll, old, a, of, t, off, s, ref, n, low, high, kl, norm, dnll, None)

    assert back(n=0) == 0
    for f in (call, back):
        for kw, word in ((dict(nll=None), b"null"), (dict(old=None), b"null"), (dict(a=None), b"null"), (dict(norm=None), b"null"), (dict(s=0), b"sequences"),
                         (dict(off=None), b"one sequence"), (dict(low=-0.1), b"clip"), (dict(low=1.1), b"clip"), (dict(high=-1.0), b"clip"),
                         (dict(high=math.nan), b"clip"), (dict(kl=math.inf), b"kl"), (dict(ref=None), b"reference"), (dict(nll=P + 2), b"aligned"),
                         (dict(t=P + 4), b"aligned"), (dict(off=P + 4), b"aligned")):
            assert refused(L, f(**kw), word), kw
    assert refused(L, call(result=None), b"null") and refused(L, call(n=5000), b"workspace") and refused(L, back(dnll=None), b"null")
    assert L.sk_policy_loss_workspace(0, 3) == L.sk_policy_loss_workspace(10, 3) == 0 and L.sk_policy_loss_workspace(10, 3000) >= 16 * 3000
    assert L.sk_policy_loss_workspace(5000, 3) >= 16 * 6


def test_policy_gradient_over_what_other_tokens_read(L):
    def back(of, dnll, dloss=None, a=P):
        return L.sk_policy_loss_backward(dloss, P, P, a, of, None, P, 2, None, 10, 0.2, 0.2, 0.0, Q, dnll, None)

    for kw in (dict(of=0, dnll=Q), dict(of=1, dnll=Q), dict(of=0, dnll=R, dloss=R), dict(of=1, dnll=R, a=R)):
        assert refused(L, back(**kw), b"one value a token"), kw


def test_workspace_of_one_gradient(L):
    """The sums of dweight's slices are asked for with dweight only."""
    def need(dx, dw, rows=30000, width=64, out=200):
        return L.sk_grouped_linear_backward_workspace(P, out, P, width, Q, width, out * width, rows, 2, width, out, dx, width, dw, width, out * width, 1)

    assert need(R, None) == 0 < need(None, 2 * R) == need(R, 2 * R)
