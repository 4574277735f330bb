"""The policy loss and its gradient at the ends of their range: references far from the policy or excluded by it, ratios that overflow with advantages of
zero. One token's value is compared, relative to its own size.

Tolerance before any run: exp of 32 bits is off by 4 E of itself, exp(e) - 1 beyond 1 by at most 6.3 E + E; kl, norm, dloss and their products
round seven times at most. 16 E.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

E = 2.0 ** -24
FAR = [-0.25, -1.0 + 2.0 ** -24, -1.0, -1.0 - 2.0 ** -23, -1.5, -5.0, -15.5, -20.0, -87.0, -104.0, -1e5, -(2.0 ** 24) - 2, -1e9, -3.4e38]
NEAR = [1e-6, 0.25, 1.0 - 2.0 ** -24, 1.0, 1.0 + 2.0 ** -23, 2.0, 30.0, 88.0]


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def vector(*values):
    return torch.tensor(values, device="cuda")


@pytest.mark.parametrize("tokens", [1, 5000])
def test_gradient_of_the_divergence_over_its_whole_range(ops, tokens):
    """kl (exp(e) - 1): -kl for a reference that gives a token next to no probability, or none."""
    e = torch.tensor(FAR + NEAR).float()                             # of whole numbers and of 32 bits: nll = 0 makes it the difference itself
    for i, v in enumerate(e.tolist() + [-math.inf, math.inf]):
        ref = torch.full((tokens,), -v, device="cuda")
        zero = torch.zeros(tokens, device="cuda")
        _, norm = ops.policy_loss(zero, zero, zero, reference_nll=ref, kl=0.25)
        got = ops.policy_loss_backward(None, zero, zero, zero, norm, reference_nll=ref, kl=0.25).double() * tokens
        want = 0.25 * (math.expm1(v) if v < 700 else math.inf)
        if math.isinf(want):
            assert bool((got == want).all()), v
        else:
            assert float((got - want).abs().max()) <= 16 * E * abs(want), (v, got[0].item(), want)


def test_gradient_of_a_token_that_the_reference_excludes_beside_others(ops):
    """Its own part stays what it is, and no other token's changes."""
    g = torch.Generator(device="cuda").manual_seed(1)
    nll, ref, a = (torch.randn(3000, generator=g, device="cuda").abs() for _ in range(3))
    old = nll + 0.05
    _, norm = ops.policy_loss(nll, old, a, reference_nll=ref, kl=0.5, clip=(0.2, 0.2))
    want = ops.policy_loss_backward(None, nll, old, a, norm, reference_nll=ref, kl=0.5)
    ref[7], ref[2500] = math.inf, 1e9
    got = ops.policy_loss_backward(None, nll, old, a, norm, reference_nll=ref, kl=0.5)
    d = old.double() - nll.double()
    for t in (7, 2500):
        value = float(norm[0].double() * (a[t].double() * torch.exp(d[t]) - 0.5))
        size = float(norm[0].double() * (a[t].double() * torch.exp(d[t]) + 0.5))
        assert abs(float(got[t]) - value) <= 16 * E * size
    got[[7, 2500]] = want[[7, 2500]]
    assert torch.equal(got, want)
