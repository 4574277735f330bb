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


# ratios that overflow, by themselves or as a difference of infinite losses, under bounds that do and do not reach them
@pytest.mark.parametrize("clip", [(0.2, 0.2), (1.0, math.inf), (0.2, 3e38), (0.2, 1e60), (0.0, 0.0)], ids=str)
@pytest.mark.parametrize("of", ["tokens", "sequences"])
@pytest.mark.parametrize("zero", [0.0, -0.0])
def test_an_advantage_of_zero_is_zero_whatever_the_ratio(ops, zero, of, clip):
    for old in (89.0, 200.0, 3e38, math.inf):
        nll, a = vector(0.0), vector(zero)
        offsets = torch.tensor([0, 1], device="cuda")
        result, norm = ops.policy_loss(nll, vector(old), a, offsets=offsets, clip=clip, advantage_of=of)
        assert result[0] == 0 and norm.tolist() == [1.0]
        assert float(result[2]) == (old > math.log1p(clip[1]))
        assert ops.policy_loss_backward(None, nll, vector(old), a, norm, offsets=offsets, clip=clip, advantage_of=of).tolist() == [0.0]


def test_advantages_of_zero_beside_others(ops):
    """A group of answers of one reward, advantages of zero, next to one with advantages: only the latter counts."""
    g = torch.Generator(device="cuda").manual_seed(2)
    nll = torch.rand(4000, generator=g, device="cuda")
    old = nll + 0.1
    offsets, a = torch.tensor([0, 1500, 4000], device="cuda"), vector(0.0, 1.5)
    args = dict(offsets=offsets, clip=(1.0, math.inf), advantage_of="sequences")
    want, norm = ops.policy_loss(nll, old, a, average="sequences", **args)
    grad = ops.policy_loss_backward(None, nll, old, a, norm, **args)
    old[:1500] += 200.0
    got, norm = ops.policy_loss(nll, old, a, average="sequences", **args)
    assert torch.equal(got, want)
    assert torch.equal(ops.policy_loss_backward(None, nll, old, a, norm, **args), grad) and not grad[:1500].any()


def test_a_ratio_that_is_no_number_stays_one(ops):
    for nll, old in ((math.nan, 1.0), (1.0, math.nan), (math.inf, math.inf)):
        result, norm = ops.policy_loss(vector(nll), vector(old), vector(0.0))
        assert math.isnan(float(result[0]))
        assert math.isnan(ops.policy_loss_backward(None, vector(nll), vector(old), vector(0.0), norm).item())


def test_divergence_over_its_whole_range(ops):
    """exp(e) - e - 1, infinite at both ends (a token that the policy or that the reference excludes). exp is 3.8 times as far off relative to the
    difference at most, 15.2 E; the difference's two roundings."""
    for v in torch.tensor(FAR + NEAR).float().tolist() + [-math.inf, math.inf]:
        zero = vector(0.0)
        for nll, ref in ((zero, vector(-v)), (vector(v), zero)):
            result, _ = ops.policy_loss(nll, nll, zero, reference_nll=ref, kl=0.5) if math.isfinite(v) else ops.policy_loss(nll, zero, zero, reference_nll=ref, kl=0.5)
            want = math.inf if v > 700 or math.isinf(v) else math.expm1(v) - v if abs(v) > 1e-3 else v * v / 2 * (1 + v / 3 * (1 + v / 4))
            if want > 3.4e38:
                assert float(result[1]) == math.inf and float(result[0]) == math.inf, (v, result)
            else:
                assert abs(float(result[1]) - want) <= 20 * E * want, (v, result)
                assert abs(float(result[0]) - 0.5 * want) <= 22 * E * 0.5 * want, (v, result)
