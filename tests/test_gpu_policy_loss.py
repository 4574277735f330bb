"""The clipped policy loss and its gradient against the formulas in 64 bits.

Tolerances before any run: exp and expm1 of 32 bits are off by at most 2 units in the last place (2^-22 relative, with the rounding of their
argument of size at most 4: 2^-22 more), each product rounds once.
"""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

E = 2.0 ** -24


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def inputs(tokens, ends, seed=0, of="tokens", spread=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")
    old = randn(tokens).abs() * 2
    nll, ref = old + spread * randn(tokens), old + randn(tokens)
    a = randn(tokens if of == "tokens" else len(ends) - 1)
    targets = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.3, -1, 5)
    return nll, old, ref, a, targets, torch.tensor(ends, dtype=torch.int64, device="cuda")


def plain(nll, old, ref, a, targets, ends, clip, kl, average, of):
    """(result, norm, gradient) in 64 bits, and the sums of magnitudes that bound what they may be off by"""
    tokens, sequences = len(nll), len(ends) - 1
    number = torch.full((tokens,), -1, device="cuda")
    for s in range(sequences):
        number[ends[s]:ends[s + 1]] = s
    live = number >= 0
    if targets is not None:
        live &= targets >= 0
    at = number.clamp(min=0)
    A = (a[at] if of == "sequences" else a).double()
    d = torch.where(live, old.double() - nll.double(), 0.0)
    r = torch.exp(d)
    low, high = 1 - clip[0], 1 + clip[1]
    cut = torch.where(A >= 0, d > math.log1p(clip[1]), d < (math.log1p(-clip[0]) if clip[0] < 1 else -math.inf))
    s = A * torch.where(cut, torch.where(A >= 0, high, low), r)
    grad = torch.where(cut, 0.0, A * r)
    k = torch.zeros_like(d)
    if ref is not None:
        e = torch.where(live, nll.double() - ref.double(), 0.0)
        k = torch.expm1(e) - e
        grad = grad + kl * torch.expm1(e)
    counts = torch.zeros(sequences, dtype=torch.float64, device="cuda").index_add_(0, at, live.double())
    if average == "tokens":
        norm = torch.full_like(counts, 1 / float(counts.sum()) if float(counts.sum()) else 0.0)
    else:
        norm = torch.where(counts > 0, 1 / (counts * max(float((counts > 0).sum()), 1.0)), 0.0)
    share = torch.where(live, norm[at], 0.0)
    values = [torch.where(live, v, 0.0) for v in (kl * k - s, k, cut.double())]
    sizes = [torch.where(live, v, 0.0) for v in ((kl * (k.abs() + 1e-3)).abs() + s.abs(), k.abs(), cut.double())]
    total, size = (torch.stack([(share * v).sum() for v in vs]) for vs in (values, sizes))
    grad_size = torch.where(live, (A * r).abs() + (abs(kl) * (torch.exp(e) + 1) if ref is not None else 0.0), 0.0)
    return total, size, norm, share * torch.where(live, grad, 0.0), share * grad_size


def check(ops, tokens, ends, average="tokens", of="tokens", masked=True, kl=0.05, clip=(0.2, 0.25), reference=True, seed=0):
    nll, old, ref, a, targets, offsets = inputs(tokens, ends, seed, of)
    targets, ref = targets if masked else None, ref if reference else None
    args = dict(targets=targets, offsets=offsets, reference_nll=ref, clip=clip, kl=kl if reference else 0.0, advantage_of=of)
    result, norm = ops.policy_loss(nll, old, a, average=average, **args)
    dloss = torch.tensor([1.7], device="cuda")
    grad = ops.policy_loss_backward(dloss, nll, old, a, norm, **args)
    want, size, n, g, gs = plain(nll, old, ref, a, targets, ends, clip, kl if reference else 0.0, average, of)
    # a token's loss: exp 8 E, products and sums 4 E; eight tokens in 32 bits 8 E; a chunk's sum, the result rounded 2 E
    assert bool(((result.double() - want).abs() <= 24 * E * size + 2.0 ** -140).all()), (result, want)
    assert bool(((norm.double() - n).abs() <= 3 * E * n).all())
    assert bool(((grad.double() - 1.7 * g).abs() <= 24 * E * 1.7 * gs + 2.0 ** -140).all())
    return result, norm, grad


ENDS = [[0, 1], [0, 5], [0, 3, 3, 10], [0, 0, 7, 7, 40, 40], [2, 9, 20], [0, 2047], [0, 2048], [0, 2049], [0, 2048, 4096], [5, 2000, 2048, 2050, 9000],
        [0, 100, 30000], [0, 1, 2, 3, 2048, 6144, 6145], list(range(0, 3001)), list(range(0, 60001, 20))]


@pytest.mark.parametrize("of", ["tokens", "sequences"])
@pytest.mark.parametrize("average", ["tokens", "sequences"])
@pytest.mark.parametrize("ends", ENDS, ids=lambda e: str(e) if len(e) < 8 else f"{len(e) - 1} sequences")
def test_policy_loss(ops, ends, average, of):
    for behind in (0, 13):
        check(ops, ends[-1] + behind, ends, average, of)
    check(ops, ends[-1], ends, average, of, masked=False)


@pytest.mark.parametrize("average", ["tokens", "sequences"])
def test_without_a_reference_and_without_clipping(ops, average):
    check(ops, 5000, [0, 100, 5000], average, reference=False)
    check(ops, 5000, [0, 100, 5000], average, kl=0.0)
    check(ops, 5000, [0, 100, 5000], average, clip=(1.0, math.inf))
    check(ops, 5000, [0, 100, 5000], average, clip=(0.0, 0.0))


def test_one_sequence_without_offsets(ops):
    for tokens in (1, 700, 5000):
        nll, old, ref, a, targets, offsets = inputs(tokens, [0, tokens])
        for average in ("tokens", "sequences"):
            one = ops.policy_loss(nll, old, a, targets, offsets, ref, kl=0.1, average=average)
            two = ops.policy_loss(nll, old, a, targets, None, ref, kl=0.1, average=average)
            assert all(torch.equal(s, t) for s, t in zip(one, two)) and one[1].shape == (1,)
            assert torch.equal(ops.policy_loss_backward(None, nll, old, a, one[1], targets, offsets, ref, kl=0.1),
                               ops.policy_loss_backward(torch.ones(1, device="cuda"), nll, old, a, two[1], targets, None, ref, kl=0.1))


@pytest.mark.parametrize("tokens", [300, 9000])
def test_nothing_takes_part(ops, tokens):
    nll, old, ref, a, targets, offsets = inputs(tokens, [0, 100, tokens])
    targets[:] = -100
    nll[:], old[3], ref[5] = math.nan, math.inf, math.nan
    for average in ("tokens", "sequences"):
        result, norm = ops.policy_loss(nll, old, a, targets, offsets, ref, kl=0.1, average=average)
        assert not result.any() and not norm.any()
        assert not ops.policy_loss_backward(None, nll, old, a, norm, targets, offsets, ref, kl=0.1).any()
    # no sequence has a token
    result, norm = ops.policy_loss(nll, old, a, None, torch.tensor([50, 50], device="cuda"), ref, kl=0.1)
    assert not result.any() and not norm.any()


@pytest.mark.parametrize("average", ["tokens", "sequences"])
def test_masked_tokens_may_hold_anything(ops, average):
    nll, old, ref, a, targets, offsets = inputs(6000, [0, 10, 2500, 6000])
    call = lambda *v: ops.policy_loss(v[0], v[1], v[3], targets, offsets, v[2], kl=0.1, average=average)
    want = call(nll, old, ref, a)
    grad = ops.policy_loss_backward(None, nll, old, a, want[1], targets, offsets, ref, kl=0.1)
    bad = [t.clone() for t in (nll, old, ref, a)]
    for t, v in zip(bad, (math.nan, math.inf, -math.inf, math.nan)):
        t[targets < 0] = v
    got = call(*bad)
    assert all(torch.equal(s, t) for s, t in zip(want, got))
    got = ops.policy_loss_backward(None, bad[0], bad[1], bad[3], want[1], targets, offsets, bad[2], kl=0.1)
    assert torch.equal(grad, got) and not got[targets < 0].any()


def test_far_ratios(ops):
    """Ratios that overflow: clipped where the advantage is not negative, infinite losses where it is; an advantage of zero gives zero."""
    nll = torch.tensor([0.0, 0.0, 0.0, 200.0], device="cuda")
    old = torch.tensor([200.0, 200.0, 200.0, 0.0], device="cuda")
    a = torch.tensor([2.0, 0.0, -1.0, -3.0], device="cuda")
    offsets = torch.arange(5, device="cuda")
    for i, (loss, clipped, g) in enumerate([(-2.4, 1, 0.0), (0.0, 1, 0.0), (math.inf, 0, -math.inf), (2.4, 1, 0.0)]):
        part = slice(i, i + 1)
        result, norm = ops.policy_loss(nll[part], old[part], a[part])
        assert result.tolist() == pytest.approx([loss, 0.0, clipped], rel=1e-6)
        assert ops.policy_loss_backward(None, nll[part], old[part], a[part], norm).tolist() == [g]


def test_small_drifts(ops):
    """exp(e) - e - 1 near zero, where 32 bits would cancel: relative to its own size."""
    e = torch.cat([torch.logspace(-7, 0.5, 400, device="cuda"), -torch.logspace(-7, 1, 400, device="cuda")])
    zero = torch.zeros_like(e)
    offsets = torch.arange(len(e) + 1, device="cuda")
    for t in range(0, len(e), 37):
        part = slice(t, t + 1)
        result, _ = ops.policy_loss(e[part], e[part], zero[part], reference_nll=zero[part])
        d = float(e[t])
        want = math.expm1(d) - d if abs(d) > 1e-3 else d * d / 2 * (1 + d / 3 * (1 + d / 4 * (1 + d / 5)))
        assert abs(float(result[1]) - want) <= 40 * E * want        # expm1 2^-23, the subtraction loses at most 2 / 0.35 of it


def test_gradient_against_differences(ops):
    nll, old, ref, a, targets, offsets = inputs(900, [0, 300, 900], spread=0.1)
    args = dict(targets=targets, offsets=offsets, reference_nll=ref, kl=0.2, clip=(0.5, 0.9))
    _, norm = ops.policy_loss(nll, old, a, average="sequences", **args)
    grad = ops.policy_loss_backward(None, nll, old, a, norm, **args).double()
    way, step = torch.randn(900, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").double(), 1e-5
    f = [float(plain(nll.double() + s * way, old, ref, a, targets, [0, 300, 900], (0.5, 0.9), 0.2, "sequences", "tokens")[0][0]) for s in (step, -step)]
    assert abs(float((grad * way).sum()) - (f[0] - f[1]) / (2 * step)) <= 1e-6 * float((grad * way).abs().sum())


def test_gradient_over_an_input(ops):
    nll, old, ref, a, targets, offsets = inputs(3000, [0, 1000, 3000])
    args = dict(targets=targets, offsets=offsets, reference_nll=ref, kl=0.2)
    _, norm = ops.policy_loss(nll, old, a, **args)
    want = ops.policy_loss_backward(None, nll, old, a, norm, **args)
    over = nll.clone()
    assert ops.policy_loss_backward(None, over, old, a, norm, dnll=over, **args) is over and torch.equal(over, want)


def test_no_tokens(ops):
    empty = torch.empty(0, device="cuda")
    offsets = torch.zeros(4, dtype=torch.int64, device="cuda")
    result, norm = ops.policy_loss(empty, empty, empty, offsets=offsets)
    assert result.tolist() == [0, 0, 0] and norm.tolist() == [0, 0, 0]
    assert ops.policy_loss_backward(None, empty, empty, empty, norm, offsets=offsets).numel() == 0


def test_bad_offsets_reach_nothing(ops):
    nll, old, ref, a, targets, _ = inputs(5000, [0, 5000])
    for e in ([-9, 100, 1 << 40], [4000, 20, 3000, 10], [5000, 0, 1 << 62], [-(1 << 62), -1, 0]):
        offsets = torch.tensor(e, device="cuda")
        for average in ("tokens", "sequences"):
            _, norm = ops.policy_loss(nll, old, a, targets, offsets, ref, average=average)
            ops.policy_loss_backward(None, nll, old, a, norm, targets, offsets, ref)
    torch.cuda.synchronize()


def test_same_bits_every_time(ops):
    first = check(ops, 300_000, [0, 9, 70_000, 70_001, 300_000], "sequences")
    for _ in range(3):
        again = check(ops, 300_000, [0, 9, 70_000, 70_001, 300_000], "sequences")
        assert all(torch.equal(s, t) for s, t in zip(first, again))
