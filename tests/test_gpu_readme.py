"""README's examples of the operators, as they stand there: they run one after the other, and the layer of experts gives what its formula says, with its gradients."""
import os
import re

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from conftest import ROOT  # noqa: E402


def blocks():
    with open(os.path.join(ROOT, "README.md")) as f:
        found = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    return [b for b in found if "operators." in b]


def randn(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def test_head_norm_and_updates():
    half = torch.bfloat16
    targets = torch.arange(40, device="cuda")
    name = dict(x=randn(1, 40, 64, dtype=half), gamma=randn(2, 64), beta=randn(3, 64), w=randn(4, 300, 64, dtype=half), targets=targets, dloss=torch.ones(40, device="cuda"),
                gradient=randn(5, 96, 64, dtype=half), m=torch.zeros(96, 64, device="cuda"))
    exec(blocks()[0], name)
    assert name["dw"].shape == (300, 64) and name["dx"].shape == (40, 64) and name["update"].shape == (96, 64)


@pytest.mark.parametrize("k", [1, 2, 3])
def test_experts_dropout_and_policy(k):
    half, tokens, width, groups = torch.bfloat16, 50, 64, 5
    x, w, dz = randn(1, tokens, width, dtype=half), randn(2, groups, width, width, dtype=half, scale=0.125), randn(3, tokens, width, dtype=half)
    experts = randn(4, tokens, groups).topk(k, 1).indices
    weights = torch.softmax(randn(5, tokens, k), 1).to(half)
    loss = randn(6, tokens).abs()
    from paper_2210_07454_b200 import operators
    name = dict(operators=operators, x=x, w=w, dz=dz, experts=experts, weights=weights, groups=groups, k=k, seed=11, loss=loss, old_loss=loss + 0.1, reference=loss - 0.2, advantages=randn(7, tokens),
                targets=torch.ones(tokens, dtype=torch.int64, device="cuda"), sequences=torch.tensor([0, 20, 50], device="cuda"))
    exec(blocks()[1], name)
    assert name["dloss"].shape == (tokens,) and bool(torch.isfinite(name["result"]).all())
    mask = operators.dropout(torch.ones(tokens, width, device="cuda"), 0.1, 11).double()
    xd, wd = x.double().requires_grad_(), w.double().requires_grad_()
    y = sum(weights[:, i:i + 1].double() * torch.einsum("tw,tow->to", xd, wd[experts[:, i]]) for i in range(k))
    z = xd + mask * y
    z.backward(dz.double())
    # some ten roundings to bf16 one after the other, 2^-9 each on average and independent of one another
    for got, want in ((name["z"], z.detach()), (name["dx"], xd.grad), (name["dw"], wd.grad)):
        assert float((got.double() - want).norm() / want.norm()) <= 10 * 2.0 ** -9
