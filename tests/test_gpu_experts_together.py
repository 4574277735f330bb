"""The operators for experts, dropout and policy tuning together, as a model uses them: gradients of a whole pass against a plain one in 64 bits, the
example, CUDA graphs, streams, threads."""
import math
import os
import sys
import threading

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from conftest import ROOT  # noqa: E402

sys.path.insert(0, os.path.join(ROOT, "examples"))


@pytest.fixture(scope="module")
def ops():
    from paper_2210_07454_b200 import operators
    return operators


def plain_losses(model, token, target, seed, experts_of, ops):
    """The example's forward pass in 64 bits with autograd, on its own choice of experts and its own mask. Returns (losses, leaves)."""
    layer = model.experts
    w, gamma, beta = (t.clone() for t in model.parts(model.x))
    leaves = [t.double().requires_grad_() for t in (w.bfloat16(), gamma, beta, layer.router, layer.up.bfloat16(), layer.down.bfloat16())]
    W, g, b, router, up, down = leaves
    e = W[token]
    top = (e @ router.T).gather(1, experts_of)
    weights = torch.softmax(top, 1)
    mixed = torch.zeros_like(e)
    for k in range(experts_of.shape[1]):
        h = torch.einsum("tw,thw->th", e, up[experts_of[:, k]])
        mixed = mixed + weights[:, k:k + 1] * torch.einsum("th,twh->tw", torch.relu(h) ** 2, down[experts_of[:, k]])
    mask = ops.dropout(torch.ones(mixed.shape, device="cuda"), model.dropout, seed).double()
    z = e + mixed * mask
    c = z - z.mean(1, keepdim=True)
    y = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * g + b
    logits = y @ W.T
    return torch.logsumexp(logits, 1) - logits.gather(1, target[:, None])[:, 0], leaves


def plain_policy(nll, old, a, target, lengths, reference, clip, kl):
    number = torch.repeat_interleave(torch.arange(len(lengths), device="cuda"), lengths)
    r = torch.exp(old.double() - nll)
    A = a.double()[number]
    e = nll - reference.double()
    token = -torch.minimum(r * A, r.clamp(1 - clip[0], 1 + clip[1]) * A) + kl * (torch.exp(e) - e - 1)
    live = (target >= 0).double()
    counts = torch.zeros(len(lengths), dtype=torch.float64, device="cuda").index_add_(0, number, live)
    return (token * live / counts[number]).sum() / len(lengths)


def test_a_whole_pass_and_its_gradients(ops):
    """Every operator in turn, forwards and backwards. Activations and their gradients are bf16 between the operators, each rounded by up to 2^-8: some ten of
    them one after the other; errors of different elements are independent, so that a gradient as a whole is off by about sqrt(10) 2^-9, and 3e-2 leaves room
    for those that are amplified by the norm and the square."""
    import policy_tuning as example
    model = example.Model(vocab=300, width=72, hidden=104, experts=5, chosen=2, dropout=0.2, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens = 413
    token, target = (torch.randint(0, 300, (tokens,), generator=g, device="cuda") for _ in range(2))
    lengths = torch.tensor([100, 13, 200, 100], device="cuda")
    offsets = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    nll, state = model.forward(token, target, seed=77)
    experts_of = state[5][2]
    want, leaves = plain_losses(model, token, target, 77, experts_of, ops)
    # losses are differences of logits of size about 4 in bf16 products of normalised rows
    assert float((nll.double() - want.detach()).norm() / want.detach().norm()) <= 1e-2
    old, reference = nll + 0.1 * torch.randn(tokens, generator=g, device="cuda"), nll + 0.3 * torch.randn(tokens, generator=g, device="cuda")
    a = torch.randn(4, generator=g, device="cuda")
    args = dict(targets=target, offsets=offsets, reference_nll=reference, clip=(0.9, 5.0), kl=0.3, advantage_of="sequences")        # nothing is clipped: both
    result, norm = ops.policy_loss(nll, old, a, average="sequences", **args)                                                         # sides are smooth here
    assert float(result[2]) == 0.0
    dnll = ops.policy_loss_backward(None, nll, old, a, norm, **args)
    row = torch.zeros(model.d, device="cuda")
    drouter, dup, ddown = model.backward(dnll, state, row)
    plain_policy(want, old, a, target, lengths, reference, (0.9, 5.0), 0.3).backward()
    got = [*model.parts(row), drouter, dup, ddown]
    for name, x, leaf in zip(("W", "gamma", "beta", "router", "up", "down"), got, leaves):
        assert float((x.double() - leaf.grad).norm() / leaf.grad.norm()) <= 3e-2, name
    ops.sync()


def test_the_example_runs():
    import policy_tuning
    rewards = policy_tuning.tune(steps=3, prompts=4, answers=4, length=5)
    assert len(rewards) == 3 and all(math.isfinite(r) and 0 <= r <= 1 for r in rewards)


def inputs(seed, tokens=500, groups=6, width=72, out=136, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")
    experts = torch.randint(-1, groups, (tokens, 2), generator=g, device="cuda")
    old = randn(tokens).abs()
    offsets = torch.sort(torch.randint(0, tokens, (9,), generator=g, device="cuda")).values
    return [experts, randn(tokens, width).to(dtype), randn(groups, out, width).to(dtype), randn(2 * tokens, out).to(dtype), randn(tokens, width),
            torch.full((1,), seed * 31, dtype=torch.int64, device="cuda"), old + 0.2 * randn(tokens), old, randn(8), offsets, old + randn(tokens)]


def everything(ops, experts, x, w, dy, residual, seed, nll, old, a, offsets, reference, stream=None):
    order, places, ends = ops.sort_by_expert(experts, len(w), stream=stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    rows = x[order // 2]
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    y = ops.grouped_linear(rows, w, ends, stream=stream)
    dx, dw = ops.grouped_linear_backward(dy, rows, w, ends, stream=stream)
    z = ops.dropout(residual, 0.3, seed, residual=residual, stream=stream)
    dz = ops.dropout_backward(residual, 0.3, seed, stream=stream)
    args = dict(offsets=offsets, reference_nll=reference, kl=0.1, advantage_of="sequences", stream=stream)
    result, norm = ops.policy_loss(nll, old, a, average="sequences", **args)
    return [order, places, ends, y, dx, dw, z, dz, result, norm, ops.policy_loss_backward(None, nll, old, a, norm, **args)]


@pytest.mark.parametrize("sizes", [dict(), dict(tokens=20000, width=64, out=48), dict(tokens=3, groups=1), dict(tokens=301, width=33, out=65, dtype=torch.float16)], ids=str)
def test_in_a_graph(ops, sizes):
    """Captured once, replayed on other inputs, other groups and another seed."""
    held = inputs(0, **sizes)
    everything(ops, *inputs(0, **sizes))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything(ops, *held)
    for seed in (1, 2, 3):
        for t, new in zip(held, inputs(seed, **sizes)):
            t.copy_(new)
        graph.replay()
        want = everything(ops, *inputs(seed, **sizes))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    ops.sync()


@pytest.mark.parametrize("tokens,groups,width,out", [(40, 6, 64, 256), (3000, 12, 136, 520), (6000, 3, 256, 128)])
def test_the_second_product_beside_the_first(ops, tokens, groups, width, out):
    """The product that gives dweight begins while the one for dx still runs; the groups change from replay to replay in the same memory. It gives the bits that it gives alone."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    experts = torch.zeros(tokens, dtype=torch.int64, device="cuda")
    x, dy = (torch.zeros(tokens, n, dtype=torch.bfloat16, device="cuda") for n in (width, out))
    w = torch.randn(groups, out, width, generator=g, device="cuda").bfloat16()

    def step():
        order, _, ends = ops.sort_by_expert(experts, groups)
        return (ends, *ops.grouped_linear_backward(dy, x, w, ends))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ends, dx, dw = step()
    for _ in range(40):
        experts.copy_(torch.randint(-1, groups, (tokens,), generator=g, device="cuda"))
        x.copy_(torch.randn(tokens, width, generator=g, device="cuda"))
        dy.copy_(torch.randn(tokens, out, generator=g, device="cuda"))
        graph.replay()
        got = dx.clone(), dw.clone()
        torch.cuda.synchronize()
        assert torch.equal(ops.grouped_linear_backward(dy, x, w, ends, dweight=False)[0], got[0])
        torch.cuda.synchronize()
        assert torch.equal(ops.grouped_linear_backward(dy, x, w, ends, dx=False)[1], got[1])
    ops.sync()


def test_two_graphs_replayed_at_once(ops):
    """Two captures of the same calls, replayed in two streams: nothing of one is the other's."""
    sets = [inputs(s, tokens=20000, width=64, out=48) for s in (1, 2)]
    want = [everything(ops, *s) for s in sets]
    torch.cuda.synchronize()
    graphs, got = [], []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got.append(everything(ops, *s))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(10):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_on_another_stream_beside_pending_work(ops):
    first, second = inputs(1, tokens=20000, width=64, out=48), inputs(2, tokens=20000, width=64, out=48)
    want, want2 = everything(ops, *first), everything(ops, *second)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        torch.cuda._sleep(20_000_000)
        pending = everything(ops, *first)            # its workspaces are free again for the current stream, and not yet used
        got = everything(ops, *second, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(pending, want)) and all(torch.equal(a, b) for a, b in zip(got, want2))


def test_from_several_threads(ops):
    """Calls of different sizes at the same time, a stream each."""
    sizes = [dict(tokens=900), dict(tokens=20000, width=64, out=48), dict(tokens=301, width=33, out=65, dtype=torch.float16), dict(tokens=40, groups=40)]
    held = [inputs(i, **s) for i, s in enumerate(sizes)]
    want = [everything(ops, *h) for h in held]
    torch.cuda.synchronize()
    wrong = []

    def work(h, w):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(30):
                got = everything(ops, *h)
            stream.synchronize()
            wrong.extend(not torch.equal(a, b) for a, b in zip(got, w))

    threads = [threading.Thread(target=work, args=p) for p in zip(held, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(wrong) == 4 * 11 and not any(wrong)
    ops.sync()


def test_outputs_of_grouped_gradients_in_a_step_gradient_array(ops):
    """dweight as a view of a row of the (n, d) gradient array, beside other parameters: off any boundary, and nothing else is written."""
    experts, x, w, dy, *_ = inputs(4)
    order, _, ends = ops.sort_by_expert(experts, len(w))
    rows = x[order // 2]
    _, want = ops.grouped_linear_backward(dy, rows, w, ends)
    for at in (0, 1, 3, 8):
        grads = torch.full((2, at + w.numel() + 5), 9.0, device="cuda")
        view = grads[1, at:at + w.numel()].view(w.shape)
        ops.grouped_linear_backward(dy, rows, w, ends, dx=False, dweight=view)
        # 32-bit sums of at most 1000 products, to be rounded as the 16-bit ones were: parts are joined in another order
        assert float((view.to(w.dtype).double() - want.double()).abs().max()) <= 2.0 ** -7 * float(want.double().abs().max())
        assert bool((grads[0] == 9).all()) and bool((grads[1, :at] == 9).all()) and bool((grads[1, at + w.numel():] == 9).all())
