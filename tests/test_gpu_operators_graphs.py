"""The operators inside a CUDA graph: captured once, replayed on new inputs."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_operators_in_a_graph():
    from paper_2210_07454_b200 import operators as ops

    def inputs(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")
        return [randn(300, 333), randn(333), randn(300, 333), randn(200, 72).bfloat16(), randn(1001, 72).bfloat16(),
                torch.randint(0, 1001, (200,), generator=g, device="cuda"), randn(90, 130), randn(2, 300, 260), randn(2, 300, 260)]

    def calls(x, w, dy, h, v, t, u, big, m):
        y, mean, rstd = ops.layer_norm(x, w)
        loss, lse = ops.linear_cross_entropy(h, v, t)
        return [y, mean, rstd, loss, lse, *ops.layer_norm_backward(dy, x, w, mean, rstd), *ops.linear_cross_entropy_backward(loss, h, v, t, lse),
                ops.orthogonalize(u), ops.orthogonalize(big, momentum=m), m]

    held = inputs(0)
    calls(*inputs(0))                                # kernels are loaded and prepared outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls(*held)
    for seed in (1, 2, 3):
        for t, new in zip(held, inputs(seed)):
            t.copy_(new)
        graph.replay()
        want = calls(*inputs(seed))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    ops.sync()
