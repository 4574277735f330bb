"""Which stream and device the memory, launches and questions of the operators for experts, dropout and policies belong to: the Python side on the host, with a
stand-in for the library and for torch's streams."""
import pytest

torch = pytest.importorskip("torch")

from test_operators_streams import World  # noqa: E402


class More(World):
    def __init__(self, monkeypatch):
        super().__init__(monkeypatch)
        monkeypatch.setattr(self.ops, "_new_on", lambda device: lambda shape, stride, dtype: self.new(shape, stride, dtype, device))

    def calls(self, device=0):
        """name, inputs, tensors given as outputs, call(stream)"""
        o, p = self.ops, lambda *shape, dtype=torch.float32: self.place(torch.zeros(*shape, dtype=dtype), device)
        half, whole = torch.bfloat16, torch.int64
        x, w, off, dy = p(4, 8, dtype=half), p(2, 6, 8, dtype=half), p(3, dtype=whole), p(4, 6, dtype=half)
        y, dx, dw, e = p(4, 6, dtype=half), p(4, 8, dtype=half), p(2, 6, 8), p(4, dtype=whole)
        v, r, z, seed = p(4, 8), p(4, 8), p(4, 8), p(1, dtype=whole)
        n, old, a, t, ref, norm, d, g = p(4), p(4), p(2), p(4, dtype=whole), p(4), p(2), p(1), p(4)
        policy = dict(targets=t, offsets=off, reference_nll=ref, kl=0.1, advantage_of="sequences")
        return [("sk_sort_by_expert", (e,), (), lambda s: o.sort_by_expert(e, 5, stream=s)),
                ("sk_grouped_linear", (x, w, off), (), lambda s: o.grouped_linear(x, w, off, stream=s)),
                ("sk_grouped_linear", (x, w, off), (y,), lambda s: o.grouped_linear(x, w, off, out=y, stream=s)),
                ("sk_grouped_linear_backward", (dy, x, w, off), (), lambda s: o.grouped_linear_backward(dy, x, w, off, stream=s)),
                ("sk_grouped_linear_backward", (dy, x, w, off), (dx, dw), lambda s: o.grouped_linear_backward(dy, x, w, off, dx=dx, dweight=dw, stream=s)),
                ("sk_dropout", (v, r, seed), (), lambda s: o.dropout(v, 0.1, seed, residual=r, stream=s)),
                ("sk_dropout", (v, seed), (z,), lambda s: o.dropout_backward(v, 0.1, seed, dx=z, stream=s)),
                ("sk_policy_loss", (n, old, a, t, off, ref), (), lambda s: o.policy_loss(n, old, a, stream=s, **policy)),
                ("sk_policy_loss_backward", (d, n, old, a, norm, t, off, ref), (), lambda s: o.policy_loss_backward(d, n, old, a, norm, stream=s, **policy)),
                ("sk_policy_loss_backward", (n, old, a, norm), (g,),
                 lambda s: o.policy_loss_backward(None, n, old, a, norm, offsets=off, advantage_of="sequences", dnll=g, stream=s))]


@pytest.fixture
def world(monkeypatch):
    from paper_2210_07454_b200 import operators
    operators._size.cache_clear()
    yield More(monkeypatch)
    operators._size.cache_clear()                    # what the stand-in answered


def test_memory_and_tensors_of_a_given_stream(world):
    for name, inputs, given, call in world.calls():
        world.allocated.clear()
        world.called.clear()
        out = call(world.side)
        assert all(s is world.side for _, s in world.allocated) and (world.allocated or given), name
        assert [c[0] for c in world.called] == [name] and world.called[0][2] == 22 and world.current is world.main
        assert all(world.side in t.recorded for t in inputs + given), name
        for t in out if isinstance(out, tuple) else (out,):
            assert t is None or any(t is g for g in given) or world.main in t.recorded, name
        call(None)
        assert world.called[-1][2] == 11


def test_a_stream_of_another_device_is_refused(world):
    from paper_2210_07454_b200.binding import SkError
    for _, _, _, call in world.calls():
        with pytest.raises(SkError):
            call(world.stream(33, device=1))
    assert not world.called


def test_tensors_written_in_place_say_so(world):
    for _, inputs, given, call in world.calls():
        for stream in (None, world.side):
            before, kept = [t._version for t in given], [t._version for t in inputs]
            call(stream)
            assert all(t._version > b for t, b in zip(given, before)) and [t._version for t in inputs] == kept


def test_another_device_than_the_current_one(world):
    for _, _, _, call in world.calls(device=1):
        call(None)
    assert {"sk_sort_by_expert_workspace", "sk_grouped_linear_workspace", "sk_grouped_linear_backward_workspace", "sk_policy_loss_workspace"} == {n for n, _ in world.asked}
    assert all(device == 1 for _, device in world.asked) and all(device == 1 for _, device, _ in world.called) and world.device == 0


def test_tensors_that_do_not_fit_are_refused(world):
    from paper_2210_07454_b200.binding import SkError
    o, p = world.ops, lambda *shape, dtype=torch.float32, device=0: world.place(torch.zeros(*shape, dtype=dtype), device)
    half, whole = torch.bfloat16, torch.int64
    x, w, off, dy = p(4, 8, dtype=half), p(2, 6, 8, dtype=half), p(3, dtype=whole), p(4, 6, dtype=half)
    n, a, v = p(4), p(2), p(4, 8)
    wrong = [lambda: o.grouped_linear(p(4, 8), w, off), lambda: o.grouped_linear(x, p(2, 6, 8, dtype=torch.float16), off), lambda: o.grouped_linear(x, p(6, 8, dtype=half), off),
             lambda: o.grouped_linear(x, p(2, 6, 9, dtype=half), off), lambda: o.grouped_linear(x, w, p(4, dtype=whole)), lambda: o.grouped_linear(x, w, p(3)),
             lambda: o.grouped_linear(p(4, 8, dtype=half, device=1), w, off), lambda: o.grouped_linear(x, w, off, out=p(4, 7, dtype=half)),
             lambda: o.grouped_linear(x, w, off, out=p(4, 6)), lambda: o.grouped_linear(x.t().contiguous().t(), w, off), lambda: o.grouped_linear(x[:1].expand(4, 8), w, off),
             lambda: o.grouped_linear_backward(p(3, 6, dtype=half), x, w, off), lambda: o.grouped_linear_backward(dy, x, w, off, dx=p(4, 7, dtype=half)),
             lambda: o.grouped_linear_backward(dy, x, w, off, dweight=p(2, 6, 8, dtype=torch.float16)),
             lambda: o.grouped_linear_backward(dy, x, w, off, dweight=p(2, 6, 9)),
             lambda: o.sort_by_expert(p(4), 3), lambda: o.sort_by_expert(p(4, dtype=whole), 0), lambda: o.sort_by_expert(p(4, dtype=whole), 2049),
             lambda: o.sort_by_expert(p(8, dtype=whole)[::2], 3),
             lambda: o.dropout(v, 0.1, None), lambda: o.dropout(v, 0.1, p(2, dtype=whole)), lambda: o.dropout(v, 0.1, p(1)), lambda: o.dropout(v, 0.1, 1, residual=p(4, 7)),
             lambda: o.dropout(v, 0.1, 1, residual=p(4, 8, dtype=half)), lambda: o.dropout(v, 0.1, 1, out=p(4, 8, dtype=half)), lambda: o.dropout(p(()), 0.1, 1),
             lambda: o.dropout(p(4, 8, dtype=whole), 0.1, 1),
             lambda: o.policy_loss(n, p(5), n), lambda: o.policy_loss(n, n, a), lambda: o.policy_loss(n, n, n, offsets=off, advantage_of="sequences"),
             lambda: o.policy_loss(n, n, n, advantage_of="rows"), lambda: o.policy_loss(n, n, n, average="rows"), lambda: o.policy_loss(n, n, n, offsets=p(1, dtype=whole)),
             lambda: o.policy_loss(n, n, n, clip=0.2), lambda: o.policy_loss(n, n, n, targets=n), lambda: o.policy_loss(p(8)[::2], n, n),
             lambda: o.policy_loss(p(4, dtype=half), n, n), lambda: o.policy_loss_backward(None, n, n, n, p(2)), lambda: o.policy_loss_backward(n, n, n, n, p(1)),
             lambda: o.policy_loss_backward(None, n, n, n, p(1), dnll=p(3))]
    for i, call in enumerate(wrong):
        with pytest.raises(SkError):
            call()
    assert not world.called
