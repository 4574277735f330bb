"""Which stream and device the operators' memory, launches and questions belong to: the Python side on the host, with a stand-in
for the library and for torch's streams, and the same on a device with work pending on the current stream."""
import contextlib
import types

import pytest

torch = pytest.importorskip("torch")


class Placed(torch.Tensor):
    """A host tensor that says it is on device `place` and writes down which streams it is recorded on."""
    place = 0
    recorded = ()

    def get_device(self):
        return self.place

    def record_stream(self, stream):
        self.recorded = self.recorded + (stream,)

    @property
    def is_cuda(self):
        return True


class World:
    """Current stream and device, what was allocated and called under which of them."""

    def __init__(self, monkeypatch):
        from paper_2210_07454_b200 import operators
        self.ops, self.device = operators, 0
        self.main, self.side = self.stream(11), self.stream(22)
        self.current = self.main
        self.allocated, self.called, self.asked = [], [], []
        monkeypatch.setattr(operators, "_raw_stream", lambda device: self.current.cuda_stream)
        monkeypatch.setattr(operators, "_current_device", lambda: self.device)
        monkeypatch.setattr(operators, "_new", self.new)
        monkeypatch.setattr(operators, "lib", lambda: self)
        monkeypatch.setattr(torch.cuda, "stream", self.under)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        monkeypatch.setattr(torch.cuda, "device", self.on)

    @staticmethod
    def stream(number, device=0):
        return types.SimpleNamespace(cuda_stream=number, device=types.SimpleNamespace(type="cuda", index=device), device_index=device)

    @contextlib.contextmanager
    def under(self, stream):
        before, self.current = self.current, stream
        yield
        self.current = before

    @contextlib.contextmanager
    def on(self, device):
        before, self.device = self.device, device
        yield
        self.device = before

    def new(self, shape, stride, dtype, device):
        t = self.place(torch.empty_strided(shape, stride, dtype=dtype), device)
        self.allocated.append((t, self.current))
        return t

    def place(self, t, device=0):
        t = t.as_subclass(Placed)
        t.place = device
        return t

    def __getattr__(self, name):                 # the library's entry points
        if not name.startswith("sk_"):
            raise AttributeError(name)

        def call(*args):
            if name.endswith("_workspace"):
                self.asked.append((name, self.device))
                return 512
            self.called.append((name, self.device, args[-1]))
            return 0
        return call

    def calls(self, device=0):
        """The five operators' calls: name, inputs, tensors given as outputs, call(stream)."""
        o, p = self.ops, lambda *shape, dtype=torch.float32: self.place(torch.zeros(*shape, dtype=dtype), device)
        x, w, dy, mean, rstd = p(4, 8), p(8), p(4, 8), p(4), p(4)
        h, v, t, d = p(4, 8, dtype=torch.float16), p(6, 8, dtype=torch.float16), p(4, dtype=torch.int64), p(4)
        u, m, y = p(3, 5), p(3, 5), p(4, 8)
        deep, dw = p(2, 4, 8), p(6, 8, dtype=torch.float16)
        return [("sk_layer_norm", (x, w), (y,), lambda s: o.layer_norm(x, w, out=y, stream=s)),
                ("sk_layer_norm", (deep, w), (), lambda s: o.layer_norm(deep, w, w, stream=s)),
                ("sk_layer_norm_backward", (dy, x, w, mean, rstd), (), lambda s: o.layer_norm_backward(dy, x, w, mean, rstd, stream=s)),
                ("sk_linear_cross_entropy", (h, v, t), (), lambda s: o.linear_cross_entropy(h, v, t, stream=s)),
                ("sk_linear_cross_entropy_backward", (d, h, v, t), (dw,), lambda s: o.linear_cross_entropy_backward(d, h, v, t, d, dweight=dw, stream=s)),
                ("sk_orthogonalize", (u,), (m,), lambda s: o.orthogonalize(u, momentum=m, stream=s))]


@pytest.fixture
def world(monkeypatch):
    return World(monkeypatch)


def test_memory_of_a_given_stream_comes_from_that_stream(world):
    """torch hands memory out again in the order of the stream it belongs to: another stream may still have kernels of the
    current one running on it."""
    for name, _, given, call in world.calls():
        world.allocated.clear()
        world.called.clear()
        out = call(world.side)
        assert world.allocated and all(s is world.side for _, s in world.allocated), name
        assert [c[0] for c in world.called] == [name] and world.called[0][2] == 22
        assert world.current is world.main
        for t in out if isinstance(out, tuple) else (out,):          # handed back: the caller goes on with them on its own stream
            assert any(t is g for g in given) or world.main in t.recorded, name
    for name, _, _, call in world.calls():
        world.allocated.clear()
        call(None)
        assert all(s is world.main for _, s in world.allocated) and world.called[-1][2] == 11


def test_a_stream_of_another_device_is_refused(world):
    from paper_2210_07454_b200.binding import SkError
    other = world.stream(33, device=1)
    for _, _, _, call in world.calls():
        with pytest.raises(SkError):
            call(other)
    assert not world.called


def test_tensors_given_to_a_stream_are_kept_for_it(world):
    """A temporary that is dropped right after the call must not be handed out again before the given stream is done with it."""
    for name, inputs, given, call in world.calls():
        call(world.side)
        for t in inputs + given:
            assert world.side in t.recorded, name


def test_tensors_written_in_place_say_so(world):
    """What a call writes into given tensors raises their version, as torch's own functions do: autograd's check for tensors that were
    changed after they were saved sees it."""
    o, p = world.ops, lambda *shape, dtype=torch.float32: world.place(torch.zeros(*shape, dtype=dtype))
    half = torch.bfloat16
    x, w, s, h, t = p(4, 8), p(8), p(4), p(4, 8, dtype=half), p(4, dtype=torch.int64)
    y, dx, dw, db, dh, dv, u, m = p(4, 8), p(4, 8), p(8), p(8), p(4, 8, dtype=half), p(4, 8), p(4, 8, dtype=half), p(4, 8)
    calls = [((y,), lambda **k: o.layer_norm(x, w, out=y, **k)),
             ((dx, dw, db), lambda **k: o.layer_norm_backward(x, x, w, s, s, dx=dx, dweight=dw, dbias=db, **k)),
             ((dh, dv), lambda **k: o.linear_cross_entropy_backward(s, h, h, t, s, dhidden=dh, dweight=dv, **k)),
             ((u, m), lambda **k: o.orthogonalize(x, momentum=m, out=u, **k))]
    inputs = (x, w, s, h, t)
    for written, call in calls:
        for kw in ({}, dict(stream=world.side)):
            before, kept = [v._version for v in written], [v._version for v in inputs]
            call(**kw)
            assert all(v._version > b for v, b in zip(written, before)) and [v._version for v in inputs] == kept


def test_sizes_are_asked_with_the_tensors_device_current(world):
    """The layer norm's workspace depends on the device's number of SMs."""
    for _, _, _, call in world.calls(device=1):
        call(None)
    assert {"sk_layer_norm_backward_workspace", "sk_linear_cross_entropy_workspace", "sk_linear_cross_entropy_backward_workspace",
            "sk_orthogonalize_workspace"} == {name for name, _ in world.asked}
    assert all(device == 1 for _, device in world.asked), world.asked
    assert all(device == 1 for _, device, _ in world.called) and world.device == 0


@pytest.mark.gpu
def test_operators_on_a_stream_take_temporaries():
    """Inputs and outputs that are dropped, and whose memory is written again, while the given stream is still busy."""
    from paper_2210_07454_b200 import operators as ops
    g = torch.Generator(device="cuda").manual_seed(2)
    x, gamma = torch.randn(4096, 512, generator=g, device="cuda"), torch.randn(512, generator=g, device="cuda")
    u = torch.randn(300, 400, generator=g, device="cuda")
    want, want_u = ops.layer_norm(x, gamma), ops.orthogonalize(u)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        copies = [x.clone(), gamma.clone(), u.clone()]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = ops.layer_norm(*copies[:2], stream=side)
        got_u = ops.orthogonalize(copies[2], stream=side)
        del copies
        over = [torch.full_like(t, 7.0) for t in (x, gamma, u, x, gamma, u)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(got_u, want_u)
        assert all(bool((t == 7).all()) for t in over)


@pytest.mark.gpu
def test_operators_on_a_stream_beside_pending_work():
    """Long work on the current stream, its memory freed while it is pending: calls on another stream that wait for none of it give
    the bits they give alone, and the pending work's results are its own."""
    from paper_2210_07454_b200 import operators as ops
    g = torch.Generator(device="cuda").manual_seed(1)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    tokens, vocab, width = 512, 4001, 96
    h, w = randn(tokens, width, dtype=torch.bfloat16), randn(vocab, width, dtype=torch.bfloat16)
    h2, w2 = randn(tokens, width, dtype=torch.bfloat16), randn(vocab, width, dtype=torch.bfloat16)
    t = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    x, dy, gamma, u, u2 = randn(3000, 333), randn(3000, 333), randn(333), randn(2, 300, 500), randn(2, 300, 500)

    def everything(h, w, u, stream=None):
        loss, lse = ops.linear_cross_entropy(h, w, t, stream=stream)
        y, mean, rstd = ops.layer_norm(x, gamma, stream=stream)
        return [loss, lse, y, mean, rstd, *ops.linear_cross_entropy_backward(loss, h, w, t, lse, stream=stream),
                *ops.layer_norm_backward(dy, x, gamma, mean, rstd, stream=stream), ops.orthogonalize(u, stream=stream)]

    want, want2 = everything(h, w, u), everything(h2, w2, u2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        torch.cuda._sleep(20_000_000)                # some ten milliseconds
        pending = everything(h, w, u)                # its workspaces are free again for the current stream, and not yet used
        got = everything(h2, w2, u2, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(pending, want))
        assert all(torch.equal(a, b) for a, b in zip(got, want2))
    ops.sync()
    ops.sync(side)
