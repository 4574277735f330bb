"""Seeds of dropout: whole numbers of any size and kind pass, whatever would have to be rounded, parsed or is no number is refused (the Python side, on the host)."""
import math

import pytest

torch = pytest.importorskip("torch")
numpy = pytest.importorskip("numpy")

from test_more_operators_streams import More  # noqa: E402


@pytest.fixture
def world(monkeypatch):
    return More(monkeypatch)


@pytest.mark.parametrize("seed", [0, 7, -1, 1 << 63, (1 << 64) + 5, True, numpy.int64(-3), numpy.uint64((1 << 64) - 1), numpy.int32(9), 3.0], ids=str)
def test_whole_numbers(world, seed):
    assert world.ops._seed(seed, 0) == (int(seed) % (1 << 64), None)


@pytest.mark.parametrize("seed", [1.5, -0.25, math.inf, -math.inf, math.nan, "7", None, numpy.float32(3.5), [1], 2j], ids=str)
def test_what_is_no_whole_number_is_refused(world, seed):
    from paper_2210_07454_b200.binding import SkError
    v = world.place(torch.zeros(4, 8), 0)
    for call in (lambda: world.ops.dropout(v, 0.1, seed), lambda: world.ops.dropout_backward(v, 0.1, seed)):
        with pytest.raises(SkError):
            call()
    assert not world.called
