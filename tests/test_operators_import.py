"""The operators without the shortcuts that a torch build may lack: they import, and give the same bits."""
import subprocess
import sys

import pytest

from conftest import ROOT

torch = pytest.importorskip("torch")

# hidden while the module is imported; torch's public functions may go through them
WITHOUT = """
import torch
torch.cuda.is_available()
kept = []
for owner, name in ((torch._C, "_cuda_getCurrentRawStream"), (torch._C, "_cuda_getDevice"), (torch._C._dynamo.guards, "_empty_strided_cuda")):
    if {which} in ("all", name) and hasattr(owner, name):
        kept.append((owner, name, getattr(owner, name)))
        delattr(owner, name)
from paper_2210_07454_b200 import operators
for owner, name, f in kept:
    setattr(owner, name, f)
    assert f not in (operators._raw_stream, operators._current_device, operators._empty_here)
"""
NAMES = ["all", "_cuda_getCurrentRawStream", "_cuda_getDevice", "_empty_strided_cuda"]


@pytest.mark.parametrize("which", NAMES)
def test_operators_import_without_private_names(which):
    code = WITHOUT.format(which=repr(which)) + "assert callable(operators._raw_stream) and callable(operators._current_device) and callable(operators._empty_here)\n"
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)


@pytest.mark.gpu
def test_operators_run_without_private_names(tmp_path):
    from paper_2210_07454_b200 import operators
    body = """
def everything(operators):
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = torch.randn(50, 96, generator=g, device="cuda"), torch.randn(96, generator=g, device="cuda")
    h, v = (torch.randn(n, 64, generator=g, device="cuda").bfloat16() for n in (50, 300))
    t = torch.randint(0, 300, (50,), generator=g, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    y, mean, rstd = operators.layer_norm(x, w)
    loss, lse = operators.linear_cross_entropy(h, v, t)
    out = [y, mean, rstd, loss, lse, *operators.layer_norm_backward(x, x, w, mean, rstd),
           *operators.linear_cross_entropy_backward(loss, h, v, t, lse), operators.orthogonalize(torch.randn(200, 150, generator=g, device="cuda"))]
    torch.cuda.synchronize()
    out += operators.linear_cross_entropy(h, v, t, stream=side)
    torch.cuda.synchronize()
    return [o.cpu() for o in out]
"""
    path = tmp_path / "out.pt"
    code = WITHOUT.format(which="'all'") + body + f"torch.save(everything(operators), {str(path)!r})\n"
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)
    names = {"torch": torch}
    exec(body, names)
    assert all(torch.equal(a, b) for a, b in zip(torch.load(path), names["everything"](operators)))
