"""The order by expert as the first call of a process, for every number of experts at which its shared memory may need the device's leave: a limit that an earlier
call with more experts has raised must not be what makes it run."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from conftest import ROOT  # noqa: E402

CODE = """
import sys, torch
from paper_2210_07454_b200 import operators as ops
for groups in (int(g) for g in sys.argv[1:]):
    for n in (500, 5000):
        experts = torch.arange(n, device="cuda") * 7 % groups
        order, places, offsets = ops.sort_by_expert(experts, groups)
        assert torch.equal(experts[order], experts.sort().values) and torch.equal(order[places], torch.arange(n, device="cuda"))
        assert torch.equal(offsets, torch.searchsorted(experts.sort().values, torch.arange(groups + 1, device="cuda")))
print("as it should be")
"""


# in rising order: none of them is helped by those before it
def test_numbers_of_experts_around_the_limit():
    groups = [*range(352, 368), 1023, 2047, 2048]
    done = subprocess.run([sys.executable, "-c", CODE, *map(str, groups)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "as it should be" in done.stdout, done.stderr[-2000:]
