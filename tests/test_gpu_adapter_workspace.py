"""Workspaces of the adapters' calls: how much of one is used, and one for calls of different sizes."""
import pytest
import torch

from test_gpu_adapter import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens", [{0: 600, 3: 1030, 49: 513}, {7: 512, 8: 1024, 9: 1025, 30: 511}, {0: 2600, 1: 513, 2: 514}, {48: 513, 49: 2600}])
def test_several_runs_of_some_of_many_adapters(dtype, tokens):
    """Parts of runs lie beside each other without overlap, wherever in the list the adapters with several runs are; the others have few tokens."""
    n = 50
    ids = [a for a, count in tokens.items() for _ in range(count)] + [t % (n + 1) - 1 for t in range(700) if t % (n + 1) - 1 not in tokens]
    g = torch.Generator().manual_seed(len(ids))
    ids = torch.tensor(ids)[torch.randperm(len(ids), generator=g)].tolist()
    c = Case(dtype, len(ids), 130, 70, [3 + a % 5 for a in range(n)], ids)
    c.forward()
    c.backward()
    c.check_backward()
