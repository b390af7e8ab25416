"""Workspaces of the adapters' calls: how much of one is used, and one for calls of different sizes."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV
from test_gpu_adapter import Case, ids_of

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


SIZES = [1, 2, 3, 16, 33, 64, 65, 130, 256, 257, 300, 511, 700, 1536, 1537, 2100]


@pytest.mark.parametrize("dtype,K,N,ranks", [("bf16", 1024, 512, [16, 40, 3]), ("f16", 130, 1733, [9, 33]), ("bf16", 72, 64, [256]), ("f16", 2050, 66, [4] * 40)])
def test_one_workspace_for_all_sizes(dtype, K, N, ranks):
    """A workspace made for the most tokens serves calls with fewer, and no call writes past its end."""
    whole = None
    for T in reversed(SIZES):
        c = Case(dtype, T, K, N, ranks, ids_of(T, len(ranks), "mixed"))
        if whole is None:
            sizes = [P.adapter_workspace(c.table, T, backward=b).numel() for b in (False, True)]
            whole = [torch.full((n + 65536,), 0xFF, dtype=torch.uint8, device=DEV) for n in sizes]
        c.forward(workspace=whole[0][: sizes[0]])
        c.check_forward(str(T))
        c.backward(workspace=whole[1][: sizes[1]])
        c.check_backward(str(T))
        need = [P.adapter_workspace(c.table, T, backward=b).numel() for b in (False, True)]
        assert need[0] <= sizes[0] and need[1] <= sizes[1]
        for w, n in zip(whole, sizes):
            assert bool((w[n:] == 0xFF).all())
        for b, n in zip((False, True), need):                                   # and the size that is asked for at this number of tokens is enough
            w = torch.full((n + 65536,), 0xFF, dtype=torch.uint8, device=DEV)
            c.backward(workspace=w[:n]) if b else c.forward(workspace=w[:n])
            assert bool((w[n:] == 0xFF).all())
