"""Sizes of the adapters' workspace."""
import ctypes

import pytest

import paper_1911_02497_amd as P
from paper_1911_02497_amd import binding as B


def size(T, back, n_in, n_out, n_adapters, max_rank):
    lst = B.AdapterList(1 << 38, n_in, n_out, n_adapters, max_rank, B.TYPE_BF16, 7)
    return P.library().condensa_adapter_workspace_bytes(ctypes.byref(lst), T, back)


def test_parts_of_gradients_are_for_adapters_with_several_runs():
    """1537 tokens are three runs at most of adapters that have more than one, whatever the list holds: 1000 of rank 64 took 2.2 GB."""
    below, above = (size(T, 1, 4608, 4096, 1000, 64) for T in (1536, 1537))
    assert above - below <= 6 * 64 * (4608 + 4096) * 4 + (1 << 20)
    assert size(1537, 1, 4608, 4096, 16384, 16) < 1 << 25


LISTS = [(4608, 4096, 64, 16), (512, 2048, 16, 8), (650, 2600, 12, 24), (64, 64, 3, 256), (63, 65, 1, 1), (1 << 20, 40000, 5, 33), (40000, 1 << 20, 5, 33), (4096, 4608, 16384, 128), (7, 3, 0, 0),
         (1 << 20, 1 << 20, 2, 4)]


@pytest.mark.parametrize("back", [0, 1])
@pytest.mark.parametrize("shape", LISTS)
def test_a_workspace_serves_fewer_tokens(shape, back):
    """The size never falls as tokens are added: 64 adapters of rank 16 beside 4608 -> 4096 took 11.5 MB at 64 tokens and 0.5 MB at 8192."""
    some = list(range(1, 3000)) + [s + d for k in range(12, 24) for s in (1 << k, 3 << (k - 1)) for d in (-1, 0, 1)] + [1 << 24]
    before = 0
    for T in sorted(some):
        now = size(T, back, *shape)
        assert now >= before, (T, now, before)
        before = now


def test_sizes_stay_in_proportion():
    assert size(8192, 0, 4608, 4096, 64, 16) < 16 << 20
    assert size(1, 0, 512, 2048, 16, 8) == 256
