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
