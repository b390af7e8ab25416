"""Lists that no condensa_adamw_list_init made are refused before anything reaches a device: addresses here are never touched."""
import ctypes

import pytest

import paper_1911_02497_amd as P
from paper_1911_02497_amd import binding as B

BASE, ARG = 1 << 40, -6


@pytest.mark.parametrize("field,value", [("n_chunks", 1 << 51), ("n_chunks", (1 << 51) + 1), ("n_chunks", 1 << 63), ("code_type", B.TYPE_F32), ("code_type", 9)])
def test_counts_that_wrap_and_types_of_no_list(field, value):
    lst = B.AdamwList(BASE, BASE + 4096, 1000, 1, 1, 32, 0, 1)
    setattr(lst, field, value)
    s = B.AdamwSettings(1e-3, 0.9, 0.999, 1e-8, 0.01, 0.0, B.ROUND_NEAREST, 1, 0, None, 0)
    assert P.library().condensa_lc_adamw_step(ctypes.byref(lst), ctypes.byref(s), None) == ARG
