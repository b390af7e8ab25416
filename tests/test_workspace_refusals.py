"""Workspaces that a caller brings: those that do not lie on the call's device, or whose elements are not one behind the other, are refused before anything is launched."""
import types

import pytest
import torch

from paper_1911_02497_amd import binding as B


class Room:
    """What a tensor says of itself."""

    def __init__(self, device=1, contiguous=True, numel=4096, size=1):
        self.get_device, self.is_contiguous = lambda: device, lambda: contiguous
        self.numel, self.element_size, self.data_ptr = lambda: numel, lambda: size, lambda: 1 << 40


BAD = {"host": torch.empty(1 << 20, dtype=torch.uint8), "another device": Room(device=0), "one byte, expanded": Room(contiguous=False)}


@pytest.fixture
def calls(monkeypatch):
    """Operands pass; what would be launched is recorded."""
    ran = []
    monkeypatch.setattr(B, "_run", lambda place, stream, entry, *args: ran.append(args))
    for name in ("_operand", "_rows", "_like"):
        monkeypatch.setattr(B, name, lambda *_: (1 << 41, 64))
    monkeypatch.setattr(B, "_place", lambda index: types.SimpleNamespace(device=torch.device("cuda", index), index=index))
    monkeypatch.setattr(B, "_norm_rows", lambda name, t: ((3, 64), torch.bfloat16, B._place(1)))
    monkeypatch.setattr(B, "_norm_weight", lambda *_: (1 << 42, 0))
    monkeypatch.setattr(B, "_token_ids", lambda *_: 1 << 43)
    monkeypatch.setattr(B, "_kept_z", lambda *_: (1 << 44, 8))
    return ran


def entry_points():
    matrix = types.SimpleNamespace(index=1, rows=3, cols=64, ref=None)
    out = torch.empty(3, 64, dtype=torch.bfloat16)
    dweight = types.SimpleNamespace(shape=(64,), dtype=torch.float32, get_device=lambda: 1, is_contiguous=lambda: True, data_ptr=lambda: 1 << 45)
    table = types.SimpleNamespace(index=1, device=torch.device("cuda", 1), n_in=64, n_out=64, max_rank=8, ref=None, grads=None, keep_for=lambda s: 7)
    return {
        "project": lambda ws: B.condensa_project_fp8(matrix, matrix, out, workspace=ws),
        "project backward": lambda ws: B.condensa_project_fp8_backward(matrix, matrix, out, workspace=ws),
        "norm backward": lambda ws: B.condensa_rms_norm_backward(out, out, out, dx=out, dweight=dweight, workspace=ws),
        "adapters": lambda ws: B.condensa_adapter_project(out, out, table, None, y=out, workspace=ws),
        "adapters backward": lambda ws: B.condensa_adapter_project_backward(out, out, out, table, None, None, dx=out, workspace=ws),
    }


@pytest.mark.parametrize("name", list(entry_points()))
def test_calls(calls, name):
    call = entry_points()[name]
    for bad in BAD.values():
        with pytest.raises(TypeError):
            call(bad)
    assert not calls
    call(Room())
    assert (1 << 40, 4096) == next(p for p in zip(calls[0], calls[0][1:]) if p[0] == 1 << 40)
    call(Room(numel=1000, size=4))
    assert (1 << 40, 4000) == next(p for p in zip(calls[1], calls[1][1:]) if p[0] == 1 << 40)


def test_a_gradient_that_needs_none(calls):
    B.condensa_rms_norm_backward(torch.empty(3, 64), torch.empty(3, 64), torch.empty(64), dx=torch.empty(3, 64), dweight=False, workspace=BAD["host"])
    assert calls[0][-2:] == (None, 0)


def test_selections():
    for bad in BAD.values():
        with pytest.raises(TypeError):
            B._workspace(B.OP_PRUNE, 1000, 0, 1, 1, B.SCOPE_GLOBAL, torch.device("cuda", 1), bad)
    good = Room()
    assert B._workspace(B.OP_PRUNE, 1000, 0, 1, 1, B.SCOPE_GLOBAL, torch.device("cuda", 1), good)[0] is good
