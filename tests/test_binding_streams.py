"""Which stream a call takes, found without a device."""
import types

import pytest
import torch

from paper_1911_02497_amd import binding as B


@pytest.fixture
def streams(monkeypatch):
    """A machine with three devices whose current streams are 100, 101 and 102; the second device is the current one."""
    B._raw_stream.cache_clear()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: types.SimpleNamespace(cuda_stream=100 + (1 if index is None else index)))
    yield monkeypatch
    B._raw_stream.cache_clear()


def test_the_public_way_where_torch_lacks_its_own(streams):
    streams.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert B._stream(None) == 101
    assert B._stream(types.SimpleNamespace(cuda_stream=7)) == 7


def test_torchs_own_way(streams):
    streams.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 200 + index, raising=False)
    assert B._stream(None) == 201
