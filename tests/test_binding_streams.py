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


def test_a_table_elsewhere_takes_the_stream_of_its_own_device(streams):
    """With the second device current, a call of a table on the third launches there, on that device's current stream."""
    entered, calls = [], []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            entered.append(self.index)

        def __exit__(self, *_):
            entered.append(None)

    streams.setattr(torch.cuda, "device", Device)
    streams.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 200 + index, raising=False)

    def entry(*args):
        calls.append((args, entered[-1] if entered else None))
        return 0

    there = types.SimpleNamespace(index=2, device=torch.device("cuda", 2))
    here = types.SimpleNamespace(index=1, device=torch.device("cuda", 1))
    B._run(there, None, entry, "a")
    B._run(here, None, entry, "b")
    assert calls == [(("a", 202), 2), (("b", 201), None)]
    side = types.SimpleNamespace(device=torch.device("cuda", 2), cuda_stream=9)
    B._run(there, side, entry, "c")
    assert calls[-1] == (("c", 9), 2)
    with pytest.raises(ValueError):
        B._run(here, side, entry, "d")


def test_tables_are_of_one_device():
    one, two = (types.SimpleNamespace(device=torch.device("cuda", i)) for i in (0, 1))
    assert B._device_of([one, one], "weights") == torch.device("cuda", 0)
    with pytest.raises(TypeError):
        B._device_of([one, two], "weights")


def test_whether_a_stream_is_captured_is_asked_of_that_stream(streams):
    """A list made on a stream that is being captured, with another one current, is not waited for; made on another one beside a capture, it is."""
    current, waited = ["outer"], []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            current.append(self.stream.name)

        def __exit__(self, *_):
            current.pop()

    streams.setattr(torch.cuda, "stream", On)
    for captured, asked, want in (("side", "side", []), ("outer", "side", ["side"])):
        waited.clear()
        streams.setattr(torch.cuda, "is_current_stream_capturing", lambda captured=captured: current[-1] == captured)
        B._wait_unless_captured(types.SimpleNamespace(name=asked, synchronize=lambda: waited.append(asked)))
        assert waited == want


def test_any_object_with_a_stream_handle(streams):
    assert B._handle_on(torch.device("cuda", 1), types.SimpleNamespace(cuda_stream=5)) == 5
    calls = []
    B._run(types.SimpleNamespace(index=1, device=torch.device("cuda", 1)), types.SimpleNamespace(cuda_stream=5), lambda *args: calls.append(args))
    assert calls == [(5,)]
