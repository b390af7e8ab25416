"""Tables on the device, and what is made for a call, where several streams are at work."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV
from test_gpu_adapter import Case

pytestmark = pytest.mark.gpu


def test_a_table_made_on_a_stream_that_is_captured():
    """Made on a captured stream while another one is current: the list is laid out by the graph and not waited for."""
    c = Case("bf16", 5, 64, 96, [8], [0] * 5)
    c.forward()
    want = c.y.clone()
    side, other, g = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        with torch.cuda.stream(other):
            table = P.adapter_table(c.adapters, stream=side)
        P.condensa_adapter_project(c.x, c.w, table, c.ids, y=c.y)
    for _ in range(3):
        c.y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.y, want)


def busy(stream):
    """Some milliseconds of work on a stream."""
    with torch.cuda.stream(stream):
        a = torch.full((4096, 4096), 1.0 / 4096, device=DEV)
        for _ in range(40):
            a = a @ a
    return a


def handed_out_again(nbytes, address):
    """Whether memory of this size that is asked for now overlaps that at `address`; nothing is written into it."""
    asked = [torch.empty(nbytes, dtype=torch.uint8, device=DEV) for _ in range(64)]
    return any(abs(t.data_ptr() - address) < nbytes for t in asked)


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("what", ["adapters", "adamw"])
def test_a_table_dropped_while_another_stream_reads_it(what, given):
    """Its list and its tensors are not handed out before the work of that stream is done, whether the stream was given or current."""
    side = torch.cuda.Stream()
    n = 1 << 21                                                     # lists and tensors with blocks of their own
    if what == "adapters":
        c = Case("bf16", 5, 64, 96, [8] * 2000, [0] * 5)
        table, c.adapters, c.grads = c.table, None, None
        c.table = None
        held = [(table._memory.data_ptr(), table._memory.numel())]
        step = lambda s: P.condensa_adapter_project(c.x, c.w, table, c.ids, y=c.y, workspace=ws, stream=s)  # noqa: E731
        ws = P.adapter_workspace(table, 5)
    else:
        t = [torch.zeros(n, device=DEV) for _ in range(4)]
        table = P.adamw_table([t[0]], [t[1]], [t[2]], [t[3]])
        held = [(x.data_ptr(), x.numel() * 4) for x in t]
        del t
        step = lambda s: P.condensa_lc_adamw_step(table, 1e-3, 1, stream=s)  # noqa: E731
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    keep = busy(side)
    if given:
        step(side)
    else:
        with torch.cuda.stream(side):
            step(None)
    done = torch.cuda.Event()
    done.record(side)
    table = step = None
    found = [handed_out_again(nbytes, address) for address, nbytes in held]
    assert not done.query()                                         # the work is still under way, so the answers mean something
    side.synchronize()
    assert not any(found)
    assert bool(torch.isfinite(keep).all())
