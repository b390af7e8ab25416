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


def test_outputs_made_for_another_stream():
    """What a call on another stream returns does not lie in memory that the current stream, still at work, was given back.  (The workspaces,
    which hold places of tokens, are the test's own: nothing but values is at stake.)"""
    T = 300
    c = Case("bf16", T, 512, 4096, [8, 16], [t % 2 for t in range(T)])
    ws, wb = P.adapter_workspace(c.table, T), P.adapter_workspace(c.table, T, backward=True)
    c.forward(workspace=ws)
    c.backward(workspace=wb)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    old = [torch.empty(t.numel(), dtype=t.dtype, device=DEV) for t in (c.y, c.z, c.dx) for _ in range(8)]
    keep = busy(torch.cuda.current_stream())
    for t in old:
        t.fill_(float("nan"))
    del old, t
    out = P.condensa_adapter_project(c.x, c.w, c.table, c.ids, z=True, workspace=ws, stream=side)
    back = P.condensa_adapter_project_backward(c.dy, c.x, c.w, c.table, c.ids, out["z"], workspace=wb, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out["y"], c.y) and torch.equal(out["z"], c.z) and torch.equal(back["dx"], c.dx)
    assert bool(torch.isfinite(keep).all())


def test_workspaces_made_for_another_stream():
    """Nor does the workspace that such a call makes: looked at by address, with no work under way."""
    T = 300
    c = Case("bf16", T, 512, 4096, [8, 16], [t % 2 for t in range(T)])
    c.forward()
    side = torch.cuda.Stream()
    for backward in (False, True):
        n = P.adapter_workspace(c.table, T, backward=backward).numel()
        old = [torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(4)]
        places = [t.data_ptr() for t in old]
        del old
        torch.cuda.synchronize()
        if backward:
            out = P.condensa_adapter_project_backward(c.dy, c.x, c.w, c.table, c.ids, c.z, dx=c.dx, stream=side)
        else:
            out = P.condensa_adapter_project(c.x, c.w, c.table, c.ids, y=c.y, stream=side)
        torch.cuda.synchronize()
        at = out["workspace"].data_ptr()
        assert not any(abs(at - p) < n for p in places)


def test_a_stream_that_is_only_a_handle():
    """As the other entry points, tables' calls take any object that has a stream's handle."""
    class Handle:
        def __init__(self, stream):
            self.cuda_stream = stream.cuda_stream

    c = Case("bf16", 300, 128, 96, [8], [0] * 300)
    c.forward()
    c.backward()
    want = [t.clone() for t in (c.y, c.z, c.dx, *c.grads[0])]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    handle = Handle(side)
    table = P.adapter_table(c.adapters, grads=c.grads, stream=handle)
    out = P.condensa_adapter_project(c.x, c.w, table, c.ids, z=True, stream=handle)
    back = P.condensa_adapter_project_backward(c.dy, c.x, c.w, table, c.ids, out["z"], stream=handle)
    torch.cuda.synchronize()
    for got, right in zip((out["y"], out["z"], back["dx"], *c.grads[0]), want):
        assert torch.equal(got, right)
