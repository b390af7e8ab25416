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
