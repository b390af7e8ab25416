"""The same refusals with tensors on a device, and workspaces of other types than bytes."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV
from test_gpu_adapter import Case, ids_of

pytestmark = pytest.mark.gpu


def bad_ones():
    return [torch.empty(1 << 24, dtype=torch.uint8), torch.empty(1, device=DEV, dtype=torch.uint8).expand(1 << 24), torch.empty(1 << 20, 2, device=DEV, dtype=torch.uint8)[:, 0]]


def calls():
    w = P.condensa_quantize_fp8_blocks(torch.randn(300, 260, device=DEV), block_rows=128)
    x, dy = P.condensa_quantize_fp8_blocks(torch.randn(100, 260, device=DEV)), P.condensa_quantize_fp8_blocks(torch.randn(100, 300, device=DEV))
    h = torch.randn(100, 260, device=DEV).to(torch.bfloat16)
    norm = torch.ones(260, device=DEV)
    c = Case("bf16", 100, 130, 70, [8, 4], ids_of(100, 2, "mixed"))
    weights = [torch.randn(100, 100, device=DEV)]
    z = P.condensa_adapter_project(c.x, c.w, c.table, c.ids, z=True)["z"]
    return [
        (lambda ws: P.condensa_project_fp8(x, w, dtype=torch.bfloat16, workspace=ws)["y"], lambda: P.project_fp8_workspace(w, 100)),
        (lambda ws: P.condensa_project_fp8_backward(dy, w, dtype=torch.bfloat16, workspace=ws)["dx"], lambda: P.project_fp8_workspace(w, 100, backward=True)),
        (lambda ws: P.condensa_rms_norm_backward(h, h, norm, workspace=ws)["dweight"], lambda: P.rms_norm_workspace(100, 260)),
        (lambda ws: P.condensa_adapter_project(c.x, c.w, c.table, c.ids, workspace=ws)["y"], lambda: P.adapter_workspace(c.table, 100)),
        (lambda ws: P.condensa_adapter_project_backward(c.dy, c.x, c.w, c.table, c.ids, z, workspace=ws)["dx"], lambda: P.adapter_workspace(c.table, 100, backward=True)),
        (lambda ws: P.condensa_prune(weights, [0.5], workspace=ws)["theta"][0][0], lambda: torch.empty(1 << 24, device=DEV, dtype=torch.uint8)),
        (lambda ws: P.condensa_lc_step(weights, [weights[0].clone()], 1e-3, 0.5, workspace=ws)["theta"][0], lambda: torch.empty(1 << 24, device=DEV, dtype=torch.uint8)),
        (lambda ws: P.condensa_neuron_prune(weights, 0.5, workspace=ws)["theta"][0], lambda: torch.empty(1 << 24, device=DEV, dtype=torch.uint8)),
        (lambda ws: P.condensa_count_nonzero(weights, workspace=ws), lambda: torch.empty(1 << 24, device=DEV, dtype=torch.uint8)),
    ]


def test_refused_and_served():
    for call, make in calls():
        want = call(None)
        for bad in bad_ones():
            with pytest.raises(TypeError):
                call(bad)
        ws = make()
        assert torch.equal(call(ws), want)
        assert torch.equal(call(ws.view(torch.float32)), want)
