"""Norm, codes, products and their backward passes as a feed-forward block uses them: stage by stage against the definitions, in a graph, on other streams, and past 32-bit offsets."""
import importlib.util
import os

import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV
from test_gpu_fp8_blocks import check_codes, norm_gradients, SUMS
from test_gpu_project_fp8 import check, matrix, values

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("feed_forward_fp8", os.path.join(os.path.dirname(__file__), "..", "examples", "feed_forward_fp8.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def made(T, width, hidden, dtype, seed=0):
    g = torch.Generator(DEV).manual_seed(seed)
    normal = lambda std, *shape: torch.randn(*shape, device=DEV, generator=g) * std  # noqa: E731
    block = example.FeedForward(normal(0.04, hidden, width), normal(0.02, width, hidden), 1 + normal(0.1, width))
    return block, [normal(s, T, width).to(dtype) for s in (1.0, 1.0, 0.1, 0.1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,width,hidden", [(1, 512, 2048), (64, 650, 2600), (300, 512, 2048), (1333, 650, 1000)])
def test_block(dtype, T, width, hidden):
    block, (x, residual, dy, dh) = made(T, width, hidden, dtype)
    y, kept = block.forward(x, residual)
    assert torch.equal(kept["h"], (x.float() + residual.float()).to(dtype))
    h = kept["h"].cpu().double()
    u = h / torch.sqrt(h.square().mean(1, keepdim=True) + float(torch.tensor(1e-6))) * block.norm.cpu().double()
    check_codes(kept["u"], u, SUMS * u.abs())
    up = P.condensa_project_fp8(kept["u"], block.w1, dtype=dtype)["y"]
    check(up, values(kept["u"]), values(block.w1), dtype, -(-width // 128))
    assert torch.equal(kept["a"], torch.relu(up))
    check(y, values(kept["codes"]), values(block.w2), dtype, -(-hidden // 128))
    dx = block.backward(dy, dh, kept)
    dyq = P.condensa_quantize_fp8_blocks(dy)
    da = P.condensa_project_fp8_backward(dyq, block.w2, dtype=dtype)["dx"]
    check(da, values(dyq), values(block.w2).t().contiguous(), dtype, -(-width // 128))
    daq = P.condensa_quantize_fp8_blocks(da * (kept["a"] > 0))
    du = P.condensa_project_fp8_backward(daq, block.w1, dtype=dtype)["dx"]
    check(du, values(daq), values(block.w1).t().contiguous(), dtype, -(-hidden // 128))
    want, size, want_w, size_w = norm_gradients(kept["h"], du, block.norm, dh, float(torch.tensor(1e-6)))
    unit, tiny = torch.finfo(dtype).eps / 2, 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -133
    assert bool(((dx.cpu().double() - want).abs() <= unit * want.abs() + 3 * SUMS * size + tiny).all())
    assert bool(((block.grad.cpu().double() - want_w).abs() <= (T + 100) * 2.0 ** -24 * size_w + 1e-30).all())
    before = block.norm.clone()
    block.step(1e-2, 1)
    moved = block.grad.abs() > 1e-5
    assert bool(((before - block.norm)[moved].sign() == block.grad[moved].sign()).all())


def test_example_runs():
    block, answer = example.main(width=256, hidden=384, tokens=20, steps=2)
    assert answer.shape == (1, 256) and bool(torch.isfinite(answer).all()) and bool(torch.isfinite(block.norm).all())


@pytest.mark.parametrize("T", [1, 100, 700])
def test_captured_and_replayed(T):
    """A forward and a backward pass in a graph, several times with other inputs, beside eager work and an eager graph of the same leaves."""
    block, (x, residual, dy, dh) = made(T, 384, 640, torch.bfloat16)

    def both():
        y, kept = block.forward(x, residual)
        return y, block.backward(dy, dh, kept), block.grad

    leaf = block.norm.clone().requires_grad_()
    alive = (leaf * 2).sum()                                              # an eager graph that lives on
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    g = torch.Generator(DEV).manual_seed(7)
    for _ in range(4):
        for t in (x, residual, dy, dh):
            t.copy_(torch.randn(t.shape, device=DEV, generator=g) * 0.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        torch.randn(1000, 1000, device=DEV) @ torch.randn(1000, 1000, device=DEV)
        block.grad.fill_(3.0)
        want = both()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    alive.backward()
    assert bool((leaf.grad == 2).all())


def test_two_captured_graphs_share_a_workspace():
    g = torch.Generator(DEV).manual_seed(5)
    w = matrix(500, 2700, 128, g)
    ws = P.project_fp8_workspace(w, 100)
    xs = [matrix(100, 2700, 1, g) for _ in range(2)]
    want = [P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"] for x in xs]
    graphs = []
    for x in xs:
        graph, y = torch.cuda.CUDAGraph(), torch.empty(100, 500, device=DEV, dtype=torch.bfloat16)
        with torch.cuda.graph(graph):
            P.condensa_project_fp8(x, w, y, workspace=ws)
        graphs.append((graph, y))
    for _ in range(3):
        for (graph, y), right in zip(graphs, want):
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, right)


def test_other_streams():
    """Calls with a stream of their own make their results and workspaces there; two at once do not meet."""
    block, (x, residual, dy, dh) = made(900, 1024, 1024, torch.bfloat16)
    y, kept = block.forward(x, residual)
    back = P.condensa_rms_norm_backward(dy, kept["h"], block.norm, codes=True)
    dx = P.condensa_project_fp8_backward(back["codes"], block.w1, dtype=torch.bfloat16)["dx"]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        got = []
        for s in streams:
            out = P.condensa_rms_norm(x, block.norm, residual=residual, codes=True, stream=s)
            up = P.condensa_project_fp8(out["codes"], block.w1, dtype=torch.bfloat16, stream=s)["y"]
            b = P.condensa_rms_norm_backward(dy, out["sum"], block.norm, codes=True, stream=s)
            d = P.condensa_project_fp8_backward(b["codes"], block.w1, dtype=torch.bfloat16, stream=s)["dx"]
            back_up = P.condensa_dequantize_fp8_blocks(P.condensa_quantize_fp8_blocks(up, stream=s), stream=s)
            got.append((out["sum"], up, b["dx"], b["dweight"], d, back_up))
        torch.cuda.synchronize()
        up = P.condensa_project_fp8(kept["u"], block.w1, dtype=torch.bfloat16)["y"]
        want = (kept["h"], up, back["dx"], back["dweight"], dx, P.condensa_dequantize_fp8_blocks(P.condensa_quantize_fp8_blocks(up)))
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


def test_offsets_past_32_bits():
    """Rows whose distance from the first passes 2^32 bytes: the last ones are as those of a call with them alone."""
    T, n = (1 << 20) + (1 << 17) + 77, 4096
    x = torch.empty(T, n, device=DEV, dtype=torch.bfloat16)
    x[:-300].fill_(0.5)
    x[-300:] = torch.randn(300, n, device=DEV).to(torch.bfloat16)
    w = (1 + 0.1 * torch.randn(n, device=DEV)).to(torch.bfloat16)
    out = P.condensa_rms_norm(x, w, residual=x, codes=True, y=True)
    few = P.condensa_rms_norm(x[-300:], w, residual=x[-300:], codes=True, y=True)
    assert torch.equal(out["sum"][-300:], few["sum"]) and torch.equal(out["y"][-300:], few["y"])
    assert torch.equal(out["codes"].q[-300:], few["codes"].q) and torch.equal(out["codes"].scale[-300:], few["codes"].scale)
    m = P.condensa_quantize_fp8_blocks(x)
    part = P.condensa_quantize_fp8_blocks(x[-300:])
    assert torch.equal(m.q[-300:], part.q) and torch.equal(P.condensa_dequantize_fp8_blocks(m, dtype=torch.bfloat16)[-300:], P.condensa_dequantize_fp8_blocks(part, dtype=torch.bfloat16))
    back = P.condensa_rms_norm_backward(x, out["sum"], w, dweight=False)["dx"]
    assert torch.equal(back[-300:], P.condensa_rms_norm_backward(x[-300:], few["sum"], w, dweight=False)["dx"])
    del back, out
    g = torch.Generator(DEV).manual_seed(2)
    W = matrix(200, n, 128, g)
    y = P.condensa_project_fp8(m, W, dtype=torch.bfloat16)["y"]
    check(y[-300:], values(part), values(W), torch.bfloat16, n // 128)
    del y
    W = matrix(n, 200, 128, g)
    dx = P.condensa_project_fp8_backward(m, W, dtype=torch.bfloat16)["dx"]
    check(dx[-300:], values(part), values(W).t().contiguous(), torch.bfloat16, n // 128)
