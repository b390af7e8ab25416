"""Matrices in 8 bits and the norm that answers in them, against their definitions in binary64.

Codes and scales of the codec are equal to the definition's.  Tolerances of the norm, elementwise: u = eps / 2 of the 16-bit type for the one rounding of an output, H = 2^-24 of the
magnitudes that it rounds for every binary32 operation: a lane adds up to 64 values, the wavefront's lanes 6 times, wavefronts 16 times, and fewer than ten operations follow, so
100 H for what a row's sums are part of.  A code is half a step off at most: 2^-4 of its value, or 2^-10 of the scale below the normal range."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
H = 2.0 ** -24
SUMS = 100 * H


def rows_of(x, pad=0, offset=0, fill=7.0):
    """x in rows with `pad` more elements in memory, `offset` elements past an aligned address; and the whole buffer."""
    r, c = x.shape
    whole = torch.full((r * (c + pad) + offset + 8,), fill, device=DEV, dtype=x.dtype)
    v = whole[offset:offset + r * (c + pad)].view(r, c + pad)[:, :c]
    v.copy_(x)
    return v, whole


def room(rows, cols, block_rows=1, pad=0, offset=0):
    q, whole = rows_of(torch.full((rows, cols), 0x55, device=DEV, dtype=torch.uint8), pad, offset, 0x7F)
    s, whole_s = rows_of(torch.full((-(-rows // block_rows), -(-cols // 128)), -3.0, device=DEV), 1, 0)
    return P.Fp8Matrix(q, s, block_rows), whole, whole_s


def definition(x, block_rows):
    """(values of the codes, scales) on the CPU in binary64; the quotients of 24-bit significands are exact enough there to tell every tie."""
    x = x.cpu().double()
    R, C = x.shape
    pad = torch.zeros(-(-R // block_rows) * block_rows, -(-C // 128) * 128, dtype=torch.float64)
    pad[:R, :C] = x
    size = torch.nan_to_num(pad.abs(), nan=0.0, posinf=0.0).view(-1, block_rows, pad.shape[1] // 128, 128)
    most = size.amax((1, 3))
    scale = torch.where(most < 2.0 ** -100, torch.zeros_like(most), most).float() / torch.tensor(448.0)
    each = torch.where(most < 2.0 ** -100, torch.full_like(most, float("inf")), most).repeat_interleave(block_rows, 0).repeat_interleave(128, 1)[:R, :C]
    q = torch.where(torch.isinf(x), torch.where(torch.isinf(each), 0.0, 448.0) * torch.sign(x), x * 448 / each)
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    return (q / step).round() * step, scale


def values(m):
    return m.q.view(torch.float8_e4m3fn).cpu().double() if m.q.is_contiguous() else m.q.contiguous().view(torch.float8_e4m3fn).cpu().double()


def same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=-999.0), torch.nan_to_num(b, nan=-999.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols,pad,offset", [(1, 1, 0, 0), (1, 512, 0, 0), (3, 127, 0, 1), (130, 129, 5, 3), (257, 650, 0, 0), (128, 1024, 0, 0), (5, 2600, 8, 0), (300, 513, 3, 2)])
def test_codec(dtype, block_rows, rows, cols, pad, offset):
    g = torch.Generator(DEV).manual_seed(rows * 1000 + cols)
    x = torch.randn(rows, cols, device=DEV, generator=g) * torch.exp(2 * torch.randn(rows, cols, device=DEV, generator=g))
    x = torch.where(torch.rand(rows, cols, device=DEV, generator=g) < 0.3, torch.zeros_like(x), x).clamp(-6e4, 6e4).to(TYPES[dtype])
    v, _ = rows_of(x, pad, offset)
    m, whole, whole_s = room(rows, cols, block_rows, pad, offset)
    assert P.condensa_quantize_fp8_blocks(v, out=m) is m
    code, scale = definition(x, block_rows)
    assert same(values(m), code) and torch.equal(m.scale.cpu(), scale)
    between = torch.ones(whole.numel(), dtype=torch.bool, device=DEV)
    between[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = False
    assert bool((whole[between] == 0x7F).all())                          # what lies between rows is left alone
    assert int((whole_s == 7.0).sum()) >= m.scale.shape[0]
    for out_type in (torch.float32, torch.bfloat16, torch.float16):
        out, whole_out = rows_of(torch.zeros(rows, cols, device=DEV, dtype=out_type), pad, offset)
        P.condensa_dequantize_fp8_blocks(m, out=out)
        each = scale.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
        assert same(out.cpu(), (code.float() * each).to(out_type))
        assert bool((whole_out[between] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_codec_of_special_values(dtype, block_rows):
    x = torch.zeros(6, 6 * 128, device=DEV)
    x[0, 0], x[0, 1], x[0, 2], x[0, 3] = float("inf"), float("-inf"), float("nan"), 2.0
    x[1, 128:256] = float("nan")
    x[2, 256:300] = float("inf")                                         # no finite magnitude: scale 0
    x[3, 384:400] = -0.0
    x[4, 512:640] = torch.arange(128, device=DEV) * 2.0 ** -7            # ties of many codes
    if dtype != "f16":
        x[5, 640:768] = 2.0 ** -101
        x[5, 512:640] = torch.finfo(TYPES[dtype]).max * (torch.arange(128, device=DEV) / 127) if block_rows == 1 else 0
    m = P.condensa_quantize_fp8_blocks(x.to(TYPES[dtype]), block_rows=block_rows)
    code, scale = definition(x.to(TYPES[dtype]), block_rows)
    assert same(values(m), code) and torch.equal(m.scale.cpu(), scale)
    if block_rows == 1:
        assert m.q[3, 384].item() == 0x80 and m.q[0, 0].item() == 0x7E and m.q[0, 1].item() == 0xFE and m.q[0, 2].item() & 0x7F == 0x7F


def test_codec_empty_and_repeated():
    m = P.condensa_quantize_fp8_blocks(torch.zeros(0, 40, device=DEV), block_rows=128)
    assert m.rows == 0 and tuple(P.condensa_dequantize_fp8_blocks(m).shape) == (0, 40)
    x = torch.randn(300, 5000, device=DEV)
    a, b = P.condensa_quantize_fp8_blocks(x), P.condensa_quantize_fp8_blocks(x)
    assert torch.equal(a.q, b.q) and torch.equal(a.scale, b.scale)


def check_codes(m, y, slack):
    """Codes and scales of y (binary64), which the kernel has with `slack` of its own (elementwise)."""
    code, scale = values(m), m.scale.cpu().double()
    R, C = y.shape
    pad = torch.zeros(R, -(-C // 128) * 128, dtype=torch.float64)
    pad[:, :C] = y.abs()
    pad_slack = torch.zeros_like(pad)
    pad_slack[:, :C] = slack
    most = pad.view(R, -1, 128).amax(2)
    off = pad_slack.view(R, -1, 128).amax(2)
    assert bool(((scale - most / 448).abs() <= off / 448 + 4 * H * most / 448 + 2.0 ** -109).all())
    each = scale.repeat_interleave(128, 1)[:, :C]
    assert bool(((code * each - y).abs() <= torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * each) * (1 + 8 * H) + 2 * slack + 8 * H * y.abs() + 2.0 ** -100).all())


NORMS = [(1, 512, 0, 0), (1, 1, 0, 0), (2, 7, 0, 1), (3, 130, 3, 1), (33, 650, 0, 0), (5, 4608, 8, 0), (9, 4097, 0, 0), (4, 8192, 0, 0), (600, 129, 7, 0), (2, 16384, 0, 0), (2, 30001, 0, 0),
         (1, 32768, 0, 0), (1537, 64, 0, 0), (700, 1030, 0, 0), (3, 1500, 0, 0), (2, 19900, 0, 0), (4200, 4608, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("weight_type", ["f32", "same"])
@pytest.mark.parametrize("T,n,pad,offset", NORMS)
def test_norm(dtype, weight_type, T, n, pad, offset):
    t = TYPES[dtype]
    u, tiny = torch.finfo(t).eps / 2, 2.0 ** -25 if dtype == "f16" else 2.0 ** -133
    g = torch.Generator(DEV).manual_seed(T + n)
    x, res = (torch.randn(T, n, device=DEV, generator=g).to(t) for _ in range(2))
    w = (1 + 0.3 * torch.randn(n, device=DEV, generator=g)).to(t if weight_type == "same" else torch.float32)
    vx, vr = rows_of(x, pad, offset)[0], rows_of(res, pad, 0)[0]
    for residual in (vr, None):
        s, whole = rows_of(torch.zeros_like(x), pad, offset)
        y = rows_of(torch.zeros_like(x), pad, 0)[0]
        m, whole_q, _ = room(T, n, 1, pad, offset)
        out = P.condensa_rms_norm(vx, w, residual=residual, eps=1e-5, sum=s, y=y, codes=m)
        assert out["sum"] is s and out["y"] is y and out["codes"] is m
        h = x if residual is None else (x.float() + res.float()).to(t)
        assert torch.equal(s, h)
        h = h.cpu().double()
        want = h / torch.sqrt(h.square().mean(1, keepdim=True) + float(torch.tensor(1e-5))) * w.cpu().double()
        assert bool(((y.cpu().double() - want).abs() <= (u + SUMS) * want.abs() + tiny).all())
        check_codes(m, want, SUMS * want.abs())
        between = torch.ones(whole.numel(), dtype=torch.bool, device=DEV)
        between[offset:offset + T * (n + pad)].view(T, n + pad)[:, :n] = False
        assert bool((whole[between] == 7.0).all()) and bool((whole_q[between] == 0x7F).all())
        over = vx.clone() if residual is None else vr.clone()
        alone = P.condensa_rms_norm(over if residual is None else vx, w, residual=None if residual is None else over, eps=1e-5, sum=over, codes=True)       # in place
        assert torch.equal(over, s) and alone["y"] is None and torch.equal(alone["codes"].q, m.q) and torch.equal(alone["codes"].scale, m.scale)


def norm_gradients(h, dy, w, dsum, eps):
    """dx, the magnitudes that its binary32 operations round, dweight and its magnitudes."""
    h, dy, w = h.cpu().double(), dy.cpu().double(), w.cpu().double()
    r = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    u, g = h * r, dy * w
    dx = r * (g - u * (g * u).mean(1, keepdim=True))
    size = r * (g.abs() + u.abs() * (g * u).abs().mean(1, keepdim=True))
    if dsum is not None:
        dx, size = dx + dsum.cpu().double(), size + dsum.cpu().double().abs()
    return dx, size, (dy * u).sum(0), (dy * u).abs().sum(0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("weight_type", ["f32", "same"])
@pytest.mark.parametrize("T,n,pad,offset", NORMS)
def test_norm_gradients(dtype, weight_type, T, n, pad, offset):
    t = TYPES[dtype]
    u, tiny = torch.finfo(t).eps / 2, 2.0 ** -25 if dtype == "f16" else 2.0 ** -133
    g = torch.Generator(DEV).manual_seed(T + n)
    h, dy, ds = (torch.randn(T, n, device=DEV, generator=g).to(t) for _ in range(3))
    w = (1 + 0.3 * torch.randn(n, device=DEV, generator=g)).to(t if weight_type == "same" else torch.float32)
    vh, vdy, vds = rows_of(h, pad, offset)[0], rows_of(dy, pad, 0)[0], rows_of(ds, pad, offset)[0]
    eps = float(torch.tensor(1e-5))
    for dsum in (vds, None):
        dx, whole = rows_of(torch.zeros_like(h), pad, offset)
        dw = torch.full((n,), 5.0, device=DEV)
        m, _, _ = room(T, n, 1, pad, offset)
        P.condensa_rms_norm_backward(vdy, vh, w, dsum=dsum, eps=1e-5, dx=dx, dweight=dw, codes=m)
        want, size, want_w, size_w = norm_gradients(h, dy, w, None if dsum is None else ds, eps)
        assert bool(((dx.cpu().double() - want).abs() <= u * want.abs() + 3 * SUMS * size + tiny).all())
        assert bool(((dw.cpu().double() - want_w).abs() <= (T + 100) * H * size_w + 1e-30).all())
        check_codes(m, want, 3 * SUMS * size)
        between = torch.ones(whole.numel(), dtype=torch.bool, device=DEV)
        between[offset:offset + T * (n + pad)].view(T, n + pad)[:, :n] = False
        assert bool((whole[between] == 7.0).all())
        again = P.condensa_rms_norm_backward(vdy, vh, w, dsum=dsum, eps=1e-5, dx=True if dsum is None else vds, codes=True)                  # dx over dsum
        assert torch.equal(again["dx"], dx) and torch.equal(again["dweight"], dw) and torch.equal(again["codes"].q, m.q)
        vds.copy_(ds)
        only = P.condensa_rms_norm_backward(vdy, vh, w, dsum=dsum, eps=1e-5, dx=False, dweight=False, codes=True)
        assert only["dx"] is None and only["dweight"] is None and torch.equal(only["codes"].q, m.q)


def test_norm_gradients_against_differences():
    """Along a direction d: (F(h + e d) - F(h - e d)) / 2 e of F = sum dy y(h) in binary64, with an error of e^2, against dx . d, and the same for the weight."""
    g = torch.Generator().manual_seed(3)
    T, n, eps = 7, 300, 1e-5
    h, dy = (torch.randn(T, n, generator=g).to(torch.bfloat16) for _ in range(2))
    w = 1 + 0.3 * torch.randn(n, generator=g)
    out = P.condensa_rms_norm_backward(dy.to(DEV), h.to(DEV), w.to(DEV), eps=eps)

    def F(h, w):
        return float((dy.double() * h / torch.sqrt(h.square().mean(1, keepdim=True) + float(torch.tensor(eps))) * w).sum())

    for seed in range(3):
        d, dw = torch.randn(T, n, generator=g).double(), torch.randn(n, generator=g).double()
        e = 1e-4
        along = (F(h.double() + e * d, w.double()) - F(h.double() - e * d, w.double())) / (2 * e)
        assert abs(along - float((out["dx"].cpu().double() * d).sum())) <= 1e-2 * float((out["dx"].cpu().double() * d).norm())
        along = (F(h.double(), w.double() + e * dw) - F(h.double(), w.double() - e * dw)) / (2 * e)
        assert abs(along - float((out["dweight"].cpu().double() * dw).sum())) <= 1e-4 * float((out["dweight"].cpu().double() * dw).norm())


def test_norm_of_special_rows():
    """Squares beyond binary32, rows of zeros, infinities and NaN: none of them reaches another row."""
    n = 1000
    x = torch.randn(8, n, device=DEV).to(torch.bfloat16)
    plain = P.condensa_rms_norm(x, torch.ones(n, device=DEV), y=True)["y"]
    s = x.clone()
    s[1] = (s[1].double() * 2.0 ** 120).to(torch.bfloat16)
    s[2] = 0
    s[3, 5] = float("inf")
    s[4, 7] = float("nan")
    s[5] = (s[5].double() * 2.0 ** -100).to(torch.bfloat16)
    w = torch.ones(n, device=DEV)
    out = P.condensa_rms_norm(s, w, y=True, codes=True)
    y = out["y"]
    assert torch.equal(y[0], plain[0]) and torch.equal(y[6:], plain[6:])
    h = s[1].cpu().double()
    want = h / h.square().mean().sqrt()
    assert bool(((y[1].cpu().double() - want).abs() <= (2.0 ** -8 / 2 * 2 + SUMS) * want.abs()).all())
    assert bool((y[2] == 0).all()) and bool((out["codes"].scale[2] == 0).all())
    assert bool(torch.isnan(y[3, 5])) and bool((torch.cat([y[3, :5], y[3, 6:]]) == 0).all())
    assert bool(torch.isnan(y[4]).all()) and bool((out["codes"].q[4] & 0x7F == 0x7F).all())
    want = s[5].cpu().double() / 1e-3
    assert bool(((y[5].cpu().double() - want).abs() <= 2.0 ** -7 * want.abs()).all())
    dy = torch.randn(8, n, device=DEV).to(torch.bfloat16)
    good = P.condensa_rms_norm_backward(dy, x, w)["dx"]
    dx = P.condensa_rms_norm_backward(dy, s, w)["dx"]
    assert torch.equal(dx[0], good[0]) and torch.equal(dx[6:], good[6:]) and bool(torch.isfinite(dx[1]).all())
    want, size, _, _ = norm_gradients(s[1:2], dy[1:2], w, None, 0.0)
    assert bool(((dx[1:2].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 3 * SUMS * size + 2.0 ** -133).all())


def test_norm_without_tokens():
    x = torch.zeros(0, 40, device=DEV, dtype=torch.bfloat16)
    out = P.condensa_rms_norm(x, torch.ones(40, device=DEV), residual=x, codes=True)
    assert out["codes"].rows == 0
    back = P.condensa_rms_norm_backward(x, x, torch.ones(40, device=DEV), dweight=torch.full((40,), 3.0, device=DEV))
    assert bool((back["dweight"] == 0).all())
