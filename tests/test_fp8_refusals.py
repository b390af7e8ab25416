"""What the entry points of matrices in 8 bits, of their products and of the norm refuse, found before anything reaches a device: addresses here are never touched."""
import ctypes

import pytest

import paper_1911_02497_amd as P
from paper_1911_02497_amd import binding as B

NULL, SIZE, DENSITY, SHAPE, WORKSPACE, ARG = -1, -2, -3, -4, -5, -6
BASE, STEP = 1 << 40, 1 << 28
F32, F16, BF16 = B.TYPE_F32, B.TYPE_F16, B.TYPE_BF16


def matrix(at=0, rows=100, cols=300, block_rows=1, **over):
    d = dict(q=BASE + at * STEP, scale=BASE + at * STEP + STEP // 2, rows=rows, cols=cols, q_stride=cols, scale_stride=-(-cols // 128), block_rows=block_rows, reserved=0)
    d.update(over)
    return B.Fp8MatrixDesc(*[d[f] for f, _ in B.Fp8MatrixDesc._fields_])


def ref(m):
    return None if m is None else ctypes.byref(m)


def encode(m, x=BASE + 8 * STEP, type_=BF16, stride=300):
    return P.library().condensa_quantize_fp8_blocks(x, type_, stride, ref(m), None)


def decode(m, x=BASE + 8 * STEP, type_=BF16, stride=300):
    return P.library().condensa_dequantize_fp8_blocks(ref(m), x, type_, stride, None)


BAD_MATRICES = [
    (dict(rows=-1), SIZE), (dict(rows=(1 << 24) + 1), SIZE), (dict(q=None), NULL), (dict(scale=None), NULL), (dict(cols=0), SHAPE), (dict(cols=(1 << 20) + 1, q_stride=1 << 21), SHAPE),
    (dict(q_stride=299), SHAPE), (dict(q_stride=(1 << 22) + 1), SHAPE), (dict(scale_stride=2), SHAPE), (dict(scale_stride=1 << 30), SHAPE), (dict(scale=BASE + STEP // 2 + 2), ARG),
    (dict(block_rows=0), ARG), (dict(block_rows=64), ARG), (dict(reserved=1), ARG),
]


@pytest.mark.parametrize("call", [encode, decode])
@pytest.mark.parametrize("over,status", BAD_MATRICES)
def test_matrices(call, over, status):
    assert call(matrix(**over)) == status


@pytest.mark.parametrize("call", [encode, decode])
@pytest.mark.parametrize("over,status", [
    (dict(x=None), NULL), (dict(type_=3), ARG), (dict(type_=-1), ARG), (dict(stride=299), SHAPE), (dict(stride=(1 << 22) + 1), SHAPE), (dict(x=BASE + 8 * STEP + 1), ARG),
    (dict(x=BASE + 8 * STEP + 2, type_=F32), ARG), (dict(x=BASE + 64), ARG), (dict(x=BASE + STEP // 2), ARG),
])
def test_codec(call, over, status):
    assert call(matrix(), **over) == status


def test_codec_sizes():
    assert encode(None) == NULL and decode(None) == NULL
    assert encode(matrix(rows=0, q=None, scale=None), x=None) == 0 and decode(matrix(rows=0, q=None, scale=None), x=None) == 0
    big = matrix(rows=1 << 24, cols=1 << 20, q_stride=1 << 20, scale_stride=1 << 13)
    assert encode(big, x=1 << 60, stride=1 << 20) == SIZE and decode(big, x=1 << 60, stride=1 << 20) == SIZE


def norm(**over):
    d = dict(x=BASE, residual=BASE + STEP, weight=BASE + 2 * STEP, sum=BASE + 3 * STEP, y=BASE + 4 * STEP, codes=None, n_tokens=100, width=300, x_stride=300, residual_stride=300,
             sum_stride=300, y_stride=300, type=BF16, weight_type=BF16, eps=1e-6, reserved=0)
    d.update(over)
    if d["codes"] is not None:
        d["codes"] = ctypes.pointer(d["codes"])
    return P.library().condensa_rms_norm(ctypes.byref(B.RmsNormCall(*[d[f] for f, _ in B.RmsNormCall._fields_])), None)


def norm_back(ws=BASE + 9 * STEP, size=1 << 27, **over):
    d = dict(dy=BASE, h=BASE + STEP, dsum=BASE + 3 * STEP, weight=BASE + 2 * STEP, dx=BASE + 4 * STEP, dweight=BASE + 5 * STEP, codes=None, n_tokens=100, width=300, dy_stride=300,
             h_stride=300, dsum_stride=300, dx_stride=300, type=BF16, weight_type=BF16, eps=1e-6, reserved=0)
    d.update(over)
    if d["codes"] is not None:
        d["codes"] = ctypes.pointer(d["codes"])
    return P.library().condensa_rms_norm_backward(ctypes.byref(B.RmsNormGradCall(*[d[f] for f, _ in B.RmsNormGradCall._fields_])), ws, size, None)


@pytest.mark.parametrize("call", [norm, norm_back])
@pytest.mark.parametrize("over,status", [
    (dict(n_tokens=-1), SIZE), (dict(n_tokens=(1 << 24) + 1), SIZE), (dict(width=0), SHAPE), (dict(width=32769), SHAPE), (dict(type=F32), ARG), (dict(type=F16), ARG),
    (dict(weight_type=F16), ARG), (dict(reserved=1), ARG), (dict(weight=None), NULL), (dict(weight=BASE + 2 * STEP + 1), ARG), (dict(weight_type=F32, weight=BASE + 2 * STEP + 2), ARG),
    (dict(eps=0.0), DENSITY), (dict(eps=-1e-6), DENSITY), (dict(eps=float("nan")), DENSITY), (dict(eps=float("inf")), DENSITY),
    (dict(codes=matrix(6, block_rows=128)), ARG), (dict(codes=matrix(6, rows=99)), SHAPE), (dict(codes=matrix(6, cols=299, q_stride=300)), SHAPE), (dict(codes=matrix(6, q=None)), NULL),
    (dict(codes=matrix(0)), ARG), (dict(codes=matrix(4)), ARG), (dict(codes=matrix(6, scale=BASE + STEP)), ARG), (dict(codes=matrix(6, scale=BASE + 6 * STEP + 300)), ARG),
])
def test_norm_arguments(call, over, status):
    assert call(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(x=None), NULL), (dict(sum=None, y=None), NULL), (dict(x_stride=299), SHAPE), (dict(residual_stride=-300), SHAPE), (dict(sum_stride=1 << 23), SHAPE), (dict(y_stride=0), SHAPE),
    (dict(x=BASE + 1), ARG), (dict(residual=BASE + STEP + 1), ARG), (dict(sum=BASE + 3 * STEP + 1), ARG), (dict(y=BASE + 4 * STEP + 1), ARG),
    (dict(y=BASE), ARG), (dict(y=BASE + STEP), ARG), (dict(y=BASE + 3 * STEP + 200), ARG), (dict(sum=BASE + STEP + 2), ARG), (dict(sum=BASE, x_stride=304), ARG),
    (dict(sum=BASE + 2 * STEP), ARG),
])
def test_norm_rows(over, status):
    assert norm(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(dy=None), NULL), (dict(h=None), NULL), (dict(dx=None, dweight=None), NULL), (dict(dy_stride=299), SHAPE), (dict(h_stride=299), SHAPE), (dict(dsum_stride=299), SHAPE),
    (dict(dx_stride=299), SHAPE), (dict(dy=BASE + 1), ARG), (dict(dweight=BASE + 5 * STEP + 2), ARG), (dict(dx=BASE), ARG), (dict(dx=BASE + STEP), ARG), (dict(dx=BASE + 3 * STEP + 2), ARG),
    (dict(dweight=BASE + STEP), ARG), (dict(ws=None), WORKSPACE), (dict(ws=BASE + 9 * STEP + 16), WORKSPACE), (dict(size=7 * 300 * 4 - 1), WORKSPACE), (dict(ws=BASE + 4 * STEP), ARG),
])
def test_norm_gradient_rows(over, status):
    assert norm_back(**over) == status


def test_norm_without_tokens():
    lib = P.library()
    assert lib.condensa_rms_norm(None, None) == NULL and lib.condensa_rms_norm_backward(None, None, 0, None) == NULL
    assert norm(n_tokens=0, x=None, residual=None, sum=None, y=None) == 0
    assert norm_back(n_tokens=0, dy=None, h=None, dsum=None, dx=None, dweight=None, codes=matrix(6, rows=0, q=None, scale=None), ws=None, size=0) == 0
    assert norm_back(n_tokens=0, dy=None, h=None, dsum=None, dx=None, dweight=None, ws=None, size=0) == 0           # dx of no tokens has no address
    size = lib.condensa_rms_norm_workspace_bytes
    assert size(-1, 64) == 0 and size((1 << 24) + 1, 64) == 0 and size(1, 0) == 0 and size(1, 32769) == 0
    sizes = [size(T, 1000) for T in (0, 1, 100, 511, 512, 513, 8192, 1 << 24)]
    assert sizes == sorted(sizes) and all(s > 0 and s % 256 == 0 for s in sizes)


def product(x=None, w=None, y=BASE + 4 * STEP, ld=1100, type_=BF16, ws=BASE + 5 * STEP, size=1 << 27, backward=False):
    x = matrix(0, rows=100, cols=1100 if backward else 1000) if x is None else x
    w = matrix(1, rows=1100, cols=1000, block_rows=128) if w is None else w
    lib = P.library()
    return (lib.condensa_project_fp8_backward if backward else lib.condensa_project_fp8)(ref(x), ref(w), y, ld, type_, ws, size, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("over,status", [
    (dict(y=None), NULL), (dict(type_=F32), ARG), (dict(type_=7), ARG), (dict(y=BASE + 4 * STEP + 1), ARG), (dict(ld=999), SHAPE), (dict(ld=1 << 23), SHAPE),
    (dict(ws=None), WORKSPACE), (dict(ws=BASE + 5 * STEP + 128), WORKSPACE), (dict(size=1000), WORKSPACE), (dict(y=BASE), ARG), (dict(y=BASE + STEP), ARG), (dict(ws=BASE), ARG),
    (dict(ws=BASE + 4 * STEP), ARG), (dict(ws=BASE + STEP // 2), ARG),
    (dict(w=matrix(1, rows=1100, cols=1000)), ARG), (dict(w=matrix(1, rows=0, cols=1000, block_rows=128)), SHAPE), (dict(x=matrix(0, rows=100, cols=1001)), SHAPE),
    (dict(x=matrix(0, rows=100, cols=1000, block_rows=128)), ARG), (dict(x=matrix(0, rows=(1 << 24) + 1, cols=1000)), SIZE),
])
def test_products(backward, over, status):
    assert product(backward=backward, **over) == status


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("over,status", [b for b in BAD_MATRICES if "q_stride" not in b[0] and "scale_stride" not in b[0]] + [(dict(q_stride=999), SHAPE), (dict(scale_stride=7), SHAPE)])
def test_matrices_of_products(backward, over, status):
    weight = dict(rows=1100, cols=1000, block_rows=128)
    assert product(w=matrix(1, **{**weight, **{k: (v + STEP if k == "scale" and v else v) for k, v in over.items()}}), backward=backward) == status


def test_products_without_tokens_and_beyond_a_launch():
    assert product(x=matrix(0, rows=0, cols=1000, q=None, scale=None), y=None, ws=None, size=0) == 0
    w = matrix(1, rows=1 << 20, cols=1 << 20, block_rows=128)
    x = matrix(0, rows=1 << 24, cols=1 << 20)
    for backward in (False, True):
        assert product(x=x, w=w, ld=1 << 20, backward=backward, size=1 << 62) == SIZE
    size = P.library().condensa_project_fp8_workspace_bytes
    w = matrix(1, rows=1100, cols=1000, block_rows=128)
    for backward in (0, 1):
        sizes = [size(ref(w), T, backward) for T in (0, 1, 17, 64, 65, 1000, 8192, 1 << 24)]
        assert sizes == sorted(sizes) and all(s > 0 and s % 256 == 0 for s in sizes)
        assert size(ref(w), -1, backward) == 0 and size(ref(w), (1 << 24) + 1, backward) == 0
    assert size(ref(matrix(1)), 100, 0) == 0 and size(None, 100, 0) == 0


def test_struct_layouts():
    assert ctypes.sizeof(B.Fp8MatrixDesc) == 56 and ctypes.sizeof(B.RmsNormCall) == 112 and ctypes.sizeof(B.RmsNormGradCall) == 120


def test_binding_checks():
    import torch
    q, s = torch.zeros(10, 300, dtype=torch.uint8), torch.zeros(10, 3)
    with pytest.raises(TypeError):
        P.Fp8Matrix(q, s)                                                 # not on a device
    with pytest.raises(TypeError):
        P.condensa_quantize_fp8_blocks(torch.zeros(10, 300))
    with pytest.raises(TypeError):
        P.condensa_rms_norm(torch.zeros(10, 300, dtype=torch.bfloat16), torch.ones(300))
    with pytest.raises(TypeError):
        P.condensa_rms_norm_backward(torch.zeros(10, 300, dtype=torch.bfloat16), torch.zeros(10, 300, dtype=torch.bfloat16), torch.ones(300))
