"""Products with matrices in 8 bits, both directions, against the values that the codes stand for in binary64.

Tolerances, elementwise: u = eps / 2 of the 16-bit type for the result's rounding.  The matrix instruction aligns eight neighbouring products of codes to the largest of their
exponents e (the sum of both codes' exponents, so 2^e is no more than the largest product) and cuts what lies below 2^(e - 13): beside 2^16, 2^3 is kept and 2^2 is not.  Eight products lose
less than 8 * 2^-13 of their largest, which is no more than the largest of eight values of x times the largest of eight of W.  Sixteen such groups, the block's scales
and the sum over blocks are binary32: H = 2^-24 (twice that where an addition cuts) of the sums' magnitude for each."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
H = 2.0 ** -24


def matrix(rows, cols, block_rows, g, pad=0, offset=0, fill=0x7F, std=1.0):
    """Codes of random values in rows with `pad` more bytes (NaN codes) in memory, `offset` bytes past an aligned address, and scales of many sizes."""
    whole = torch.full((rows * (cols + pad) + offset + 32,), fill, device=DEV, dtype=torch.uint8)
    q = whole[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v = torch.randn(rows, cols, device=DEV, generator=g) * 60
    v = torch.where(torch.rand(rows, cols, device=DEV, generator=g) < 0.2, torch.zeros_like(v), v)
    q.copy_(v.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    s = torch.full((-(-rows // block_rows), -(-cols // 128) + 1), float("nan"), device=DEV)
    s[:, :-1] = std / 60 * torch.exp(0.5 * torch.randn(s.shape[0], s.shape[1] - 1, device=DEV, generator=g))
    return P.Fp8Matrix(q, s[:, :-1], block_rows)


def values(m):
    by = m.scale.double().repeat_interleave(m.block_rows, 0)[:m.rows].repeat_interleave(128, 1)[:, :m.cols]
    return m.q.contiguous().view(torch.float8_e4m3fn).double() * by


def largest_of8(v):
    """Of eight neighbouring values of a row."""
    return torch.nn.functional.pad(v.abs(), (0, -v.shape[1] % 8)).view(v.shape[0], -1, 8).amax(2)


def check(out, x, w, t, steps):
    """w: [outputs, sum]"""
    u, tiny = torch.finfo(t).eps / 2, 2.0 ** -25 if t == torch.float16 else 2.0 ** -133
    product = lambda a, b: a @ b.t().contiguous()  # noqa: E731
    want, size, cut = product(x, w), product(x.abs(), w.abs()), product(largest_of8(x), largest_of8(w)) * 2.0 ** -10
    far = (out.double() - want).abs() - (u * want.abs() + cut + (2 * 16 + 2 * steps + 32) * H * size + tiny)
    assert bool((far <= 0).all()), float(far.max())


SIZES = [(1, 512, 2048), (1, 1, 1), (1, 130, 70), (2, 128, 64), (5, 257, 129), (16, 4608, 256), (17, 1000, 333), (31, 64, 4096), (64, 4608, 1024), (65, 200, 65), (96, 2048, 512),
         (129, 650, 2600), (200, 640, 640), (257, 1024, 520), (300, 2600, 650), (1000, 384, 384), (1024, 1024, 1024), (2048, 520, 2048), (1333, 650, 1000), (3584, 200, 3520), (3500, 3584, 300), (400, 520, 4096), (1800, 4096, 333),
         (100, 2700, 500), (70, 600, 2600), (1100, 1003, 1999), (4000, 2100, 4400), (4000, 4400, 2100)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("rows", ["aligned", "contiguous", "any"])
def test_products(dtype, T, K, N, rows):
    t = TYPES[dtype]
    g = torch.Generator(DEV).manual_seed(T * 7 + K + N)
    pads = lambda c: dict(aligned=(-c % 16, 0), contiguous=(0, 0), any=(5, 3))[rows]  # noqa: E731
    w = matrix(N, K, 128, g, *pads(K), std=0.05)
    x, dy = matrix(T, K, 1, g, *pads(K)), matrix(T, N, 1, g, *pads(N))
    whole = torch.full((T * (N + 3) + 8,), 7.0, device=DEV, dtype=t)
    y = whole[1:1 + T * (N + 3)].view(T, N + 3)[:, :N] if rows == "any" else torch.full((T, N), 7.0, device=DEV, dtype=t)
    out = P.condensa_project_fp8(x, w, y)
    assert out["y"] is y
    W = values(w)
    check(y, values(x), W, t, -(-K // 128))
    if rows == "any":
        left = torch.ones_like(whole, dtype=torch.bool)
        left[1:1 + T * (N + 3)].view(T, N + 3)[:, :N] = False
        assert bool((whole[left] == 7.0).all())
    back = P.condensa_project_fp8_backward(dy, w, dtype=t)["dx"]
    check(back, values(dy), W.t().contiguous(), t, -(-N // 128))
    assert torch.equal(P.condensa_project_fp8(x, w, dtype=t)["y"], y) and torch.equal(P.condensa_project_fp8_backward(dy, w, dtype=t)["dx"], back)      # equal bits


@pytest.mark.parametrize("T", [1, 3, 16, 40, 100, 700])
def test_specials_stay_in_their_rows(T):
    """NaN codes and scales of infinity reach their token's outputs and those of their row (block) of W, and no others."""
    K, N = 300, 400
    g = torch.Generator(DEV).manual_seed(T)
    w, x, dy = matrix(N, K, 128, g, 20, 0), matrix(T, K, 1, g, 20, 0), matrix(T, N, 1, g)
    y, dx = (P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"], P.condensa_project_fp8_backward(dy, w, dtype=torch.bfloat16)["dx"])
    x.q[T // 2, 299], dy.q[T // 2, 0] = 0x7F, 0xFF
    bad, bad_dx = (P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"], P.condensa_project_fp8_backward(dy, w, dtype=torch.bfloat16)["dx"])
    rest = torch.arange(T, device=DEV) != T // 2
    for was, now in ((y, bad), (dx, bad_dx)):
        assert bool(torch.isnan(now[T // 2]).all()) and torch.equal(now[rest], was[rest])
    x.q[T // 2, 299], dy.q[T // 2, 0] = 0, 0
    y, dx = (P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"], P.condensa_project_fp8_backward(dy, w, dtype=torch.bfloat16)["dx"])
    w.q[399, 7] = 0x7F
    bad, bad_dx = (P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"], P.condensa_project_fp8_backward(dy, w, dtype=torch.bfloat16)["dx"])
    assert bool(torch.isnan(bad[:, 399]).all()) and torch.equal(bad[:, :399], y[:, :399])
    assert bool(torch.isnan(bad_dx[:, 7]).all()) and torch.equal(bad_dx[:, 8:], dx[:, 8:]) and torch.equal(bad_dx[:, :7], dx[:, :7])


def test_zero_tokens_and_a_kept_workspace():
    g = torch.Generator(DEV).manual_seed(1)
    w = matrix(700, 900, 128, g)
    assert P.condensa_project_fp8(matrix(0, 900, 1, g), w, dtype=torch.float16)["y"].shape == (0, 700)
    ws = P.project_fp8_workspace(w, 900), P.project_fp8_workspace(w, 900, backward=True)
    for T in (900, 300, 129, 64, 16, 1):
        x, dy = matrix(T, 900, 1, g), matrix(T, 700, 1, g)
        assert torch.equal(P.condensa_project_fp8(x, w, dtype=torch.float16, workspace=ws[0])["y"], P.condensa_project_fp8(x, w, dtype=torch.float16)["y"])
        assert torch.equal(P.condensa_project_fp8_backward(dy, w, dtype=torch.float16, workspace=ws[1])["dx"], P.condensa_project_fp8_backward(dy, w, dtype=torch.float16)["dx"])


@pytest.mark.parametrize("T", [1, 40, 100, 700])
def test_scales_of_infinity_stay_in_their_rows_and_blocks(T):
    K, N = 300, 400
    g = torch.Generator(DEV).manual_seed(T)
    w, x = matrix(N, K, 128, g, 20, 0), matrix(T, K, 1, g, 20, 0)
    y = P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"]
    was = float(x.scale[T // 2, 1])
    x.scale[T // 2, 1] = float("inf")
    bad = P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"]
    rest = torch.arange(T, device=DEV) != T // 2
    assert not bool(torch.isfinite(bad[T // 2]).any()) and torch.equal(bad[rest], y[rest])
    x.scale[T // 2, 1] = was
    w.scale[2, 0] = float("inf")                                          # rows 256 .. 383 of W
    bad = P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"]
    assert not bool(torch.isfinite(bad[:, 256:384]).any()) and torch.equal(bad[:, :256], y[:, :256]) and torch.equal(bad[:, 384:], y[:, 384:])
