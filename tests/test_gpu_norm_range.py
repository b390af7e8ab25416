"""The norm and its gradients over the whole range of binary32, against their definitions in binary64.

Tolerances are those of test_gpu_fp8_blocks.py, elementwise: u = eps / 2 of bfloat16 for the one rounding of an output, SUMS = 100 * 2^-24 of what a row's sums are part of.  The
factor 1 / sqrt(mean of h^2 + eps) is below binary32's normal range where the root is above 2^126; it is then up to 2^-22 off, four of those hundred units."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV
from test_gpu_fp8_blocks import H, SUMS, norm_gradients, rows_of, values

pytestmark = pytest.mark.gpu

B16 = torch.bfloat16
MOST = torch.finfo(B16).max                                               # almost 2^128
# one value a row, rows of one and of several wavefronts, of one, two and four pieces a wavefront, odd and aligned ones
WIDTHS = [1, 512, 650, 1000, 4608, 8192, 16384, 30001, 32768]


def large_rows(n, g):
    """Rows of one size and either sign, one of values of many sizes, one with a single large value among ordinary ones, and an ordinary one."""
    sign = torch.where(torch.rand(7, n, device=DEV, generator=g) < 0.5, -1.0, 1.0)
    h = sign * torch.tensor([MOST, 2.0 ** 127, 2.0 ** 124, 2.0 ** 122, 1.0, 1.0, 1.0], device=DEV)[:, None]
    h[4] *= 2.0 ** (127 * torch.rand(n, device=DEV, generator=g))
    h[5:] *= torch.rand(2, n, device=DEV, generator=g) + 0.5
    h[5, n // 2] = MOST
    return h.to(B16)


def factor(h, eps):
    return torch.sqrt(h.square().mean(1, keepdim=True) + float(torch.tensor(eps)))


def check_codes(m, y, slack):
    """Codes and scales of y (binary64), which the kernel has with `slack` of its own (elementwise).  A block whose largest magnitude is below 2^-100 has scale 0, and its values
    are taken for zeros: 2^-100 / 448 is what a scale may be off for that, and 2^-100 a value."""
    code, scale = values(m), m.scale.cpu().double()
    R, C = y.shape
    blocks = lambda t: torch.nn.functional.pad(t, (0, -C % 128)).view(R, -1, 128).amax(2)  # noqa: E731
    most, off = blocks(y.abs()), blocks(slack)
    far = (scale - most / 448).abs() - (off / 448 + 4 * H * most / 448 + 2.0 ** -100 / 448)
    assert bool((far <= 0).all()), (scale[far > 0][:4], most[far > 0][:4] / 448)
    each = scale.repeat_interleave(128, 1)[:, :C]
    assert bool(((code * each - y).abs() <= torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * each) * (1 + 8 * H) + 2 * slack + 8 * H * y.abs() + 2.0 ** -100).all())


def check_forward(h, w, eps):
    out = P.condensa_rms_norm(h, w, eps=eps, y=True, codes=True)
    h, w = h.cpu().double(), w.cpu().double()
    want = h / factor(h, eps) * w
    # h * weight below 2^-126 is a multiple of 2^-149, so up to 2^-150 off before it is divided: of 2^-133, the least value, that is 2^-17, which is more than SUMS
    slack = SUMS * want.abs() + 2.0 ** -150 / factor(h, eps)
    assert bool(((out["y"].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + slack + 2.0 ** -133).all())
    check_codes(out["codes"], want, slack)


def check_backward(h, dy, w, dsum, eps):
    T = h.shape[0]
    out = P.condensa_rms_norm_backward(dy, h, w, dsum=dsum, eps=eps, codes=True)
    want, size, want_w, size_w = norm_gradients(h, dy, w, dsum, float(torch.tensor(eps)))
    assert bool(((out["dx"].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 3 * SUMS * size + 2.0 ** -133).all())
    assert bool(((out["dweight"].cpu().double() - want_w).abs() <= (T + 100) * H * size_w + 1e-30).all())
    check_codes(out["codes"], want, 3 * SUMS * size)


@pytest.mark.parametrize("weight_type", [torch.float32, B16])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("n", WIDTHS)
def test_rows_up_to_the_largest_value(n, pad, weight_type):
    """Sums of squares up to 2^271.  (The gradients are small where h is large: dy is, too.)"""
    g = torch.Generator(DEV).manual_seed(n)
    h = rows_of(large_rows(n, g), pad)[0]
    w = (1 + 0.3 * torch.randn(n, device=DEV, generator=g)).to(weight_type)
    check_forward(h, w, 1e-6)
    dy = (torch.randn(h.shape, device=DEV, generator=g) * 2.0 ** 20).to(B16)
    for dsum in (None, (torch.randn(h.shape, device=DEV, generator=g) * 2.0 ** -100).to(B16)):
        check_backward(h, rows_of(dy, pad)[0], w, dsum, 1e-6)


def test_a_large_eps_beside_large_rows():
    g = torch.Generator(DEV).manual_seed(1)
    h, w = large_rows(1000, g), torch.ones(1000, device=DEV)
    for eps in (1e20, 3e38):
        check_forward(h, w, eps)
        check_backward(h, torch.randn(7, 1000, device=DEV, generator=g).to(B16), w, None, eps)


@pytest.mark.parametrize("weight_type", [torch.float32, B16])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("n", WIDTHS)
def test_products_of_h_and_its_gradient_beyond_the_range(n, pad, weight_type):
    """The sum of dy * weight * h leaves binary32 where neither the squares nor dy * weight do, and where the squares do as well."""
    g = torch.Generator(DEV).manual_seed(n)
    h = torch.randn(7, n, device=DEV, generator=g)
    dy = torch.randn(7, n, device=DEV, generator=g)
    # rows 1 and 2: products beyond the range; 3: their sum alone, since dy follows h; 4 and 5: squares too; 6: one product of many
    dy[3] = h[3]
    size = torch.tensor([[0, 0], [50, 86], [60, 100], [0, 115], [120, 70], [100, 110], [0, 60]], device=DEV)
    h, dy = h * 2.0 ** size[:, :1], dy * 2.0 ** size[:, 1:]
    h[6, n // 2], dy[6, n // 2] = 2.0 ** 62, 2.0 ** 80
    h, dy = h.to(B16), dy.to(B16)
    w = (1 + 0.3 * torch.randn(n, device=DEV, generator=g)).to(weight_type)
    for dsum in (None, torch.randn(7, n, device=DEV, generator=g).to(B16)):
        check_backward(rows_of(h, pad)[0], rows_of(dy, pad)[0], w, dsum, 1e-6)


@pytest.mark.parametrize("weight_type", [torch.float32, B16])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("n", WIDTHS)
def test_squares_below_the_range(n, pad, weight_type):
    """h of 2^-74 and an eps of as little as a square of it: neither is lost."""
    g = torch.Generator(DEV).manual_seed(n)
    h = torch.randn(5, n, device=DEV, generator=g) * 2.0 ** torch.tensor([-74.0, -70.0, -60.0, -40.0, -133.0], device=DEV)[:, None]
    h = rows_of(h.to(B16), pad)[0]
    w = (1 + 0.3 * torch.randn(n, device=DEV, generator=g)).to(weight_type)
    dy = torch.randn(5, n, device=DEV, generator=g).to(B16)
    for eps in (1e-44, 1e-40, 1e-30):
        check_forward(h, w, eps)
        check_backward(h, dy, w, None, eps)
