"""Codes of quotients that are the middle of two codes, and of their neighbours in binary32, against the exact quotient; and the weight's gradient of a norm in the order of its sums.

x 448 / top is the middle of two codes m where x = m top / 448, which binary32 has where the product of the odd parts of m (17 to 31, or 1 to 15 below the smallest normal code) and of
top / 448 has 24 bits or fewer.  The quotients are formed in binary64: x 448 has 33 bits, and a quotient by 24 bits that is not m is 2^-30 away from it at least, so that it is rounded to m
only where it is m."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV
from test_gpu_fp8_blocks import H, TYPES, definition, norm_gradients, same, values

pytestmark = pytest.mark.gpu

# largest values, and how many of the candidates below tie where binary32 has them: all 126 middles where the 448th part has few bits, those with small odd parts where it has 21, and 22 to 24
TOPS = [(448.0, 252), (7.0, 252), (112 / 128, 252), (7 * 3.0, 252), (7 * 1365 / 64, 252), (7 * 1398103 / 2 ** 20, 12), (7 * (2 ** 21 + 1) / 2 ** 23, 8), (1 - 2.0 ** -24, 8), (7 * 2.0 ** 70, 252),
        (7 * 5 * 2.0 ** -99, 252), (448 * 2.0 ** 100, 252), (448 * 2.0 ** 110, 252)]


def middles():
    normal = [(8 + k + 0.5) * 2.0 ** (e - 3) for e in range(-6, 9) for k in range(8) if (8 + k + 0.5) * 2.0 ** (e - 3) < 448]
    return torch.tensor([(k + 0.5) * 2.0 ** -9 for k in range(8)] + normal, dtype=torch.float64)


def candidates(top):
    """Values next to m top / 448 for every middle m: that one in binary32, two neighbours on either side, and both signs."""
    x = (middles() * top / 448).float()
    bits = x.view(torch.int32)
    x = torch.cat([(bits + d).view(torch.float32) for d in (-2, -1, 0, 1, 2)])
    x = x[(x.abs() <= top) & (x > 0)]
    return torch.cat([x, -x])


def tied(x, top):
    """Which quotients are the middle of two codes, and whether the even one is below."""
    q = (x.double() * 448 / top).abs()
    m = middles()
    at = torch.searchsorted(m, q).clamp(max=len(m) - 1)
    return m[at] == q, (at % 2 == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("top,count", TOPS)
def test_ties(top, count, block_rows, dtype):
    t = TYPES[dtype]
    if float(torch.tensor(top, dtype=torch.float64).to(t)) != top:
        return                                                           # the type has no such value
    x = candidates(top)
    x = x[x.to(t).float() == x]
    ties, even_below = tied(x, top)
    assert int(ties.sum()) == count and int(even_below[ties].sum()) == count // 2
    rows = torch.zeros(128, 128)                                         # each row that has any: the largest value and 127 candidates
    rows[:-(-len(x) // 127), 0] = top
    for i in range(0, len(x), 127):
        part = x[i:i + 127]
        rows[i // 127, 1:1 + len(part)] = part
    v = rows.to(t).to(DEV)
    m = P.condensa_quantize_fp8_blocks(v, block_rows=block_rows)
    code, scale = definition(v, block_rows)
    assert same(values(m), code) and torch.equal(m.scale.cpu(), scale)
    assert torch.equal(m.q.cpu() >> 7, (rows < 0).to(torch.uint8))


@pytest.mark.parametrize("T,n", [(4200, 64), (4200, 650), (4200, 1500), (4200, 4608), (8192, 2048), (20000, 512)])
def test_weight_gradient_in_the_order_of_its_sums(T, n):
    """A value goes through as many additions as its wavefront takes rows in turn (17 at most at these sizes), then 8 for wavefronts with rows of their own, 16 for 1024 workgroups, 16 and 2 for
    the threads that add them up: 59, of 2^-24 of the magnitudes' sum each.  u = h r beside it: r is half as far off as the sum of squares, whose values go through 8 additions in a lane, 6 over lanes
    and 4 over wavefronts, and five operations follow: 14.  100 leaves room for a quarter more."""
    g = torch.Generator(DEV).manual_seed(T + n)
    h, dy = (torch.randn(T, n, device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
    w = torch.ones(n, device=DEV)
    got = P.condensa_rms_norm_backward(dy, h, w, eps=1e-5)["dweight"].cpu().double()
    _, _, want, size = norm_gradients(h, dy, w, None, float(torch.tensor(1e-5)))
    assert bool(((got - want).abs() <= 100 * H * size).all()), float(((got - want).abs() / size).max() / H)


def blocks_of(top):
    """Candidates in blocks of one row, the largest value first in each."""
    x = candidates(top)
    row = torch.zeros(-(-len(x) // 127), 128)
    row[:, 0] = top
    row[:, 1:] = torch.nn.functional.pad(x, (0, -len(x) % 127)).view(-1, 127)
    return row.view(1, -1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("top", [top for top, _ in TOPS])
def test_ties_in_a_gradient(top, dtype):
    """Where h is zero, dy and eps are one, the gradient is the weight."""
    w = blocks_of(top)
    n = w.shape[1]
    for T in (1, 3):
        dy, h = torch.ones(T, n, device=DEV, dtype=dtype), torch.zeros(T, n, device=DEV, dtype=dtype)
        m = P.condensa_rms_norm_backward(dy, h, w[0].to(DEV), eps=1.0, dx=False, dweight=False, codes=True)["codes"]
        code, scale = definition(w, 1)
        assert same(values(m), code.expand(T, n)) and torch.equal(m.scale.cpu(), scale.expand(T, n // 128))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("top", [top for top, _ in TOPS if 2.0 ** -99 <= top <= 2.0 ** 100])
def test_ties_in_a_norm(top, dtype):
    """Where h is one, codes are those of the weight, whatever the row's factor is."""
    w = blocks_of(top)
    for T in (1, 5):
        m = P.condensa_rms_norm(torch.ones(T, w.shape[1], device=DEV, dtype=dtype), w[0].to(DEV), eps=0.3, codes=True)["codes"]
        assert same(values(m), definition(w, 1)[0].expand(T, w.shape[1]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_products_of_16_bits_next_to_a_tie(dtype):
    """Rows of h whose products with the weight have a quotient within 2^-24 of the middle of two codes, but not on it, or on it: found among many, since they cannot be made."""
    g = torch.Generator(DEV).manual_seed(5)
    w = (1 + 0.3 * torch.randn(128, device=DEV, generator=g)).to(dtype)
    m = middles().to(DEV)
    found = []
    for _ in range(8):
        h = torch.randn(100000, 128, device=DEV, generator=g).to(dtype)
        y = h.double() * w.double()                                      # exact, and in binary32 as well
        q = (y * 448 / y.abs().amax(1, keepdim=True)).abs()
        at = torch.bucketize(q, m).clamp(max=len(m) - 1)
        near = torch.minimum((m[at] - q).abs(), (m[(at - 1).clamp(min=0)] - q).abs()) <= q * 2.0 ** -24
        found.append(h[near.any(1)])
    h = torch.cat(found)[:20000]
    assert len(h) >= 100
    codes = P.condensa_rms_norm(h, w, codes=True)["codes"]
    assert same(values(codes), definition(h.double() * w.double(), 1)[0])
