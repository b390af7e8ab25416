"""What z and dz carry into y and dx: more bits than the 16-bit type has, and float16's whole way from far below its range to far above it,
however many tokens there are.

Tolerances as in the tests of the formulas, u = eps / 2: the sums in binary32, one rounding of the result, and for z and dz what two
16-bit values leave of a number, u^2 of it; of float16, whose second value ends at 2^-25 where the largest of 32 is at least 2^14, 2^-39 of that one
besides."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV
from test_gpu_adapter import H, TYPES, Case, ids_of

pytestmark = pytest.mark.gpu

# tokens, inputs and outputs of forward passes whose sum is not split, of one that is, and of the largest tiles
SIZES = [(300, 136, 1728), (200, 136, 1728), (3330, 1032, 3528)]


def share(c, at, z, size, m, terms):
    """(z M^T, its tolerance before rounding) for tokens whose z has the summed magnitudes `size` over `terms` products."""
    mt = m.double().t().contiguous()
    dz = 2 * c.u ** 2 * z.abs() + (terms + 16) * H * size
    if c.t == torch.float16:
        dz = dz + 2.0 ** -38 * z.abs().amax(1, keepdim=True)
    return z @ mt, 1.01 * (dz @ mt.abs() + (m.shape[1] + 64) * H * (z.abs() @ mt.abs()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_the_share_is_rounded_once(dtype, T, K, N):
    """Beside a W of zeros y and dx are the adapters' shares alone."""
    c = Case(dtype, T, K, N, [1, 16, 40], ids_of(T, 3, "mixed"))
    back = Case(dtype, T, N, K, [1, 16, 40], ids_of(T, 3, "mixed"))
    c.w.zero_()
    back.w.zero_()
    c.forward()
    back.forward()
    back.backward()
    for a in range(3):
        at = c.tokens(a)
        A, B, s = c.adapters[a]
        x = c.x[at].double()
        y, tol = share(c, at, s * (x @ A.double().t().contiguous()), abs(s) * (x.abs() @ A.double().abs().t().contiguous()), B, K)
        c.within(c.y[at], y, tol + 1.01 * c.u * y.abs() + c.tiny, f"y {a}")
        A, B, s = back.adapters[a]
        dy = back.dy[at].double()
        dx, tol = share(back, at, s * (dy @ B.double()), abs(s) * (dy.abs() @ B.double().abs()), A.t(), K)
        back.within(back.dx[at], dx, tol + 1.01 * back.u * dx.abs() + back.tiny, f"dx {a}")


@pytest.mark.parametrize("T,K,N", SIZES)
@pytest.mark.parametrize("big", [True, False])
def test_values_that_float16_does_not_reach(T, K, N, big):
    """Sums above 65504 or among float16's last bits whose products with the other matrix are ordinary values."""
    up, down = (30.0, 2.0 ** -9) if big else (2.0 ** -14, 2.0 ** 14)
    c, back = Case("f16", T, K, N, [3, 40], ids_of(T, 2, "mixed")), Case("f16", T, N, K, [3, 40], ids_of(T, 2, "mixed"))
    for case in (c, back):
        case.w.mul_(2.0 ** -4)
    c.x.abs_().mul_(up)
    back.dy.abs_().mul_(10 * up)
    for i in range(2):
        A, B, _ = c.adapters[i]
        A.abs_().mul_(up * K ** 0.5 * 4)
        B.mul_(down)
        A, B, _ = back.adapters[i]
        B.abs_().mul_(40 * up)
        A.mul_(down)
    c.forward()
    back.z = torch.zeros(T, 40, device=DEV, dtype=torch.float16)
    back.backward()
    for a in range(2):
        at = c.tokens(a)
        A, B, s = c.adapters[a]
        x, w = c.x[at].double(), c.w.double()
        z, zs = s * (x @ A.double().t().contiguous()), abs(s) * (x.abs() @ A.double().abs().t().contiguous())
        assert bool((z.abs() > 65536).any()) if big else bool((z.abs() < 2.0 ** -14).any())
        y, tol = share(c, at, z, zs, B, K)
        y = y + x @ w.t().contiguous()
        tol = tol + (K + 300) * H * (x.abs() @ w.abs().t().contiguous()) + H * y.abs()
        assert bool((y.abs() < 60000).all())
        c.within(c.y[at], y, tol + 1.01 * c.u * y.abs() + c.tiny, f"y {a}")
        A, B, s = back.adapters[a]
        dy, w = back.dy[at].double(), back.w.double()
        dz, dzs = s * (dy @ B.double()), abs(s) * (dy.abs() @ B.double().abs())
        assert bool((dz.abs() > 65536).any()) if big else bool((dz.abs() < 2.0 ** -8).any())
        dx, tol = share(back, at, dz, dzs, A.t(), K)
        dx = dx + dy @ w
        tol = tol + (K + 300) * H * (dy.abs() @ w.abs()) + H * dx.abs()
        assert bool((dx.abs() < 60000).all())
        back.within(back.dx[at], dx, tol + 1.01 * back.u * dx.abs() + back.tiny, f"dx {a}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,K,N", SIZES[:2])
def test_infinities_of_an_adapter_keep_their_sign(dtype, T, K, N):
    """A finite z times an infinity of B is an infinity of its sign, and dz times one of A."""
    c, back = Case(dtype, T, K, N, [1], [0] * T), Case(dtype, T, N, K, [1], [0] * T)
    c.adapters[0][1][5, 0] = float("inf")
    back.adapters[0][0][0, 5] = float("inf")
    c.forward()
    back.forward()
    back.backward()
    for got, by in ((c.y, c.x.double() @ c.adapters[0][0].double().t()), (back.dx, back.dy.double() @ back.adapters[0][1].double())):
        want = torch.sign(by[:, 0] * 0.5) * float("inf")
        assert torch.equal(got[:, 5].double(), want)
        rest = got.double()
        rest[:, 5] = 0
        assert bool(torch.isfinite(rest).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_what_the_workspace_held_does_not_matter(dtype, T, K, N):
    """Bytes of NaN in the workspace: what is read of it has been written by the call."""
    for how in ("mixed", "none"):
        c = Case(dtype, T, K, N, [3, 40, 70], ids_of(T, 3, how))
        ws = [P.adapter_workspace(c.table, T, backward=b) for b in (False, True)]
        for w in ws:
            w.fill_(255)
        c.forward(workspace=ws[0])
        c.check_forward(how)
        c.backward(workspace=ws[1])
        c.check_backward(how)
        back = Case(dtype, T, N, K, [3, 40, 70], ids_of(T, 3, how))
        w = P.adapter_workspace(back.table, T, backward=True).fill_(255)
        back.forward(workspace=P.adapter_workspace(back.table, T).fill_(255))
        back.check_forward(how)
        back.backward(workspace=w)
        back.check_backward(how)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [2.0 ** 126, 2.0 ** -112])
def test_gradients_beside_scales_of_any_size(dtype, scale):
    """dz near both ends of binary32: the gradients' 16-bit values are scaled as far as it takes."""
    T, K, N, r = 150, 96, 64, 9
    c = Case(dtype, T, K, N, [r], [0] * T, scale_x=0.1)
    A, B, _ = c.adapters[0]
    c.x.mul_(2.0 ** -6)
    table = P.adapter_table([(A, B, scale)], grads=c.grads)
    z = torch.zeros(T, r, device=DEV, dtype=c.t)
    P.condensa_adapter_project_backward(c.dy, c.x, c.w, table, c.ids, z, dx=False)
    dy, x = c.dy.double(), c.x.double()
    dz, dzs = scale * (dy @ B.double()), scale * (dy.abs() @ B.double().abs())
    tol = 1.01 * (((N + 16) * H * dzs + 2 * c.u ** 2 * dz.abs()).t().contiguous() @ x.abs() + (2 * T + 16) * H * (dz.abs().t().contiguous() @ x.abs()))
    tol = tol + 2.0 ** -38 * dz.abs().max() * x.abs().sum(0)[None] + 2.0 ** -140 * T
    c.within(c.grads[0][0], dz.t().contiguous() @ x, tol, "grad_A")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_infinities_of_x_keep_their_sign_in_gradients(dtype):
    """dz times an infinity of x is an infinity of its sign, also where dz needs no more than one 16-bit value."""
    T, K, N, r = 70, 64, 48, 6
    c = Case(dtype, T, K, N, [r], [0] * T)
    A, B, s = c.adapters[0]
    B[:, 0] = 0
    B[3, 0] = 1                                                      # dz of rank 0 is a value of dy times the scale
    c.z = torch.zeros(T, r, device=DEV, dtype=c.t)
    c.x[5, 7], c.x[5, 9] = float("inf"), float("-inf")
    assert bool((c.dy[5, 3] != 0).all())
    c.backward()
    dz = s * (c.dy.double() @ B.double())
    got = c.grads[0][0].double()
    assert torch.equal(got[:, 7], torch.sign(dz[5]) * float("inf")) and torch.equal(got[:, 9], torch.sign(dz[5]) * float("-inf"))
    got[:, 7] = got[:, 9] = 0
    assert bool(torch.isfinite(got).all()) and bool(torch.isfinite(c.grads[0][1]).all())
