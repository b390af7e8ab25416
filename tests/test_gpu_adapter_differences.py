"""The adapters' gradients against differences of the loss, with steps along the gradient so that a wrong one shows.

L = <dy, y> is linear in A, in B and in x, so L(p + m) - L(p - m) = <gradient, (p + m) - (p - m)> for steps of any size.  What may differ: y is off by
u |y| and by (K + 300) 2^-24 and z's 2 u^2 of the magnitudes that it sums; the gradient of A by 2 u^2 + (N + T + 40) 2^-24 of its magnitudes, that of B
by u of them, since z comes in 16 bits, and dx by u of itself and 2 u^2 + (N + 300) 2^-24 of its magnitudes.  Steps are four times the parameter's deviation along
the gradient's sign, which makes the difference four times all that or more: zeros or half of a gradient are far outside."""
import pytest
import torch

from test_gpu_adapter import H, Case, ids_of

pytestmark = pytest.mark.gpu


def loss_and_error(c):
    """<dy, y> of a forward pass and a bound on what rounding does to it."""
    c.forward()
    y = c.y.double()
    size = c.x.double().abs() @ c.w.double().abs().t()
    for a, (A, B, s) in enumerate(c.adapters):
        at = c.tokens(a)
        size[at] += abs(s) * (c.x[at].double().abs() @ A.double().abs().t()) @ B.double().abs().t()
    err = 1.01 * (c.u * y.abs() + ((c.K + 300) * H + 2 * c.u ** 2) * size) + c.tiny
    return (c.dy.double() * y).sum(), (c.dy.double().abs() * err).sum()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T,K,N", [(90, 64, 48), (300, 136, 1736), (1700, 72, 80)])
def test_steps_along_the_gradient(dtype, T, K, N):
    c = Case(dtype, T, K, N, [8, 4], ids_of(T, 2, "blocks"))
    c.forward()
    c.dy.copy_((c.y.float() * 0.1).to(c.t))                          # every token adds to the loss, as where training lowers one
    c.backward()
    parameters, dx_size = [], c.dy.double().abs() @ c.w.double().abs()
    for a, (A, B, s) in enumerate(c.adapters):
        at, r = c.tokens(a), A.shape[0]
        dy, dz = c.dy[at].double().abs(), abs(s) * (c.dy[at].double().abs() @ B.double().abs())
        dx_size[at] += dz @ A.double().abs()
        parameters.append((A, c.grads[a][0].clone(), (2 * c.u ** 2 + (N + T + 40) * H) * (dz.t() @ c.x[at].double().abs())))
        parameters.append((B, c.grads[a][1].clone(), 1.01 * c.u * (dy.t() @ c.z[at, :r].double().abs())))
    parameters.append((c.x, c.dx.clone(), c.u * c.dx.double().abs() + (2 * c.u ** 2 + (N + 300) * H) * dx_size + c.tiny))
    for i, (p, grad, err) in enumerate(parameters):
        save, step = p.clone(), grad.float().sign() * p.float().std() * 4
        moved, loss, tol = 0.0, 0.0, 0.0
        for sign in (1, -1):
            p.copy_((save.float() + sign * step).to(c.t))
            value, rounding = loss_and_error(c)
            moved, loss, tol = moved + sign * p.double(), loss + sign * value, tol + rounding
        p.copy_(save)
        want, tol = (grad.double() * moved).sum(), tol + (err * moved.abs()).sum()
        assert abs(loss - want) <= tol, (i, float(loss), float(want), float(tol))
        assert want > 4 * tol, (i, float(want), float(tol))
