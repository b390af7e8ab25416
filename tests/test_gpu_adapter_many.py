"""Lists as long as they may be."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV

pytestmark = pytest.mark.gpu


def test_gradients_of_the_longest_list():
    """16384 adapters, one of rank 256 far down the list, beside 2048 -> 2048: more workgroups of gradients than a launch holds."""
    n, K, N, T, wide = 16384, 2048, 2048, 90, 16000
    g = torch.Generator(DEV).manual_seed(3)
    normal = lambda std, *shape: (torch.randn(*shape, device=DEV, generator=g) * std).bfloat16()  # noqa: E731
    small, big = (normal(K ** -0.5, 1, K), normal(0.1, N, 1)), (normal(K ** -0.5, 256, K), normal(0.1, N, 256))
    ga, gb = torch.full((n, 1, K), 5.0, device=DEV), torch.full((n, N, 1), 5.0, device=DEV)
    wide_grads = torch.full((256, K), 5.0, device=DEV), torch.full((N, 256), 5.0, device=DEV)
    table = P.adapter_table([(*big, 1.0) if i == wide else (*small, 1.0) for i in range(n)],
                            grads=[wide_grads if i == wide else (ga[i], gb[i]) for i in range(n)])
    ids = torch.tensor([(wide, 16383, 0)[t % 3] for t in range(T)], dtype=torch.int32, device=DEV)
    x, dy, w = normal(1.0, T, K), normal(0.1, T, N), normal(0.05, N, K)
    z = P.condensa_adapter_project(x, w, table, ids, z=True)["z"]
    dx = P.condensa_adapter_project_backward(dy, x, w, table, ids, z)["dx"]
    h, u = 2.0 ** -24, 2.0 ** -8
    for a, (A, B), got in ((wide, big, wide_grads), (16383, small, (ga[16383], gb[16383])), (0, small, (ga[0], gb[0]))):
        at = torch.nonzero(ids == a).flatten()
        xa, ya, za = x[at].double(), dy[at].double(), z[at, : A.shape[0]].double()
        dz, size = ya @ B.double(), ya.abs() @ B.double().abs()
        tol = ((N + 16) * h * size + 2 * u ** 2 * dz.abs()).t() @ xa.abs() + (2 * T + 16) * h * (dz.abs().t() @ xa.abs())
        assert bool(((got[0].double() - dz.t() @ xa).abs() <= 1.01 * tol).all())
        assert bool(((got[1].double() - ya.t() @ za).abs() <= 1.01 * (T + 16) * h * (ya.abs().t() @ za.abs())).all())
        want = ya @ w.double() + dz @ A.double()
        tol = u * want.abs() + ((N + 16) * h * size + u * dz.abs()) @ A.double().abs() + (N + 300) * h * (ya.abs() @ w.double().abs() + dz.abs() @ A.double().abs())
        assert bool(((dx[at].double() - want).abs() <= 1.01 * tol).all())
    others = torch.ones(n, dtype=torch.bool, device=DEV)
    others[[0, wide, 16383]] = False
    assert not bool(ga[others].any()) and not bool(gb[others].any())
