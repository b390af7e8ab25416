"""Adapters beside a shared projection, forward and backward, against the formulas in binary64.

Tolerances, elementwise: u = eps / 2 of the 16-bit type for every rounding to it (the result, and z or dz where it enters y or dx),
2^-24 a term for binary32 sums (products of 16-bit values are exact), each of the sum of magnitudes that it rounds.  What lies below
the normal range of float16 is rounded by half of 2^-24 at most."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
H = 2.0 ** -24


class Case:
    def __init__(self, dtype, T, K, N, ranks, ids, seed=0, pad=0, offset=0, scale_x=1.0, scale_dy=0.1):
        g = torch.Generator(DEV).manual_seed(seed)
        t = TYPES[dtype]

        def rows(r, c, std):
            """[r, c] with `pad` more columns in memory, `offset` elements past an aligned address."""
            whole = torch.full((r * (c + pad) + offset + 8,), 7.0, device=DEV, dtype=t)
            v = whole[offset:offset + r * (c + pad)].view(r, c + pad)[:, :c]
            v.copy_((torch.randn(r, c, device=DEV, generator=g) * std).to(t))
            return v

        self.t, self.T, self.K, self.N, self.u = t, T, K, N, torch.finfo(t).eps / 2
        self.tiny = 2.0 ** -25 if t == torch.float16 else 1e-38
        self.x, self.w, self.dy = rows(T, K, scale_x), rows(N, K, 0.05), rows(T, N, scale_dy)
        self.y, self.dx = rows(T, N, 0.0), rows(T, K, 0.0)
        self.adapters = [((torch.randn(r, K, device=DEV, generator=g) * K ** -0.5).to(t), (torch.randn(N, r, device=DEV, generator=g) * 0.1).to(t),
                          (0.5, 1.0, -2.0)[i % 3]) for i, r in enumerate(ranks)]
        self.grads = [(torch.full((r, K), 5.0, device=DEV), torch.full((N, r), 5.0, device=DEV)) for r in ranks]
        self.ids = torch.tensor(ids, dtype=torch.int32, device=DEV) if T else torch.empty(0, dtype=torch.int32, device=DEV)
        assert self.ids.numel() == T
        kw = {} if ranks else {"n_in": K, "n_out": N, "dtype": t}
        self.table = P.adapter_table(self.adapters, grads=self.grads, **kw)

    def tokens(self, a):
        return torch.nonzero(self.ids == a).flatten()

    def forward(self, z_width=None, **kw):
        width = max(max((a.shape[0] for a, _, _ in self.adapters), default=1), z_width or 0)
        self.z = torch.full((self.T, width), 9.0, device=DEV, dtype=self.t)
        return P.condensa_adapter_project(self.x, self.w, self.table, self.ids, y=self.y, z=self.z, **kw)

    def check_forward(self, what=""):
        x, w = self.x.double(), self.w.double()
        y, size = x @ w.t().contiguous(), x.abs() @ w.abs().t().contiguous()
        z, tz = torch.zeros_like(self.z, dtype=torch.float64), torch.zeros_like(self.z, dtype=torch.float64)
        extra = torch.zeros_like(y)
        for a, (A, B, s) in enumerate(self.adapters):
            at, r = self.tokens(a), A.shape[0]
            if at.numel() == 0:
                continue
            za = s * (x[at] @ A.double().t().contiguous())
            zs = abs(s) * (x[at].abs() @ A.double().abs().t().contiguous())
            z[at, :r] = za
            tz[at, :r] = self.u * za.abs() + (self.K + 16) * H * zs + self.tiny
            bt = B.double().t().contiguous()
            y[at] += za @ bt
            size[at] += za.abs() @ bt.abs()
            extra[at] = 1.01 * (tz[at, :r] @ bt.abs())
        tol = 1.01 * (self.u * y.abs() + extra + (self.K + 300) * H * size) + self.tiny
        self.within(self.z, z, 1.01 * tz, f"{what} z")
        self.within(self.y, y, tol, f"{what} y")

    def within(self, got, want, tol, what):
        bad = ~((got.double() - want).abs() <= tol)
        assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist(), tol[bad][:3].tolist())

    def backward(self, **kw):
        return P.condensa_adapter_project_backward(self.dy, self.x, self.w, self.table, self.ids, self.z, dx=self.dx, **kw)

    def check_backward(self, what=""):
        x, w, dy = self.x.double(), self.w.double(), self.dy.double()
        dx, size = dy @ w, dy.abs() @ w.abs()
        extra = torch.zeros_like(dx)
        split = self.u ** 2 * 2
        for a, (A, B, s) in enumerate(self.adapters):
            at, r = self.tokens(a), A.shape[0]
            dz, dzs = s * (dy[at] @ B.double()), abs(s) * (dy[at].abs() @ B.double().abs())
            tdz = (self.N + 16) * H * dzs
            dx[at] += dz @ A.double()
            size[at] += dz.abs() @ A.double().abs()
            extra[at] = 1.01 * ((self.u * dz.abs() + tdz + self.tiny) @ A.double().abs())
            xa, ya, z = x[at], dy[at], self.z[at, :r].double()
            mags = dz.abs().t().contiguous() @ xa.abs()
            tol = 1.01 * ((tdz + split * dz.abs()).t().contiguous() @ xa.abs() + (2 * at.numel() + 16) * H * mags)
            if self.t == torch.float16 and at.numel():
                tol = tol + 2.0 ** -38 * dz.abs().max() * xa.abs().sum(0)[None]
            self.within(self.grads[a][0], dz.t().contiguous() @ xa, tol + 1e-38, f"{what} grad_A {a}")
            self.within(self.grads[a][1], ya.t().contiguous() @ z, 1.01 * (at.numel() + 16) * H * (ya.abs().t().contiguous() @ z.abs()) + 1e-38,
                        f"{what} grad_B {a}")
        self.within(self.dx, dx, 1.01 * (self.u * dx.abs() + extra + (self.N + 300) * H * size) + self.tiny, f"{what} dx")

    def padding_untouched(self):
        for t in (self.y, self.dx):
            whole = t._base if t._base is not None else t
            n, (r, c) = whole.numel(), t.shape
            inside = torch.zeros(n, dtype=torch.bool, device=DEV)
            for i in range(0, r):
                at = t.storage_offset() + i * t.stride(0)
                inside[at:at + c] = True
            assert bool((whole.flatten()[~inside] == 7.0).all())


def ids_of(T, n, how):
    if how == "blocks":
        return [(t * (n + 1) // max(T, 1)) - 1 for t in range(T)]
    if how == "mixed":
        return [(t * 7 + t // 3) % (n + 1) - 1 for t in range(T)]
    if how == "none":
        return [-1] * T
    if how == "wild":
        return [(0, n, -5, 2 ** 31 - 1, -2 ** 31, n - 1)[t % 6] for t in range(T)]
    return [how] * T


RANKS = {"one": [8], "odd": [1, 3, 24, 33], "wide": [64, 65, 16], "widest": [256, 130, 5], "many": [4] * 40, "zero": []}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T", [1, 2, 16, 17, 33, 64, 65, 130, 257, 600])
@pytest.mark.parametrize("shape", [(64, 64), (72, 136), (33, 31), (650, 260), (512, 1024)])
@pytest.mark.parametrize("ranks,how", [("odd", "mixed"), ("one", "blocks")])
def test_sizes(dtype, T, shape, ranks, how):
    n = len(RANKS[ranks])
    c = Case(dtype, T, *shape, RANKS[ranks], ids_of(T, n, how))
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("ranks", list(RANKS))
@pytest.mark.parametrize("how", ["blocks", "mixed", "none", "wild", 0])
@pytest.mark.parametrize("T", [7, 200])
def test_ranks_and_owners(dtype, ranks, how, T):
    n = len(RANKS[ranks])
    c = Case(dtype, T, 96, 200, RANKS[ranks], ids_of(T, n, how) if n or how == "none" else [3] * T, seed=1)
    c.forward(z_width=300)
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("T", [20, 300])
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (8, 0), (2, 2), (0, 4), (5, 3)])
@pytest.mark.parametrize("shape", [(128, 192), (66, 130)])
def test_strides_and_addresses(T, pad, offset, shape):
    c = Case("bf16", T, *shape, [16, 7], ids_of(T, 2, "mixed"), pad=pad, offset=offset)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    c.padding_untouched()


@pytest.mark.parametrize("dtype,T,K,N", [("bf16", 1100, 640, 384), ("f16", 1700, 250, 330), ("bf16", 2304, 2048, 2304)])
def test_long(dtype, T, K, N):
    """Several runs of tokens of one adapter, and the largest tiles."""
    c = Case(dtype, T, K, N, [16, 20, 8], [0 if t < 900 else (2 if t % 5 else -1) for t in range(T)])
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scale_dy", [1e-6, 1e3])
def test_gradients_of_any_size(dtype, scale_dy):
    """Gradients keep their relative accuracy where dy is far from 1 (float16's dz alone would not)."""
    if dtype == "f16" and scale_dy < 1e-5:
        scale_dy = 3e-5                                                  # dy itself is float16
    c = Case(dtype, 150, 128, 96, [8, 4], ids_of(150, 2, "blocks"), scale_x=0.1, scale_dy=scale_dy)
    c.forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("T", [40, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_is_not_finite_stays_with_its_request(T, dtype):
    """An adapter that holds infinities and NaN, and a token that does, spoil their own tokens and gradients and nobody else's."""
    c = Case(dtype, T, 128, 128, [8, 8, 8], ids_of(T, 3, "mixed"))
    c.adapters[1][0][3, 5] = float("nan")
    c.adapters[1][1][7, :] = float("inf")
    bad_token = int(c.tokens(2)[1])
    c.x[bad_token, 9] = float("inf")
    c.dy[bad_token, 9] = float("nan")
    c.forward()
    c.backward()
    good = (c.ids != 1).clone()
    good[bad_token] = False
    assert bool(torch.isfinite(c.y[good].float()).all()) and bool(torch.isfinite(c.dx[good].float()).all()) and bool(torch.isfinite(c.z[good].float()).all())
    assert not bool(torch.isfinite(c.y[c.ids == 1].float()).all(1).any())
    for g in c.grads[0]:
        assert bool(torch.isfinite(g).all())
    clean = Case(dtype, T, 128, 128, [8, 8, 8], ids_of(T, 3, "mixed"))
    clean.forward()
    clean.backward()
    assert torch.equal(clean.y[good], c.y[good]) and torch.equal(clean.dx[good], c.dx[good])
    assert torch.equal(clean.grads[0][0], c.grads[0][0]) and torch.equal(clean.grads[0][1], c.grads[0][1])


def test_no_tokens():
    c = Case("bf16", 0, 64, 96, [8, 4], [])
    c.forward()
    c.backward()
    for a, b in c.grads:
        assert not bool(a.any()) and not bool(b.any())


def test_without_dx_and_without_z():
    c = Case("bf16", 100, 64, 96, [8], [0] * 100)
    c.forward()
    y = P.condensa_adapter_project(c.x, c.w, c.table, c.ids)
    assert torch.equal(y["y"], c.y) and y["z"] is None
    out = P.condensa_adapter_project_backward(c.dy, c.x, c.w, c.table, c.ids, c.z, dx=False)
    assert out["dx"] is None
    c.backward()
    c.check_backward()


def test_gradients_against_differences():
    """<dL/dA, dA'> against (L(A + h dA') - L(A - h dA')) / 2h for L = <dy, y>, exact in h since y is linear in A and in B; the tolerance is
    what y's rounding to 16 bits can do to L, 2 u sum |dy| |y| / 2h, with steps as large as the parameters."""
    c = Case("f16", 90, 64, 48, [8, 4], ids_of(90, 2, "blocks"))
    c.forward()
    c.backward()
    grads = [(a.clone(), b.clone()) for a, b in c.grads]
    for a in range(2):
        for k in range(2):
            p = c.adapters[a][k]
            save, step = p.clone(), (torch.randn_like(p.float()) * p.float().std()).half()
            loss = []
            for sign in (1, -1):
                p.copy_((save.float() + sign * step.float()).half())
                c.forward()
                loss.append((c.dy.double() * c.y.double()).sum())
                moved = p.float() - save.float() if sign == 1 else moved - (p.float() - save.float())
                noise = 3 * c.u * (c.dy.double().abs() * (c.y.double().abs() + 1)).sum()
            p.copy_(save)
            want = (grads[a][k].double() * moved.double()).sum()
            assert abs(loss[0] - loss[1] - want) <= 2 * noise, (a, k)


@pytest.mark.parametrize("T", [5, 300])
def test_equal_calls_give_equal_bits_on_any_stream(T):
    c = Case("bf16", T, 256, 320, [16, 8], ids_of(T, 2, "mixed"))
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    keep = [t.clone() for t in (c.y, c.z, c.dx, *c.grads[0], *c.grads[1])]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.forward(stream=s)
    c.backward(stream=s)
    s.synchronize()
    for a, b in zip(keep, (c.y, c.z, c.dx, *c.grads[0], *c.grads[1])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [5, 300])
def test_graphs(T):
    """A captured forward and backward pass replays with new tokens, adapters and values, between eager calls."""
    c = Case("bf16", T, 128, 192, [16, 8], ids_of(T, 2, "mixed"))
    ws, wb = P.adapter_workspace(c.table, T), P.adapter_workspace(c.table, T, backward=True)
    c.forward(workspace=ws)
    z = c.z
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P.condensa_adapter_project(c.x, c.w, c.table, c.ids, y=c.y, z=z, workspace=ws)
        P.condensa_adapter_project_backward(c.dy, c.x, c.w, c.table, c.ids, z, dx=c.dx, workspace=wb)
    other = Case("bf16", 77, 64, 64, [4], [0] * 77, seed=5)
    for k in range(3):
        c.x.copy_(torch.randn(T, 128, device=DEV).bfloat16())
        c.dy.copy_(torch.randn(T, 192, device=DEV).bfloat16())
        c.ids.copy_(torch.tensor(ids_of(T, 2, ("blocks", "mixed", "none")[k]), dtype=torch.int32))
        c.adapters[0][0].mul_(-0.5)
        g.replay()
        torch.cuda.synchronize()
        c.z = z
        c.check_forward(f"replay {k}")
        c.check_backward(f"replay {k}")
        other.forward()
        other.check_forward()


def test_inputs_beyond_32_bits():
    """Rows of x, y and W further apart than 2^32 bytes in all."""
    T, K, N, far = 1100, 64, 72, 1 << 22
    c = Case("bf16", T, K, N, [8], [0] * T)
    x = torch.empty(T * far, device=DEV, dtype=torch.bfloat16).view(T, far)[:, :K]
    x.copy_(c.x)
    y = torch.empty(T * far, device=DEV, dtype=torch.bfloat16).view(T, far)[:, :N]
    c.x, c.y = x, y
    c.forward()
    c.check_forward()
    c.dy = y.clone()
    c.dx = torch.empty(T * far, device=DEV, dtype=torch.bfloat16).view(T, far)[:, :K]
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("T", [1, 2, 3, 4])
@pytest.mark.parametrize("K,N,ranks,pad", [(512, 2048, [8], 0), (1, 1, [1], 0), (7, 33, [5, 3], 3), (4609, 65, [2], 0), (520, 40, [250, 16], 8), (4608, 300, [16, 40], 0)])
def test_single_tokens(dtype, T, K, N, ranks, pad):
    """Decoding: a token or a few, with adapters of their own or without, of small and large A."""
    for ids in ([0] * T, [t % (len(ranks) + 1) - 1 for t in range(T)], [len(ranks) - 1 - t % len(ranks) for t in range(T)]):
        c = Case(dtype, T, K, N, ranks, ids, pad=pad)
        c.forward(z_width=max(ranks) + 3)
        c.check_forward(str(ids))
        y = P.condensa_adapter_project(c.x, c.w, c.table, c.ids)["y"]
        assert torch.equal(y, c.y)


@pytest.mark.parametrize("T", [64, 65, 66, 300])
@pytest.mark.parametrize("K,N", [(63, 72), (72, 65), (1, 1), (129, 7), (7, 129)])
def test_rows_of_odd_length(T, K, N):
    """Rows that no load of 16 bytes fits, on both sides of where they are copied, with rows of x and y apart and infinities next to them."""
    c = Case("bf16", T, K, N, [9, 33], ids_of(T, 2, "mixed"), pad=3)
    c.x._base.view(T * (K + 3) + 8)[: T * (K + 3)].view(T, K + 3)[:, K:].fill_(float("inf"))
    c.dy._base.view(T * (N + 3) + 8)[: T * (N + 3)].view(T, N + 3)[:, N:].fill_(float("nan"))
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


def test_long_runs_of_one_adapter():
    """Runs on both sides of one pass, of the length that is summed in parts, and an adapter without a token."""
    for T in (255, 256, 257, 1536, 1537, 2600):
        c = Case("f16", T, 130, 70, [20, 40, 3], [0] * (T - 5) + [2] * 5)
        c.forward()
        c.backward()
        c.check_backward(str(T))
        assert not bool(c.grads[1][0].any()) and not bool(c.grads[1][1].any())
