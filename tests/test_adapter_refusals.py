"""What the adapter entry points refuse, found before anything reaches a device: addresses here are never touched."""
import ctypes

import pytest

import paper_1911_02497_amd as P
from paper_1911_02497_amd import binding as B

NULL, SIZE, DENSITY, SHAPE, WORKSPACE, ARG = -1, -2, -3, -4, -5, -6
BASE, STEP = 1 << 40, 1 << 28


def adapter(at=0, rank=8, grads=False, **over):
    a = B.Adapter(BASE + at * 4 * STEP, BASE + (at * 4 + 1) * STEP, None, None, 1.0, rank)
    if grads:
        a.grad_a, a.grad_b = BASE + (at * 4 + 2) * STEP, BASE + (at * 4 + 3) * STEP
    for k, v in over.items():
        setattr(a, k, v)
    return a


def init(adapters, n=None, type_=B.TYPE_BF16, n_in=64, n_out=96, ws=BASE >> 1, size=1 << 20, out=True):
    arr = (B.Adapter * max(len(adapters), 1))(*adapters)
    lst = B.AdapterList()
    return P.library().condensa_adapter_list_init(arr if adapters else None, len(adapters) if n is None else n, type_, n_in, n_out, ws, size, None,
                                                  ctypes.byref(lst) if out else None)


@pytest.mark.parametrize("call,status", [
    (lambda: init([adapter()], out=False), NULL),
    (lambda: init([], n=1), NULL),
    (lambda: init([adapter()], n=-1), SIZE),
    (lambda: init([adapter()], n=16385), SIZE),
    (lambda: init([adapter()], type_=B.TYPE_F32), ARG),
    (lambda: init([adapter()], n_in=0), SHAPE),
    (lambda: init([adapter()], n_out=(1 << 20) + 1), SHAPE),
    (lambda: init([adapter()], ws=None), WORKSPACE),
    (lambda: init([adapter()], ws=(BASE >> 1) + 16), WORKSPACE),
    (lambda: init([adapter()], size=32), WORKSPACE),
    (lambda: init([adapter(rank=0)]), SHAPE),
    (lambda: init([adapter(rank=257)]), SHAPE),
    (lambda: init([adapter(a=None)]), NULL),
    (lambda: init([adapter(b=None)]), NULL),
    (lambda: init([adapter(grad_a=BASE * 2)]), NULL),
    (lambda: init([adapter(a=BASE + 1)]), ARG),
    (lambda: init([adapter(grads=True, grad_a=BASE * 2 + 2)]), ARG),
    (lambda: init([adapter(scale=float("inf"))]), DENSITY),
    (lambda: init([adapter(scale=float("nan"))]), DENSITY),
    (lambda: init([adapter(grads=True, grad_a=BASE + 64)]), ARG),                   # a gradient in A
    (lambda: init([adapter(grads=True), adapter(at=1, grads=True, grad_b=BASE + 3 * STEP + 400)]), ARG),
    (lambda: init([adapter()], ws=BASE), ARG),
])
def test_lists(call, status):
    assert call() == status


def the_list(**over):
    d = dict(table_dev=BASE >> 2, n_in=64, n_out=96, n_adapters=3, max_rank=8, type=B.TYPE_BF16, flags=7)
    d.update(over)
    return B.AdapterList(*[d[f] for f, _ in B.AdapterList._fields_])


def project(lst=None, **over):
    d = dict(x=BASE, ldx=64, T=100, w=BASE + STEP, ldw=64, ids=BASE + 2 * STEP, y=BASE + 3 * STEP, ldy=96, z=None, ldz=0, ws=BASE + 4 * STEP, size=1 << 27)
    d.update(over)
    lst = the_list() if lst is None else lst
    return P.library().condensa_adapter_project(ctypes.byref(lst) if lst else None, *d.values(), None)


def backward(lst=None, **over):
    d = dict(dy=BASE, lddy=96, x=BASE + STEP, ldx=64, T=100, w=BASE + 2 * STEP, ldw=64, ids=BASE + 3 * STEP, z=BASE + 4 * STEP, ldz=8, dx=BASE + 5 * STEP, lddx=64,
             ws=BASE + 6 * STEP, size=1 << 27)
    d.update(over)
    lst = the_list() if lst is None else lst
    return P.library().condensa_adapter_project_backward(ctypes.byref(lst) if lst else None, *d.values(), None)


@pytest.mark.parametrize("call", [project, backward])
@pytest.mark.parametrize("over,status", [
    (dict(T=-1), SIZE), (dict(T=(1 << 24) + 1), SIZE), (dict(x=None), NULL), (dict(w=None), NULL), (dict(ids=None), NULL),
    (dict(ldx=63), SHAPE), (dict(ldw=63), SHAPE), (dict(ldx=-64), SHAPE), (dict(ldx=1 << 40), SHAPE),
    (dict(x=BASE + 7 * STEP + 1), ARG), (dict(ids=BASE + 8 * STEP + 2), ARG),
    (dict(ws=None), WORKSPACE), (dict(ws=BASE + 9 * STEP + 128), WORKSPACE), (dict(size=128), WORKSPACE),
])
def test_shared_arguments(call, over, status):
    assert call(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(y=None), NULL), (dict(ldy=95), SHAPE), (dict(y=BASE + 3 * STEP + 1), ARG), (dict(z=BASE + 5 * STEP, ldz=7), SHAPE),
    (dict(y=BASE), ARG), (dict(y=BASE + 99 * 128 + 126), ARG), (dict(z=BASE + 3 * STEP + 64, ldz=8), ARG), (dict(ws=BASE + STEP), ARG),
    (dict(ws=BASE >> 2), ARG), (dict(y=BASE + 2 * STEP), ARG),
])
def test_forward(over, status):
    assert project(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(dy=None), NULL), (dict(z=None), NULL), (dict(lddy=95), SHAPE), (dict(ldz=7), SHAPE), (dict(lddx=63), SHAPE),
    (dict(dx=BASE), ARG), (dict(dx=BASE + STEP), ARG), (dict(dx=BASE + 4 * STEP), ARG), (dict(ws=BASE + 2 * STEP), ARG),
])
def test_backward(over, status):
    assert backward(**over) == status


@pytest.mark.parametrize("over,status", [
    (dict(table_dev=None), ARG), (dict(n_in=0), ARG), (dict(n_out=1 << 21), ARG), (dict(n_adapters=-1), ARG), (dict(max_rank=300), ARG), (dict(type=0), ARG),
])
def test_lists_that_are_none(over, status):
    assert project(the_list(**over)) == status and backward(the_list(**over)) == status
    assert P.library().condensa_adapter_workspace_bytes(ctypes.byref(the_list(**over)), 100, 0) == 0


def test_no_list_and_no_gradients():
    lib = P.library()
    assert lib.condensa_adapter_project(None, BASE, 64, 1, BASE, 64, BASE, BASE, 96, None, 0, BASE, 1 << 20, None) == NULL
    assert backward(the_list(flags=3)) == NULL                            # adapters without gradient buffers


def test_nothing_to_do():
    assert project(T=0, x=None, y=None, ids=None, ws=None, size=0) == 0
    assert backward(the_list(n_adapters=0, max_rank=0), T=0, ldz=0, x=None, dy=None, z=None, ids=None, ws=None, size=0) == 0


def test_workspace_sizes():
    lib, lst = P.library(), the_list()
    size = lambda T, back: lib.condensa_adapter_workspace_bytes(ctypes.byref(lst), T, back)  # noqa: E731
    for T in (0, 1, 64, 65, 1000, 1 << 24):
        for back in (0, 1):
            assert size(T, back) > 0 and size(T, back) % 256 == 0
    assert size(-1, 0) == 0 and size((1 << 24) + 1, 1) == 0
    assert lib.condensa_adapter_list_bytes(-1) == 0 and lib.condensa_adapter_list_bytes(16385) == 0 and lib.condensa_adapter_list_bytes(0) == 256
    assert ctypes.sizeof(B.Adapter) == 40 and ctypes.sizeof(B.AdapterList) == 40


def test_binding_checks():
    import torch
    a, b = torch.zeros(8, 64, dtype=torch.bfloat16), torch.zeros(96, 8, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        P.adapter_table([(a, b, 1.0)])                                    # not on a device
    with pytest.raises(TypeError):
        P.adapter_table([(a.float(), b.float(), 1.0)])
    with pytest.raises(TypeError):
        P.adapter_table([], n_in=64, n_out=64)


def test_grids_beyond_the_largest_launch():
    big = the_list(n_in=1 << 20, n_out=1 << 20)
    assert project(big, T=1 << 24, ldx=1 << 20, ldw=1 << 20, ldy=1 << 20, size=1 << 62) == SIZE
    assert backward(big, T=1 << 24, lddy=1 << 20, ldx=1 << 20, ldw=1 << 20, lddx=1 << 20, size=1 << 62) == SIZE
