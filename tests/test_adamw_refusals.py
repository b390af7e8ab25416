"""What the AdamW entry points refuse, found before anything reaches a device: addresses here are never touched."""
import ctypes

import pytest

import paper_1911_02497_amd as P
from paper_1911_02497_amd import binding as B

NULL, SIZE, DENSITY, WORKSPACE, ARG = -1, -2, -3, -5, -6
BASE = 1 << 40


def tensor(n=1000, at=0, bits=32, **over):
    t = B.AdamwTensor()
    for i, f in enumerate(("w", "grad", "exp_avg", "exp_avg_sq")):
        setattr(t, f, BASE + (at * 16 + i) * (1 << 24))
    if bits == 8:
        t.exp_avg_scale, t.exp_avg_sq_scale = BASE + (at * 16 + 4) * (1 << 24), BASE + (at * 16 + 5) * (1 << 24)
    t.n = n
    for k, v in over.items():
        setattr(t, k, v)
    return t


def init(tensors, bits=32, grad=B.TYPE_F32, code=B.TYPE_BF16, ws=BASE >> 1, size=1 << 20, n=None, out=True):
    arr = (B.AdamwTensor * max(len(tensors), 1))(*tensors)
    lst = B.AdamwList()
    return P.library().condensa_adamw_list_init(arr, len(tensors) if n is None else n, bits, grad, code, ws, size, None,
                                                ctypes.byref(lst) if out else None)


@pytest.mark.parametrize("call,status", [
    (lambda: init([tensor()], out=False), NULL),
    (lambda: init([tensor()], n=-1), SIZE),
    (lambda: init([tensor()], n=65537), SIZE),
    (lambda: init([tensor(n=(3 << 32) + 1)]), SIZE),
    (lambda: init([tensor(n=3 << 32, at=0), tensor(n=1, at=1)]), SIZE),
    (lambda: init([tensor()], bits=16), ARG),
    (lambda: init([tensor()], grad=3), ARG),
    (lambda: init([tensor()], code=B.TYPE_F32), ARG),
    (lambda: init([tensor()], ws=None), WORKSPACE),
    (lambda: init([tensor()], ws=(BASE >> 1) + 128), WORKSPACE),
    (lambda: init([tensor()], size=256), WORKSPACE),
    (lambda: init([tensor(w=None)]), NULL),
    (lambda: init([tensor(grad=None)]), NULL),
    (lambda: init([tensor(exp_avg=None)]), NULL),
    (lambda: init([tensor(exp_avg_sq=None)]), NULL),
    (lambda: init([tensor(theta=BASE << 1)]), NULL),
    (lambda: init([tensor(lambda_=BASE << 1)]), NULL),
    (lambda: init([tensor()], bits=8), NULL),
    (lambda: init([tensor(bits=8)], bits=32), ARG),
    (lambda: init([tensor(w=BASE + 2)]), ARG),
    (lambda: init([tensor(grad=BASE + (1 << 24) + 2)]), ARG),
    (lambda: init([tensor(grad=BASE + (1 << 24) + 1)], grad=B.TYPE_F16), ARG),
    (lambda: init([tensor(codes=BASE + (9 << 24) + 1)]), ARG),
    (lambda: init([tensor(grad=BASE)]), ARG),                                       # gradients in the weights
    (lambda: init([tensor(exp_avg=BASE + 3996)]), ARG),                             # states in the last weight
    (lambda: init([tensor(codes=BASE + (2 << 24) + 100)]), ARG),
    (lambda: init([tensor(), tensor(at=1, w=BASE + 400)]), ARG),                    # weights of two tensors
    (lambda: init([tensor()], ws=BASE + 256 * 4), ARG),
    (lambda: init([tensor(bits=8, exp_avg_scale=BASE + (2 << 24))], bits=8), ARG),
])
def test_lists(call, status):
    assert call() == status


def settings(**over):
    s = B.AdamwSettings(1e-3, 0.9, 0.999, 1e-8, 0.01, 0.0, B.ROUND_NEAREST, 1, 0, None, 0)
    for k, v in over.items():
        setattr(s, k, v)
    return s


@pytest.mark.parametrize("over,status", [
    (dict(step=0), ARG), (dict(step=-3), ARG), (dict(reserved=1), ARG), (dict(rounding=2), ARG), (dict(rounding=-1), ARG),
    (dict(rounding=1), ARG),                                             # states in 32 bits are not rounded by random bits
    (dict(lr=float("nan")), DENSITY), (dict(lr=float("inf")), DENSITY), (dict(beta1=1.0), DENSITY), (dict(beta1=-0.1), DENSITY),
    (dict(beta2=1.0), DENSITY), (dict(beta2=float("nan")), DENSITY), (dict(eps=-1e-8), DENSITY), (dict(eps=float("inf")), DENSITY),
    (dict(weight_decay=float("nan")), DENSITY), (dict(mu=-1.0), DENSITY), (dict(mu=float("inf")), DENSITY), (dict(grad_scale_dev=BASE + 2), ARG),
])
def test_settings(over, status):
    lst = B.AdamwList(BASE, BASE + 4096, 1000, 1, 1, 32, 0, 1)
    assert P.library().condensa_lc_adamw_step(ctypes.byref(lst), ctypes.byref(settings(**over)), None) == status


def test_lists_that_are_none():
    lib, s = P.library(), settings()
    assert lib.condensa_lc_adamw_step(None, ctypes.byref(s), None) == NULL
    assert lib.condensa_lc_adamw_step(ctypes.byref(B.AdamwList()), ctypes.byref(s), None) == NULL
    lst = B.AdamwList(BASE, BASE + 4096, 1000, 1, 1, 32, 0, 1)
    assert lib.condensa_lc_adamw_step(ctypes.byref(lst), None, None) == NULL
    for k, v in (("state_bits", 16), ("grad_type", 5), ("n_chunks", 1 << 40)):
        bad = B.AdamwList(BASE, BASE + 4096, 1000, 1, 1, 32, 0, 1)
        setattr(bad, k, v)
        assert lib.condensa_lc_adamw_step(ctypes.byref(bad), ctypes.byref(s), None) == ARG, k
    empty = B.AdamwList(BASE, BASE + 4096, 0, 0, 0, 32, 0, 1)
    assert lib.condensa_lc_adamw_step(ctypes.byref(empty), ctypes.byref(s), None) == 0          # nothing to do, nothing launched


def test_sizes_of_lists():
    lib = P.library()
    assert lib.condensa_adamw_list_bytes(None, 1) == 0 and lib.condensa_adamw_list_bytes(None, -1) == 0
    assert lib.condensa_adamw_list_bytes(None, 0) == 512
    arr = (B.AdamwTensor * 2)(tensor(n=8193), tensor(n=0))
    assert lib.condensa_adamw_list_bytes(arr, 2) == 512
    assert ctypes.sizeof(B.AdamwTensor) == 80 and ctypes.sizeof(B.AdamwList) == 48 and ctypes.sizeof(B.AdamwSettings) == 80


def test_binding_checks():
    import torch
    w = [torch.zeros(10)]
    with pytest.raises(TypeError):
        P.adamw_table(w, w, w, w)                                        # not on a device
    with pytest.raises(ValueError):
        P.adamw_table(w, [], w, w)
    with pytest.raises(ValueError):
        P.adamw_table(w, w, [torch.zeros(10, dtype=torch.uint8)], w)     # 8-bit states without scales
    with pytest.raises(TypeError):
        P.adamw_table(w, [w[0].double()], w, w)
