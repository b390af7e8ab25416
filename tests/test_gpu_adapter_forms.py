"""Every form of the wide product: tiles of 64 to 256 rows, rows at any address, more tokens than the parts of a split sum serve.

The rules that choose a form are in adapter.hip; beside each size stands the form that it takes.  A backward pass of (tokens, outputs, inputs) has the
wide product of the forward pass of (tokens, inputs, outputs), so both directions run each size."""
import pytest
import torch

from test_gpu_adapter import Case, ids_of

pytestmark = pytest.mark.gpu

# tokens, summed values, columns of the result, padding of rows
FORMS = {
    "256x256": (3330, 1032, 3528, 0),          # 14 x 14 tiles; neither rows, columns nor the sum are whole tiles
    "256x192": (3330, 1032, 5576, 0),          # 14 x 30
    "128x128, four steps": (1333, 648, 2600, 0),
    "128x128, four steps, copied rows": (1333, 650, 2600, 0),
    "128x128, two steps": (1333, 200, 4000, 0),
    "128x128, rows of 4 bytes": (3000, 200, 2816, 2),
    "64x64, eight steps": (300, 136, 1728, 0),
    "64x64, four steps": (300, 136, 4104, 0),
    "64x64, three steps": (600, 72, 4104, 0),
    "64x64, rows of 4 bytes": (300, 136, 1736, 2),
    "64x64, rows at any address": (300, 136, 1736, 1),
}


def both(form, dtype, ranks, how, check=True, **kw):
    """Cases whose forward (first) and backward pass (second) take the form."""
    T, n_sum, n_wide, pad = FORMS[form]
    ids = how if isinstance(how, list) else ids_of(T, len(ranks), how)
    cases = [Case(dtype, T, n_sum, n_wide, ranks, ids, pad=pad, **kw), Case(dtype, T, n_wide, n_sum, ranks, ids, pad=pad, **kw)]
    if check:
        for c, what in zip(cases, ("forward", "backward")):
            c.forward()
            c.check_forward(f"{form} {what}")
            c.backward()
            c.check_backward(f"{form} {what}")
            c.padding_untouched()
            del c
    return cases


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("how", ["mixed", "blocks"])
@pytest.mark.parametrize("form", list(FORMS))
def test_several_adapters_in_a_tile(form, how, dtype):
    both(form, dtype, [256, 130, 65, 64, 33, 16, 1], how)


@pytest.mark.parametrize("form", ["256x192", "128x128, two steps", "64x64, eight steps", "64x64, rows of 4 bytes"])
def test_forty_adapters(form):
    both(form, "bf16", [4] * 40, "mixed")


@pytest.mark.parametrize("how", ["none", "wild"])
@pytest.mark.parametrize("form", ["256x256", "128x128, four steps, copied rows", "64x64, three steps", "64x64, rows at any address"])
def test_tokens_without_an_adapter(form, how):
    both(form, "f16", [8, 24, 3], how)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("form", ["256x256", "256x192", "128x128, four steps", "64x64, eight steps", "64x64, rows of 4 bytes", "64x64, rows at any address"])
def test_what_is_not_finite_stays_with_its_request(form, dtype):
    """As the test of this name at fewer tokens: an adapter that holds infinities and NaN, and a token that does, spoil nobody else's."""
    ranks = [8, 8, 8]
    for c, clean in zip(both(form, dtype, ranks, "mixed", check=False), both(form, dtype, ranks, "mixed", check=False)):
        c.adapters[1][0][3, 5] = float("nan")
        c.adapters[1][1][7, :] = float("inf")
        bad = int(c.tokens(2)[1])
        c.x[bad, 9] = float("inf")
        c.dy[bad, 9] = float("nan")
        good = c.ids != 1
        good[bad] = False
        for case in (c, clean):
            case.forward()
            case.backward()
        assert not bool(torch.isfinite(c.y[c.ids == 1].float()).all(1).any())
        for got, want in ((c.y, clean.y), (c.dx, clean.dx), (c.z, clean.z)):
            assert bool(torch.isfinite(got[good].float()).all()) and torch.equal(got[good], want[good])
        for got, want in zip(c.grads[0], clean.grads[0]):
            assert bool(torch.isfinite(got).all()) and torch.equal(got, want)


@pytest.mark.parametrize("form", list(FORMS))
def test_equal_calls_give_equal_bits(form):
    for c in both(form, "bf16", [16, 40, 8], "mixed", check=False):
        c.forward()
        c.backward()
        keep = [t.clone() for t in (c.y, c.z, c.dx, *(g for pair in c.grads for g in pair))]
        for _ in range(3):
            c.y.zero_(), c.dx.zero_()
            c.forward()
            c.backward()
            for a, b in zip(keep, (c.y, c.z, c.dx, *(g for pair in c.grads for g in pair))):
                assert torch.equal(a, b)
