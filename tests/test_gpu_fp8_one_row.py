"""Products with matrices of a single row, whose stride says nothing: tolerances are those of test_gpu_project_fp8.py, and NaN codes follow the row in memory."""
import pytest
import torch

import paper_1911_02497_amd as P
from gpu_util import DEV
from test_gpu_project_fp8 import check, matrix, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("offset", [0, 3])
@pytest.mark.parametrize("n_in,n_out", [(650, 2600), (512, 650), (4608, 4090), (130, 129), (70, 1), (1, 70), (1, 1), (5000, 1999)])
def test_one_token_backward(n_in, n_out, offset, dtype):
    g = torch.Generator(DEV).manual_seed(n_in + n_out)
    w, dy = matrix(n_out, n_in, 128, g, -n_in % 128, 0, std=0.05), matrix(1, n_out, 1, g, 40, offset)
    dx = P.condensa_project_fp8_backward(dy, w, dtype=dtype)["dx"]
    check(dx, values(dy), values(w).t().contiguous(), dtype, -(-n_out // 128))
    y = P.condensa_project_fp8(matrix(1, n_in, 1, g, 40, offset), w, dtype=dtype)["y"]
    assert y.shape == (1, n_out) and bool(torch.isfinite(y).all())


@pytest.mark.parametrize("T", [1, 40, 100, 700])
@pytest.mark.parametrize("n_in", [1, 650, 2600])
def test_one_row_of_weights(T, n_in):
    g = torch.Generator(DEV).manual_seed(T + n_in)
    w, x, dy = matrix(1, n_in, 128, g, 40, 0), matrix(T, n_in, 1, g, -n_in % 16, 0), matrix(T, 1, 1, g, 15, 0)
    check(P.condensa_project_fp8(x, w, dtype=torch.bfloat16)["y"], values(x), values(w), torch.bfloat16, -(-n_in // 128))
    check(P.condensa_project_fp8_backward(dy, w, dtype=torch.bfloat16)["dx"], values(dy), values(w).t().contiguous(), torch.bfloat16, 1)


def test_an_aligned_row_is_not_copied():
    """One token's gradient in rows of 128 bytes: the product's parts and their sum, and no copy before them."""
    w = P.condensa_quantize_fp8_blocks(torch.randn(2600, 650, device=DEV), block_rows=128)
    dy = P.condensa_quantize_fp8_blocks(torch.randn(1, 2600, device=DEV))
    before = P.condensa_launch_count()
    P.condensa_project_fp8_backward(dy, w, dtype=torch.bfloat16)
    assert P.condensa_launch_count() - before == 2
