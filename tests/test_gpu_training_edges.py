"""Layer norms and distillation losses at the ends of their ranges, against the formulas in 64 bits."""
import math

import pytest
import torch

from rows_util import HALF, buffers, grad, put

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [9, 130, 257, 700, 1301, 3000, 5000, 9001])
def test_rows_of_one_large_value(cols, dtype):
    """A row of 2^67 alone has no variance; with an eps of 1e-37 its mean times rstd is beyond the largest float, and nothing of that reaches the gradients."""
    n, rows = 1, 3
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(n, [(cols, 1), (cols, 1)])
    gain, dy = torch.rand(n, cols, generator=gen) + 0.5, torch.randn(n, rows, cols, generator=gen).to(dtype)
    put(gb, 0, gain.unsqueeze(-1)), put(gb, 1, torch.zeros(n, cols, 1))
    x = torch.full((n, rows, cols), 2.0 ** 67, dtype=dtype, device="cuda")
    y, total, mean, rstd = gb.layer_norm(0, x, bias=1, eps=1e-37)
    assert not y.any() and bool((mean == 2.0 ** 67).all())
    dx = gb.layer_norm_backward(0, dy.cuda(), total, mean, rstd, bias=1).cpu().double()
    r = rstd.cpu().double().unsqueeze(-1)
    gdy = gain.double().unsqueeze(1) * dy.double()
    want = r * (gdy - gdy.mean(-1, keepdim=True))
    # the mean of cols products: as many additions, their roundings and the division; a difference and a product behind it
    off = U * r * ((cols + 4) * gdy.abs().mean(-1, keepdim=True) + 4 * gdy.abs())
    assert bool(((dx - want).abs() <= off + HALF[dtype] * (want.abs() + off)).all())
    assert not grad(gb, 0).any()
    gb.close()
