"""Layer norms and distillation losses at the ends of their ranges, against the formulas in 64 bits."""
import math
from decimal import Decimal, localcontext

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


def divergences(t, z, u):
    """sum p log(p / q) of every row in 40 digits: at u = 2^20 it is 10^-12 and less, of logarithms that 64 bits hold to 10^-16."""
    with localcontext() as ctx:
        ctx.prec = 40

        def one(t, z):
            t, z = ([Decimal(v) / Decimal(u) for v in row] for row in (t, z))
            a, b = [v.exp() for v in t], [v.exp() for v in z]
            return float(sum(p * (v - w) for p, v, w in zip(a, t, z)) / sum(a) - sum(a).ln() + sum(b).ln())
        return torch.tensor([[[one(*rows)] for rows in zip(*pair)] for pair in zip(t.tolist(), z.tolist())], dtype=torch.float64)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("labelled", [False, True])
@pytest.mark.parametrize("temperature", [4.0, 30.0, 1000.0, 2.0 ** 20])
@pytest.mark.parametrize("rows,cols", [(40, 3), (7, 10), (5, 128), (3, 300), (3, 513), (2, 1024)])
def test_a_teacher_of_all_classes(rows, cols, temperature, labelled, dtype):
    """Softmaxes at a high temperature lie within 1 / temperature of each other; the loss is the square of that, times the temperature's square."""
    print("case", rows, cols, temperature, labelled, dtype, flush=True)
    n, u, hard, soft = 2, temperature, 0.5, 0.75
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(n, [(4, 4)])
    z = (2 * torch.randn(n, rows, cols, generator=gen)).to(dtype)
    index = torch.rand(n, rows, cols, generator=gen).argsort(-1).int()
    teacher = 2 * torch.randn(n, rows, cols, generator=gen)
    labels = torch.randint(0, cols, (n, rows), generator=gen, dtype=torch.int32) if labelled else None
    weights = torch.rand(n, rows, generator=gen) + 0.5
    loss, dz = gb.distill(z.cuda(), index.cuda(), teacher.cuda(), None if labels is None else labels.cuda(), temperature=u, hard=hard, soft=soft,
                          weights=weights.cuda())
    gb.close()
    z, w = z.double(), weights.double().unsqueeze(-1)
    t = torch.zeros_like(z).scatter_(-1, index.long(), teacher.double())
    zd, td = z - z.amax(-1, keepdim=True), t - t.amax(-1, keepdim=True)
    d = (zd - td) / u
    p = torch.softmax(t / u, -1)
    m = (p * d).sum(-1, keepdim=True)
    x, kl = d - m, divergences(t, z, u)
    f = torch.expm1(x) - x                                                       # kl = log(1 + sum p f)
    off_p = U * (cols + 4 * td.abs() / u + 20)                                   # relative: exponential, sum, quotient
    off_d = U * ((zd.abs() + td.abs()) / u + 2 * d.abs())
    off_x = off_d + U * x.abs() + (p * (off_d + d.abs() * (off_p + (cols + 4) * U))).sum(-1, keepdim=True)
    off_kl = (p * (torch.expm1(x).abs() * off_x + f * (off_p + (cols + 20) * U))).sum(-1, keepdim=True) + 6 * U * kl
    want_l, off_l = w * soft * u * u * kl, w * soft * u * u * off_kl
    y = x - kl
    want, off = w * soft * u * p * torch.expm1(y), w * soft * u * p * (torch.expm1(y).abs() * (off_p + 8 * U) + torch.exp(y) * (off_x + off_kl + U * y.abs()))
    if labelled:
        at = labels.long().unsqueeze(-1)
        s, log_s = torch.softmax(z, -1), torch.log_softmax(z, -1)
        want_l = want_l - w * hard * log_s.gather(-1, at)
        off_l = off_l + w * hard * U * (cols + 40 + 8 * zd.abs().amax(-1, keepdim=True))
        want = want + w * hard * s.scatter_add(-1, at, -torch.ones_like(w))
        off = off + w * hard * s * U * (cols + 40 + 4 * zd.abs()) + torch.zeros_like(z).scatter_(-1, at, 4 * U * w * hard)
    loss, dz = loss.cpu().double().unsqueeze(-1), dz.cpu().double()
    assert bool(((loss - want_l).abs() <= off_l + 4 * U * want_l.abs()).all()), float(((loss - want_l).abs() / want_l.abs()).max())
    off = off + 4 * U * want.abs()
    assert bool(((dz - want).abs() <= off + HALF[dtype] * (want.abs() + off)).all()), float((dz - want).abs().max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [2, 10, 128, 300, 1000])
def test_a_teacher_of_all_classes_that_is_sure(cols, dtype):
    """Weights that round to 0 have no logarithm and their classes still count in the student's; distances beyond the series; classes the student rules out."""
    from test_gpu_distill import check, inputs
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(2, [(4, 4)])
    z, labels, index, teacher, weights = inputs(gen, 2, 6, cols, cols, dtype)
    teacher[0, 0, 0] = teacher[0, 1, : cols // 2] = -1e4                            # weights of 0
    teacher[0, 2] *= 50                                                           # far from the student
    z[0, 3] *= 60
    teacher[0, 4], z[0, 4] = 0.0, 0.0                                             # alike: no loss
    labels[0, 5] = -1
    for temperature, hard in ((2.0, 0.5), (7.0, 0.0), (100.0, 0.5)):
        loss, dz = check(gb, z, labels, index, teacher, weights, temperature, hard, 0.75)
        assert hard or loss[0, 4] == 0 and not dz[0, 4].any()
    z[1, 0, 0] = -math.inf                                                        # but not by the teacher
    loss, dz = gb.distill(z.cuda(), index.cuda(), teacher.cuda(), temperature=4.0)
    gb.close()
    assert loss[1, 0] == math.inf and bool(loss[1, 1:].isfinite().all()) and bool(dz.isfinite().all())
