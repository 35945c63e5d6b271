"""Layer norms of rows of activations, forward and backward, against their formulas in 64 bits."""
import math

import pytest
import torch

from rows_util import HALF, buffers, grad, held, mask, put

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
SUM = 48     # roundings on the way of one element of a row into its sum: 16 in a lane, 6 across a wavefront, 16 across wavefronts, a few before and behind
COLS = [1, 2, 7, 8, 9, 31, 65, 128, 129, 256, 300, 513, 650, 1024, 1301, 2048, 2049, 5000, 8191, 8192, 8193, 16384]


def setup(n, cols, gen):
    gb = buffers(n, [(cols, 1), (cols, 1)])
    g, b = 1 + 0.3 * torch.randn(n, cols, 1, generator=gen), torch.randn(n, cols, 1, generator=gen)
    put(gb, 0, g), put(gb, 1, b)
    return gb, g.double().transpose(1, 2), b.double().transpose(1, 2)


def few(n, rows, ragged):
    return torch.tensor([rows * (i + 1) // (n + 1) if i else 0 for i in range(n)], dtype=torch.int32, device="cuda") if ragged else None


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", COLS)
def test_forward(cols, dtype):
    n, rows = 3, 5 if cols > 2000 else 19
    print("case", cols, dtype, flush=True)
    gen = torch.Generator().manual_seed(cols)
    gb, g, b = setup(n, cols, gen)
    for residual, ragged in ((False, False), (True, True)):
        x = (torch.randn(n, rows, cols, generator=gen) * 2 + 5 * torch.randn(n, rows, 1, generator=gen)).to(dtype)
        r = torch.randn(n, rows, cols, generator=gen).to(dtype) if residual else None
        counts = few(n, rows, ragged)
        there = mask(n, rows, counts)
        out = torch.full((n, rows, cols), 7.0, dtype=dtype, device="cuda")
        mean, rstd = (torch.full((n, rows), 7.0, device="cuda") for _ in range(2))
        y, total, m, s = gb.layer_norm(0, x.cuda(), bias=1, residual=None if r is None else r.cuda(), counts=counts, out=out, mean_out=mean, rstd_out=rstd)
        v = x.double() if r is None else (x.float() + r.float()).to(dtype).double()
        assert total.dtype == dtype and torch.equal(torch.where(there, total.cpu().double(), v), v)
        want_m = v.mean(-1, keepdim=True)
        d = v - want_m
        want_s = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-5)
        h = d * want_s
        want = h * g + b
        off_m = 2 * U * want_m.abs() + SUM * U * d.abs().mean(-1, keepdim=True)
        off_s = SUM * 2 * U        # of the squares' mean, halved by the root, and of the mean in them, which enters by its square
        assert bool(((m.cpu().double()[..., None] - want_m).abs() <= off_m)[there].all())
        assert bool(((s.cpu().double()[..., None] - want_s).abs() <= off_s * want_s)[there].all())
        off = g.abs() * want_s * (off_m + U * d.abs()) + (off_s + 4 * U) * (h * g).abs() + U * b.abs()
        assert bool(((y.cpu().double() - want).abs() <= off + HALF[dtype] * (want.abs() + off))[there.expand_as(want)].all())
        gone = ~there
        assert bool((y.cpu()[gone.expand_as(want)] == 7).all()) and bool((m.cpu()[gone[..., 0]] == 7).all()) and bool((s.cpu()[gone[..., 0]] == 7).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", COLS)
def test_backward(cols, dtype):
    n, rows = 3, 5 if cols > 2000 else 37
    print("case", cols, dtype, flush=True)
    gen = torch.Generator().manual_seed(cols + 1)
    gb, g, _ = setup(n, cols, gen)
    for residual, ragged, accumulate in ((False, False, False), (True, True, True)):
        v = (torch.randn(n, rows, cols, generator=gen) * 2 + 3 * torch.randn(n, rows, 1, generator=gen)).to(dtype)
        dy = torch.randn(n, rows, cols, generator=gen).to(dtype)
        r = torch.randn(n, rows, cols, generator=gen).to(dtype) if residual else None
        mean, rstd = v.double().mean(-1).float(), (1 / torch.sqrt(v.double().var(-1, unbiased=False) + 1e-5)).float()
        counts = few(n, rows, ragged)
        there = mask(n, rows, counts)
        before = [grad(gb, l).transpose(1, 2) for l in (0, 1)]
        out = torch.full((n, rows, cols), 7.0, dtype=dtype, device="cuda")
        dx = gb.layer_norm_backward(0, dy.cuda(), v.cuda(), mean.cuda(), rstd.cuda(), bias=1, residual=None if r is None else r.cuda(), counts=counts,
                                    accumulate=accumulate, out=out).cpu().double()
        s, u = rstd.double()[..., None], torch.where(there, dy.double(), 0.0)
        h = (v.double() - mean.double()[..., None]) * s
        gy = g * u
        m1, m2 = gy.mean(-1, keepdim=True), (gy * h).mean(-1, keepdim=True)
        want = s * (gy - m1 - h * m2) + (0 if r is None else r.double())
        off = s * (4 * U * gy.abs() + (SUM + 4) * U * gy.abs().mean(-1, keepdim=True) + h.abs() * (SUM + 12) * U * (gy * h).abs().mean(-1, keepdim=True))
        off = off + U * want.abs()
        assert bool(((dx - want).abs() <= off + HALF[dtype] * (want.abs() + off))[there.expand_as(want)].all())
        assert bool((dx[~there.expand_as(want)] == 7).all())
        for l, part in ((0, u * h), (1, u)):
            sum_ = part.sum(1, keepdim=True) + (before[l] if accumulate else 0)
            off = (rows + 12) * U * part.abs().sum(1, keepdim=True) + U * sum_.abs()
            assert bool(((grad(gb, l).transpose(1, 2) - sum_).abs() <= off).all())
    gb.close()


@pytest.mark.parametrize("n,rows,cols", [(2, 3000, 40), (3, 700, 650), (1, 2500, 2100)])
def test_many_rows_of_integers_sum_exactly(n, rows, cols):
    """Integers below 2^24: the bias's gradient has one right answer, and so has the gain's where h is +-1; twice the same bits, and added to itself twice that."""
    gen = torch.Generator().manual_seed(rows)
    gb = buffers(n, [(cols, 1), (cols, 1)])
    put(gb, 0, torch.ones(n, cols, 1))
    dy = torch.randint(-30, 31, (n, rows, cols), generator=gen).float()
    v = torch.randint(0, 2, (n, rows, cols), generator=gen).float() * 2 + 4            # 4 or 6: h = v - 5
    mean, rstd = torch.full((n, rows), 5.0).cuda(), torch.ones(n, rows).cuda()
    first = gb.layer_norm_backward(0, dy.cuda(), v.cuda(), mean, rstd, bias=1)
    dg, db = (dy.double() * (v.double() - 5)).sum(1)[..., None], dy.double().sum(1)[..., None]
    assert torch.equal(grad(gb, 0), dg) and torch.equal(grad(gb, 1), db)
    second = gb.layer_norm_backward(0, dy.cuda(), v.cuda(), mean, rstd, bias=1, accumulate=True)
    assert torch.equal(grad(gb, 0), 2 * dg) and torch.equal(grad(gb, 1), 2 * db) and torch.equal(first, second)
    gb.layer_norm_backward(0, dy.cuda(), v.cuda(), mean, rstd)                            # without a bias its gradient stays
    assert torch.equal(grad(gb, 0), dg) and torch.equal(grad(gb, 1), 2 * db)
    gb.g[0].fill_(3.0)
    third = gb.layer_norm_backward(0, dy.cuda(), v.cuda(), mean, rstd, bias=1, want_grads=False)
    assert torch.equal(first, third) and bool((gb.g[0] == 3).all())
    gb.layer_norm_backward(0, dy[:, :0].cuda(), v[:, :0].cuda(), mean[:, :0].contiguous(), rstd[:, :0].contiguous(), bias=1)
    assert not grad(gb, 0).any() and not grad(gb, 1).any()                               # no rows: nothing is added to zero
    gb.close()


def test_rows_far_from_zero():
    """A mean 2^14 times the spread: squares of the values themselves would have lost the variance."""
    n, rows, cols = 2, 9, 2048
    gen = torch.Generator().manual_seed(5)
    gb, g, b = setup(n, cols, gen)
    x = torch.randn(n, rows, cols, generator=gen) + 16384.0
    y, _, m, s = gb.layer_norm(0, x.cuda(), bias=1)
    v = x.double()
    d = v - v.mean(-1, keepdim=True)
    want_s = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-5)
    assert bool(((s.cpu().double()[..., None] - want_s).abs() <= 2 * SUM * U * want_s).all())
    off = g.abs() * want_s * (2 * U * 16384 + SUM * U * d.abs().mean(-1, keepdim=True)) + (2 * SUM + 6) * U * (d * want_s * g).abs() + 2 * U * b.abs() + 4 * U
    assert bool(((y.cpu().double() - (d * want_s * g + b)).abs() <= off).all())
    gb.close()


def test_in_place_strides_and_kept_results():
    n, rows, cols = 3, 11, 96
    gen = torch.Generator().manual_seed(6)
    gb, g, b = setup(n, cols, gen)
    x = torch.randn(n, rows, cols, generator=gen).cuda()
    want = gb.layer_norm(0, x, bias=1)[0].clone()
    wide = torch.full((rows, n, 2 * cols + 3), 9.0, device="cuda")
    view = wide[:, :, 1:cols + 1].transpose(0, 1)
    view.copy_(x)
    y, total, _, _ = gb.layer_norm(0, view, bias=1, out=view)
    assert torch.equal(y, want) and y.data_ptr() == view.data_ptr() and torch.equal(total, x)
    assert bool((wide[:, :, 0] == 9).all()) and bool((wide[:, :, cols + 1:] == 9).all())
    keep = gb.checkpoint(rows, cols)
    none, _, _, _ = gb.layer_norm(0, x, bias=1, keep=keep)
    assert none is None
    # what is kept is the 8-bit form of the result in float
    assert torch.equal(gb.checkpoint_load(keep, dtype=F32).cpu(), held(want.cpu())[0].float())
    one = torch.randn(1, 1, cols, generator=gen).cuda().expand(n, rows, cols)            # an input that repeats
    assert torch.equal(gb.layer_norm(0, one, bias=1)[0], gb.layer_norm(0, one.contiguous(), bias=1)[0])
    dy, mean, rstd = torch.randn(n, rows, cols, generator=gen).cuda(), torch.zeros(n, rows, device="cuda"), torch.ones(n, rows, device="cuda")
    apart = gb.layer_norm_backward(0, dy, x, mean, rstd, bias=1).clone()
    assert torch.equal(gb.layer_norm_backward(0, dy, x, mean, rstd, bias=1, out=dy), apart)
    gb.close()


def test_what_is_not_finite_stays_in_its_row():
    n, rows, cols = 2, 6, 70
    gen = torch.Generator().manual_seed(7)
    gb, g, b = setup(n, cols, gen)
    x = torch.randn(n, rows, cols, generator=gen)
    clean = gb.layer_norm(0, x.cuda(), bias=1)[0].cpu()
    x[0, 1, 3], x[1, 2, 69], x[1, 4] = math.nan, math.inf, 3.0
    y, _, m, s = (t.cpu() for t in gb.layer_norm(0, x.cuda(), bias=1))
    bad = torch.zeros(n, rows, dtype=torch.bool)
    bad[0, 1] = bad[1, 2] = True
    assert bool(y[bad].isnan().all()) and bool(s[bad].isnan().all())
    same = ~bad
    same[1, 4] = False
    assert torch.equal(y[same], clean[same])
    # a constant row: its bias, and no more than rounding of 1 / sqrt(eps)
    assert bool((y[1, 4].double() - b[1, 0]).abs().max() <= U * b[1, 0].abs().max()) and m[1, 4] == 3
    assert abs(float(s[1, 4]) * math.sqrt(1e-5) - 1) <= 8 * U
    gb.close()


def test_gradient_against_differences():
    n, rows, cols = 1, 2, 10
    gen = torch.Generator().manual_seed(8)
    gb, g, b = setup(n, cols, gen)
    x, dy = torch.randn(n, rows, cols, generator=gen), torch.randn(n, rows, cols, generator=gen)
    _, total, mean, rstd = gb.layer_norm(0, x.cuda(), bias=1)
    dx = gb.layer_norm_backward(0, dy.cuda(), total, mean, rstd, bias=1).cpu().double()

    def loss(v, gain, bias):
        return (torch.nn.functional.layer_norm(v, (cols,), eps=1e-5) * gain + bias).mul(dy.double()).sum()

    def differences(args, k):
        out = torch.zeros_like(args[k])
        for i in range(out.numel()):
            moved = []
            for step in (1e-4, -1e-4):
                now = [t.clone() for t in args]
                now[k].view(-1)[i] += step
                moved.append(loss(*now))
            out.view(-1)[i] = (moved[0] - moved[1]) / 2e-4
        return out
    args = [x.double(), g, b]
    # central differences: the third derivative, some tens here, times 1e-8 / 6; and some hundreds of float roundings of terms of a few units
    for got, k in ((dx, 0), (grad(gb, 0).transpose(1, 2), 1), (grad(gb, 1).transpose(1, 2), 2)):
        assert bool(((got - differences(args, k)).abs() <= 1e-6 + 400 * U).all())
    gb.close()
