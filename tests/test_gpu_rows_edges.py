"""The operators on rows of activations at the edges of what they take: several tables and streams, values that are not finite or the largest
finite ones, rows that do not exist, results in the place of inputs, and the kernels of large products with all they fuse."""
import math

import pytest
import torch

from paper_2008_01425_amd import binding as B
from rows_util import HALF, act, buffers, grad, held, mask, product_error, put, slope

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def integers(gen, shape, top):
    return torch.randint(-top, top + 1, shape, generator=gen).double()


def test_two_sets_of_buffers_on_two_streams():
    """A call with other buffers on another stream, while calls on the first ones still wait on theirs: each writes to and reads from its own."""
    n, rows, p, q = 3, 60, 40, 50
    gen = torch.Generator().manual_seed(21)
    gb = buffers(n, [(p, q), (p, 1)])
    w, x, dz = integers(gen, (n, p, q), 3), integers(gen, (n, rows, q), 4), integers(gen, (n, rows, p), 3)
    put(gb, 0, w)
    xd, dzd = x.float().cuda(), dz.float().cuda()
    one = (gb.x, gb.ptrs, gb.g, gb.gptrs)
    two = ([2 * t for t in gb.x], None, [torch.zeros_like(t) for t in gb.g], None)
    two = (two[0], [t.data_ptr() for t in two[0]], two[2], [t.data_ptr() for t in two[2]])

    def take(buffers):
        gb.x, gb.ptrs, gb.g, gb.gptrs = buffers
    side = torch.cuda.Stream()
    for first, second in ((one, two), (two, one)):
        for g in one[2] + two[2]:
            g.fill_(7.0)
        take(first)
        gb.linear_backward(0, dzd, xd, bias=1)              # the first set's tables
        for g in first[2]:
            g.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)                  # some 50 ms
            y1 = gb.linear(0, xd)
            dx1 = gb.linear_backward(0, dzd, xd, bias=1)
        take(second)
        y2 = gb.linear(0, xd)
        dx2 = gb.linear_backward(0, 2 * dzd, xd, bias=1)
        torch.cuda.synchronize()
        f1, f2 = (1, 2) if first is one else (2, 1)
        assert torch.equal(y1.cpu().double(), f1 * (x @ w.transpose(1, 2))) and torch.equal(y2.cpu().double(), f2 * (x @ w.transpose(1, 2)))
        assert torch.equal(dx1.cpu().double(), f1 * (dz @ w)) and torch.equal(dx2.cpu().double(), 2 * f2 * (dz @ w))
        dw = dz.transpose(1, 2) @ x
        take(first)
        assert torch.equal(grad(gb, 0), dw)
        take(second)
        assert torch.equal(grad(gb, 0), 2 * dw)
    take(one)
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
def test_what_is_not_finite_in_a_checkpoint_comes_back_through_the_activation(name, dtype):
    """A checkpoint holds infinities as NaN; the slope there is NaN, so a gradient that went through such a value is NaN and no other one."""
    n, rows, p, q = 2, 40, 33, 70
    gen = torch.Generator().manual_seed(9)
    gb = buffers(n, [(p, q), (p, 1)])
    w, z = integers(gen, (n, p, q), 3), integers(gen, (n, rows, q), 4)
    put(gb, 0, w)
    z[0, 3, 5], z[0, 3, 6], z[1, 39, 69], z[1, 0, 0] = math.nan, math.inf, -math.inf, math.nan
    odd = ~torch.isfinite(z)
    z8 = gb.checkpoint_store(z.float().cuda())
    dz, dy = integers(gen, (n, rows, p), 3), integers(gen, (n, rows, q), 3)
    dy[0, 3, 6] = 0.0
    got = gb.activation_backward(name, dy.to(dtype).cuda(), z8).cpu()
    assert torch.equal(torch.isnan(got), odd) and bool(torch.isfinite(got[~odd]).all())
    got = gb.linear_backward(0, dz.to(dtype).cuda(), torch.zeros(n, rows, q, dtype=dtype, device="cuda"), bias=1, act=name, z=z8).cpu()
    assert torch.equal(torch.isnan(got), odd) and bool(torch.isfinite(got[~odd]).all())
    if name == "relu":
        want = torch.where(z > 0, dz @ w, 0.0).float().to(dtype)
        assert torch.equal(got[~odd], want[~odd])
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_norm_in_place_returns_the_sum_it_was_taken_of(dtype):
    n, rows, cols = 2, 9, 70
    gen = torch.Generator().manual_seed(12)
    gb = buffers(n, [(cols, 1)])
    put(gb, 0, torch.randn(n, cols, 1, generator=gen))
    x = torch.randn(n, rows, cols, generator=gen).to(dtype).cuda()
    dy = torch.randn(n, rows, cols, generator=gen).to(dtype).cuda()
    y, total, rstd = gb.norm(0, x)
    want = gb.norm_backward(0, dy, total, rstd)
    there = x.clone()
    y2, total2, rstd2 = gb.norm(0, there, out=there)
    assert y2 is there and torch.equal(y2, y) and torch.equal(rstd, rstd2)
    assert torch.equal(total2, x)
    assert torch.equal(gb.norm_backward(0, dy, total2, rstd2), want)
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_do_not_exist_are_zero_in_what_is_allocated(dtype):
    """A checkpoint stored with counts and read back, or multiplied, without."""
    n, rows, p, q = 3, 50, 20, 70
    gen = torch.Generator().manual_seed(11)
    gb = buffers(n, [(p, q), (p, 1)])
    w, x = integers(gen, (n, p, q), 2), integers(gen, (n, rows, q), 4)
    put(gb, 0, w)
    junk = [torch.full((1 << 14,), 255, dtype=torch.uint8, device="cuda") for _ in range(8)]
    del junk                                                    # what an allocation may find
    counts = torch.tensor([0, 17, 50], dtype=torch.int32, device="cuda")
    kept = gb.checkpoint_store(x.to(dtype).cuda(), counts=counts)
    there = mask(n, rows, counts)
    x = torch.where(there, x, 0.0)
    assert torch.equal(gb.checkpoint_load(kept, dtype=F32).cpu().double(), x)
    assert torch.equal(gb.linear(0, kept, dtype=dtype).cpu(), (x @ w.transpose(1, 2)).float().to(dtype))
    gb.close()


def test_the_largest_floats_go_through_a_product():
    """Times one, in either operand of every product: their pieces never sum to more than they are."""
    most = torch.finfo(F32).max
    v = torch.tensor([[most, -most, 1.0, most * 0.9995], [most * 0.998, 3.0, -most * 0.9999, 0.0], [2.0, 0.0, 0.0, -most * 0.996]], dtype=torch.float64).float()
    one = torch.eye(4)[None]
    gb = buffers(1, [(4, 4), (4, 1), (3, 4), (3, 1)])
    put(gb, 0, one)
    assert torch.equal(gb.linear(0, v[None].cuda()).cpu()[0], v)                           # as rows of a forward product
    dx = gb.linear_backward(0, v[None].cuda(), torch.eye(3, 4)[None].cuda(), bias=1)
    assert torch.equal(dx.cpu()[0], v)                                                     # of an input gradient
    assert torch.equal(grad(gb, 0)[0, :, :3].float(), v.t())                               # of a weight gradient
    put(gb, 2, v[None])
    assert torch.equal(gb.linear(2, one.cuda()).cpu()[0], v.t())                           # as weights
    dx = gb.linear_backward(2, torch.eye(3)[None].cuda(), v[None].cuda(), bias=3)
    assert torch.equal(dx.cpu()[0], v) and torch.equal(grad(gb, 2)[0].float(), v)          # ... and as the weight gradient's input
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_the_largest_finite_values_in_a_checkpoint(dtype):
    """From 248 * 2^120 on the nearest e4m3 value is 256 * 2^120 = 2^128, which no float holds: whatever reads it reads an infinity."""
    most = torch.finfo(dtype).max
    border = 248.0 * 2.0 ** 120
    x = torch.tensor([most, -most, border, -border, 247.0 * 2.0 ** 120, 2.0 ** 127, -2.0 ** 120, math.inf, math.nan, 1.0], dtype=torch.float64)
    x = x.to(dtype).view(1, 10, 1)
    want = held(x)[0].float()
    assert torch.equal(torch.isinf(want[0, :4]), torch.ones(4, 1, dtype=torch.bool)) and bool(torch.isfinite(want[0, 4:7]).all())
    gb = buffers(1, [(1, 1), (1, 1)])
    put(gb, 0, torch.ones(1, 1, 1))
    kept = gb.checkpoint_store(x.cuda())
    same = lambda a, b: torch.equal(a.cpu().float().nan_to_num(nan=7.0, posinf=8.0, neginf=9.0), b.nan_to_num(nan=7.0, posinf=8.0, neginf=9.0))  # noqa: E731
    assert same(gb.checkpoint_load(kept, dtype=F32), want) and same(gb.checkpoint_load(kept), want)
    assert same(gb.linear(0, kept, dtype=dtype), want)                          # as a product takes them
    for sign in (1.0, -1.0):                                                    # ... and as a weight gradient does
        two = gb.checkpoint_store(sign * x[:, :4:2].abs().contiguous().cuda())
        gb.linear_backward(0, torch.ones(1, 2, 1, dtype=dtype, device="cuda"), two, bias=1, want_dx=False)
        assert float(grad(gb, 0)) == sign * math.inf
    keep = gb.checkpoint(10, 1)
    gb.linear(0, x.cuda(), keep=keep)                                           # as a product leaves them
    assert same(gb.checkpoint_load(keep, dtype=F32), want)
    got = gb.activation_backward("relu", torch.ones(1, 10, 1, dtype=dtype, device="cuda"), kept)
    assert same(got, torch.where(torch.isnan(want), math.nan, (want > 0).float()))
    gb.close()


@pytest.mark.parametrize("cols", [5, 33, 650, 1041])
def test_padding_of_a_kept_norm_is_zero_also_where_its_row_is_not_a_number(cols):
    n, rows = 2, 4
    gb = buffers(n, [(cols, 1)])
    put(gb, 0, torch.ones(n, cols, 1))
    x = torch.ones(n, rows, cols)
    x[0, 1, 3], x[1, 2, cols - 1], x[1, 3, 0] = math.nan, math.inf, math.nan
    keep = gb.checkpoint(rows, cols)
    keep.data.fill_(255)
    gb.norm(0, x.cuda(), keep=keep)
    pitch = (cols + 31) // 32 * 32
    codes = keep.data[:n * rows * pitch].cpu().view(n, rows, pitch)
    assert bool((codes[..., cols:] == 0).all())
    assert bool(torch.isnan(gb.checkpoint_load(keep)[0, 1]).all())
    gb.close()


def test_no_rows_leave_accumulated_gradients_bit_for_bit():
    gb = buffers(2, [(6, 5), (6, 1), (5, 1)])
    for g in gb.g:
        g.fill_(-0.0)
    none = lambda c: torch.zeros(2, 0, c, device="cuda")  # noqa: E731
    gb.linear_backward(0, none(6), none(5), bias=1, accumulate=True)
    gb.norm_backward(2, none(5), none(5), torch.zeros(2, 0, device="cuda"), accumulate=True)
    assert all(bool((torch.signbit(g)).all()) for g in gb.g)
    gb.close()


def test_types_that_do_not_agree_are_refused():
    gb = buffers(2, [(6, 5), (6, 1)])
    x = torch.zeros(2, 4, 5, device="cuda")
    kept = gb.checkpoint_store(x)
    with pytest.raises(ValueError):
        gb.linear(0, x, dtype=BF16)
    with pytest.raises(ValueError):
        gb.linear(0, kept, dtype=BF16, out=torch.zeros(2, 4, 6, device="cuda"))
    with pytest.raises(TypeError):
        gb.linear(0, kept, dtype=torch.float16)
    with pytest.raises(TypeError):
        gb.checkpoint_load(kept, out=torch.zeros(2, 4, 5, device="cuda", dtype=torch.float16))
    with pytest.raises(ValueError):
        gb.checkpoint_load(kept, dtype=BF16, out=torch.zeros(2, 4, 5, device="cuda"))
    assert gb.linear(0, x, dtype=F32).dtype == F32 and gb.linear(0, kept).dtype == BF16 and gb.linear(0, kept, dtype=F32).dtype == F32
    assert gb.linear(0, kept, out=torch.zeros(2, 4, 6, device="cuda")).dtype == F32
    assert gb.checkpoint_load(kept).dtype == BF16 and gb.checkpoint_load(kept, out=torch.zeros(2, 4, 5, device="cuda")).dtype == F32
    gb.close()


def test_more_workers_than_one_side_of_a_grid():
    """70 000 workers, a gain of 40 entries each."""
    from paper_2008_01425_amd.device import GossipBuffers
    n, rows, cols = 70000, 2, 40
    gb = GossipBuffers(n, [], [], [(cols, 1)], 1, 1)
    gen = torch.Generator().manual_seed(31)
    g = integers(gen, (n, cols), 3)
    x, dy = integers(gen, (n, rows, cols), 3), integers(gen, (n, rows, cols), 3)
    params, grads = torch.zeros(n, gb.N, device="cuda"), torch.full((n, gb.N), 7.0, device="cuda")
    gb.ptrs, gb.gptrs = ([t.data_ptr() for t in buf] for buf in (params, grads))
    gb.layer_of(params, 0)[:, :, 0] = g.float().cuda()
    one = torch.ones(n, rows, device="cuda")
    dx = gb.norm_backward(0, dy.float().cuda(), x.float().cuda(), one)
    assert torch.equal(gb.layer_of(grads, 0)[:, :, 0].cpu().double(), (dy * x).sum(1))
    want = g[:, None] * dy - x * (g[:, None] * dy * x).mean(-1, keepdim=True)
    # a mean of integers, a product and a difference: three roundings
    assert bool(((dx.cpu().double() - want).abs() <= 3 * 2.0 ** -24 * (want.abs() + (g[:, None] * dy).abs() + x.abs() * (g[:, None] * dy * x).mean(-1, keepdim=True).abs())).all())
    y, _, rstd = gb.norm(0, x.float().cuda(), eps=1.0)
    want = 1 / torch.sqrt(x.square().mean(-1) + 1.0)
    assert bool(((rstd.cpu().double() - want).abs() <= 4 * 2.0 ** -23 * want).all())
    gb.close()


@pytest.mark.parametrize("e", [-100, -110, -118, -126, -134, -141])
def test_products_of_the_smallest_floats(e):
    """Operands around 2^e, times others that bring the sums back into the middle of the range.  A float below 2^-110 enters to 2^-134, half a step of
    the smallest bf16 values; all else costs what it costs elsewhere."""
    n, rows, p, q = 2, 70, 66, 130
    gen = torch.Generator().manual_seed(200 - e)
    gb = buffers(n, [(p, q), (p, 1)])

    def small(*shape):
        return ((torch.rand(*shape, generator=gen).double() + 1) * torch.randn(*shape, generator=gen).sign() * 2.0 ** e).float()

    def large(*shape):
        return (torch.randn(*shape, generator=gen).double() * 2.0 ** 90).float()

    def near(got, a, b, lost_a, lost_b):
        a, b = a.double(), b.double()
        off = product_error(a, b, F32)
        off = off + 2.0 ** -134 * (lost_a * b.abs().sum(1, keepdim=True) + lost_b * a.abs().sum(2, keepdim=True))
        want = a @ b
        assert bool(((got.cpu().double() - want).abs() <= off + HALF[F32] * (want.abs() + off) + 2.0 ** -140).all())
    w, x, dz = small(n, p, q), large(n, rows, q), large(n, rows, p)
    put(gb, 0, w)
    near(gb.linear(0, x.cuda()), x, w.transpose(1, 2), 0, 1)
    near(gb.linear_backward(0, dz.cuda(), small(n, rows, q).cuda(), bias=1), dz, w, 0, 1)
    w, x, dz = large(n, p, q), small(n, rows, q), small(n, rows, p)
    put(gb, 0, w)
    near(gb.linear(0, x.cuda()), x, w.transpose(1, 2), 1, 0)
    x = large(n, rows, q)
    near(gb.linear_backward(0, dz.cuda(), x.cuda(), bias=1), dz, w, 1, 0)
    near(grad(gb, 0), dz.transpose(1, 2), x, 1, 0)
    gb.close()


def some(n, rows, ragged):
    """Counts: none, or counts that end inside tiles, steps and splits; with several workers one of them has no rows, or says more than there are, or fewer than none."""
    if not ragged:
        return None
    of = {1: [rows * 2 // 3 + 1], 2: [min(37, rows), rows - rows // 9], 3: [-3, 1, rows + 5]}
    counts = of.get(n) or [(-2, rows // 2 + 1, rows, min(3, rows), 2 * rows + 7, 0, rows // 3 + 1)[i % 7] for i in range(n)]
    assert sum(min(max(k, 0), rows) for k in counts) > 0
    return torch.tensor(counts, dtype=torch.int32, device="cuda")


def check_fused(n, rows, p, q, dtype, kept, ragged):
    """Integers and relu: one right answer for the result, for what is kept and for every gradient, with all that the products fuse."""
    print("case", n, rows, p, q, dtype, kept, ragged, flush=True)
    gen = torch.Generator().manual_seed(n * 1000 + rows + p + q)
    gb = buffers(n, [(p, q), (p, 1)])
    w, b = integers(gen, (n, p, q), 2), integers(gen, (n, p, 1), 50)
    x, dz, z = integers(gen, (n, rows, q), 4), integers(gen, (n, rows, p), 3), integers(gen, (n, rows, q), 4)
    r, rx = integers(gen, (n, rows, p), 9), integers(gen, (n, rows, q), 9)
    put(gb, 0, w), put(gb, 1, b)
    counts = some(n, rows, ragged)
    there = mask(n, rows, counts)
    given = gb.checkpoint_store(x.to(dtype).cuda()) if kept else x.to(dtype).cuda()
    keep = gb.checkpoint(rows, p)
    keep.data.fill_(77)
    out = torch.full((n, rows, p), 7.0, dtype=dtype, device="cuda")
    y = gb.linear(0, given, bias=1, act="relu", residual=r.to(dtype).cuda(), keep=keep, counts=counts, out=out)
    sums = x @ w.transpose(1, 2) + b.transpose(1, 2)
    assert torch.equal(y.cpu(), torch.where(there, sums.clamp(min=0) + r, 7.0).float().to(dtype))
    back = torch.full((n, rows, p), 7.0, device="cuda")
    gb.checkpoint_load(keep, counts=counts, out=back)
    assert torch.equal(back.cpu(), torch.where(there, held(sums)[0], 7.0).float())
    pitch = (p + 31) // 32 * 32
    codes = keep.data[:n * rows * pitch].cpu().view(n, rows, pitch)
    assert bool((codes[~there.expand(n, rows, pitch)] == 77).all()) and bool((codes[..., p:][there.expand(n, rows, pitch - p)] == 0).all())
    z8, dzd = gb.checkpoint_store(z.float().cuda()), dz.to(dtype).cuda()
    for g in gb.g:
        g.fill_(7.0)
    dx = torch.full((n, rows, q), 7.0, dtype=dtype, device="cuda")
    gb.linear_backward(0, dzd, bias=1, act="relu", z=z8, residual=rx.to(dtype).cuda(), want_grads=False, counts=counts, out=dx)
    assert all(bool((g == 7.0).all()) for g in gb.g)                         # dX alone
    want = torch.where(there, (dz @ w) * (z > 0) + rx, 7.0).float().to(dtype)
    assert torch.equal(dx.cpu(), want)
    dx.fill_(7.0)
    gb.linear_backward(0, dzd, given, bias=1, act="relu", z=z8, residual=rx.to(dtype).cuda(), counts=counts, out=dx)
    assert torch.equal(dx.cpu(), want)
    dz0 = torch.where(there, dz, 0.0)
    dw, db = dz0.transpose(1, 2) @ x, dz0.sum(1)[..., None]
    assert torch.equal(grad(gb, 0), dw) and torch.equal(grad(gb, 1), db)
    gb.linear_backward(0, dzd, given, accumulate=True, want_dx=False, counts=counts)
    assert torch.equal(grad(gb, 0), 2 * dw) and torch.equal(grad(gb, 1), db)
    gb.close()


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype,kept", [(F32, False), (F32, True), (BF16, False), (BF16, True)])
@pytest.mark.parametrize("n,rows,p,q", [(1, 1, 1, 1), (1, 2, 64, 32), (3, 5, 33, 65), (2, 40, 129, 127), (1, 300, 257, 96), (2, 257, 384, 31), (17, 9, 40, 70),
                                        (40, 70, 34, 50)])
def test_fused_products_of_integers_are_exact(n, rows, p, q, dtype, kept, ragged):
    check_fused(n, rows, p, q, dtype, kept, ragged)


@pytest.mark.parametrize("splits", [1, 4])
@pytest.mark.parametrize("tile", [32, 64, 128, 256])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype,kept", [(F32, False), (F32, True), (BF16, False), (BF16, True)])
@pytest.mark.parametrize("n,rows,p,q", [(1, 515, 131, 258), (2, 515, 270, 520), (3, 70, 520, 140)])
def test_fused_products_on_every_tile(n, rows, p, q, dtype, kept, ragged, tile, splits):
    """Every tile forced, its steps split or not: a count inside the first of the weight gradient's splits leaves the later ones empty."""
    from parity_util import env_settings
    with env_settings(dict(PG_LINEAR_TILE=tile, PG_LINEAR_SPLITS=splits)):
        check_fused(n, rows, p, q, dtype, kept, ragged)


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("tile", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_smooth_activations_on_every_tile(name, dtype, tile, splits):
    """Input in 8 bits, pre-activation kept, residual; the input gradient back through a kept activation.  Beside a kept result bf16 weights enter in two
    pieces, each within 2^-8 of what is left of them: 2^-16."""
    from parity_util import env_settings
    n, rows, p, q = 2, 290, 270, 390
    gen = torch.Generator().manual_seed(tile + splits)
    with env_settings(dict(PG_LINEAR_TILE=tile, PG_LINEAR_SPLITS=splits)):
        gb = buffers(n, [(p, q), (p, 1)])
    w, b = torch.randn(n, p, q, generator=gen) * 2 / math.sqrt(q), torch.randn(n, p, 1, generator=gen)
    put(gb, 0, w), put(gb, 1, b)
    x, r = held(torch.randn(n, rows, q, generator=gen))[0], torch.randn(n, rows, p, generator=gen).to(dtype)
    x8, keep = gb.checkpoint_store(x.float().cuda()), gb.checkpoint(rows, p)
    y = gb.linear(0, x8, bias=1, act=name, residual=r.cuda(), keep=keep).cpu().double()
    wt = w.double().transpose(1, 2)
    z = x @ wt + b.double().transpose(1, 2)
    off = product_error(x, wt, F32) + (2.0 ** -16 * (x.abs() @ wt.abs()) if dtype == BF16 else 0.0) + 2.0 ** -23 * z.abs()
    want = act(name, z) + r.double()
    # |act'| <= 1.13; the functions themselves to a few units of float at the size of z
    assert bool(((y - want).abs() <= 1.13 * off + 2.0 ** -20 * z.abs() + 2.0 ** -23 + HALF[dtype] * (want.abs() + 2 * off)).all())
    kept = gb.checkpoint_load(keep, dtype=F32).cpu().double()
    step = (2.0 ** -9 * 2.0 ** held(z)[1]).repeat_interleave(32, -1)[..., :p]   # a block's maximum at a border may go to the next scale
    assert bool(((kept - z).abs() <= off + 2.0 ** -4 * (z.abs() + off) + step).all())

    z = held(torch.randn(n, rows, q, generator=gen) * 2)[0]
    z8, dz, r = gb.checkpoint_store(z.float().cuda()), torch.randn(n, rows, p, generator=gen).to(dtype), torch.randn(n, rows, q, generator=gen).to(dtype)
    dx = gb.linear_backward(0, dz.cuda(), x8, bias=1, act=name, z=z8, residual=r.cuda()).cpu().double()
    plain, size, s = dz.double() @ w.double(), product_error(dz.double(), w.double(), dtype), slope(name, z)
    want = plain * s + r.double()
    off = size * s.abs() + 2.0 ** -20 * plain.abs() + 2.0 ** -22 * (plain.abs() + r.double().abs())
    assert bool(((dx - want).abs() <= off + HALF[dtype] * (want.abs() + off)).all())
    # the weights' gradient has no rounding but its sum's: both operands enter exactly
    dzt = dz.double().transpose(1, 2)
    assert bool(((grad(gb, 0) - dzt @ x).abs() <= product_error(dzt, x, F32) + 2.0 ** -24 * (dzt @ x).abs()).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,rows,cols", [(1, 7, 1030), (1, 10, 2049), (1, 9, 4100), (1, 8, 8200), (1, 6, 16384), (3, 50, 33), (17, 9, 70), (40, 21, 650)])
def test_norms_of_some_of_their_rows(n, rows, cols, dtype):
    """Counts inside a worker's rows, and the backward pass without the gain's gradient.  Integers: sums of squares and of products are exact."""
    print("case", n, rows, cols, dtype, flush=True)
    gen = torch.Generator().manual_seed(cols + n)
    gb = buffers(n, [(cols, 1)])
    g, x, r, dy = integers(gen, (n, cols, 1), 2), integers(gen, (n, rows, cols), 3), integers(gen, (n, rows, cols), 3), integers(gen, (n, rows, cols), 3)
    put(gb, 0, g)
    counts = some(n, rows, True)
    there = mask(n, rows, counts)
    xd, rd, dyd = (t.to(dtype).cuda() for t in (x, r, dy))
    old = lambda: torch.full((n, rows, cols), 7.0, dtype=dtype, device="cuda")  # noqa: E731
    y, total, rstd = gb.norm(0, xd, residual=rd, eps=0.25, counts=counts, out=old(), sum_out=old(), rstd_out=torch.full((n, rows), 7.0, device="cuda"))
    s = x + r
    assert torch.equal(total.cpu().double(), torch.where(there, s, 7.0))
    want = torch.where(there[..., 0], 1 / torch.sqrt(s.square().mean(-1) + 0.25), 7.0)
    assert bool(((rstd.cpu().double() - want).abs() <= 5 * 2.0 ** -24 * want).all())        # a division, a sum, a root, a division
    want = torch.where(there, s * want[..., None] * g.transpose(1, 2), 7.0)
    assert bool(((y.cpu().double() - want).abs() <= (8 * 2.0 ** -24 + HALF[dtype]) * want.abs()).all())
    for buf in gb.g:
        buf.fill_(7.0)
    one, sd = torch.full((n, rows), 0.5, device="cuda"), s.to(dtype).cuda()
    dx = gb.norm_backward(0, dyd, sd, one, counts=counts, want_grads=False, out=old())
    assert all(bool((buf == 7.0).all()) for buf in gb.g)
    h, gd = s * 0.5, g.transpose(1, 2)
    mean = (gd * dy * h).mean(-1, keepdim=True)
    want = 0.5 * (gd * dy - h * mean)
    off = 0.5 * (h * mean).abs() * 3 * 2.0 ** -24 + 2.0 ** -24 * want.abs()                  # a division, a product, a difference
    assert bool((torch.where(there, (dx.cpu().double() - want).abs() - (off + HALF[dtype] * (want.abs() + off)), 0.0) <= 0).all())
    assert bool((dx.cpu() == 7.0)[~there.expand_as(dx)].all())
    again = gb.norm_backward(0, dyd, sd, one, counts=counts, out=old())
    assert torch.equal(dx, again)
    assert torch.equal(grad(gb, 0)[..., 0], torch.where(there, dy * h, 0.0).sum(1))
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_checkpoints_and_activations_of_some_of_their_rows(dtype):
    for n, rows, cols in ((1, 50, 70), (17, 9, 33), (40, 30, 100)):
        gen = torch.Generator().manual_seed(n)
        gb = buffers(n, [(2, 2)])
        z, dy = integers(gen, (n, rows, cols), 8), integers(gen, (n, rows, cols), 3)
        counts = some(n, rows, True)
        there = mask(n, rows, counts)
        z8 = gb.checkpoint_store(z.to(dtype).cuda(), counts=counts)
        assert torch.equal(gb.checkpoint_load(z8, dtype=F32, counts=counts).cpu().double(), torch.where(there, z, 0.0))
        out = torch.full((n, rows, cols), 7.0, dtype=dtype, device="cuda")
        gb.activation_backward("relu", dy.to(dtype).cuda(), z8, counts=counts, out=out)
        assert torch.equal(out.cpu().double(), torch.where(there, dy * (z > 0), 7.0))
        gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,rows,d,wide", [(2, 33, 70, 130), (1, 20, 2100, 40), (2, 9, 8200, 33)])
def test_results_in_the_place_of_what_they_are_made_of(n, rows, d, wide, dtype):
    """Every pair of arguments that may be the very same rows, on a stream of the caller's: bit for bit what results of their own hold."""
    gen = torch.Generator().manual_seed(d)
    gb = buffers(n, [(wide, d), (wide, 1), (d, 1)])
    for l, s in enumerate(gb.shapes):
        put(gb, l, torch.randn(n, *s, generator=gen))
    x, r, dy, dr = (torch.randn(n, rows, d, generator=gen).to(dtype).cuda() for _ in range(4))
    dz, rz = (torch.randn(n, rows, wide, generator=gen).to(dtype).cuda() for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, total, rstd = gb.norm(2, x, residual=r)
    lin = gb.linear(0, x, bias=1, act="silu", residual=rz)
    z8 = gb.checkpoint_store(x)
    dx = gb.linear_backward(0, dz, x, bias=1, act="silu", z=z8, residual=dr)
    linear_grads = grad(gb, 0), grad(gb, 1)
    ds, dg = gb.norm_backward(2, dy, total, rstd, residual=dr), grad(gb, 2)
    da = gb.activation_backward("gelu", dy, z8)
    torch.cuda.synchronize()
    for which in ("sum", "y", "both"):                       # x + r where x was, or r; the result where x was
        a, b = x.clone(), r.clone()
        side.wait_stream(torch.cuda.current_stream())
        got = gb.norm(2, a, residual=b, sum_out=a if which == "sum" else b if which == "both" else None, out=a if which != "sum" else None, stream=side)
        side.synchronize()
        assert torch.equal(got[0], y) and torch.equal(got[1], total) and torch.equal(got[2], rstd)
        assert got[0 if which != "sum" else 1] is a
    a = rz.clone()
    side.wait_stream(torch.cuda.current_stream())
    gb.linear(0, x, bias=1, act="silu", residual=a, out=a, stream=side)
    b = dr.clone()
    side.wait_stream(torch.cuda.current_stream())
    gb.linear_backward(0, dz, x, bias=1, act="silu", z=z8, residual=b, out=b, stream=side)
    side.synchronize()
    assert torch.equal(a, lin) and torch.equal(b, dx) and torch.equal(grad(gb, 0), linear_grads[0]) and torch.equal(grad(gb, 1), linear_grads[1])
    for take in (0, 1):                                      # dx where dy was, or where the passing gradient was
        a, b = dy.clone(), dr.clone()
        side.wait_stream(torch.cuda.current_stream())
        got = gb.norm_backward(2, a, total, rstd, residual=b, out=(a, b)[take], stream=side)
        side.synchronize()
        assert torch.equal(got, ds) and torch.equal(grad(gb, 2), dg)
    a = dy.clone()
    side.wait_stream(torch.cuda.current_stream())
    gb.activation_backward("gelu", a, z8, out=a, stream=side)
    side.synchronize()
    assert torch.equal(a, da)
    gb.close()
