"""The operators on rows of activations against plain statements in 64 bits: sizes around every tile, rows that do not exist, strides, types,
values that are not finite, graphs, streams, and a training step of all of them."""
import math

import pytest
import torch

from paper_2008_01425_amd import binding as B
from rows_util import HALF, act, buffers, grad, held, mask, product_error, put, slope

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SIZES = [(1, 1, 1, 1), (4, 1, 64, 32), (3, 5, 33, 65), (2, 16, 129, 127), (2, 31, 130, 258), (1, 33, 127, 40), (2, 129, 100, 333),
         (1, 300, 257, 96), (5, 64, 8, 1028), (2, 257, 384, 31)]


def integers(gen, shape, top):
    return torch.randint(-top, top + 1, shape, generator=gen).double()


def few(n, rows, ragged):
    if not ragged:
        return None
    return torch.tensor([(rows * (i + 2)) // (n + 2) if i else 0 for i in range(n)], dtype=torch.int32, device="cuda")


def check_products(n, rows, p, q, dtype, kept, ragged):
    print("case", n, rows, p, q, dtype, kept, ragged, flush=True)
    gen = torch.Generator().manual_seed(n * 1000 + rows + p + q)
    gb = buffers(n, [(p, q), (p, 1)])
    w, b = integers(gen, (n, p, q), 2), integers(gen, (n, p, 1), 50)
    x, dz = integers(gen, (n, rows, q), 4 if kept else 8), integers(gen, (n, rows, p), 3)
    if dtype == F32 and not kept:      # two numbers of 20 bits, at most one of them in any sum of products
        x[:, 0, 0] = 2 ** 20 - 1
        dz[:, min(1, rows - 1), 0] = 1 - 2 ** 20 if rows > 1 else 3
    r, rx = integers(gen, (n, rows, p), 9), integers(gen, (n, rows, q), 9)
    put(gb, 0, w), put(gb, 1, b)
    counts = few(n, rows, ragged)
    there = mask(n, rows, counts)
    xd = x.to(dtype).cuda()
    given = gb.checkpoint_store(xd) if kept else xd
    out = torch.full((n, rows, p), 7.0, dtype=dtype, device="cuda")
    y = gb.linear(0, given, bias=1, residual=r.to(dtype).cuda(), counts=counts, out=out)
    want = torch.where(there, x @ w.transpose(1, 2) + b.transpose(1, 2) + r, 7.0)
    assert torch.equal(y.cpu(), want.float().to(dtype))
    dx = torch.full((n, rows, q), 7.0, dtype=dtype, device="cuda")
    dzd = dz.to(dtype).cuda()
    gb.linear_backward(0, dzd, given, bias=1, residual=rx.to(dtype).cuda(), counts=counts, out=dx)
    want = torch.where(there, dz @ w + rx, 7.0)
    assert torch.equal(dx.cpu(), want.float().to(dtype))
    dz0 = torch.where(there, dz, 0.0)
    dw, db = dz0.transpose(1, 2) @ x, dz0.sum(1)[..., None]
    assert torch.equal(grad(gb, 0), dw) and torch.equal(grad(gb, 1), db)
    gb.linear_backward(0, dzd, given, bias=1, accumulate=True, want_dx=False, counts=counts)
    assert torch.equal(grad(gb, 0), 2 * dw) and torch.equal(grad(gb, 1), 2 * db)
    gb.close()


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype,kept", [(F32, False), (F32, True), (BF16, False), (BF16, True)])
@pytest.mark.parametrize("n,rows,p,q", SIZES)
def test_products_of_integers_are_exact(n, rows, p, q, dtype, kept, ragged):
    """Integers whose sums fit 24 bits: every product, forward and backward, has one right answer.  In float some need all three pieces."""
    check_products(n, rows, p, q, dtype, kept, ragged)


@pytest.mark.parametrize("splits", [1, 4])
@pytest.mark.parametrize("tile", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype,kept", [(F32, False), (F32, True), (BF16, False), (BF16, True)])
@pytest.mark.parametrize("n,rows,p,q", [(2, 3, 5, 7), (2, 290, 270, 520), (1, 515, 131, 258)])
def test_products_on_every_tile(n, rows, p, q, dtype, kept, tile, splits):
    """The same with each tile forced, and its steps split or not."""
    from parity_util import env_settings
    with env_settings(dict(PG_LINEAR_TILE=tile, PG_LINEAR_SPLITS=splits)):
        check_products(n, rows, p, q, dtype, kept, rows > 500)


@pytest.mark.parametrize("tile", [32, 64, 128, 256])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_kept_results_on_every_tile(dtype, tile):
    """Integers again: what is kept beside a result is the 8-bit form of the one right sum; infinities of a column as NaN, whether split or not."""
    from parity_util import env_settings
    n, rows, p, q = 2, 270, 300, 390
    gen = torch.Generator().manual_seed(tile)
    w, b, x = integers(gen, (n, p, q), 2), integers(gen, (n, p, 1), 50), integers(gen, (n, rows, q), 8)
    w[1, 7, 3] = math.inf
    z = x @ w.transpose(1, 2) + b.transpose(1, 2)
    want = held(torch.where(torch.isfinite(z), z, math.nan))[0].float().nan_to_num(nan=1e30)
    for splits in (1, 3):
        with env_settings(dict(PG_LINEAR_TILE=tile, PG_LINEAR_SPLITS=splits)):
            gb = buffers(n, [(p, q), (p, 1)])
        put(gb, 0, w), put(gb, 1, b)
        keep = gb.checkpoint(rows, p)
        y = gb.linear(0, x.to(dtype).cuda(), bias=1, keep=keep)
        assert torch.equal(y.cpu().nan_to_num(nan=7e30), z.float().to(dtype).nan_to_num(nan=7e30))
        assert torch.equal(gb.checkpoint_load(keep, dtype=F32).cpu().nan_to_num(nan=1e30), want)
        gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("n,rows,p,q", [(3, 5, 33, 65), (2, 40, 130, 100), (1, 150, 260, 190)])
def test_linear_with_its_activation_and_what_it_keeps(n, rows, p, q, name, dtype):
    gen = torch.Generator().manual_seed(rows)
    gb = buffers(n, [(p, q), (p, 1)])
    w, b = torch.randn(n, p, q, generator=gen) * 2 / math.sqrt(q), torch.randn(n, p, 1, generator=gen)
    x, r = torch.randn(n, rows, q, generator=gen).to(dtype), torch.randn(n, rows, p, generator=gen).to(dtype)
    put(gb, 0, w), put(gb, 1, b)
    keep = gb.checkpoint(rows, p)
    y = gb.linear(0, x.cuda(), bias=1, act=name, residual=r.cuda(), keep=keep).cpu().double()
    xw = x.double(), w.double().transpose(1, 2)
    z = xw[0] @ xw[1] + b.double().transpose(1, 2)
    off = product_error(*xw, dtype) + 2.0 ** -23 * z.abs()
    # |act'| <= 1.13; the functions themselves to a few units of float at the size of z
    want = act(name, z) + r.double()
    assert bool(((y - want).abs() <= 1.13 * off + 2.0 ** -20 * z.abs() + 2.0 ** -23 + HALF[dtype] * (want.abs() + 2 * off)).all())
    kept = gb.checkpoint_load(keep, dtype=F32).cpu().double()
    _, e = held(z)
    step = (2.0 ** -9 * 2.0 ** e).repeat_interleave(32, -1)[..., :p]       # a block's maximum at a border may go to the next scale
    assert bool(((kept - z).abs() <= off + 2.0 ** -4 * (z.abs() + off) + step).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("n,rows,p,q", [(2, 7, 65, 70), (2, 140, 190, 130)])
def test_gradients_through_kept_activations(n, rows, p, q, name, dtype):
    gen = torch.Generator().manual_seed(p)
    gb = buffers(n, [(p, q), (p, 1)])
    w = torch.randn(n, p, q, generator=gen)
    put(gb, 0, w)
    z = held(torch.randn(n, rows, q, generator=gen) * 2)[0]
    x, dz = held(act(name, z))[0], torch.randn(n, rows, p, generator=gen).to(dtype)
    z8, x8 = gb.checkpoint_store(z.float().cuda()), gb.checkpoint_store(x.float().cuda())
    r = torch.randn(n, rows, q, generator=gen).to(dtype)
    dx = gb.linear_backward(0, dz.cuda(), x8, bias=1, act=name, z=z8, residual=r.cuda()).cpu().double()
    plain, size = dz.double() @ w.double(), product_error(dz.double(), w.double(), dtype)
    s = slope(name, z)
    want = plain * s + r.double()
    off = size * s.abs() + 2.0 ** -20 * plain.abs() + 2.0 ** -22 * (plain.abs() + r.double().abs())
    assert bool(((dx - want).abs() <= off + HALF[dtype] * (want.abs() + off)).all())
    # the weights' gradient has no rounding but its sum's: both operands enter exactly
    dw = dz.double().transpose(1, 2) @ x
    assert bool(((grad(gb, 0) - dw).abs() <= product_error(dz.double().transpose(1, 2), x, F32) + 2.0 ** -24 * dw.abs()).all())
    db = dz.double().sum(1)[..., None]
    assert bool(((grad(gb, 1) - db).abs() <= rows * 2.0 ** -24 * dz.double().abs().sum(1)[..., None]).all())
    dy = torch.randn(n, rows, q, generator=gen).to(dtype)
    got = gb.activation_backward(name, dy.cuda(), z8).cpu().double()
    want = dy.double() * s
    assert bool(((got - want).abs() <= HALF[dtype] * want.abs() + 2.0 ** -20 * dy.double().abs()).all())
    gb.close()


@pytest.mark.parametrize("name", ["none", "gelu", "silu"])
def test_gradients_are_those_of_differences(name):
    """Central differences of sum(linear * c) along random directions, step h: h^2 / 6 of a third derivative (below 2 for these functions, times |d z|^3) and the
    rounding of two sums of 1e3 terms of size 1 in float, 2^-24 / h of each."""
    n, rows, p, q, h = 2, 24, 40, 32, 2.0 ** -6
    gen = torch.Generator().manual_seed(3)
    gb = buffers(n, [(p, q), (p, 1)])
    w, b = torch.randn(n, p, q, generator=gen) / math.sqrt(q), torch.randn(n, p, 1, generator=gen)
    x, c = torch.randn(n, rows, q, generator=gen).cuda(), torch.randn(n, rows, p, generator=gen).cuda()
    put(gb, 0, w), put(gb, 1, b)
    keep = gb.checkpoint(rows, p)
    gb.linear(0, x, bias=1, act=name, keep=keep)
    z = gb.linear(0, x, bias=1)
    # act'(z) from the exact z here: what 8 bits make of it is tested above
    dz = (c.double() * slope(name, z.double())).float()
    dx = gb.linear_backward(0, dz, x, bias=1)
    for _ in range(4):
        d, dw, db = torch.randn(n, rows, q, generator=gen), torch.randn(n, p, q, generator=gen) / math.sqrt(q), torch.randn(n, p, 1, generator=gen)
        ends = []
        for sign in (1, -1):
            put(gb, 0, w + sign * h * dw), put(gb, 1, b + sign * h * db)
            ends.append(float((gb.linear(0, x + sign * h * d.cuda(), bias=1, act=name).double() * c.double()).sum()))
        put(gb, 0, w), put(gb, 1, b)
        told = float((dx.cpu().double() * d.double()).sum() + (grad(gb, 0) * dw.double()).sum() + (grad(gb, 1) * db.double()).sum())
        # z moves by h times dz along d, dw, db (a few units each) and h^2 d dw: second order, cancelled by the central difference
        dzd = d.double() @ w.double().transpose(1, 2) + x.cpu().double() @ dw.double().transpose(1, 2) + db.double().transpose(1, 2)
        bent = (d.double() @ dw.double().transpose(1, 2)).abs()
        third = (c.cpu().double().abs() * (2 * dzd.abs() ** 3 / 6 + 1.2 * bent * dzd.abs())).sum()
        assert abs((ends[0] - ends[1]) / (2 * h) - told) <= float(third) * h * h + 2.0 ** -24 / h * float(c.cpu().double().abs().sum()) * 32
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,rows,cols", [(1, 1, 1), (3, 5, 8), (2, 9, 33), (2, 6, 512), (2, 7, 650), (1, 5, 1030), (2, 3, 2049), (1, 4, 4100),
                                         (1, 3, 8200), (1, 2, 16384)])
@pytest.mark.parametrize("ragged", [False, True])
def test_norm_and_its_gradients(n, rows, cols, dtype, ragged):
    print("case", n, rows, cols, dtype, ragged, flush=True)
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(n, [(cols, 1)])
    g = torch.randn(n, cols, 1, generator=gen)
    put(gb, 0, g)
    x, r = (torch.randn(n, rows, cols, generator=gen).to(dtype) for _ in range(2))
    counts = few(n, rows, ragged)
    there = mask(n, rows, counts)
    eps = 1e-5
    keep = gb.checkpoint(rows, cols)
    old = lambda: torch.full((n, rows, cols), 7.0, dtype=dtype, device="cuda")  # noqa: E731
    rstd_out = torch.full((n, rows), 7.0, device="cuda")
    y, total, rstd = gb.norm(0, x.cuda(), residual=r.cuda(), eps=eps, keep=keep, counts=counts, out=old(), sum_out=old(), rstd_out=rstd_out)
    s = (x.double() + r.double()).float().to(dtype)
    assert torch.equal(total.cpu(), torch.where(there, s, torch.tensor(7.0, dtype=dtype)))
    s = s.double()
    want_rstd = 1 / torch.sqrt(s.square().mean(-1, keepdim=True) + eps)
    tiny = (cols + 8) * 2.0 ** -24         # a sum of squares (all of one sign) in float, then a root and a division
    got = torch.where(there, rstd.cpu().double()[..., None], want_rstd)
    assert bool(((got - want_rstd).abs() <= tiny * want_rstd).all())
    assert bool((rstd.cpu()[~there[..., 0]] == 7.0).all())
    want = s * want_rstd * g.double().transpose(1, 2)
    err = (y.cpu().double() - want).abs()
    assert bool((torch.where(there, err, 0.0) <= (tiny + 2.0 ** -22) * want.abs() + HALF[dtype] * want.abs()).all())
    assert bool((y.cpu() == 7.0)[~there.expand_as(y)].all())
    kept = gb.checkpoint_load(keep, dtype=F32, counts=counts).cpu().double()
    _, e = held(want)
    step = (2.0 ** -9 * 2.0 ** e).repeat_interleave(32, -1)[..., :cols]
    assert bool(((torch.where(there, kept - want, 0.0)).abs() <= (2.0 ** -4 + tiny + 2.0 ** -22) * want.abs() + step).all())

    dy, dr = (torch.randn(n, rows, cols, generator=gen).to(dtype) for _ in range(2))
    rs = want_rstd.float()
    dx = gb.norm_backward(0, dy.cuda(), s.to(dtype).cuda(), rs[..., 0].contiguous().cuda(), residual=dr.cuda(), counts=counts, out=old())
    rs, gd = rs.double(), g.double().transpose(1, 2)
    h = s * rs
    parts = gd * dy.double() * h
    want = rs * (gd * dy.double() - h * parts.mean(-1, keepdim=True)) + dr.double()
    off = (rs * ((gd * dy.double()).abs() + h.abs() * parts.abs().mean(-1, keepdim=True)) + dr.double().abs()) * (cols + 8) * 2.0 ** -24
    assert bool((torch.where(there, (dx.cpu().double() - want).abs() - HALF[dtype] * want.abs(), 0.0) <= (1 + HALF[dtype]) * off).all())
    assert bool((dx.cpu() == 7.0)[~there.expand_as(dx)].all())
    terms = torch.where(there, dy.double() * h, 0.0)
    dg = terms.sum(1)[..., None]
    off = terms.abs().sum(1)[..., None] * (rows + 4) * 2.0 ** -24
    assert bool(((grad(gb, 0) - dg).abs() <= off).all())
    gb.norm_backward(0, dy.cuda(), s.to(dtype).cuda(), rs[..., 0].float().contiguous().cuda(), counts=counts, accumulate=True)
    assert bool(((grad(gb, 0) - 2 * dg).abs() <= 3 * off).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_checkpoint_holds_what_its_definition_says(dtype):
    """Every e4m3 value and the middles between them, scales over the whole range, borders of the scale, zeros, infinities, NaN."""
    rows = []
    codes = [m * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8, 16)] + [m * 2.0 ** -9 for m in range(8)]
    codes = sorted({c for c in codes if c <= 448})
    middles = [(a + b) / 2 for a, b in zip(codes, codes[1:])]
    every = torch.tensor(codes + [-c for c in codes] + middles + [-m for m in middles], dtype=torch.float64)
    every = torch.cat([every.reshape(-1), torch.zeros(-len(every) % 31)]).view(-1, 31)
    rows.append(torch.cat([torch.full((len(every), 1), 448.0), every], 1).reshape(-1))           # scale 1
    for e in (-140, -126, -117, -100, -30, 0, 5, 100, 118):
        g = torch.Generator().manual_seed(e + 200)
        rows.append((torch.randn(rows[0].numel(), generator=g).double().clamp(-3.9, 3.9)) * 2.0 ** e)
    for top in (1.75, 1.7578125, 1.0, 1.9921875):
        v = torch.full((rows[0].numel(),), 0.3)
        v[::32] = top
        rows.append(v.double())
    odd = rows[0].clone()
    odd[3::32], odd[7::64], odd[9::96] = math.inf, -math.inf, math.nan
    rows += [torch.zeros_like(odd), odd, torch.full_like(odd, math.nan)]
    x = torch.stack(rows).float().to(dtype)[None]
    cols = x.shape[2] - 5                       # the last block is a short one
    x = x[:, :, :cols].contiguous()
    gb = buffers(1, [(2, 2)])
    kept = gb.checkpoint_store(x.cuda())
    want, e = held(x)
    got = gb.checkpoint_load(kept, dtype=F32).cpu()
    assert torch.equal(got.nan_to_num(nan=1e30), want.float().nan_to_num(nan=1e30))
    assert torch.equal(gb.checkpoint_load(kept).cpu().float().nan_to_num(nan=1e30), want.float().nan_to_num(nan=1e30))  # bf16 holds them too
    pitch = (cols + 31) // 32 * 32
    codes_end = (x.shape[1] * pitch + 255) // 256 * 256
    scales = kept.data[codes_end:codes_end + x.shape[1] * pitch // 32].cpu().view(x.shape[1], -1)
    assert torch.equal(scales.double() - 127, e[0])
    again = gb.checkpoint_store(got.cuda())     # what it holds it holds again
    assert torch.equal(gb.checkpoint_load(again, dtype=F32).cpu().nan_to_num(nan=1e30), got.nan_to_num(nan=1e30))
    gb.close()


@pytest.mark.parametrize("cols", [1, 7, 31, 32, 33, 64, 100, 511, 520, 1301])
@pytest.mark.parametrize("ragged", [False, True])
def test_checkpoints_of_any_width(cols, ragged):
    n, rows = 3, 19
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(n, [(2, 2)])
    x = torch.randn(n, rows, cols, generator=gen)
    counts = few(n, rows, ragged)
    kept = gb.checkpoint(rows, cols)
    kept.data.fill_(255)
    gb.checkpoint_store(x.cuda(), counts=counts, out=kept)
    out = torch.full((n, rows, cols), 7.0, device="cuda")
    gb.checkpoint_load(kept, counts=counts, out=out)
    there = mask(n, rows, counts)
    assert torch.equal(out.cpu(), torch.where(there, held(x)[0].float(), 7.0))
    pitch = (cols + 31) // 32 * 32
    codes = kept.data[:n * rows * pitch].cpu().view(n, rows, pitch)
    assert bool((codes[..., cols:][there.expand(n, rows, pitch - cols)] == 0).all())
    assert bool((codes[~there.expand(n, rows, pitch)] == 255).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_nan_go_through(dtype):
    """What is not finite stays in the rows and columns it belongs to; infinities keep their sign and become NaN against zero or each other."""
    n, rows, p, q = 1, 140, 150, 96
    gen = torch.Generator().manual_seed(1)
    gb = buffers(n, [(p, q), (p, 1)])
    w, x = integers(gen, (n, p, q), 3), integers(gen, (n, rows, q), 3)
    w[0, 5, 7], w[0, 9, 40], w[0, 20, 3] = math.inf, -math.inf, math.nan
    x[0, 11, 7], x[0, 33, 50], x[0, 130, 2] = math.inf, -math.inf, math.nan
    if dtype == F32:
        w[0, 30, 8] = 3.4e38           # finite, but infinite once rounded to bf16
        x[0, :, 8] = x[0, :, 8].sign()
        w = w.float().double()
    put(gb, 0, w)
    dz = integers(gen, (n, rows, p), 3)
    dz[0, 70, 100], dz[0, 71, 5] = math.inf, 0.0
    keep = gb.checkpoint(rows, p)
    y = gb.linear(0, x.to(dtype).cuda()).cpu()
    assert torch.equal(gb.linear(0, x.to(dtype).cuda(), keep=keep).cpu().nan_to_num(nan=7e30), y.nan_to_num(nan=7e30))
    want = (x @ w.transpose(1, 2))
    z = x @ w.transpose(1, 2)
    z, kept = torch.where(torch.isfinite(z), z, math.nan), gb.checkpoint_load(keep, dtype=F32).cpu()
    assert torch.equal(kept.nan_to_num(nan=1e300), held(z.float())[0].float().nan_to_num(nan=1e300))
    dx = gb.linear_backward(0, dz.to(dtype).cuda(), x.to(dtype).cuda()).cpu()
    for got, ref in ((y, want), (dx, dz @ w), (grad(gb, 0), dz.transpose(1, 2) @ x)):
        ref = ref.float()
        if got.dtype == BF16:
            ref = ref.to(dtype)
        got, ref = got.double(), ref.double()
        assert torch.equal(torch.isnan(got), torch.isnan(ref))
        ref, got = ref.nan_to_num(nan=0.0, posinf=1e300, neginf=-1e300), got.nan_to_num(nan=0.0, posinf=1e300, neginf=-1e300)
        big = ref.abs() > 1e30
        assert torch.equal(got[~big], ref[~big])
        assert bool(((got - ref).abs()[big] <= 2.0 ** -22 * ref.abs()[big]).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_of_inputs_and_outputs(dtype):
    """Rows inside wider ones at odd offsets, workers interleaved, one input for all workers, results beside untouched elements."""
    n, rows, p, q = 3, 37, 45, 51
    gen = torch.Generator().manual_seed(2)
    gb = buffers(n, [(p, q), (p, 1)])
    w, b = integers(gen, (n, p, q), 2), integers(gen, (n, p, 1), 5)
    put(gb, 0, w), put(gb, 1, b)
    x, dz, r = integers(gen, (1, rows, q), 4), integers(gen, (n, rows, p), 3), integers(gen, (1, 1, p), 9)
    xd = torch.zeros(rows, q + 3, dtype=dtype, device="cuda")[:, 3:].unsqueeze(0).expand(n, -1, -1)
    xd[0].copy_(x[0])
    dzd = torch.zeros(rows, n, p + 2, dtype=dtype, device="cuda")[:, :, 1:p + 1].transpose(0, 1)
    dzd.copy_(dz)
    rd = r.to(dtype).cuda().expand(n, rows, p)
    room = torch.full((rows, n, p + 5), 7.0, dtype=dtype, device="cuda")
    gb.linear(0, xd, bias=1, residual=rd, out=room[:, :, 1:p + 1].transpose(0, 1))
    want = torch.full((rows, n, p + 5), 7.0, dtype=torch.float64)
    want[:, :, 1:p + 1] = (x @ w.transpose(1, 2) + b.transpose(1, 2) + r).transpose(0, 1)
    assert torch.equal(room.cpu().double(), want.float().to(dtype).double())
    room = torch.full((n, rows, q + 1), 7.0, dtype=dtype, device="cuda")
    gb.linear_backward(0, dzd, xd, bias=1, out=room[:, :, 1:])
    assert torch.equal(room[:, :, 1:].cpu().double(), (dz @ w).float().to(dtype).double()) and bool((room[:, :, 0] == 7).all())
    assert torch.equal(grad(gb, 0), dz.transpose(1, 2) @ x.expand(n, -1, -1))
    # the very same rows as the residual
    y = rd.contiguous()
    gb.linear(0, xd, bias=1, residual=y, out=y)
    assert torch.equal(y.cpu().double(), (x @ w.transpose(1, 2) + b.transpose(1, 2) + r).float().to(dtype).double())
    kept = gb.checkpoint_store(dzd)
    assert torch.equal(gb.checkpoint_load(kept, dtype=F32).cpu().double(), dz)
    gb.close()


def test_padded_parameter_rows_and_their_padding():
    """A torus at rank 4 pads the rows of its layers; products take the stride, and write nothing between rows."""
    from paper_2008_01425_amd import workloads as W
    from paper_2008_01425_amd.device import GossipBuffers
    edges = W.torus_edges(3, 3)
    gb = GossipBuffers(9, edges, [0.2] * len(edges), [(70, 100), (70, 1)], 4, 1)
    assert B.pg_layer_stride(gb.ctx, 0) == 128
    gb.alloc_grads()
    for g in gb.g:
        g.fill_(7.0)
    gen = torch.Generator().manual_seed(4)
    w, x, dz = integers(gen, (9, 70, 100), 2), integers(gen, (9, 20, 100), 4), integers(gen, (9, 20, 70), 3)
    put(gb, 0, w)
    for X in gb.x:                          # what lies between the rows is no part of them
        X[:70 * 128].view(70, 128)[:, 100:] = math.nan
    y = gb.linear(0, x.float().cuda())
    dx = gb.linear_backward(0, dz.float().cuda(), x.float().cuda(), bias=1)
    assert torch.equal(y.cpu().double(), x @ w.transpose(1, 2)) and torch.equal(dx.cpu().double(), dz @ w)
    assert torch.equal(grad(gb, 0), dz.transpose(1, 2) @ x)
    for g in gb.g:
        assert bool((g[:70 * 128].view(70, 128)[:, 100:] == 7.0).all())
    gb.close()


def test_no_rows_at_all():
    gb = buffers(2, [(6, 5), (6, 1), (5, 1)])
    for g in gb.g:
        g.fill_(7.0)
    none = lambda c: torch.zeros(2, 0, c, device="cuda")  # noqa: E731
    assert gb.linear(0, none(5), bias=1).shape == (2, 0, 6)
    gb.linear_backward(0, none(6), none(5), bias=1, accumulate=True)
    gb.norm_backward(2, none(5), none(5), torch.zeros(2, 0, device="cuda"), accumulate=True)
    assert all(bool((grad(gb, l) == 7.0).all()) for l in range(3))
    gb.linear_backward(0, none(6), none(5), bias=1)
    gb.norm_backward(2, none(5), none(5), torch.zeros(2, 0, device="cuda"))
    assert all(bool((grad(gb, l) == 0.0).all()) for l in range(3))
    y, _, rstd = gb.norm(2, none(5))
    assert y.shape == (2, 0, 5) and rstd.shape == (2, 0)
    assert gb.checkpoint_load(gb.checkpoint_store(none(5))).shape == (2, 0, 5)
    gb.close()


def _room(gigabytes):
    if torch.cuda.mem_get_info()[0] < gigabytes << 30:
        pytest.skip(f"needs {gigabytes} GB")


@pytest.mark.parametrize("n,rows,row,worker", [(2, 40, 200, (1 << 31) + 72), (1, 2100, 1 << 21, 0)])
def test_strides_beyond_thirty_two_bits(n, rows, row, worker):
    """Workers more than 2^31 elements apart, rows that end beyond 2^32 bytes: the same bits as from compact tensors."""
    _room(40)
    p, q = 70, 96
    gen = torch.Generator().manual_seed(8)
    gb = buffers(n, [(p, q), (p, 1), (q, 1)])
    for l, s in enumerate(gb.shapes):
        put(gb, l, torch.randn(n, *s, generator=gen))

    def far(x):
        size = (n - 1) * worker + (rows - 1) * row + x.shape[2]
        out = torch.empty(size, dtype=x.dtype, device="cuda").as_strided(x.shape, (worker or size, row, 1))
        out.copy_(x)
        return out

    x, r, dz, rq = (torch.randn(n, rows, c, generator=gen).to(BF16).cuda() for c in (q, p, p, q))
    out = far(torch.zeros_like(r))
    gb.linear(0, far(x), bias=1, residual=r, out=out)
    assert torch.equal(out, gb.linear(0, x, bias=1, residual=r))
    del out
    want, grads = gb.linear_backward(0, dz, x, bias=1, residual=rq), [g.clone() for g in gb.g]
    out = far(torch.zeros_like(x))
    gb.linear_backward(0, far(dz), far(x), bias=1, residual=rq, out=out)
    assert torch.equal(out, want) and all(torch.equal(gb.layer_of(a, l), gb.layer_of(b, l)) for a, b in zip(gb.g, grads) for l in (0, 1))
    y, total, rstd = gb.norm(2, x, residual=rq)
    gb.norm(2, far(x), residual=rq, out=out)
    assert torch.equal(out, y)
    want = gb.norm_backward(2, x, total, rstd)
    gb.norm_backward(2, far(x), total, rstd, out=out)
    assert torch.equal(out, want)
    gb.checkpoint_load(gb.checkpoint_store(far(x)), out=out)
    assert torch.equal(out, gb.checkpoint_load(gb.checkpoint_store(x)))
    gb.close()


def test_checkpoints_and_norms_of_very_many_rows():
    """More than 2^32 bytes of codes, and more work-groups than one side of a grid takes."""
    _room(40)
    gb = buffers(1, [(8, 1)])
    put(gb, 0, torch.ones(1, 8, 1))
    for rows, cols in (((1 << 20) + 3, 4100), ((1 << 26) + 70, 3)):
        x = torch.randn(1, 1, cols, device="cuda").expand(1, rows, cols)
        kept = gb.checkpoint_store(x)
        back = gb.checkpoint_load(kept)
        assert torch.equal(back[0, 0].cpu().float(), held(x[0, :1].cpu())[0][0].float())
        for part in back.split(1 << 18, 1):
            assert bool((part == back[:, :1]).all())
        del kept, back
    rows = (1 << 24) + 5
    x = torch.randn(1, rows, 8, device="cuda", dtype=BF16)
    y = gb.norm(0, x)[0]
    half = rows // 2
    assert torch.equal(y[:, :half], gb.norm(0, x[:, :half])[0]) and torch.equal(y[:, half:], gb.norm(0, x[:, half:])[0])
    gb.close()


class Block:
    """A residual block of all workers: y = s + W2 act(W1 norm(s)), s = x + r, in the layers (gain, W1, b1, W2, b2) of a context."""

    def __init__(self, n, rows, d, wide, dtype, seed, name="gelu"):
        gen = torch.Generator().manual_seed(seed)
        self.n, self.rows, self.d, self.wide, self.dtype, self.name = n, rows, d, wide, dtype, name
        self.shapes = [(d, 1), (wide, d), (wide, 1), (d, wide), (d, 1)]
        self.gb = buffers(n, self.shapes)
        self.params = [(torch.randn(n, *s, generator=gen) * (0.3 / math.sqrt(s[1])) + (1 if k == 0 else 0)).float() for k, s in enumerate(self.shapes)]
        self.x, self.r = (torch.randn(n, rows, d, generator=gen).to(dtype) for _ in range(2))
        self.dy = (torch.randn(n, rows, d, generator=gen) / rows).to(dtype)
        for l, w in enumerate(self.params):
            put(self.gb, l, w)
        self.gb.q.normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
        self.xd, self.rd, self.dyd = self.x.cuda(), self.r.cuda(), self.dy.cuda()

    def step(self, eta=None):
        gb = self.gb
        h, z = gb.checkpoint(self.rows, self.d), gb.checkpoint(self.rows, self.wide)
        _, s, rstd = gb.norm(0, self.xd, residual=self.rd, keep=h)
        a = gb.linear(1, h, bias=2, act=self.name, keep=z, dtype=self.dtype)
        y = gb.linear(3, a, bias=4, residual=s)
        dz = gb.linear_backward(3, self.dyd, a, bias=4, act=self.name, z=z)
        dh = gb.linear_backward(1, dz, h, bias=2)
        ds = gb.norm_backward(0, dh, s, rstd, residual=self.dyd)
        if eta is not None:
            gb.round_sgd(eta)
        return y, ds

    def oracle(self):
        """The same block in 64 bits by autograd, its 8-bit values in the places where the library keeps them: the forward pass sees norm(s) in
        8 bits, the activation's slope z in 8 bits."""
        p = [w.double().requires_grad_(True) for w in self.params]
        s = (self.x.double() + self.r.double()).float().to(self.dtype).double().requires_grad_(True)
        hn = s / torch.sqrt(s.square().mean(-1, keepdim=True) + 1e-6) * p[0].transpose(1, 2)
        h = hn + (held(hn.detach())[0] - hn.detach())
        z = h @ p[1].transpose(1, 2) + p[2].transpose(1, 2)
        z8 = held(z.detach())[0]
        a = act(self.name, z).detach() + slope(self.name, z8) * (z - z.detach())
        y = a @ p[3].transpose(1, 2) + p[4].transpose(1, 2) + s
        (y * self.dy.double()).sum().backward()
        return y.detach(), s.grad, [w.grad for w in p]


def near(got, want, dtype):
    """In norm.  bf16: each of at most eight steps of the chain rounds by 2^-8 at most, two operands at a time.  float: a value of either 8-bit
    checkpoint may fall on the other side of a border, one in 1e5 by 2^-3 of itself; 1e-3 is far more than that and far less than any mistake."""
    got, want = got.cpu().double(), want.double()
    assert float((got - want).norm()) <= (16 * 2.0 ** -8 if dtype == BF16 else 1e-3) * float(want.norm())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,rows,d,wide", [(4, 50, 96, 160), (3, 7, 33, 70), (2, 200, 64, 300)])
def test_a_training_step_of_all_of_them(n, rows, d, wide, dtype):
    """Forward, backward and the gossip round that takes the gradients: the round's parameters are those of the same round on the 64-bit gradients."""
    blk = Block(n, rows, d, wide, dtype, seed=rows)
    y, ds = blk.step()
    want_y, want_ds, want_g = blk.oracle()
    near(y, want_y, dtype), near(ds, want_ds, dtype)
    for l in range(5):
        near(grad(blk.gb, l), want_g[l], dtype)
    other = Block(n, rows, d, wide, dtype, seed=rows)
    for l in range(5):
        for i in range(n):
            other.gb.set_grad_layer(i, l, want_g[l][i].float().numpy())
    eta = 0.5
    before = [blk.gb.layer_of(torch.stack(blk.gb.x), l).cpu().double() for l in range(5)]
    blk.gb.round_sgd(eta), other.gb.round_sgd(eta)
    for l in range(5):
        got, want = (blk.gb.layer_of(torch.stack(g.x), l).cpu().double() for g in (blk.gb, other.gb))
        moved = eta * want_g[l]
        assert float((got - want).norm()) <= (16 * 2.0 ** -8 if dtype == BF16 else 1e-3) * float(moved.norm()) + 1e-6 * float(before[l].norm())
        assert float((want - before[l]).norm()) > 0
    blk.gb.close(), other.gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_replays_of_a_captured_step_equal_the_direct_call(dtype):
    """A whole step in a graph, replayed between eager steps on other inputs: the same bits every time; two graphs have workspaces of their own."""
    blk = Block(3, 200, 64, 130, dtype, seed=5)
    y, ds = blk.step()
    torch.cuda.synchronize()
    want = [y.clone(), ds.clone()] + [g.clone() for g in blk.gb.g]
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = blk.step()
        graphs.append((graph, outs))
    x = blk.xd.clone()
    for replay in range(3):
        for graph, outs in graphs:
            for g in blk.gb.g:
                g.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            for got, ref in zip(list(outs) + blk.gb.g, want):
                for l in range(5) if got.dim() == 1 else [None]:
                    a, b = (got, ref) if l is None else (blk.gb.layer_of(t, l) for t in (got, ref))
                    assert torch.equal(a, b), f"replay {replay}"
            blk.xd.mul_(0.5)
            blk.step()
            blk.xd.copy_(x)
            torch.cuda.synchronize()
    blk.gb.close()


def test_a_stream_of_the_callers():
    blk = Block(2, 150, 64, 100, BF16, seed=6)
    y, ds = blk.step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    gb = blk.gb
    with torch.cuda.stream(s):
        y2, ds2 = blk.step()
    h = gb.checkpoint_store(blk.xd, stream=s)
    back = gb.checkpoint_load(h, dtype=F32, stream=s)
    s.synchronize()
    assert torch.equal(y, y2) and torch.equal(ds, ds2)
    assert torch.equal(back.cpu(), held(blk.x)[0].float())
    gb.close()


def test_the_profile_names_them():
    blk = Block(2, 40, 64, 100, F32, seed=7)
    blk.step()
    B.pg_profile_enable(blk.gb.ctx, True)
    blk.step()
    got = {k["name"]: k for k in B.pg_profile_collect(blk.gb.ctx)}
    assert set(got) == {"norm", "linear", "linear_dx", "linear_dw", "norm_backward"}
    assert got["linear"]["launches"] == 2 and got["linear"]["bytes"] == 4.0 * 2 * 2 * 64 * 100 and got["linear_dw"]["ms"] > 0
    B.pg_profile_enable(blk.gb.ctx, False)
    blk.gb.close()


def test_what_the_python_side_refuses():
    gb = buffers(2, [(6, 5), (6, 1), (5, 1)])
    x = torch.zeros(2, 4, 5, device="cuda")
    for bad in (x.half(), x.double()):
        with pytest.raises(TypeError):
            gb.linear(0, bad)
    for bad in (torch.zeros(2, 4, 6, device="cuda"), torch.zeros(3, 4, 5, device="cuda"), torch.zeros(2, 4, 5), torch.zeros(2, 5, 4, device="cuda").transpose(1, 2)):
        with pytest.raises(ValueError):
            gb.linear(0, bad)
    with pytest.raises(ValueError):
        gb.linear(0, x[0])
    with pytest.raises(ValueError):
        gb.linear(0, x, residual=torch.zeros(2, 4, 6, device="cuda", dtype=BF16))
    with pytest.raises(ValueError):
        gb.linear(0, x, keep=gb.checkpoint(4, 5))
    with pytest.raises(ValueError):
        from paper_2008_01425_amd.device import Checkpoint
        gb.linear(0, x, keep=Checkpoint(2, 4, 6, torch.zeros(8, dtype=torch.uint8, device="cuda")))
    with pytest.raises(ValueError):
        gb.linear(0, x, counts=torch.zeros(2, device="cuda", dtype=torch.int64))
    with pytest.raises(ValueError):
        gb.norm(0, x)
    with pytest.raises(ValueError):
        gb.norm(2, x, rstd_out=torch.zeros(2, 5, device="cuda"))
    with pytest.raises(B.PGError):
        gb.linear(0, x, bias=2)
    with pytest.raises(B.PGError):
        gb.linear(0, x, out=torch.zeros(1, 1, 6, device="cuda").expand(2, 4, 6))     # an output that meets itself
    with pytest.raises(B.PGError):
        gb.linear_backward(0, torch.zeros(2, 4, 6, device="cuda"), None)
    with pytest.raises(B.PGError):
        gb.activation_backward("none", x, gb.checkpoint(4, 5))
    gb.close()
