"""Losses and their gradients against the formulas in 64 bits: labels, a teacher's top logits, both; entries and rows that do not exist."""
import math

import pytest
import torch

from rows_util import HALF, buffers, mask

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def statement(z, labels, hard, index, teacher, temperature, soft, weights):
    """(loss, gradient, what float arithmetic may put each off by), row by row in 64 bits."""
    n, rows, cols = z.shape
    loss, dz, off_l, off_g = (torch.zeros(s, dtype=torch.float64) for s in ((n, rows), (n, rows, cols), (n, rows), (n, rows, cols)))
    line = 8 * max(20, math.ceil(cols / 8192)) + 40    # roundings on an element's way into its row's sum: those in a lane (20 eights, or all), across lanes and wavefronts, a few more

    def softmax(x):
        """(distribution, log sum, distances, relative error of an entry of the distribution, of the sum)"""
        d = x - x.max()
        e = torch.exp(d)
        near = torch.where(e > 0, d, 0.0).abs()
        off = U * (4 * near + 4)                       # distance, its product with log2(e) / temperature, the exponential itself
        s = e.sum()
        off_s = float((e * off).sum() / s) + U * line
        return e / s, torch.log(s), d, off + off_s + 2 * U, off_s
    for i in range(n):
        for t in range(rows):
            w = 1.0 if weights is None else float(weights[i, t])
            if w == 0:
                continue
            c = -1 if labels is None else int(labels[i, t])
            if hard and 0 <= c < cols:
                s, log_s, d, off, off_s = softmax(z[i, t])
                loss[i, t] += w * hard * (log_s - d[c])
                off_l[i, t] += abs(w * hard) * (off_s + U * (4 * abs(log_s) + 2 * abs(d[c]) + 4 * abs(log_s - d[c])))
                dz[i, t] += w * hard * s
                dz[i, t, c] -= w * hard
                off_g[i, t] += abs(w * hard) * s * (off + 4 * U)
                off_g[i, t, c] += abs(w * hard) * 2 * U
            if index is None or not soft:
                continue
            there = [j for j in range(index.shape[-1]) if 0 <= int(index[i, t, j]) < cols and float(teacher[i, t, j]) > -math.inf]
            if not there:
                continue
            at = index[i, t, there].long()
            p, log_p, dp, off_p, off_sp = softmax(teacher[i, t, there].double() / temperature)
            q, log_q, d, off, off_s = softmax(z[i, t] / temperature)
            a, b = dp - log_p, d[at] - log_q
            u = w * soft * temperature
            part = torch.where(p > 0, p * (a - b), 0.0)
            loss[i, t] += u * temperature * part.sum()
            size = 6 * (dp.abs() + log_p.abs() + torch.where(p > 0, d[at], 0.0).abs() + log_q.abs())
            off_l[i, t] += abs(u * temperature) * ((p * (U * size + off_s + off_sp) + part.abs() * (off_p + (len(there) + 6) * U)).sum() + 4 * U * part.abs().sum())
            dz[i, t] += u * q
            dz[i, t].index_add_(0, at, -u * p)
            off_g[i, t] += abs(u) * q * (off + 6 * U)
            off_g[i, t].index_add_(0, at, abs(u) * p * (off_p + (len(there) + 6) * U))
    off_g += 2 * U * dz.abs()                           # two parts added
    return loss, dz, off_l + 2 * U * loss.abs(), off_g


def inputs(gen, n, rows, cols, top, dtype):
    z = (2 * torch.randn(n, rows, cols, generator=gen)).to(dtype)
    labels = torch.randint(0, cols, (n, rows), generator=gen, dtype=torch.int32)
    index = torch.rand(n, rows, cols, generator=gen).topk(top, -1)[1].int() if top else None
    teacher = 2 * torch.randn(n, rows, top, generator=gen) if top else None
    weights = torch.rand(n, rows, generator=gen) + 0.5
    return z, labels, index, teacher, weights


def cuda(x):
    return None if x is None else x.cuda()


def check(gb, z, labels, index, teacher, weights, temperature, hard, soft, counts=None):
    n, rows, cols = z.shape
    dtype = z.dtype
    there = mask(n, rows, counts)
    out, loss_out = torch.full((n, rows, cols), 7.0, dtype=dtype, device="cuda"), torch.full((n, rows), 7.0, device="cuda")
    loss, dz = gb.distill(z.cuda(), cuda(index), cuda(teacher), cuda(labels), temperature=temperature, hard=hard, soft=soft, weights=cuda(weights),
                          counts=counts, out=out, loss_out=loss_out)
    loss, dz = loss.cpu().double(), dz.cpu().double()
    want_l, want, off_l, off = statement(z.double(), labels, hard, index, teacher, temperature, soft, weights)
    least = 2.0 ** -120                            # what is below the smallest floats
    assert bool(((loss - want_l).abs() <= off_l + least)[there[..., 0]].all()), float((loss - want_l).abs().max())
    assert bool(((dz - want).abs() <= off + HALF[dtype] * (want.abs() + off) + least)[there.expand_as(want)].all())
    assert bool((dz[~there.expand_as(want)] == 7).all()) and bool((loss[~there[..., 0]] == 7).all())
    alone, none = gb.distill(z.cuda(), cuda(index), cuda(teacher), cuda(labels), temperature=temperature, hard=hard, soft=soft, weights=cuda(weights),
                             counts=counts, want_grad=False)
    assert none is None and torch.equal(alone.cpu().double()[there[..., 0]], loss[there[..., 0]])
    return loss, dz


SIZES = [(1, 1, 1, 1), (3, 5, 2, 2), (2, 40, 10, 3), (3, 7, 127, 8), (2, 9, 128, 128), (2, 9, 129, 20), (1, 6, 512, 32), (2, 5, 513, 64), (1, 5, 2048, 128),
         (2, 3, 2049, 1), (1, 3, 8192, 1024), (1, 3, 8193, 33), (2, 2, 16384, 20), (1, 3, 16385, 65), (1, 2, 33278, 32), (1, 2, 40960, 5), (1, 2, 40961, 7),
         (2, 1, 150001, 50)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,rows,cols,top", SIZES)
def test_losses_and_gradients(n, rows, cols, top, dtype):
    print("case", n, rows, cols, top, dtype, flush=True)
    gen = torch.Generator().manual_seed(cols + top)
    gb = buffers(n, [(4, 4)])
    z, labels, index, teacher, weights = inputs(gen, n, rows, cols, top, dtype)
    counts = torch.tensor([max(0, rows - i) for i in range(n)], dtype=torch.int32, device="cuda")
    check(gb, z, labels, index, teacher, weights, 2.0, 0.5, 0.75)                    # both, two temperatures
    check(gb, z, labels, index, teacher, None, 1.0, 1.0, 1.0, counts)                # both, one
    check(gb, z, labels, None, None, weights, 1.0, 0.25, 1.0, counts)                # cross entropy
    check(gb, z, None, index, teacher, weights, 3.5, 1.0, 1.0)                       # the teacher alone
    check(gb, z, labels, index, teacher, weights, 0.5, 0.0, -1.5)                    # a label that counts nothing
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols,top", [(600, 3), (1024, 256), (1025, 257), (2048, 20), (2049, 5), (4096, 256), (4097, 1024), (8192, 8), (8193, 20), (16384, 1), (16385, 32),
                                      (24576, 9), (24577, 10), (32768, 11), (33278, 32), (36865, 12), (40960, 13), (40961, 14), (65536, 15), (65537, 16)])
def test_among_many_rows(cols, top, dtype):
    """Where there are more rows than a chip takes at once, fewer lanes share one; a few of them exist."""
    print("case", cols, top, dtype, flush=True)
    n, rows = 3, 200
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(n, [(4, 4)])
    there = [4, 0, 2]
    z = torch.zeros(n, rows, cols, dtype=dtype)
    z[:, :4] = (2 * torch.randn(n, 4, cols, generator=gen)).to(dtype)
    labels = torch.randint(0, cols, (n, rows), generator=gen, dtype=torch.int32)
    index = torch.zeros(n, rows, top, dtype=torch.int32)
    index[:, :4] = torch.rand(n, 4, cols, generator=gen).topk(top, -1)[1].int()
    index[0, 1, -1] = int(labels[0, 1])
    teacher, weights = 2 * torch.randn(n, rows, top, generator=gen), torch.rand(n, rows, generator=gen) + 0.5
    weights[2, 1] = 0.0
    counts = torch.tensor(there, dtype=torch.int32, device="cuda")

    def cut(t):
        return None if t is None else t[:, :4]
    for how in (dict(labels=labels, index=index, teacher=teacher, temperature=2.0), dict(labels=labels, index=index, teacher=teacher, temperature=1.0),
                dict(labels=labels, index=None, teacher=None, temperature=1.0)):
        out, loss_out = torch.full((n, rows, cols), 7.0, dtype=dtype, device="cuda"), torch.full((n, rows), 7.0, device="cuda")
        loss, dz = gb.distill(z.cuda(), cuda(how["index"]), cuda(how["teacher"]), labels.cuda(), temperature=how["temperature"], hard=0.5, soft=0.75,
                              weights=weights.cuda(), counts=counts, out=out, loss_out=loss_out)
        want_l, want, off_l, off = statement(z[:, :4].double(), cut(labels), 0.5, cut(how["index"]), cut(how["teacher"]), how["temperature"], 0.75, cut(weights))
        for i, count in enumerate(there):
            assert bool((dz[i, count:] == 7).all()) and bool((loss[i, count:] == 7).all())
            got, l = dz[i, :count].cpu().double(), loss[i, :count].cpu().double()
            assert bool(((l - want_l[i, :count]).abs() <= off_l[i, :count] + 2.0 ** -120).all())
            w, o = want[i, :count], off[i, :count]
            assert bool(((got - w).abs() <= o + HALF[dtype] * (w.abs() + o) + 2.0 ** -120).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols,top", [(12, 12), (300, 90), (3000, 200), (50000, 64)])
def test_entries_that_repeat_or_do_not_exist(cols, top, dtype):
    """The same class several times, the label among them or not, classes out of range, logits of -infinity, rows without any entry or label."""
    n, rows = 2, 8
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(n, [(4, 4)])
    z, labels, index, teacher, weights = inputs(gen, n, rows, cols, top, dtype)
    index = index % min(cols, 7) if cols > 12 else index % 5                          # each class many times
    index[0, 1, ::2], index[0, 2, 1::2] = -1, cols
    index[0, 3], labels[0, 4], labels[0, 3] = -5, cols, -1                            # no entries and no label; entries without a label
    teacher[1, 0, ::3] = -math.inf
    teacher[1, 1] = -math.inf
    index[1, 2], teacher[1, 2] = int(labels[1, 2]), 0.0                               # nothing but the label
    weights[1, 3] = 0.0
    index[1, 4, 1:] = -7                                                              # one entry
    index[1, 5], labels[1, 5] = -2 ** 31, 2 ** 31 - 1
    loss, dz = check(gb, z, labels, index, teacher, weights, 2.0, 0.5, 0.75)
    for i, t in ((0, 3), (1, 3), (1, 5)):
        assert loss[i, t] == 0 and not dz[i, t].any()
    check(gb, z, labels, index, teacher, weights, 1.0, 0.5, 0.75)
    check(gb, z, None, index, teacher, weights, 1.5, 0.0, 1.0)
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [9, 400, 1500, 33278, 60000])
def test_what_is_not_finite(cols, dtype):
    n, rows, top = 1, 9, 3
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(n, [(4, 4)])
    z, labels, index, teacher, weights = inputs(gen, n, rows, cols, top, dtype)
    for t in range(rows):
        labels[0, t], index[0, t] = 0, torch.tensor([1, 2, 3])
    z[0, 0, 5], z[0, 1, 5], z[0, 2], z[0, 3, 5:] = math.nan, math.inf, -math.inf, -math.inf
    z[0, 4, 0], z[0, 5, 2], teacher[0, 6, 1], z[0, 7], weights[0, 7] = -math.inf, -math.inf, math.nan, math.nan, 0.0
    labels[0, 8], index[0, 8], z[0, 8, 4] = -1, -1, math.nan                          # neither label nor entry: not a part of the loss
    args = [cuda(t) for t in (z, index, teacher, labels)]
    loss, dz = (t.cpu().double() for t in gb.distill(*args, temperature=2.0, hard=0.5, soft=0.5, weights=weights.cuda()))
    for t in (0, 1, 2, 6):
        assert math.isnan(loss[0, t]), t
    for t in (0, 1, 2):
        assert bool(dz[0, t].isnan().all()), t
    assert bool(dz[0, 6, 1:4].isnan().all())
    for t in (7, 8):
        assert loss[0, t] == 0 and not dz[0, t].any()
    want_l, want, off_l, off = statement(z[:, 3:6].double(), labels[:, 3:6], 0.5, index[:, 3:6], teacher[:, 3:6], 2.0, 0.5, weights[:, 3:6])
    assert abs(loss[0, 3] - want_l[0, 0]) <= off_l[0, 0] and loss[0, 4] == math.inf and loss[0, 5] == math.inf
    assert not dz[0, 3, 5:].any()
    assert bool(((dz[:, 3:6] - want).abs() <= off + HALF[dtype] * (want.abs() + off)).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cols", [10, 333, 1777, 33278, 50003])
def test_in_place_and_strides(cols, dtype):
    n, rows, top = 2, 5, 4
    gen = torch.Generator().manual_seed(cols)
    gb = buffers(n, [(4, 4)])
    z, labels, index, teacher, weights = (cuda(t) for t in inputs(gen, n, rows, cols, top, dtype))
    how = dict(top_index=index, top_logits=teacher, labels=labels, weights=weights, temperature=2.0, hard=0.5, soft=0.5)
    loss, want = gb.distill(z, **how)
    wide = torch.full((rows, n, cols + 5), 9.0, dtype=dtype, device="cuda")
    view = wide[:, :, 3:cols + 3].transpose(0, 1)
    view.copy_(z)
    again, dz = gb.distill(view, out=view, **how)
    assert torch.equal(loss, again) and torch.equal(dz, want)
    assert bool((wide[:, :, :3] == 9).all()) and bool((wide[:, :, cols + 3:] == 9).all())
    one = z[:1, :1].expand(n, rows, cols)
    assert torch.equal(gb.distill(one, **how)[1], gb.distill(one.contiguous(), **how)[1])
    empty, none = gb.distill(z[:, :0], labels=labels[:, :0].contiguous())
    assert empty.shape == (n, 0) and none.shape == (n, 0, cols)
    gb.close()


def test_gradient_against_differences():
    n, rows, cols, top = 1, 2, 9, 3
    gen = torch.Generator().manual_seed(9)
    gb = buffers(n, [(4, 4)])
    z, labels, index, teacher, weights = inputs(gen, n, rows, cols, top, F32)
    _, dz = gb.distill(z.cuda(), index.cuda(), teacher.cuda(), labels.cuda(), temperature=2.0, hard=0.5, soft=0.5, weights=weights.cuda())
    want = torch.zeros(z.shape, dtype=torch.float64)
    for k in range(z.numel()):
        ends = []
        for step in (1e-4, -1e-4):
            moved = z.double()
            moved.view(-1)[k] += step
            ends.append(statement(moved, labels, 0.5, index, teacher, 2.0, 0.5, weights)[0].sum())
        want.view(-1)[k] = (ends[0] - ends[1]) / 2e-4
    # central differences are off by 1e-8 / 6 times the third derivative, which is below 1 for either part here; and some tens of float roundings
    assert bool(((dz.cpu().double() - want).abs() <= 1e-8 + 100 * U).all())
    gb.close()


def test_arguments_are_checked():
    gb = buffers(2, [(4, 4)])
    z = torch.zeros(2, 3, 10, device="cuda")
    index, teacher, labels = torch.zeros(2, 3, 2, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, 2, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    for how in (dict(top_index=index), dict(top_logits=teacher), dict(top_index=index.long(), top_logits=teacher), dict(top_index=index, top_logits=teacher.bfloat16()),
                dict(top_index=index[:, :2], top_logits=teacher), dict(labels=labels.long()), dict(labels=labels[:1]), dict(labels=labels.cpu()),
                dict(labels=labels, weights=labels), dict(labels=labels, loss_out=teacher), dict(labels=labels, out=z.bfloat16()),
                dict(top_index=index.transpose(0, 1).contiguous().transpose(0, 1), top_logits=teacher)):
        with pytest.raises(ValueError):
            gb.distill(z, **how)
    gb.close()
