"""Attention to an encoder's states against its formulas in 64 bits, forward and backward: lengths from one position and state to splits of many, odd widths, shared
heads, states and positions that do not exist, masks that leave nothing."""
import math

import pytest
import torch

from rows_util import HALF, buffers

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
# workers, sequences, positions, states, heads, key heads, width
SIZES = [(1, 1, 1, 1, 1, 1, 1), (2, 2, 3, 5, 2, 1, 16), (1, 3, 33, 65, 4, 2, 37), (2, 1, 7, 130, 8, 8, 64), (1, 2, 140, 70, 6, 2, 80), (1, 1, 300, 513, 2, 2, 128),
         (2, 1, 1, 1000, 16, 4, 128), (1, 1, 2, 700, 8, 1, 192), (1, 1, 65, 200, 3, 3, 256), (1, 2, 200, 3, 4, 1, 65), (3, 2, 40, 64, 4, 4, 96),
         (1, 1, 1, 4100, 8, 2, 256), (1, 1, 4000, 40, 2, 1, 32), (1, 1, 30, 2000, 2, 2, 15), (2, 1, 129, 127, 2, 1, 33), (1, 1, 128, 128, 1, 1, 2), (1, 1, 20, 333, 2, 1, 160)]


class Case:
    def __init__(self, size, dtype, ragged, masked, seed=0, spread=1.0):
        n, B, T, S, H, G, d = self.size = size
        gen = torch.Generator().manual_seed(sum(size) + seed)
        self.dtype, self.scale = dtype, spread / math.sqrt(d)

        def rows(count, cols):
            return torch.randn(n, B * count, cols, generator=gen).to(dtype)
        self.q, self.k, self.v, self.dy = rows(T, H * d), rows(S, G * d), rows(S, G * d), rows(T, H * d)
        self.counts = self.states = self.mask = None
        if ragged:
            self.counts = torch.randint(0, T + 1, (n * B,), generator=gen, dtype=torch.int32)
            self.states = torch.randint(0, S + 1, (n * B,), generator=gen, dtype=torch.int32)
            self.counts[0], self.states[0] = T, S
            if n * B > 2:
                self.states[1], self.counts[2] = 0, 0
        if masked:
            self.mask = (torch.rand(n * B, S, generator=gen) > 0.4).to(torch.uint8)
            if n * B > 1:
                self.mask[-1] = 0

    def asked(self, b):
        return self.size[2] if self.counts is None else int(self.counts[b])

    def seen(self, b):
        S = self.size[3]
        seen = torch.arange(S) < (S if self.states is None else int(self.states[b]))
        return seen if self.mask is None else seen & (self.mask[b] != 0)

    def heads(self, x, which):
        """(sequences, length, heads, width) in double"""
        n, B, T, S, H, G, d = self.size
        return x.double().view(n * B, *((T, H) if which == "q" else (S, G)), d)

    def how(self):
        n, B, T, S, H, G, d = self.size
        gpu = [None if t is None else t.cuda() for t in (self.counts, self.states, self.mask)]
        return dict(heads=H, kv_heads=G, sequences=B, scale=self.scale, counts=gpu[0], memory_counts=gpu[1], mask=gpu[2])

    def spoil(self):
        """What does not exist or is hidden is not a number."""
        n, B, T, S, H, G, d = self.size
        for b in range(n * B):
            self.q.view(n * B, T, -1)[b, self.asked(b):] = math.nan
            self.dy.view(n * B, T, -1)[b, self.asked(b):] = math.nan
            for t in (self.k, self.v):
                t.view(n * B, S, -1)[b, ~self.seen(b)] = math.nan

    def pairs(self):
        """Every sequence and query head: its index, rows that ask, states that are seen, key head."""
        n, B, T, S, H, G, d = self.size
        for b in range(n * B):
            for h in range(H):
                yield b, h, h // (H // G), slice(0, self.asked(b)), self.seen(b).nonzero()[:, 0]

    def score(self, q, k):
        """Scores and what float may put each off by: a sum of `width` products, the scale, its logarithm's base."""
        s = q @ k.t() * self.scale
        return s, self.scale * (self.size[6] + 2) * U * (q.abs() @ k.abs().t()) + 4 * U * s.abs()


def weight_error(case, s, off, lse):
    """Relative: the score's distance to the sum, formed in logarithms to the base 2, and the exponential itself."""
    return off + U * (4 * (s - lse).abs() + 3 * s.abs() + 3 * lse.abs() + 8)


def forward(case, spoiled=True):
    n, B, T, S, H, G, d = case.size
    gb = buffers(n, [(4, 4)])
    if spoiled:
        case.spoil()
    out, lse_out = torch.full((n, B * T, H * d), 7.0, dtype=case.dtype, device="cuda"), torch.full((n, B * T, H), 7.0, device="cuda")
    y, lse = gb.attention(case.q.cuda(), case.k.cuda(), case.v.cuda(), out=out, lse_out=lse_out, **case.how())
    return gb, y.cpu(), lse.cpu()


def rounding(case, p):
    """Of a weight to the activations' type, where that is not float."""
    return HALF[BF16] * p if case.dtype == BF16 else 0.0


@pytest.mark.parametrize("ragged,masked", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, dtype, ragged, masked):
    print("case", size, dtype, ragged, masked, flush=True)
    case = Case(size, dtype, ragged, masked)
    n, B, T, S, H, G, d = size
    gb, y, lse = forward(case)
    ys, sums = case.heads(y, "q"), lse.double().view(n * B, T, H)
    q, k, v = case.heads(case.q, "q"), case.heads(case.k, "k"), case.heads(case.v, "k")
    for b, h, g, rows, seen in case.pairs():
        assert bool((ys[b, case.asked(b):, h] == 7).all()) and bool((sums[b, case.asked(b):, h] == 7).all())
        if seen.numel() == 0:
            assert not ys[b, rows, h].any() and bool((sums[b, rows, h] == -math.inf).all())
            continue
        s, off = case.score(q[b, rows, h], k[b, seen, g])
        want_lse = torch.logsumexp(s, 1, keepdim=True)
        p = torch.exp(s - want_lse)
        e = weight_error(case, s, off, want_lse)
        # of the sum: that of its terms, and its additions, which go one after the other in two halves
        e_sum = (p * e).sum(1, keepdim=True) + (seen.numel() / 2 + 80) * U
        assert bool(((sums[b, rows, h, None] - want_lse).abs() <= e_sum + 3 * U * want_lse.abs() + 4 * U * s.abs().amax(1, keepdim=True)).all())
        want = p @ v[b, seen, g]
        off = (p * (e + e_sum) + rounding(case, p) + (seen.numel() + 80) * U * p) @ v[b, seen, g].abs()
        assert bool(((ys[b, rows, h] - want).abs() <= off + HALF[dtype] * (want.abs() + off)).all()), (b, h)
    gb.close()


@pytest.mark.parametrize("ragged,masked", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_backward(size, dtype, ragged, masked):
    print("case", size, dtype, ragged, masked, flush=True)
    case = Case(size, dtype, ragged, masked, seed=1)
    n, B, T, S, H, G, d = size
    gb, y, lse = forward(case)
    for b in range(n * B):
        y.view(n * B, T, -1)[b, case.asked(b):] = math.nan
        lse.view(n * B, T, H)[b, case.asked(b):] = math.nan
    inputs = [t.cuda() for t in (case.dy, case.q, case.k, case.v, y, lse)]
    outs = [torch.full(t.shape, 7.0, dtype=dtype, device="cuda") for t in (case.q, case.k, case.v)]
    got = [t.cpu() for t in gb.attention_backward(*inputs, dq=outs[0], dk=outs[1], dv=outs[2], **case.how())]
    alone = gb.attention_backward(*inputs, want_dkv=False, **case.how())
    assert alone[1] is None and alone[2] is None
    states = gb.attention_backward(*inputs, want_dq=False, **case.how())
    assert states[0] is None
    dq, dk, dv = case.heads(got[0], "q"), case.heads(got[1], "k"), case.heads(got[2], "k")
    q, k, v, dy, ys = case.heads(case.q, "q"), case.heads(case.k, "k"), case.heads(case.v, "k"), case.heads(case.dy, "q"), case.heads(y, "q")
    sums = lse.double().view(n * B, T, H)
    want_k, want_v, off_k, off_v = (torch.zeros(n * B, S, G, d, dtype=torch.float64) for _ in range(4))
    for b, h, g, rows, seen in case.pairs():
        assert bool((dq[b, case.asked(b):, h] == 7).all())
        there = torch.arange(S) < (S if case.states is None else int(case.states[b]))
        assert bool((dk[b, ~there] == 7).all()) and bool((dv[b, ~there] == 7).all())
        if seen.numel() == 0:
            assert not dq[b, rows, h].any()
            continue
        qs, ks, vs, ds = q[b, rows, h], k[b, seen, g], v[b, seen, g], dy[b, rows, h]
        s, off = case.score(qs, ks)
        at = sums[b, rows, h, None]
        p = torch.exp(s - at)
        e = weight_error(case, s, off, at)
        dp, delta = ds @ vs.t(), (ds * ys[b, rows, h]).sum(1, keepdim=True)
        off_d = (d + 2) * U * (ds * ys[b, rows, h]).abs().sum(1, keepdim=True)
        if (S if case.states is None else int(case.states[b])) <= 32:
            # from the weights: each off by its own error and its product's, at most 32 + 2 additions
            delta = (p * dp).sum(1, keepdim=True)
            off_d = (p * (dp.abs() * (e + 36 * U) + (d + 2) * U * (ds.abs() @ vs.abs().t()))).sum(1, keepdim=True)
        off_p = (d + 2) * U * (ds.abs() @ vs.abs().t()) + off_d + 2 * U * (dp - delta).abs()
        grad = p * (dp - delta)
        off_g = p * ((dp - delta).abs() * e + off_p) + rounding(case, grad.abs())
        adds = (seen.numel() + 80) * U
        want = case.scale * grad @ ks
        off_q = case.scale * (off_g + adds * grad.abs()) @ ks.abs() + 3 * U * want.abs()
        assert bool(((dq[b, rows, h] - want).abs() <= off_q + HALF[dtype] * (want.abs() + off_q)).all()), (b, h)
        adds = (case.asked(b) * (H // G) + 80) * U
        want_k[b, :, g].index_add_(0, seen, case.scale * grad.t() @ qs)
        off_k[b, :, g].index_add_(0, seen, case.scale * (off_g + (adds + 3 * U) * grad.abs()).t() @ qs.abs())
        want_v[b, :, g].index_add_(0, seen, p.t() @ ds)
        off_v[b, :, g].index_add_(0, seen, (p * (e + adds) + rounding(case, p)).t() @ ds.abs())
    for name, have, want, off in (("dk", dk, want_k, off_k), ("dv", dv, want_v, off_v)):
        for b in range(n * B):
            count = S if case.states is None else int(case.states[b])
            w, o = want[b, :count], off[b, :count]
            assert bool(((have[b, :count] - w).abs() <= o + HALF[dtype] * (w.abs() + o)).all()), (name, b)
            assert not have[b, :count][~case.seen(b)[:count]].any()
    for b in range(n * B):       # each gradient alone: the same bits where there are any
        assert torch.equal(alone[0].cpu().view(n * B, T, -1)[b, :case.asked(b)], got[0].view(n * B, T, -1)[b, :case.asked(b)])
    for one, both in ((states[1], got[1]), (states[2], got[2])):
        diff = (one.cpu().double() - both.double()).abs()
        kept = both != 7
        # dy . y comes from a kernel of its own there, and may differ in its last bits
        assert bool((diff[kept] <= 1e-2 * both.double().abs().amax() + 1e-30).all())
    gb.close()


@pytest.mark.parametrize("splits", [1, 3, 64])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(1, 2, 50, 700, 4, 2, 40), (2, 1, 300, 270, 2, 1, 128), (1, 1, 3, 4500, 2, 1, 96), (1, 1, 700, 260, 1, 1, 200), (1, 3, 129, 400, 6, 2, 25),
                                  (8, 1, 20, 300, 2, 2, 64), (1, 1, 150, 600, 1, 1, 256)])
def test_parts(size, dtype, splits):
    """The other side in one part, a few, or as many as there are steps for; parts without any state among them."""
    from parity_util import env_settings
    with env_settings(dict(PG_ATTENTION_SPLITS=splits)):
        test_forward(size, dtype, True, False)
        test_forward(size, dtype, False, True)
        test_backward(size, dtype, True, False)
        test_backward(size, dtype, False, True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,S,H,G,d", [(5, 64, 4, 2, 48), (200, 256, 2, 1, 130), (1, 2048, 8, 8, 64), (40, 512, 1, 1, 256)])
def test_equal_weights_are_exact(T, S, H, G, d, dtype):
    """Queries of zeros weigh a power of two of states alike: means of integers, sums of integers; every element has one right value."""
    gen = torch.Generator().manual_seed(S)
    gb = buffers(2, [(4, 4)])
    k = torch.randn(2, S, G * d, generator=gen).to(dtype)
    v = torch.randint(-8, 9, (2, S, G * d), generator=gen).to(dtype)
    dy = torch.randint(-8, 9, (2, T, H * d), generator=gen).to(dtype)
    q = torch.zeros(2, T, H * d, dtype=dtype)
    y, lse = gb.attention(q.cuda(), k.cuda(), v.cuda(), H, G)
    mean = v.double().view(2, S, G, d).mean(1).repeat_interleave(H // G, 1).view(2, 1, H * d)
    assert torch.equal(y.cpu(), mean.float().to(dtype).expand_as(y)) and bool(((lse.cpu().double() - math.log(S)).abs() <= 4 * U * math.log(S)).all())
    # dv sums 1 / S of each integer: lse's logarithm and its exponential are off by some units of float
    _, dk, dv = (t.cpu().double() for t in gb.attention_backward(dy.cuda(), q.cuda(), k.cuda(), v.cuda(), y, lse, H, G))
    want = dy.double().view(2, T, G, H // G, d).sum((1, 3)).view(2, 1, G * d) / S
    size = dy.double().abs().view(2, T, G, H // G, d).sum((1, 3)).view(2, 1, G * d) / S
    assert bool(((dv - want).abs() <= (32 + T * H) * U * size + rounding_of(dtype) * size + HALF[dtype] * (want.abs() + size * HALF[dtype])).all())
    assert not dk.any()
    gb.close()


def rounding_of(dtype):
    return HALF[BF16] if dtype == BF16 else 0.0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_scores(dtype):
    """Scores of hundreds, growing along the states: the running maximum moves many times; one state in the end takes it all."""
    n, T, S, d = 1, 70, 600, 64
    gen = torch.Generator().manual_seed(3)
    gb = buffers(n, [(4, 4)])
    q = torch.ones(n, T, d).to(dtype)
    k = (torch.arange(S).view(1, S, 1) * 0.5).expand(n, S, d).contiguous().to(dtype)
    v = torch.randn(n, S, d, generator=gen).to(dtype)
    for order in (torch.arange(S), torch.arange(S - 1, -1, -1), torch.randperm(S, generator=gen)):
        y, lse = gb.attention(q.cuda(), k[:, order].contiguous().cuda(), v[:, order].contiguous().cuda(), 1)
        s = (q.double() @ k.double()[:, order].transpose(1, 2)) / 8
        p = torch.softmax(s, -1)
        want = p @ v.double()[:, order]
        # scores below 2^12, sums of 64 products of one sign: each off by at most 68 units of float of itself
        e = 140 * U * s.abs().amax()
        assert bool(((lse.cpu().double() - torch.logsumexp(s, -1).view(n, T, 1)).abs() <= e).all())
        off = (2 * e + 1000 * U + rounding_of(dtype)) * (p @ v.double()[:, order].abs())
        assert bool(((y.cpu().double() - want).abs() <= off + HALF[dtype] * want.abs() * 2).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_is_not_finite(dtype):
    """NaN and infinities reach the positions and states that meet them, and no others."""
    size = (1, 2, 40, 70, 2, 1, 24)
    case = Case(size, dtype, False, False, seed=4)
    gb, clean, _ = forward(case)
    case.q.view(2, 40, 2, 24)[0, 3, 1, 5] = math.nan
    case.k.view(2, 70, 24)[1, 69, 0] = math.nan
    y, lse = (t.cpu() for t in gb.attention(case.q.cuda(), case.k.cuda(), case.v.cuda(), **case.how()))
    ys, before = y.view(2, 40, 2, 24), clean.view(2, 40, 2, 24)
    assert bool(ys[1].isnan().all()) and bool(ys[0, 3, 1].isnan().all()) and bool(lse.view(2, 40, 2)[0, 3, 1].isnan())
    good = torch.ones(40, 2, dtype=torch.bool)
    good[3, 1] = False
    assert torch.equal(ys[0][good], before[0][good])
    case.k.view(2, 70, 24)[1, 69, 0] = 0.0
    case.v.view(2, 70, 24)[1, 7, 11] = math.inf
    y = gb.attention(case.q.cuda(), case.k.cuda(), case.v.cuda(), **case.how())[0].cpu().view(2, 40, 2, 24)
    assert bool((y[1, :, :, 11] == math.inf).all()) and bool(y[1][..., torch.arange(24) != 11].isfinite().all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    """Keys and values side by side in one tensor at odd places, workers inside rows, states that all sequences share."""
    size = n, B, T, S, H, G, d = (2, 2, 30, 50, 4, 2, 20)
    case = Case(size, dtype, False, True, seed=5)
    gb = buffers(n, [(4, 4)])
    q, k, v, dy = (t.cuda() for t in (case.q, case.k, case.v, case.dy))
    y, lse = gb.attention(q, k, v, **case.how())
    dq, dk, dv = gb.attention_backward(dy, q, k, v, y, lse, **case.how())

    def wide(x, at, width):
        w = torch.full((x.shape[1], n, width), 9.0, dtype=dtype, device="cuda")
        view = w[:, :, at:at + x.shape[2]].transpose(0, 1)
        view.copy_(x)
        return w, view
    both, _ = wide(torch.zeros(n, B * S, 1, device="cuda", dtype=dtype), 0, 2 * G * d + 7)
    keys, values = both[:, :, 1:1 + G * d].transpose(0, 1), both[:, :, 3 + G * d:3 + 2 * G * d].transpose(0, 1)
    keys.copy_(k), values.copy_(v)
    _, qv = wide(q, 3, H * d + 5)
    outs = [wide(t * 0, 1, t.shape[2] + 3) for t in (q, q, k, v)]
    y2, lse2 = gb.attention(qv, keys, values, out=outs[0][1], **case.how())
    assert torch.equal(y2, y) and torch.equal(lse2, lse)
    got = gb.attention_backward(wide(dy, 1, H * d + 1)[1], qv, keys, values, y2, lse2, dq=outs[1][1], dk=outs[2][1], dv=outs[3][1], **case.how())
    for a, b in zip(got, (dq, dk, dv)):
        assert torch.equal(a, b)
    for w, view in outs:
        assert bool((w[:, :, 0] == 9).all()) and bool((w[:, :, 1 + view.shape[2]:] == 9).all())
    # the same states for all workers
    one = k[:1].expand(n, -1, -1), v[:1].expand(n, -1, -1)
    assert torch.equal(gb.attention(q, *one, **case.how())[0], gb.attention(q, *(t.contiguous() for t in one), **case.how())[0])
    gb.close()


def test_gradients_against_differences():
    """Of the sum of dy y, by central differences of the definition in 64 bits."""
    size = n, B, T, S, H, G, d = (1, 2, 3, 5, 4, 2, 6)
    case = Case(size, F32, False, True, seed=6)
    case.mask[:] = torch.tensor([1, 0, 1, 1, 0], dtype=torch.uint8)
    gb, y, lse = forward(case, spoiled=False)
    got = [t.cpu().double() for t in gb.attention_backward(*(t.cuda() for t in (case.dy, case.q, case.k, case.v, y, lse)), **case.how())]

    def loss(q, k, v):
        total = 0.0
        q, k, v = q.view(B, T, H, d), k.view(B, S, G, d), v.view(B, S, G, d)
        for b, h, g, rows, seen in case.pairs():
            total = total + ((torch.softmax(q[b, :, h] @ k[b, seen, g].t() * case.scale, 1) @ v[b, seen, g]) * case.heads(case.dy, "q")[b, :, h]).sum()
        return total
    args = [case.q.double(), case.k.double(), case.v.double()]
    for which, have in enumerate(got):
        want = torch.zeros_like(args[which])
        for i in range(want.numel()):
            ends = []
            for step in (1e-4, -1e-4):
                now = [t.clone() for t in args]
                now[which].view(-1)[i] += step
                ends.append(loss(*now))
            want.view(-1)[i] = (ends[0] - ends[1]) / 2e-4
        # differences: 1e-8 / 6 times a third derivative of some tens; the kernels: some hundreds of float roundings of terms of a few units
        assert bool(((have - want).abs() <= 1e-6 + 1000 * U).all())
    gb.close()


def test_the_same_call_gives_the_same_bits_and_empty_ones_nothing():
    case = Case((2, 2, 100, 300, 4, 1, 64), BF16, True, True, seed=7)
    gb, y, lse = forward(case)
    n, B, T, S, H, G, d = case.size
    again = gb.attention(case.q.cuda(), case.k.cuda(), case.v.cuda(), **case.how())
    for b in range(n * B):
        rows = slice(0, case.asked(b))
        assert torch.equal(again[0].cpu().view(n * B, T, -1)[b, rows], y.view(n * B, T, -1)[b, rows])
    inputs = [t.cuda() for t in (case.dy, case.q, case.k, case.v, y, lse)]
    first, second = (gb.attention_backward(*inputs, **case.how()) for _ in range(2))
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    q, none = case.q.cuda(), case.k.cuda()[:, :0]
    y, lse = gb.attention(q, none, none, H, G, sequences=B)
    assert not y.any() and bool((lse == -math.inf).all())
    dq, dk, dv = gb.attention_backward(q, q, none, none, y, lse, H, G, sequences=B)
    assert not dq.any() and dk.shape == none.shape
    nobody, k = q[:, :0], case.k.cuda()
    y, lse = gb.attention(nobody, k, k, H, G, sequences=B)
    assert y.shape == nobody.shape
    dq, dk, dv = gb.attention_backward(nobody, nobody, k, k, y, lse, H, G, sequences=B)
    assert not dk.any() and not dv.any() and dk.shape == k.shape
    gb.close()


def test_arguments_are_checked():
    gb = buffers(2, [(4, 4)])
    q, k = torch.zeros(2, 6, 32, device="cuda"), torch.zeros(2, 4, 16, device="cuda")
    ok = dict(heads=4, kv_heads=2, sequences=2)
    gb.attention(q, k, k, **ok)
    counts = torch.ones(4, dtype=torch.int32, device="cuda")
    for how in (dict(ok, heads=3), dict(ok, kv_heads=4), dict(ok, kv_heads=0), dict(ok, heads=0), dict(ok, sequences=4), dict(ok, sequences=0), dict(ok, heads=8),
                dict(ok, counts=counts.long()), dict(ok, counts=counts[:2]), dict(ok, memory_counts=counts.cpu()), dict(ok, mask=counts),
                dict(ok, mask=torch.ones(4, 3, dtype=torch.uint8, device="cuda")), dict(ok, out=k), dict(ok, lse_out=torch.zeros(2, 6, 2, device="cuda"))):
        with pytest.raises(ValueError):
            gb.attention(q, k, k, **how)
    for bad in ((q, k, k.bfloat16()), (q, k.cpu(), k), (q[0], k, k), (q, k, k[:, :2])):
        with pytest.raises(ValueError):
            gb.attention(*bad, **ok)
    from paper_2008_01425_amd import binding as B
    for scale in (0.0, -1.0, math.inf, math.nan):
        with pytest.raises(B.PGError):
            gb.attention(q, k, k, scale=scale, **ok)
    wide = torch.zeros(2, 3, 257, device="cuda")
    with pytest.raises(B.PGError):
        gb.attention(wide, wide, wide, heads=1)
    gb.close()


@pytest.mark.parametrize("S", [1, 5, 32])
@pytest.mark.parametrize("T,H,G,d", [(1, 2, 1, 192), (3, 4, 4, 37), (16, 4, 2, 64), (2, 2, 2, 128)])
def test_few_weights_keep_sixteen_bits(T, H, G, d, S):
    """Calls of few weights in bf16 are off by their results' own rounding (half a step of 2^-8) and by what two parts of a weight leave out of it: 2^-8 of 2^-8, doubled for
    the float roundings beside it (scores, exponentials, sums of 32: below 2^-18 of the sums of magnitudes)."""
    gen = torch.Generator().manual_seed(100 * S + T)
    n = 2
    q, dy = (torch.randn(n, T, H * d, generator=gen).bfloat16() for _ in range(2))
    k, v = (torch.randn(n, S, G * d, generator=gen).bfloat16() for _ in range(2))
    gb = buffers(n, [(4, 4)])
    gpu = [t.cuda() for t in (dy, q, k, v)]
    y, lse = gb.attention(*gpu[1:], H, G)
    dq, dk, dv = gb.attention_backward(*gpu, y, lse, H, G)
    gb.close()
    heads = lambda t, h: t.double().view(n, -1, h, d).transpose(1, 2)   # noqa: E731
    Q, D = heads(q, H), heads(dy, H)
    K, V = (heads(t, G).repeat_interleave(H // G, 1) for t in (k, v))
    scale, most = 1 / math.sqrt(d), 2.0 ** -15
    p = torch.softmax(scale * Q @ K.transpose(2, 3), -1)
    dp, size = D @ V.transpose(2, 3), D.abs() @ V.abs().transpose(2, 3)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    unsure = p * (size + (p * size).sum(-1, keepdim=True))      # magnitudes behind a weight's gradient
    shared = lambda t: t.view(n, G, H // G, S, d).sum(2)        # noqa: E731
    for got, want, room in ((heads(y.cpu(), H), p @ V, p @ V.abs()), (heads(dq.cpu(), H), scale * ds @ K, scale * unsure @ K.abs()),
                            (heads(dk.cpu(), G), shared(scale * ds.transpose(2, 3) @ Q), shared(scale * unsure.transpose(2, 3) @ Q.abs())),
                            (heads(dv.cpu(), G), shared(p.transpose(2, 3) @ D), shared(p.transpose(2, 3) @ D.abs()))):
        assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + most * room).all())
