"""Attention where infinities meet what has no weight, and the kernels of calls of many weights, against the formulas in 64 bits."""
import math

import pytest
import torch

from parity_util import env_settings
from rows_util import HALF, buffers
from test_gpu_attention import BF16, F32, SIZES, U, Case, forward, rounding, test_forward as check_forward, weight_error

pytestmark = pytest.mark.gpu
FEW = 2 ** 17       # weights of a call in bf16 up to which they keep 16 bits


def weights(size):
    n, B, T, S, H, G, d = size
    return n * B * H * T * S


def left_out(case):
    """Of a product of floats whose pieces leave three products out: two of at most 2^-7 x 2^-15 of it, one of 2^-30."""
    return 8.5 * U if case.dtype == F32 and case.size[6] <= 128 else 0.0


def statement(case, y, lse, by_weights):
    """{gradient: (values, what float arithmetic may put each off by)} in 64 bits, from the y and lse that the forward call left.  by_weights(states of a sequence): whether
    dy . y is formed from the weights."""
    n, B, T, S, H, G, d = case.size
    q, k, v, dy, ys = case.heads(case.q, "q"), case.heads(case.k, "k"), case.heads(case.v, "k"), case.heads(case.dy, "q"), case.heads(y, "q")
    sums = lse.double().view(n * B, T, H)
    zeros = [torch.zeros(n * B, *shape, d, dtype=torch.float64) for shape in ((T, H), (T, H), (S, G), (S, G), (S, G), (S, G))]
    want_q, off_q, want_k, off_k, want_v, off_v = zeros
    for b, h, g, rows, seen in case.pairs():
        if seen.numel() == 0:
            continue
        qs, ks, vs, ds = q[b, rows, h], k[b, seen, g], v[b, seen, g], dy[b, rows, h]
        s, off = case.score(qs, ks)
        off = off + case.scale * left_out(case) * (qs.abs() @ ks.abs().t())
        at = sums[b, rows, h, None]
        p = torch.exp(s - at)
        e = weight_error(case, s, off, at)
        dp = ds @ vs.t()
        size = ((d + 2) * U + left_out(case)) * (ds.abs() @ vs.abs().t())
        if by_weights(S if case.states is None else int(case.states[b])):
            delta = (p * dp).sum(1, keepdim=True)
            off_d = (p * (dp.abs() * (e + 36 * U) + size)).sum(1, keepdim=True)     # at most 32 + 2 additions
        else:
            delta = (ds * ys[b, rows, h]).sum(1, keepdim=True)
            off_d = (d + 2) * U * (ds * ys[b, rows, h]).abs().sum(1, keepdim=True)
        grad = p * (dp - delta)
        off_g = p * ((dp - delta).abs() * e + size + off_d + 2 * U * (dp - delta).abs()) + rounding(case, grad.abs())
        want_q[b, rows, h] = case.scale * grad @ ks
        off_q[b, rows, h] = case.scale * (off_g + ((seen.numel() + 80) * U + left_out(case)) * grad.abs()) @ ks.abs() + 3 * U * want_q[b, rows, h].abs()
        adds = (case.asked(b) * (H // G) + 80) * U + left_out(case)
        want_k[b, :, g].index_add_(0, seen, case.scale * grad.t() @ qs)
        off_k[b, :, g].index_add_(0, seen, case.scale * (off_g + (adds + 3 * U) * grad.abs()).t() @ qs.abs())
        want_v[b, :, g].index_add_(0, seen, p.t() @ ds)
        off_v[b, :, g].index_add_(0, seen, (p * (e + adds) + rounding(case, p)).t() @ ds.abs())
    return dict(dq=(want_q, off_q), dk=(want_k, off_k), dv=(want_v, off_v))


def near(case, name, have, want, rows):
    """Of the rows that exist; the others still hold what was there."""
    have, (want, off) = case.heads(have, "q" if name == "dq" else "k"), want
    for b in range(have.shape[0]):
        w, o = want[b, :rows(b)], off[b, :rows(b)]
        assert bool(((have[b, :rows(b)] - w).abs() <= o + HALF[case.dtype] * (w.abs() + o)).all()), (name, b)
        assert bool((have[b, rows(b):] == 7).all()), (name, b)


def backward(gb, case, y, lse, **more):
    inputs = [t.cuda() for t in (case.dy, case.q, case.k, case.v, y, lse)]
    outs = {name: torch.full(t.shape, 7.0, dtype=case.dtype, device="cuda") for name, t in (("dq", case.q), ("dk", case.k), ("dv", case.v))}
    return [None if t is None else t.cpu() for t in gb.attention_backward(*inputs, **outs, **case.how(), **more)]


@pytest.mark.parametrize("want_dq", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("S,H,G,d", [(7, 2, 2, 24), (300, 8, 8, 64), (90, 3, 1, 37), (600, 8, 4, 128), (70, 2, 2, 200), (700, 8, 4, 256)])
@pytest.mark.parametrize("T", [31, 32, 33])
def test_states_that_nothing_weighs(T, S, H, G, d, dtype, want_dq):
    """A key with an infinite component that every query scores -infinity: its weights are 0, and so are its gradients, also where the last tile of queries is not full."""
    size = (1, 2, T, S, H, G, d)
    print("case", size, dtype, want_dq, flush=True)
    case = Case(size, dtype, False, False, seed=11)
    case.q.view(2, T, H, d)[..., 0] = -case.q.view(2, T, H, d)[..., 0].abs() - 0.5
    lost = [0, S // 2, S - 1]
    case.k.view(2, S, G, d)[1, lost, :, 0] = math.inf
    gb, y, lse = forward(case, spoiled=False)
    assert bool(y.isfinite().all()) and bool(lse.isfinite().all())
    dq, dk, dv = backward(gb, case, y, lse, want_dq=want_dq)
    gb.close()
    case.mask = torch.ones(2, S, dtype=torch.uint8)     # the same statement: these states are not there
    case.mask[1, lost] = 0
    want = statement(case, y, lse, lambda count: count <= 32)
    for name, have in (("dk", dk), ("dv", dv)):
        assert not have.view(2, S, -1)[1, lost].any(), name
        near(case, name, have, want[name], lambda b: S)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,S,H,G,d", [(5, 1, 2, 1, 16), (40, 2, 4, 4, 48), (3, 64, 2, 2, 128), (200, 512, 2, 1, 64), (9, 4, 2, 2, 200), (300, 256, 4, 2, 256)])
def test_infinite_values_and_gradients_stay_infinite(T, S, H, G, d, dtype):
    """Weights of a power of two have nothing behind their first bits, and a value that is infinite is infinite times all of a weight."""
    assert S & (S - 1) == 0
    size = (1, 1, T, S, H, G, d)
    case = Case(size, dtype, False, False, seed=12)
    case.q.zero_()
    case.v.view(S, G, d)[S - 1, 0, 3] = math.inf
    gb, y, lse = forward(case, spoiled=False)
    ys = y.view(T, G, H // G, d)
    assert bool((ys[:, 0, :, 3] == math.inf).all())
    ys[:, 0, :, 3] = 0.0
    assert bool(ys.isfinite().all())
    case.v.view(S, G, d)[S - 1, 0, 3] = 1.0
    y, lse = (t.cpu() for t in gb.attention(case.q.cuda(), case.k.cuda(), case.v.cuda(), **case.how()))
    case.dy.view(T, H, d)[T - 1, 0, 5] = -math.inf
    dv = backward(gb, case, y, lse)[2].view(S, G, d)
    gb.close()
    assert bool((dv[:, 0, 5] == -math.inf).all())
    dv[:, 0, 5] = 0.0
    assert bool(dv.isfinite().all())


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,S,H,G,d", [(5, 9, 2, 1, 16), (40, 70, 4, 4, 48), (33, 700, 8, 4, 128), (9, 40, 2, 2, 200), (130, 300, 4, 2, 256)])
def test_positions_without_a_state_have_no_gradient(T, S, H, G, d, dtype, bad):
    """Where the mask hides all states of a sequence, dq is 0 whatever comes back to its positions, as where no state exists."""
    size = (1, 3, T, S, H, G, d)
    case = Case(size, dtype, False, False, seed=13)
    case.mask = torch.ones(3, S, dtype=torch.uint8)
    case.mask[1] = 0
    case.states = torch.tensor([S, S, 0], dtype=torch.int32)
    case.dy.view(3, T, H, d)[1:, 0, 0, 1] = bad
    gb, y, lse = forward(case, spoiled=False)
    dq, dk, dv = backward(gb, case, y, lse)
    gb.close()
    assert not dq.view(3, T, -1)[1:].any()
    assert not dk.view(3, S, -1)[1].any() and not dv.view(3, S, -1)[1].any()
    want = statement(case, y, lse, lambda count: count <= 32)
    dq.view(3, T, -1)[1:] = 0
    near(case, "dq", dq, want["dq"], lambda b: T)
    near(case, "dk", dk, want["dk"], lambda b: int(case.states[b]))


# More than FEW weights.  Every width that kernels are built for and odd ones, shared heads, and few states under many positions.
MANY = [(1, 4, 200, 200, 2, 2, 24), (2, 2, 300, 130, 2, 1, 37), (2, 4, 70, 300, 2, 2, 64), (1, 4, 150, 260, 2, 1, 65), (1, 4, 200, 250, 2, 1, 80), (2, 3, 150, 170, 2, 2, 96),
        (2, 2, 130, 150, 4, 2, 100), (1, 4, 129, 300, 3, 1, 128), (1, 4, 130, 300, 2, 2, 160), (1, 5, 129, 200, 2, 1, 192), (1, 4, 150, 290, 1, 1, 256), (1, 4, 160, 250, 1, 1, 250),
        (2, 2, 9000, 1, 4, 2, 64), (1, 4, 900, 20, 2, 1, 128), (2, 2, 600, 32, 2, 1, 96), (1, 4, 600, 32, 2, 2, 200), (1, 4, 1100, 5, 8, 2, 37)]
HOW = [(False, False), (True, False), (False, True), (True, True)]


def ragged_too(case):
    """A short sequence that positions ask, among those that are drawn."""
    n, B, T, S, H, G, d = case.size
    if case.states is not None and n * B > 3:
        case.counts[3], case.states[3] = T // 2 + 1, min(S, 17)


@pytest.mark.parametrize("ragged,masked", HOW)
@pytest.mark.parametrize("size", MANY)
def test_forward_of_many_weights(size, ragged, masked):
    assert weights(size) > FEW
    check_forward(size, BF16, ragged, masked)


@pytest.mark.parametrize("ragged,masked", HOW)
@pytest.mark.parametrize("dtype,size", [(BF16, size) for size in MANY] + [(dtype, size) for size in SIZES for dtype in (F32, BF16)])
def test_gradients_with_and_without_that_of_queries(dtype, size, ragged, masked):
    """dk and dv alone, whose dy . y comes from a kernel of its own where sequences have room for more than 32 states, hold to the same bounds; dv, which has none of it, to its bits."""
    print("case", size, dtype, ragged, masked, flush=True)
    case = Case(size, dtype, ragged, masked, seed=21)
    ragged_too(case)
    n, B, T, S, H, G, d = size
    gb, y, lse = forward(case)
    for b in range(n * B):
        y.view(n * B, T, -1)[b, case.asked(b):] = math.nan
        lse.view(n * B, T, H)[b, case.asked(b):] = math.nan
    dq, dk, dv = backward(gb, case, y, lse)
    none, dk_alone, dv_alone = backward(gb, case, y, lse, want_dq=False)
    dq_alone, *nothing = backward(gb, case, y, lse, want_dkv=False)
    gb.close()
    assert none is None and nothing == [None, None] and torch.equal(dv, dv_alone) and torch.equal(dq, dq_alone)
    there = [S if case.states is None else int(case.states[b]) for b in range(n * B)]
    for b in range(n * B):      # what is not there is not read below either
        case.q.view(n * B, T, -1)[b, case.asked(b):] = 0
        for t in (case.k, case.v):
            t.view(n * B, S, -1)[b, ~case.seen(b)] = 0
    want = statement(case, y, lse, lambda count: count <= 32)
    near(case, "dq", dq, want["dq"], case.asked)
    near(case, "dk", dk, want["dk"], lambda b: there[b])
    near(case, "dv", dv, want["dv"], lambda b: there[b])
    near(case, "dk", dk_alone, statement(case, y, lse, lambda count: S <= 32)["dk"], lambda b: there[b])
    for b in range(n * B):
        hidden = ~case.seen(b)[:there[b]]
        for t in (dk, dv, dk_alone):
            assert not t.view(n * B, S, -1)[b, :there[b]][hidden].any()


@pytest.mark.parametrize("splits", [3, 64])
@pytest.mark.parametrize("size", [(1, 4, 60, 700, 4, 2, 40), (2, 2, 150, 270, 2, 1, 128), (1, 4, 20, 4500, 2, 1, 96), (1, 4, 700, 130, 1, 1, 200), (2, 2, 64, 600, 3, 1, 256)])
def test_parts_of_many_weights(size, splits):
    assert weights(size) > FEW
    with env_settings(dict(PG_ATTENTION_SPLITS=splits)):
        for ragged, masked in ((True, False), (False, True)):
            check_forward(size, BF16, ragged, masked)
            test_gradients_with_and_without_that_of_queries(BF16, size, ragged, masked)


@pytest.mark.parametrize("d", [24, 100, 128, 192])
def test_what_is_not_finite_among_many_weights(d):
    """NaN and infinities reach the positions and states that meet them, and no others, forward and back."""
    size = n, B, T, S, H, G, _ = (1, 2, 130, 270, 2, 1, d)
    assert weights(size) > FEW
    case = Case(size, BF16, False, False, seed=4)
    gb, clean, sums = forward(case)
    grads = backward(gb, case, clean, sums)
    case.q.view(2, T, 2, d)[0, 3, 1, 5] = math.nan
    case.k.view(2, S, d)[1, S - 1, 0] = math.nan
    y, lse = (t.cpu() for t in gb.attention(case.q.cuda(), case.k.cuda(), case.v.cuda(), **case.how()))
    ys, before = y.view(2, T, 2, d), clean.view(2, T, 2, d)
    assert bool(ys[1].isnan().all()) and bool(ys[0, 3, 1].isnan().all()) and bool(lse.view(2, T, 2)[0, 3, 1].isnan())
    good = torch.ones(T, 2, dtype=torch.bool)
    good[3, 1] = False
    assert torch.equal(ys[0][good], before[0][good])
    case.k.view(2, S, d)[1, S - 1, 0] = 0.0
    case.v.view(2, S, d)[1, 7, 11] = math.inf
    y, lse = (t.cpu() for t in gb.attention(case.q.cuda(), case.k.cuda(), case.v.cuda(), **case.how()))
    ys = y.view(2, T, 2, d)
    assert bool((ys[1, :, :, 11] == math.inf).all()) and bool(ys[1][..., torch.arange(d) != 11].isfinite().all())
    # back: the position of NaN reaches its own dq and all states of its sequence; the other sequence is as it was
    case.v.view(2, S, d)[1, 7, 11] = 1.0
    y, lse = (t.cpu() for t in gb.attention(case.q.cuda(), case.k.cuda(), case.v.cuda(), **case.how()))
    dq, dk, dv = backward(gb, case, y, lse)
    assert bool(dq.view(2, T, 2, d)[0, 3, 1].isnan().all()) and bool(dk.view(2, S, d)[0].isnan().all()) and bool(dv.view(2, S, d)[0].isnan().all())
    assert torch.equal(dq.view(2, T, 2, d)[0][good], grads[0].view(2, T, 2, d)[0][good])
    for t in (dq, dk, dv):
        assert bool(t.view(2, -1)[1].isfinite().all())
    gb.close()


def test_strides_of_many_weights():
    """Keys and values side by side in one tensor at odd places, workers inside rows, outputs in wider ones."""
    size = n, B, T, S, H, G, d = (2, 2, 130, 150, 4, 2, 20)
    assert weights(size) > FEW
    case = Case(size, BF16, False, True, seed=5)
    gb = buffers(n, [(4, 4)])
    q, k, v, dy = (t.cuda() for t in (case.q, case.k, case.v, case.dy))
    y, lse = gb.attention(q, k, v, **case.how())
    want = gb.attention_backward(dy, q, k, v, y, lse, **case.how())

    def wide(x, at, width):
        w = torch.full((x.shape[1], n, width), 9.0, dtype=BF16, device="cuda")
        view = w[:, :, at:at + x.shape[2]].transpose(0, 1)
        view.copy_(x)
        return w, view
    both = torch.full((B * S, n, 2 * G * d + 7), 9.0, dtype=BF16, device="cuda")
    keys, values = both[:, :, 1:1 + G * d].transpose(0, 1), both[:, :, 3 + G * d:3 + 2 * G * d].transpose(0, 1)
    keys.copy_(k), values.copy_(v)
    qv = wide(q, 3, H * d + 5)[1]
    outs = [wide(t * 0, 1, t.shape[2] + 3) for t in (q, q, k, v)]
    y2, lse2 = gb.attention(qv, keys, values, out=outs[0][1], **case.how())
    assert torch.equal(y2, y) and torch.equal(lse2, lse)
    got = gb.attention_backward(wide(dy, 1, H * d + 1)[1], qv, keys, values, y2, lse2, dq=outs[1][1], dk=outs[2][1], dv=outs[3][1], **case.how())
    gb.close()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for w, view in outs:
        assert bool((w[:, :, 0] == 9).all()) and bool((w[:, :, 1 + view.shape[2]:] == 9).all())


def test_many_weights_beyond_thirty_two_bits():
    """Rows of states 2^17 elements apart: the last ones lie past 4 GiB of the first, and so do a second worker's."""
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    n, rows, width, apart, memory = 2, 9, 64, 1 << 17, 18000
    assert weights((n, 1, rows, memory, 1, 1, width)) > FEW and memory * apart * 2 > 1 << 32
    gen = torch.Generator().manual_seed(9)
    gb = buffers(n, [(4, 4)])
    room = torch.empty(n * memory * apart, dtype=BF16, device="cuda").view(n, memory, apart)
    k, v = room[:, :, :width], room[:, :, 100:100 + width]
    for t in (k, v):
        t.copy_(torch.randn(n, memory, width, generator=gen).to(BF16))
    q, dy = (torch.randn(n, rows, width, generator=gen).to(BF16).cuda() for _ in range(2))
    kc, vc = k.contiguous(), v.contiguous()
    y, lse = gb.attention(q, k, v, 1)
    y2, lse2 = gb.attention(q, kc, vc, 1)
    assert torch.equal(y, y2) and torch.equal(lse, lse2)
    want = gb.attention_backward(dy, q, kc, vc, y, lse, 1)
    got = gb.attention_backward(dy, q, k, v, y, lse, 1, dk=room[:, :, 200:200 + width], dv=room[:, :, 300:300 + width])
    gb.close()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [(1, 4, 200, 200, 2, 2, 24), (1, 4, 150, 260, 2, 1, 65), (1, 4, 129, 300, 3, 1, 128), (1, 5, 129, 200, 2, 1, 192), (1, 4, 160, 250, 1, 1, 250),
                                  (1, 2, 20, 90, 2, 1, 96), (1, 2, 9, 40, 2, 2, 200)])
def test_values_with_a_mean(size, dtype):
    """Values around 16: dy . y is far from 0 and cancels in every gradient, so that a percent of it, or a column left out of it, is ten times the bounds and more also in bf16."""
    case = Case(size, dtype, False, False, seed=22)
    case.v.add_(16)
    gb, y, lse = forward(case, spoiled=False)
    for how in (dict(), dict(want_dq=False)):
        dq, dk, dv = backward(gb, case, y, lse, **how)
        want = statement(case, y, lse, lambda count: False)
        for name, have in (("dq", dq), ("dk", dk), ("dv", dv)):
            if have is not None:
                near(case, name, have, want[name], lambda b: size[3] if name != "dq" else size[2])
    gb.close()
