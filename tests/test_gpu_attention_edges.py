"""Attention where infinities meet what has no weight, and the kernels of calls of many weights, against the formulas in 64 bits."""
import math

import pytest
import torch

from rows_util import HALF, buffers
from test_gpu_attention import BF16, F32, U, Case, forward, rounding, weight_error

pytestmark = pytest.mark.gpu
FEW = 2 ** 17       # weights of a call in bf16 up to which they keep 16 bits


def weights(size):
    n, B, T, S, H, G, d = size
    return n * B * H * T * S


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
        at = sums[b, rows, h, None]
        p = torch.exp(s - at)
        e = weight_error(case, s, off, at)
        dp = ds @ vs.t()
        size = (d + 2) * U * (ds.abs() @ vs.abs().t())
        if by_weights(S if case.states is None else int(case.states[b])):
            delta = (p * dp).sum(1, keepdim=True)
            off_d = (p * (dp.abs() * (e + 36 * U) + size)).sum(1, keepdim=True)
        else:
            delta = (ds * ys[b, rows, h]).sum(1, keepdim=True)
            off_d = (d + 2) * U * (ds * ys[b, rows, h]).abs().sum(1, keepdim=True)
        grad = p * (dp - delta)
        off_g = p * ((dp - delta).abs() * e + size + off_d + 2 * U * (dp - delta).abs()) + rounding(case, grad.abs())
        want_q[b, rows, h] = case.scale * grad @ ks
        off_q[b, rows, h] = case.scale * (off_g + (seen.numel() + 80) * U * grad.abs()) @ ks.abs() + 3 * U * want_q[b, rows, h].abs()
        adds = (case.asked(b) * (H // G) + 80) * U
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
