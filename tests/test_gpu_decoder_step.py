"""Layer norms, linear layers, attention to an encoder's states and the distillation loss together: a training step of a decoder and the gossip round that takes its
gradients, captured, on other streams, beside other calls; single positions; more rows, workers and bytes than 32 bits or a grid's side count."""
import math

import pytest
import torch

from paper_2008_01425_amd import binding as B
from rows_util import HALF, buffers, grad, put

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def near(got, want, dtype):
    """A chain of a dozen operators, each off by a few units of its type: in norm, 16 half steps of bfloat16, or the thousandth that leaves float room for it."""
    got, want = got.cpu().double(), want.double()
    assert float((got - want).norm()) <= (16 * 2.0 ** -8 if dtype == BF16 else 1e-4) * float(want.norm())


class Decoder:
    """x + attention(norm(x), states) through a norm and a last layer into the loss.  Layers: 0, 1 gain and bias, 2, 3 queries, 4, 5 keys and values side by side, 6, 7 back to
    the width of x, 8, 9 gain and bias, 10, 11 the last layer."""

    def __init__(self, n, sequences, rows, memory, d, heads, kv_heads, width, words, top, dtype, seed):
        self.size = n, sequences, rows, memory, d, heads, kv_heads, width, words, top
        self.dtype = dtype
        gen = torch.Generator().manual_seed(seed)
        q, kv = heads * width, kv_heads * width
        shapes = [(d, 1), (d, 1), (q, d), (q, 1), (2 * kv, d), (2 * kv, 1), (d, q), (d, 1), (d, 1), (d, 1), (words, d), (words, 1)]
        self.gb = buffers(n, shapes)
        self.w = []
        for l, (p, c) in enumerate(shapes):
            w = torch.randn(n, p, c, generator=gen) / math.sqrt(c) if c > 1 else 0.1 * torch.randn(n, p, 1, generator=gen)
            if l in (0, 8):
                w = w + 1
            if dtype == BF16 and c > 1:
                w = w.bfloat16().float()        # weights that enter as they are
            self.w.append(w)
            put(self.gb, l, w)
        self.x = torch.randn(n, sequences * rows, d, generator=gen).to(dtype)
        self.states = torch.randn(n, sequences * memory, d, generator=gen).to(dtype)
        self.counts = torch.full((n * sequences,), rows, dtype=torch.int32)
        self.lengths = torch.randint(memory // 2, memory + 1, (n * sequences,), generator=gen, dtype=torch.int32)
        self.labels = torch.randint(-1, words, (n, sequences * rows), generator=gen, dtype=torch.int32)
        self.teacher, index = (2 * torch.randn(n, sequences * rows, words, generator=gen)).topk(top, -1)
        self.index = index.int()
        self.weights = torch.rand(n, sequences * rows, generator=gen)
        self.scale = 1.0 / (sequences * rows)
        gpu = lambda t: t.cuda()    # noqa: E731
        self.xd, self.sd = gpu(self.x), gpu(self.states)
        self.loss_in = [gpu(t) for t in (self.index, self.teacher, self.labels)]
        self.wd, self.ld = gpu(self.weights), gpu(self.lengths)

    def step(self, stream=None):
        n, sequences, rows, memory, d, heads, kv_heads, width, words, top = self.size
        gb, kv = self.gb, kv_heads * width
        how = dict(heads=heads, kv_heads=kv_heads, sequences=sequences, memory_counts=self.ld, stream=stream)
        h, _, m1, r1 = gb.layer_norm(0, self.xd, bias=1, stream=stream)
        q = gb.linear(2, h, bias=3, stream=stream)
        both = gb.linear(4, self.sd, bias=5, stream=stream)
        k, v = both[:, :, :kv], both[:, :, kv:]
        y, lse = gb.attention(q, k, v, **how)
        o = gb.linear(6, y, bias=7, stream=stream)
        g, total, m2, r2 = gb.layer_norm(8, o, bias=9, residual=self.xd, stream=stream)
        z = gb.linear(10, g, bias=11, stream=stream)
        loss, dz = gb.distill(z, *self.loss_in, temperature=2.0, hard=0.5 * self.scale, soft=0.5 * self.scale, weights=self.wd, stream=stream, out=z)
        dg = gb.linear_backward(10, dz, g, bias=11, stream=stream)
        dtotal = gb.layer_norm_backward(8, dg, total, m2, r2, bias=9, stream=stream)
        dy = gb.linear_backward(6, dtotal, y, bias=7, stream=stream)
        dboth = torch.zeros_like(both)
        dq, _, _ = gb.attention_backward(dy, q, k, v, y, lse, dk=dboth[:, :, :kv], dv=dboth[:, :, kv:], **how)
        ds = gb.linear_backward(4, dboth, self.sd, bias=5, stream=stream)
        dh = gb.linear_backward(2, dq, h, bias=3, stream=stream)
        dx = gb.layer_norm_backward(0, dh, self.xd, m1, r1, bias=1, residual=dtotal, stream=stream)
        return loss, dx, ds

    def oracle(self):
        n, sequences, rows, memory, d, heads, kv_heads, width, words, top = self.size
        w = [t.double().requires_grad_() for t in self.w]
        x, s = self.x.double().requires_grad_(), self.states.double().requires_grad_()
        norm = lambda v, a, b: torch.nn.functional.layer_norm(v, (d,), eps=1e-5) * w[a].transpose(1, 2) + w[b].transpose(1, 2)    # noqa: E731
        linear = lambda v, a, b: v @ w[a].transpose(1, 2) + w[b].transpose(1, 2)    # noqa: E731
        q, both = linear(norm(x, 0, 1), 2, 3), linear(s, 4, 5)
        q = q.view(n * sequences, rows, heads, width).transpose(1, 2)
        k, v = (t.reshape(n * sequences, memory, kv_heads, width).transpose(1, 2).repeat_interleave(heads // kv_heads, 1) for t in both.chunk(2, -1))
        score = q @ k.transpose(2, 3) / math.sqrt(width)
        score = score.masked_fill(torch.arange(memory) >= self.lengths[:, None, None, None], -math.inf)
        y = (torch.softmax(score, -1) @ v).transpose(1, 2).reshape(n, sequences * rows, heads * width)
        z = linear(norm(x + linear(y, 6, 7), 8, 9), 10, 11)
        lab = self.labels.long()
        hard = torch.where(lab >= 0, -torch.log_softmax(z, -1).gather(-1, lab.clamp(min=0)[..., None])[..., 0], 0.0)
        logp = torch.log_softmax(self.teacher.double() / 2, -1)
        soft = 4 * (logp.exp() * (logp - torch.log_softmax(z / 2, -1).gather(-1, self.index.long()))).sum(-1)
        loss = self.weights.double() * 0.5 * self.scale * (hard + soft)
        loss.sum().backward()
        return loss.detach(), x.grad, s.grad, [t.grad for t in w]


SIZES = [(2, 2, 7, 19, 40, 4, 2, 12, 50, 5), (3, 1, 150, 260, 96, 4, 1, 64, 700, 20), (1, 3, 64, 96, 64, 2, 2, 32, 1100, 8)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", SIZES)
def test_a_training_step(size, dtype):
    print("case", size, dtype, flush=True)
    dec = Decoder(*size, dtype, seed=size[2])
    loss, dx, ds = dec.step()
    want_loss, want_dx, want_ds, want_g = dec.oracle()
    near(loss, want_loss, dtype), near(dx, want_dx, dtype), near(ds, want_ds, dtype)
    for l in range(12):
        near(grad(dec.gb, l), want_g[l], dtype)
    other = Decoder(*size, dtype, seed=size[2])
    for l in range(12):
        for i in range(size[0]):
            other.gb.set_grad_layer(i, l, want_g[l][i].float().numpy())
    before = [dec.gb.layer_of(torch.stack(dec.gb.x), l).cpu().double() for l in range(12)]
    dec.gb.round_sgd(0.5), other.gb.round_sgd(0.5)
    for l in range(12):
        got, want = (dec.gb.layer_of(torch.stack(g.x), l).cpu().double() for g in (dec.gb, other.gb))
        assert float((got - want).norm()) <= (16 * 2.0 ** -8 if dtype == BF16 else 1e-3) * float(0.5 * want_g[l].norm()) + 1e-6 * float(before[l].norm())
    dec.gb.close(), other.gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_replays_of_a_captured_step_equal_the_direct_call(dtype):
    """Two graphs of a whole step, replayed in turn between eager steps on other inputs: the same bits every time."""
    dec = Decoder(*SIZES[1], dtype, seed=3)
    outs = dec.step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs] + [g.clone() for g in dec.gb.g]
    graphs, side = [], torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = dec.step()
        graphs.append((graph, got))
    x = dec.xd.clone()
    for replay in range(3):
        for graph, got in graphs:
            for g in dec.gb.g:
                g.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(got, want):
                assert torch.equal(a, b), f"replay {replay}"
            for a, b in zip(dec.gb.g, want[3:]):
                for l in range(12):
                    assert torch.equal(dec.gb.layer_of(a, l), dec.gb.layer_of(b, l)), f"replay {replay}, layer {l}"
            dec.xd.mul_(0.5)
            dec.step()
            dec.xd.copy_(x)
            torch.cuda.synchronize()
    # both on their way at the same time, on streams of their own: each has its workspaces; the gradient buffers they share get the same values from both
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, (graph, got) in zip(streams, graphs):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for _, got in graphs:
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    dec.gb.close()


def test_a_stream_of_the_callers():
    dec = Decoder(*SIZES[0], BF16, seed=6)
    first = dec.step()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        second = dec.step()
    third = dec.step(stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)
    dec.gb.close()


def test_the_profile_names_them():
    dec = Decoder(*SIZES[0], F32, seed=7)
    dec.step()
    B.pg_profile_enable(dec.gb.ctx, True)
    dec.step()
    names = {k["name"]: k["launches"] for k in B.pg_profile_collect(dec.gb.ctx)}
    assert {k: names.get(k) for k in ("layer_norm", "layer_norm_backward", "attention", "attention_dq", "attention_dkv", "distill")} == {
        "layer_norm": 2, "layer_norm_backward": 2, "attention": 1, "attention_dq": 1, "attention_dkv": 1, "distill": 1}
    dec.gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_position_at_a_time(dtype):
    """Answering: every position alone gives what it gives among the others, to the rounding of sums in another order."""
    n, sequences, rows, memory, heads, kv_heads, width = 2, 3, 9, 1500, 8, 2, 64
    gen = torch.Generator().manual_seed(8)
    gb = buffers(n, [(4, 4)])
    q = torch.randn(n, sequences * rows, heads * width, generator=gen).to(dtype).cuda()
    k, v = (torch.randn(n, sequences * memory, kv_heads * width, generator=gen).to(dtype).cuda() for _ in range(2))
    lengths = torch.tensor([1500, 1, 700, 33, 0, 1499], dtype=torch.int32, device="cuda")
    y, lse = gb.attention(q, k, v, heads, kv_heads, sequences, memory_counts=lengths)
    y, lse = y.view(n, sequences, rows, -1), lse.view(n, sequences, rows, heads)
    for t in range(rows):
        one = q.view(n, sequences, rows, -1)[:, :, t].contiguous()
        y1, lse1 = gb.attention(one, k, v, heads, kv_heads, sequences, memory_counts=lengths)
        # weights sum to 1, so a sum of 1500 of them in another order moves y by 1500 roundings of the largest value at most, in float; and one rounding of the result
        most = float(v.float().abs().max())
        assert bool(((y1 - y[:, :, t]).float().abs() <= 3000 * 2.0 ** -24 * most + (2 * 2.0 ** -8 * most if dtype == BF16 else 0.0)).all())
        same = lse1 == lse[:, :, t]
        assert bool((same | ((lse1 - lse[:, :, t]).abs() <= 3000 * 2.0 ** -24 + 2.0 ** -22 * lse1.abs())).all())
    gb.close()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_states_beyond_thirty_two_bits(dtype):
    """Rows of states 2^17 elements apart: the last ones lie past 4 GiB of the first, and so do a second worker's."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    n, rows, width, apart = 2, 3, 64, 1 << 17
    per = 4 if dtype == F32 else 2
    memory = 9000 * 4 // per
    gen = torch.Generator().manual_seed(9)
    gb = buffers(n, [(4, 4)])
    assert memory * apart * per > 1 << 32
    room = torch.empty(n * memory * apart, dtype=dtype, device="cuda").view(n, memory, apart)
    k, v = room[:, :, :width], room[:, :, 100:100 + width]
    k.copy_(torch.randn(n, memory, width, generator=gen).to(dtype)), v.copy_(torch.randn(n, memory, width, generator=gen).to(dtype))
    q, dy = (torch.randn(n, rows, width, generator=gen).to(dtype).cuda() for _ in range(2))
    y, lse = gb.attention(q, k, v, 1)
    kc, vc = k.contiguous(), v.contiguous()
    y2, lse2 = gb.attention(q, kc, vc, 1)
    assert torch.equal(y, y2) and torch.equal(lse, lse2)
    want = gb.attention_backward(dy, q, kc, vc, y, lse, 1)
    dk, dv = room[:, :, 200:200 + width], room[:, :, 300:300 + width]
    got = gb.attention_backward(dy, q, k, v, y, lse, 1, dk=dk, dv=dv)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    del room, k, v, dk, dv, got
    # logits and their gradient: rows and workers past 4 GiB
    rows, cols = 2100, 300
    wide = torch.empty((n * rows) << 21, dtype=dtype, device="cuda")
    z = torch.as_strided(wide, (n, rows, cols), (rows << 21, 1 << 21, 1))
    z.copy_(torch.randn(n, rows, cols, generator=gen).to(dtype))
    labels = torch.randint(0, cols, (n, rows), generator=gen, dtype=torch.int32).cuda()
    loss, dz = gb.distill(z.contiguous(), labels=labels)
    loss2, dz2 = gb.distill(z, labels=labels, out=z)
    assert torch.equal(loss, loss2) and torch.equal(dz, dz2)
    gb.close()


def test_more_workers_than_one_side_of_a_grid():
    n, cols = 70000, 6
    gb = buffers(n, [(cols, 1), (cols, 1)])
    gen = torch.Generator().manual_seed(11)
    x = torch.randn(n, 1, cols, generator=gen).cuda()
    flat = torch.zeros(n, gb.N, device="cuda")
    gb.x, gb.ptrs = list(flat), [flat.data_ptr() + 4 * gb.N * i for i in range(n)]
    gflat = torch.zeros(n, gb.N, device="cuda")
    gb.g, gb.gptrs = list(gflat), [gflat.data_ptr() + 4 * gb.N * i for i in range(n)]
    gb.layer_of(flat, 0).fill_(1.0)
    y, _, mean, rstd = gb.layer_norm(0, x, bias=1)
    want = torch.nn.functional.layer_norm(x.double(), (cols,), eps=1e-5)
    assert bool(((y.double() - want).abs() <= 1e-5).all())          # 40 roundings of values up to 3, rstd among them
    gb.layer_norm_backward(0, x, x, mean, rstd, bias=1)
    assert torch.equal(gb.layer_of(gflat, 1)[:, :, 0], x[:, 0])
    loss, dz = gb.distill(x, labels=torch.zeros(n, 1, dtype=torch.int32, device="cuda"))
    want = -torch.log_softmax(x.double(), -1)[:, :, 0]
    assert bool(((loss.double() - want).abs() <= 1e-5).all())
    q = x[:, :, :4].contiguous()
    out, lse = gb.attention(q, x[:, :, :4].contiguous(), x[:, :, 2:].contiguous(), 2, 2)
    # one state: its values, times a weight near 1, over that weight.  Three products of parts below 2^-24 are left out, six are summed (a rounding each, of the weight's
    # too), and the division's reciprocal and product round twice: 12 roundings.
    assert bool(((out - x[:, :, 2:]).abs() <= 12 * 2.0 ** -24 * x[:, :, 2:].abs()).all())
    dq, dk, dv = gb.attention_backward(q, q, q, x[:, :, 2:].contiguous(), out, lse, 2, 2)
    # a weight of 1 to the roundings of a score of up to 50 and its logarithm, in an exponential
    assert bool(((dv - q).abs() <= 1e-5 * q.abs()).all())
    gb.close()
