"""What the library's norms with a mean, attention to an encoder's states and distillation losses are measured on: what a
training step of n workers needs between its linear layers and behind the last one.

Layer norm: S = X + R, Y = (S - mean) rstd gain + bias.  Attention: queries of `rows` positions read `memory` states of an encoder,
`sequences` of both per worker, query heads share key heads; counts and a mask hide states.  Distillation: cross entropy against
a label and Kullback-Leibler divergence from a teacher's `top` logits, loss and gradient of the logits.

`own` false computes the plain form: whole-batch torch operations in float32, rounded once."""
import math

import torch
import torch.nn.functional as F

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _norm(op, workers, rows, cols, dtype, residual=False, ragged=False):
    return dict(op=op, workers=workers, rows=rows, cols=cols, dtype=dtype, residual=residual, ragged=ragged)


def _attention(op, workers, sequences, rows, memory, heads, kv_heads, width, dtype, ragged=False, mask=False):
    return dict(op=op, workers=workers, sequences=sequences, rows=rows, memory=memory, heads=heads, kv_heads=kv_heads, width=width,
                dtype=dtype, ragged=ragged, mask=mask)


def _distill(workers, rows, cols, top, dtype, labels=True, ragged=False):
    return dict(op="distill", workers=workers, rows=rows, cols=cols, top=top, dtype=dtype, labels=labels, ragged=ragged)


def listed():
    """Per operator from the smallest calls to the largest."""
    return [
        # one step of 20 sequences in front of a layer of the language model: latency
        dict(_norm("norm", 16, 20, 650, "f32", residual=True), name="norm_step"),
        # in front of a residual block's wide layer
        dict(_norm("norm", 8, 8192, 2048, "bf16", residual=True), name="norm_block"),
        # sequences of different lengths, rows of odd length, back
        dict(_norm("norm_backward", 16, 700, 1301, "f32", ragged=True), name="norm_ragged_backward"),
        # the block's norm, back
        dict(_norm("norm_backward", 8, 8192, 2048, "bf16", residual=True), name="norm_block_backward"),
        # a few positions over a few states, the smallest worth a call: latency
        dict(_attention("attention", 4, 1, 7, 13, 2, 2, 16, "f32"), name="attention_small"),
        # answering: the one newest position of each sequence over a long input, four query heads to a key head
        dict(_attention("attention", 8, 4, 1, 4096, 16, 4, 128, "bf16", ragged=True), name="attention_token"),
        # a long output over a longer input
        dict(_attention("attention", 2, 1, 4096, 8192, 16, 4, 128, "bf16"), name="attention_long"),
        # a training batch: padded sequences
        dict(_attention("attention_backward", 8, 4, 512, 1024, 16, 16, 64, "bf16", ragged=True), name="attention_batch_backward"),
        # a long output over a longer input, back, heads shared
        dict(_attention("attention_backward", 2, 1, 2048, 4096, 16, 4, 128, "bf16"), name="attention_long_backward"),
        # in float, head width and lengths odd, single states hidden
        dict(_attention("attention_backward", 4, 2, 333, 777, 8, 2, 80, "f32", mask=True), name="attention_float_backward"),
        # an image classifier taught by a larger one: latency
        dict(_distill(8, 128, 10, 3, "f32"), name="distill_classifier"),
        # the language model's decoder, 20 sequences of 35 positions, the teacher's 32 likeliest words
        dict(_distill(16, 700, 33278, 32, "bf16"), name="distill_words"),
    ]


def draw(rng):
    """One more case: any operator and type, from one row on one worker to cases like the listed ones."""
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    op = rng.choice(["norm", "norm_backward", "attention", "attention", "attention_backward", "attention_backward", "distill", "distill"])
    n, dtype, ragged = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice(["f32", "bf16", "bf16"]), rng.random() < 0.3
    if op.startswith("norm"):
        rows, cols = size(1, 8192), size(8, 16384)
        if rng.random() < 0.4:
            cols = 64 * max(1, cols // 64)
        while n * rows * cols > 1.3e8:
            rows = max(1, rows // 2)
        return _norm(op, n, rows, cols, dtype, rng.random() < 0.5, ragged)
    if op == "distill":
        rows, cols = size(1, 4096), size(2, 150000)
        while n * rows * cols > 3.7e8:
            rows = max(1, rows // 2)
        top = min(cols, rng.choice([0, 1, 8, 20, 32, 64, 128]))
        return _distill(n, rows, cols, top, dtype, rng.random() < 0.6 or top == 0, ragged)
    sequences, kv_heads = rng.choice([1, 1, 2, 4]), rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 8])
    rows, memory = 1 if rng.random() < 0.2 else size(1, 4096), size(2, 8192)   # a single state's weight has no gradient but rounding
    width = rng.choice([16, 32, 64, 64, 80, 96, 128, 128, 65, 37, 192, 256])
    most = 2.7e11 if op == "attention_backward" else 5.4e11      # operations
    while ((10.0 if op == "attention_backward" else 4.0) * n * sequences * heads * rows * memory * width * (4.0 if dtype == "f32" else 1.0) > most
           or n * sequences * heads * rows * memory > 5e8 or n * sequences * max(rows * heads, memory * kv_heads) * width > 2e8):
        rows, memory = max(1, rows // 2), max(2, memory * 3 // 4)
    return _attention(op, n, sequences, rows, memory, heads, kv_heads, width, dtype, ragged and memory > 3, rng.random() < 0.3 and memory > 15)


# ---- inputs -------------------------------------------------------------------------------

class State:
    """What a training program holds between two calls."""

    def __del__(self):
        if getattr(self, "gb", None) is not None:
            self.gb.close()


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _library(s)
    return s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, op, dtype = case["workers"], case["op"], TYPES[case["dtype"]]

    def normal(*shape, scale=1.0, mean=0.0, dtype=dtype):
        return torch.empty(shape, device="cuda").normal_(mean, scale, generator=gen).to(dtype)

    def lengths(count, most):    # padded to the longest
        c = torch.randint(most // 2, most + 1, (count,), device="cuda", generator=gen, dtype=torch.int32)
        c[0] = most
        return c

    s = State()
    s.case, s.dtype, s.gb, s.counts = case, dtype, None, None
    T = case["rows"]
    if op.startswith("norm"):
        q = case["cols"]
        s.counts = lengths(n, T) if case["ragged"] else None
        s.g, s.b = normal(n, q, scale=0.1, mean=1.0, dtype=torch.float32), normal(n, q, scale=0.1, dtype=torch.float32)
        # rows with means of their own, as residual streams have them
        s.x = (normal(n, T, q, dtype=torch.float32) + normal(n, T, 1, dtype=torch.float32)).to(dtype)
        s.r = normal(n, T, q, scale=0.02 if op == "norm_backward" else 0.5) if case["residual"] else None
        if op == "norm_backward":
            s.dy = normal(n, T, q, scale=0.02)
            v = s.x.double()
            s.mean = v.mean(-1)
            s.rstd = (v.sub_(s.mean.unsqueeze(-1)).square_().mean(-1) + EPS).rsqrt().float()
            s.mean = s.mean.float()
    elif op == "distill":
        V, k = case["cols"], case["top"]
        s.counts = lengths(n, T) if case["ragged"] else None
        z = normal(n, T, V, scale=2.0, dtype=torch.float32)
        if k:      # a teacher that the student follows from afar
            s.t, at = (z * 0.8 + normal(n, T, V, scale=1.5, dtype=torch.float32)).topk(k, -1)
            s.at = at.int()
        else:
            s.t = s.at = None
        s.z = z.to(dtype)
        s.labels = None
        if case["labels"]:      # positions without a label among them
            s.labels = torch.randint(0, V, (n, T), device="cuda", generator=gen, dtype=torch.int32)
            s.labels[torch.rand(n, T, device="cuda", generator=gen) < 0.05] = -1
        s.weights = torch.rand(n, T, device="cuda", generator=gen) + 0.5
        s.hard, s.soft, s.tau = (0.5 if case["labels"] else 0.0), (0.5 if k else 0.0), 2.0
    else:
        B, S, H, G, d = case["sequences"], case["memory"], case["heads"], case["kv_heads"], case["width"]
        s.q, s.k, s.v = normal(n, B * T, H * d), normal(n, B * S, G * d), normal(n, B * S, G * d)
        s.scale = 1.0 / math.sqrt(d)
        s.memory_counts = s.mask = None
        if case["ragged"]:
            s.counts, s.memory_counts = lengths(n * B, T), lengths(n * B, S)
            if n * B > 4:      # one without an input
                s.memory_counts[3] = 0
        if case["mask"]:
            s.mask = (torch.rand(n * B, S, device="cuda", generator=gen) > 0.2).to(torch.uint8)
        if op == "attention_backward":     # behind a forward pass: what that left is an input
            s.dy = normal(n, B * T, H * d, scale=0.02)
            s.y, s.lse = _attend(s)[:2]
    return s


def _library(s):
    """The same inputs where a program of this library has them: parameters and gradients in its buffers, rows behind a
    sequence's end zero in the outputs."""
    from paper_2008_01425_amd.device import GossipBuffers
    case, op = s.case, s.case["op"]
    n, T = case["workers"], case["rows"]
    shapes = [(case["cols"], 1)] * 2 if op.startswith("norm") else [(8, 8)]
    edges = [[i, (i + 1) % n] for i in range(n)] if n > 2 else [[0, 1]][:n - 1]
    s.gb = gb = GossipBuffers(n, edges, [1.0 / 3.0] * len(edges), shapes, 1, 1)
    x, g = torch.zeros(n, gb.N, device="cuda"), torch.zeros(n, gb.N, device="cuda")
    gb.x, gb.ptrs = list(x), [t.data_ptr() for t in x]
    gb.g, gb.gptrs = list(g), [t.data_ptr() for t in g]

    def rows(count, width, dtype=s.dtype):
        return torch.zeros(n, count, width, device="cuda", dtype=dtype)

    if op.startswith("norm"):
        s.params, s.grads = ([gb.layer_of(flat, l) for l in range(2)] for flat in (x, g))
        s.params[0].copy_(s.g.unsqueeze(-1))
        s.params[1].copy_(s.b.unsqueeze(-1))
        s.y = rows(T, case["cols"])
        if op == "norm":
            s.sum = rows(T, case["cols"]) if case["residual"] else None
            s.mean, s.rstd = torch.zeros(n, T, device="cuda"), torch.zeros(n, T, device="cuda")
    elif op == "distill":
        s.dz, s.loss = rows(T, case["cols"]), torch.zeros(n, T, device="cuda")
    else:
        B = case["sequences"]
        if op == "attention":
            s.out, s.out_lse = rows(B * T, case["heads"] * case["width"]), rows(B * T, case["heads"], torch.float32)
        else:
            s.lse = s.lse.contiguous()      # as the forward call leaves it
            s.dq, s.dk, s.dv = torch.zeros_like(s.q), torch.zeros_like(s.k), torch.zeros_like(s.v)


# ---- one pass -----------------------------------------------------------------------------

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    gb, case, op = s.gb, s.case, s.case["op"]
    if op == "norm":
        gb.layer_norm(0, s.x, bias=1, residual=s.r, eps=EPS, counts=s.counts, out=s.y, sum_out=s.sum, mean_out=s.mean, rstd_out=s.rstd)
        return [s.y, s.mean, s.rstd] if s.r is None else [s.y, s.mean, s.rstd, s.sum]
    if op == "norm_backward":
        gb.layer_norm_backward(0, s.dy, s.x, s.mean, s.rstd, bias=1, residual=s.r, counts=s.counts, out=s.y)
        return [s.y, s.grads[0][:, :, 0], s.grads[1][:, :, 0]]
    if op == "distill":
        gb.distill(s.z, top_index=s.at, top_logits=s.t, labels=s.labels, temperature=s.tau, hard=s.hard, soft=s.soft, weights=s.weights,
                   counts=s.counts, out=s.dz, loss_out=s.loss)
        return [s.loss, s.dz]
    how = dict(heads=case["heads"], kv_heads=case["kv_heads"], sequences=case["sequences"], scale=s.scale, counts=s.counts,
               memory_counts=s.memory_counts, mask=s.mask)
    if op == "attention":
        return list(gb.attention(s.q, s.k, s.v, out=s.out, lse_out=s.out_lse, **how))
    return list(gb.attention_backward(s.dy, s.q, s.k, s.v, s.y, s.lse, dq=s.dq, dk=s.dk, dv=s.dv, **how))


def _valid(counts, rows):
    """1 for the rows of a sequence, 0 behind its end."""
    return (torch.arange(rows, device="cuda") < counts[:, None]).float().unsqueeze(-1)


def _heads(s, x, count, heads):
    """(workers * sequences, query heads, count, width) in float; key heads once for each query head that shares them."""
    case = s.case
    x = x.float().view(case["workers"] * case["sequences"], count, heads, case["width"]).transpose(1, 2)
    return x if heads == case["heads"] else x.repeat_interleave(case["heads"] // heads, 1)


def _attend(s):
    """y, lse, and the weights of every position, with the inputs by heads."""
    case = s.case
    n, B, T, S, H, G, d = (case[k] for k in ("workers", "sequences", "rows", "memory", "heads", "kv_heads", "width"))
    q, k, v = _heads(s, s.q, T, H), _heads(s, s.k, S, G), _heads(s, s.v, S, G)
    score = torch.matmul(q, k.transpose(2, 3)).mul_(s.scale)
    seen = torch.ones(n * B, S, dtype=torch.bool, device="cuda")
    if s.memory_counts is not None:
        seen &= torch.arange(S, device="cuda") < s.memory_counts[:, None]
    if s.mask is not None:
        seen &= s.mask != 0
    score.masked_fill_(~seen[:, None, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    weight = weight.div_(torch.where(total > 0, total, 1.0))
    y = torch.matmul(weight, v)
    if s.counts is not None:
        end = _valid(s.counts, T).unsqueeze(1)
        y, weight, lse = y * end, weight.mul_(end), torch.where(end > 0, lse, 0.0)
    y = y.transpose(1, 2).reshape(n, B * T, H * d).to(s.dtype)
    return y, lse.squeeze(-1).transpose(1, 2).reshape(n, B * T, H), weight, q, k, v


def _plain(s):
    case, op = s.case, s.case["op"]
    if op == "attention":
        return list(_attend(s)[:2])
    if op == "attention_backward":
        n, B, T, S, H, G, d = (case[k] for k in ("workers", "sequences", "rows", "memory", "heads", "kv_heads", "width"))
        weight, q, k, v = _attend(s)[2:]
        dy = _heads(s, s.dy, T, H)
        if s.counts is not None:
            dy = dy * _valid(s.counts, T).unsqueeze(1)
        dv = torch.matmul(weight.transpose(2, 3), dy)
        dw = torch.matmul(dy, v.transpose(2, 3))
        ds = dw.sub_((dw * weight).sum(-1, keepdim=True)).mul_(weight).mul_(s.scale)
        dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)

        def rows(x, heads):
            return x.transpose(1, 2).reshape(n, -1, heads * d).to(s.dtype)

        def shared(x):
            return rows(x.view(n * B, G, H // G, S, d).sum(2), G)
        return [rows(dq, H), shared(dk), shared(dv)]
    end = (lambda t: t) if s.counts is None else (lambda t, m=_valid(s.counts, case["rows"]): t * m)
    if op == "norm":
        total = s.x if s.r is None else (s.x.float() + s.r.float()).to(s.dtype)
        v = total.float()
        mean = v.mean(-1, keepdim=True)
        v = v - mean
        rstd = (v.square().mean(-1, keepdim=True) + EPS).rsqrt()
        y = v * rstd * s.g.unsqueeze(1) + s.b.unsqueeze(1)
        out = [end(y).to(s.dtype), end(mean).squeeze(-1), end(rstd).squeeze(-1)]
        return out if s.r is None else out + [end(total).to(s.dtype)]
    if op == "norm_backward":
        dy, rstd = end(s.dy.float()), s.rstd.unsqueeze(-1)
        h, gdy = (s.x.float() - s.mean.unsqueeze(-1)) * rstd, dy * s.g.unsqueeze(1)
        dx = rstd * (gdy - gdy.mean(-1, keepdim=True) - h * (gdy * h).mean(-1, keepdim=True))
        if s.r is not None:
            dx = dx + end(s.r.float())
        return [dx.to(s.dtype), (dy * h).sum(1), dy.sum(1)]
    z = s.z.float()
    loss, dz = torch.zeros_like(s.weights), torch.zeros_like(z)
    if s.labels is not None:
        given = (s.labels >= 0).float()
        at = s.labels.clamp(min=0).long().unsqueeze(-1)
        c = z - z.amax(-1, keepdim=True)
        e = c.exp()
        total = e.sum(-1, keepdim=True)
        loss = loss + s.hard * given * (total.log() - c.gather(-1, at)).squeeze(-1)
        dz = e.div_(total).scatter_add_(-1, at, -torch.ones_like(total)).mul_((s.hard * given).unsqueeze(-1))
    if s.t is not None:
        c = (z - z.amax(-1, keepdim=True)) / s.tau
        e = c.exp()
        total = e.sum(-1, keepdim=True)
        t = (s.t - s.t.amax(-1, keepdim=True)) / s.tau
        p = t.exp()
        sum_p = p.sum(-1, keepdim=True)
        p = p / sum_p
        at = s.at.long()
        loss = loss + s.soft * s.tau ** 2 * (p * ((t - sum_p.log()) - (c.gather(-1, at) - total.log()))).sum(-1)
        dz = dz + e.div_(total).scatter_add_(-1, at, -p).mul_(s.soft * s.tau)
    return [end((loss * s.weights).unsqueeze(-1)).squeeze(-1), end(dz * s.weights.unsqueeze(-1)).to(s.dtype)]


# ---- the definition in 64 bits ------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    op, n, T = case["op"], case["workers"], case["rows"]

    def zeros(*shape):
        return torch.zeros(shape, device="cuda", dtype=torch.float64)

    if op.startswith("attention"):
        return _exact_attention(s)
    ends = [T] * n if s.counts is None else s.counts.tolist()
    q = case["cols"]
    if op == "norm":
        y, total, mean, rstd = zeros(n, T, q), zeros(n, T, q), zeros(n, T), zeros(n, T)
        for i, t in enumerate(ends):
            v = s.x[i, :t].double()
            if s.r is not None:
                v = v + s.r[i, :t].double()
            total[i, :t] = v
            v = v.to(s.dtype).double()     # the norm is that of the sum as it is stored
            mean[i, :t] = v.mean(1)
            rstd[i, :t] = 1.0 / torch.sqrt(v.var(1, unbiased=False) + EPS)
            y[i, :t] = F.layer_norm(v, (q,), s.g[i].double(), s.b[i].double(), EPS)
        return [y, mean, rstd] if s.r is None else [y, mean, rstd, total]
    if op == "norm_backward":
        dx, dg, db = zeros(n, T, q), zeros(n, q), zeros(n, q)
        for i, t in enumerate(ends):
            dy, r = s.dy[i, :t].double(), s.rstd[i, :t].double()[:, None]
            h = (s.x[i, :t].double() - s.mean[i, :t].double()[:, None]) * r
            u = dy * s.g[i].double()
            dx[i, :t] = r / q * (q * u - u.sum(1, keepdim=True) - h * (u * h).sum(1, keepdim=True))
            if s.r is not None:
                dx[i, :t] += s.r[i, :t].double()
            dg[i], db[i] = (dy * h).sum(0), dy.sum(0)
        return [dx, dg, db]
    loss, dz = zeros(n, T), zeros(n, T, q)
    for i, end in enumerate(ends):
        z, line = s.z[i, :end].double(), torch.arange(end, device="cuda")
        if s.labels is not None:
            lab = s.labels[i, :end].long()
            keep = lab >= 0
            logq = F.log_softmax(z, -1)
            loss[i, :end] += torch.where(keep, -s.hard * logq[line, lab.clamp(min=0)], 0.0)
            grad = logq.exp()
            grad[line, lab.clamp(min=0)] -= 1.0
            dz[i, :end] += s.hard * grad * keep[:, None]
        if s.t is not None:
            at, logp = s.at[i, :end].long(), F.log_softmax(s.t[i, :end].double() / s.tau, -1)
            logq = F.log_softmax(z / s.tau, -1)
            loss[i, :end] += s.soft * s.tau ** 2 * F.kl_div(logq.gather(1, at), logp, reduction="none", log_target=True).sum(1)
            dz[i, :end] += s.soft * s.tau * logq.exp().scatter_add(1, at, -logp.exp())
        w = s.weights[i, :end].double()
        loss[i, :end] *= w
        dz[i, :end] *= w[:, None]
    return [loss, dz]


def _exact_attention(s):
    """A worker's sequence and query head at a time, over the states that it sees alone."""
    case = s.case
    n, B, T, S, H, G, d = (case[k] for k in ("workers", "sequences", "rows", "memory", "heads", "kv_heads", "width"))
    back = case["op"] == "attention_backward"

    def zeros(*shape):
        return torch.zeros(shape, device="cuda", dtype=torch.float64)

    def by_sequence(x, heads):
        return x.view(n * B, -1, heads, d)

    y, lse = zeros(n * B, T, H, d), zeros(n * B, T, H)
    dq, dk, dv = (zeros(n * B, T, H, d), zeros(n * B, S, G, d), zeros(n * B, S, G, d)) if back else (None,) * 3
    rows = [T] * (n * B) if s.counts is None else s.counts.tolist()
    states = [S] * (n * B) if s.memory_counts is None else s.memory_counts.tolist()
    for b in range(n * B):
        seen = torch.arange(states[b], device="cuda")
        if s.mask is not None:
            seen = seen[s.mask[b, :states[b]].bool()]
        t = rows[b]
        if seen.numel() == 0:
            lse[b, :t] = -math.inf
            continue
        for h in range(H):
            g = h // (H // G)
            q = by_sequence(s.q, H)[b, :t, h].double()
            k, v = by_sequence(s.k, G)[b, seen, g].double(), by_sequence(s.v, G)[b, seen, g].double()
            score = q @ k.t() * s.scale
            lse[b, :t, h] = torch.logsumexp(score, 1)
            p = torch.softmax(score, 1)
            if not back:
                y[b, :t, h] = p @ v
                continue
            dy = by_sequence(s.dy, H)[b, :t, h].double()
            dp = dy @ v.t()
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) * s.scale
            dq[b, :t, h] = ds @ k
            dk[b, :, g].index_add_(0, seen, ds.t() @ q)
            dv[b, :, g].index_add_(0, seen, p.t() @ dy)
    if back:
        return [dq.view(n, B * T, H * d), dk.view(n, B * S, G * d), dv.view(n, B * S, G * d)]
    return [y.view(n, B * T, H * d), lse.view(n, B * T, H)]


def work(case):
    """Each input read once, each output written once; rows behind a sequence's end left out by their expectation (a quarter), hidden
    states (a fifth) kept in the bytes and left out of the operations."""
    n, op = case["workers"], case["op"]
    t = 4.0 if case["dtype"] == "f32" else 2.0
    if op.startswith("attention"):
        n *= case["sequences"]
        share = (3 * n + 1) / (4 * n) if case["ragged"] else 1.0
        T, S, H, G, d = case["rows"] * share, case["memory"] * share, case["heads"], case["kv_heads"], case["width"]
        products = 2.0 * n * H * T * S * d * (0.8 if case["mask"] else 1.0)
        queries, states = n * T * H * d * t, n * S * G * d * t
        if op == "attention":
            return {"bytes": 2 * queries + 2 * states + 4.0 * n * T * H, "flops": 2 * products}
        return {"bytes": 4 * queries + 4 * states + 4.0 * n * T * H, "flops": 5 * products}
    T, q = case["rows"] * ((3 * n + 1) / (4 * n) if case["ragged"] else 1.0), case["cols"]
    if op == "norm":
        return {"bytes": n * T * q * t * (2 + 2 * case["residual"]) + 8.0 * n * (T + q), "flops": 8.0 * n * T * q}
    if op == "norm_backward":
        return {"bytes": n * T * q * t * (3 + case["residual"]) + 4.0 * n * (2 * T + 3 * q), "flops": 12.0 * n * T * q}
    return {"bytes": 2 * n * T * q * t + n * T * (8.0 * case["top"] + 4.0 * case["labels"] + 8.0), "flops": 8.0 * n * T * q}
