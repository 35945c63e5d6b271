"""Plain statements in 64 bits of the operators on rows of activations, and what their arithmetic may cost."""
import math

import torch

from paper_2008_01425_amd import workloads as W

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # half a step, relative


def buffers(n, shapes):
    """A context over n workers with gradient buffers, ring or less."""
    from paper_2008_01425_amd.device import GossipBuffers
    edges = W.ring_edges(n)
    gb = GossipBuffers(n, edges, [1.0 / 3.0] * len(edges), shapes, 1, 1)
    gb.alloc_grads()
    return gb


def put(gb, l, w):
    for i in range(gb.n):
        gb.set_layer(i, l, w[i].float().numpy())


def grad(gb, l):
    return torch.stack([gb.layer_of(g, l).cpu() for g in gb.g]).double()


def held(x):
    """(values, exponents) of an 8-bit checkpoint of x, element by element from the definition."""
    q = x.shape[-1]
    v = torch.nn.functional.pad(x.double(), (0, -q % 32)).unflatten(-1, (-1, 32))
    fin = torch.isfinite(v)
    top = torch.where(fin, v.abs(), 0.0).amax(-1, keepdim=True)
    e = torch.full_like(top, -117.0)
    while bool((top > 448.0 * 2.0 ** e).any()):
        e = torch.where(top > 448.0 * 2.0 ** e, e + 1, e)
    u = torch.where(fin, v * 2.0 ** -e, 0.0)
    k = torch.floor(torch.log2(u.abs().clamp(min=2.0 ** -6)))
    step = 2.0 ** (k - 3)
    u = torch.round(u / step) * step
    return torch.where(fin, u * 2.0 ** e, math.nan).flatten(-2)[..., :q], e.squeeze(-1)


def act(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    return z * torch.sigmoid(z) if name == "silu" else z


def slope(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        g = torch.sigmoid(z)
        return g * (1 + z * (1 - g))
    return torch.ones_like(z)


def product_error(x, w, dtype):
    """What a product x w may be off by, from the sums of the products' sizes: float accumulation of K terms, K 2^-24 of that; pieces
    left out, 2^-24; a weight rounded to bf16, 2^-8."""
    size = torch.matmul(x.abs(), w.abs())
    return size * (x.shape[-1] * 2.0 ** -24 + (2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8))


def mask(n, rows, counts):
    return torch.arange(rows)[None, :, None] < (torch.full((n,), rows) if counts is None else counts.cpu().clamp(0, rows))[:, None, None]
