"""What the C entry points of layer norms and distillation losses refuse, without a GPU: every refusal comes before any HIP call, so the addresses here
are only numbers."""
import math

import numpy as np
import pytest
import torch

from paper_2008_01425_amd import binding as B
from paper_2008_01425_amd import workloads as W
from test_rows_api import ANY, AT, LAYER, N, Q, T, WORKERS, bad_rows, rows
from test_rows_refusals import accepted, status, table

GRADS = table(2 * AT, N, 1 << 20)


@pytest.fixture
def ctx():
    # 0: weights, 1: bias, 2: gain, 3: a gain too long, 4: the bias of the norm
    shapes = [(6, Q), (6, 1), (Q, 1), (16385, 1), (Q, 1)]
    c = B.pg_init(N, W.ring_edges(N), np.full((N,), 0.3, np.float32), [s[0] for s in shapes], [s[1] for s in shapes], 1, 1)
    yield c
    B.pg_destroy(c)


NORM = dict(params=WORKERS, layer=2, bias=4, rows=T, counts=None, type=B.PG_F32, eps=1e-5, x=rows(Q), residual=rows(Q), sum=rows(Q), y=rows(Q), y8=AT,
            mean=AT, rstd=2 * AT)
BACKWARD = dict(params=WORKERS, grads=GRADS, layer=2, bias=4, rows=T, counts=None, type=B.PG_F32, dy=rows(Q), sum=rows(Q), mean=AT, rstd=AT,
                residual=rows(Q), dx=rows(Q), accumulate=0, ws=AT)
DISTILL = dict(rows=T, cols=Q, counts=None, type=B.PG_F32, logits=rows(Q), labels=AT, hard=0.5, top=2, index=AT, top_logits=AT, temperature=2.0, soft=0.5,
               weights=AT, loss=2 * AT, dlogits=rows(Q))

CASES = [
    (B.pg_layer_norm, NORM, LAYER + [dict(layer=0), dict(layer=3), dict(bias=0), dict(bias=1), dict(bias=-2), dict(bias=5), dict(eps=0.0), dict(eps=-1.0),
                                     dict(eps=math.inf), dict(eps=math.nan), dict(y=None, y8=None), dict(y8=AT + 8), dict(mean=AT + 2), dict(rstd=AT + 1),
                                     dict(mean=2 * AT)]
     + bad_rows("x", Q, False, True) + bad_rows("residual", Q, False, False) + bad_rows("sum", Q, True, False) + bad_rows("y", Q, True, False),
     [dict(bias=-1), dict(bias=2), dict(mean=None), dict(rstd=None, mean=None), dict(y=None), dict(y8=None), dict(sum=None), dict(residual=None), dict(rows=0, x=rows(Q, 0))]),
    (B.pg_layer_norm_backward, BACKWARD, LAYER + [dict(layer=0), dict(layer=3), dict(bias=2), dict(bias=1), dict(bias=-2), dict(accumulate=-1), dict(mean=None),
                                                  dict(rstd=None), dict(mean=AT + 2), dict(rstd=AT + 2), dict(ws=None), dict(ws=AT + 64),
                                                  dict(grads=[0] + GRADS[1:]), dict(grads=[GRADS[0], GRADS[0] + 16, GRADS[2]])]
     + bad_rows("dy", Q, False, True) + bad_rows("sum", Q, False, True) + bad_rows("residual", Q, False, False) + bad_rows("dx", Q, True, True),
     [dict(bias=-1), dict(grads=None, ws=None), dict(grads=None, bias=2), dict(residual=None), dict(accumulate=1)]),
    (B.pg_distill, DISTILL, ANY + [dict(cols=0), dict(cols=(1 << 21) + 1), dict(top=-1), dict(top=Q + 1), dict(index=None), dict(top_logits=None), dict(labels=AT + 1),
                                   dict(index=AT + 2), dict(top_logits=AT + 2), dict(weights=AT + 2), dict(loss=AT + 2), dict(hard=math.nan), dict(soft=math.inf),
                                   dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf),
                                   dict(temperature=2.0 ** -21), dict(temperature=2.0 ** 21), dict(loss=None, dlogits=None), dict(loss=AT)]
     + bad_rows("logits", Q, False, True) + bad_rows("dlogits", Q, True, False),
     [dict(labels=None), dict(top=0, index=None, top_logits=None), dict(weights=None), dict(loss=None), dict(dlogits=None), dict(temperature=2.0 ** -20),
      dict(temperature=2.0 ** 20), dict(hard=0.0, soft=-1.0), dict(top=Q)]),
]


@pytest.mark.parametrize("call,good,bad,fine", CASES, ids=[c[0].__name__ for c in CASES])
def test_bad_arguments_are_refused(ctx, call, good, bad, fine):
    for change in bad:
        assert set(change) <= set(good), change
        assert status(call, ctx, *{**good, **change}.values()) == B.PG_ERR_ARG, change
    assert status(call, None, *good.values()) == B.PG_ERR_ARG
    if torch.cuda.is_available():
        return
    for change in [{}] + fine:
        assert set(change) <= set(good) and accepted(call, ctx, *{**good, **change}.values()), change


def test_entries_of_a_teacher_end_at_1024():
    c = B.pg_init(1, np.zeros((0, 2), np.int32), np.zeros(0, np.float32), [4], [4], 1, 1)
    good = dict(DISTILL, cols=5000, logits=B.pg_rows(AT, 5000, 0), dlogits=B.pg_rows(AT, 5000, 0))
    assert status(B.pg_distill, c, *dict(good, top=1025).values()) == B.PG_ERR_ARG
    assert torch.cuda.is_available() or accepted(B.pg_distill, c, *dict(good, top=1024).values())
    B.pg_destroy(c)


def test_sizes(ctx):
    none = (1 << 64) - 1
    assert B.pg_layer_norm_workspace_bytes(ctx, 2, T) == 2 * B.pg_norm_workspace_bytes(ctx, 2, T)
    for bad in ((0, T), (3, T), (9, T), (-1, T), (2, -1), (2, 1 << 30)):
        assert B.pg_layer_norm_workspace_bytes(ctx, *bad) == none
    assert B.pg_layer_norm_workspace_bytes(None, 2, T) == none


def test_kernels_have_their_kinds_and_registers():
    import code_objects
    from paper_2008_01425_amd.rocprof_summary import kernel_kind
    assert kernel_kind("pg::norm_kernel<1, 256, 1, true>") == "layer_norm" and kernel_kind("pg::norm_kernel<1, 256, 1, false>") == "norm"
    assert kernel_kind("pg::norm_backward_kernel<1, 256, 1, true>") == "layer_norm_backward"
    assert kernel_kind("pg::norm_backward_kernel<1, 256, 1, false>") == "norm_backward"
    assert kernel_kind("pg::distill_kernel<1, 1024, 5, true>") == "distill"
    kernels = code_objects.kernels(B.LIB_PATH)
    found = [k for name, k in kernels.items() if name.startswith("pg::distill_kernel<")]
    assert len(found) >= 20 and all(k[".private_segment_fixed_size"] == 0 for k in found)


def shape(**change):
    s = dict(sequences=2, rows=3, memory=4, heads=4, kv_heads=2, width=5, scale=0.5, counts=None, memory_counts=None, mask=None)
    return B.pg_attention_shape(*{**s, **change}.values())


def strided(cols, count, row=None, worker=None, data=AT):
    row = cols if row is None else row
    return B.pg_rows(data, row, count * row if worker is None else worker)


def bad_strides(name, cols, count, output, needed):
    at = 5 * AT if output else AT
    out = [strided(cols, count, data=at + 2), strided(cols, count, row=-1, data=at), strided(cols, count, row=(1 << 21) + 1, data=at),
           strided(cols, count, worker=-1, data=at), strided(cols, count, worker=(1 << 40) + 1, data=at)]
    if output:
        out += [strided(cols, count, row=0, data=at), strided(cols, count, row=cols - 1, data=at), strided(cols, count, worker=0, data=at),
                strided(cols, count, worker=count * cols - 1, data=at), B.pg_rows(at, 2 * cols, cols)]
    if needed:
        out += [None, strided(cols, count, data=0)]
    return [dict([(name, r)]) for r in out]


BAD_SHAPES = [dict(shape=None)] + [dict(shape=shape(**s)) for s in (
    dict(sequences=0), dict(sequences=-1), dict(rows=-1), dict(memory=-1), dict(heads=3), dict(heads=0), dict(kv_heads=0), dict(kv_heads=-2), dict(kv_heads=8),
    dict(width=0), dict(width=257), dict(heads=1 << 14, width=256), dict(scale=0.0), dict(scale=-0.5), dict(scale=math.inf), dict(scale=math.nan), dict(counts=AT + 2),
    dict(memory_counts=AT + 1), dict(rows=1 << 28), dict(memory=1 << 28), dict(sequences=1 << 29), dict(heads=1 << 12, kv_heads=1, rows=1 << 20))]
ATTENTION = dict(shape=shape(counts=AT, memory_counts=AT, mask=AT + 1), type=B.PG_BF16, q=strided(20, 6), k=strided(10, 8), v=strided(10, 8), y=strided(20, 6, data=2 * AT), lse=AT, ws=AT)
ATTENTION_BACKWARD = dict(shape=shape(), type=B.PG_F32, dy=strided(20, 6), q=strided(20, 6), k=strided(10, 8), v=strided(10, 8), y=strided(20, 6), lse=AT,
                          dq=strided(20, 6, data=2 * AT), dk=strided(10, 8, data=3 * AT), dv=strided(10, 8, data=4 * AT), ws=AT)


def test_attention_refuses_bad_arguments(ctx):
    odd = [dict([(name, strided(20, 6, data=AT + 1))]) for name in ("q", "y")] + [dict(y=strided(20, 6))]
    bad = BAD_SHAPES + [dict(type=2), dict(type=-1), dict(lse=AT + 2), dict(ws=AT + 128)] + odd
    for name, cols, count, output in (("q", 20, 6, False), ("k", 10, 8, False), ("v", 10, 8, False), ("y", 20, 6, True)):
        bad += [c for c in bad_strides(name, cols, count, output, True) if c[name] is None or (c[name].data or 0) % 4 != 2]      # fine for bf16
    back = BAD_SHAPES + [dict(type=2), dict(lse=AT + 2), dict(lse=None), dict(ws=AT + 128), dict(ws=None), dict(dk=None), dict(dv=None), dict(dq=None, dk=None, dv=None),
                         dict(dq=strided(20, 6)), dict(dk=strided(10, 8)), dict(dv=strided(10, 8)), dict(dv=strided(10, 8, data=3 * AT)), dict(dk=strided(10, 8, data=2 * AT))]
    for name, cols, count, output in (("dy", 20, 6, False), ("q", 20, 6, False), ("k", 10, 8, False), ("v", 10, 8, False), ("y", 20, 6, False), ("dq", 20, 6, True),
                                      ("dk", 10, 8, True), ("dv", 10, 8, True)):
        back += bad_strides(name, cols, count, output, name[1:] not in ("q", "k", "v"))
    for call, good, changes in ((B.pg_attention, ATTENTION, bad), (B.pg_attention_backward, ATTENTION_BACKWARD, back)):
        for change in changes:
            assert set(change) <= set(good), change
            assert status(call, ctx, *{**good, **change}.values()) == B.PG_ERR_ARG, (call.__name__, change)
        assert status(call, None, *good.values()) == B.PG_ERR_ARG
    if torch.cuda.is_available():
        return
    for change in ({}, dict(lse=None), dict(ws=None), dict(shape=shape()), dict(shape=shape(memory=0), k=strided(10, 0, data=0), v=strided(10, 0, data=0))):
        assert accepted(B.pg_attention, ctx, *{**ATTENTION, **change}.values()), change
    for change in ({}, dict(dq=None), dict(dk=None, dv=None)):
        assert accepted(B.pg_attention_backward, ctx, *{**ATTENTION_BACKWARD, **change}.values()), change


def test_attention_workspaces(ctx):
    none = (1 << 64) - 1
    for bad in BAD_SHAPES:
        assert B.pg_attention_workspace_bytes(ctx, bad["shape"], B.PG_BF16, False) == none
    assert B.pg_attention_workspace_bytes(ctx, shape(), 2, False) == B.pg_attention_workspace_bytes(None, shape(), 0, False) == none
    assert B.lib.pg_attention_workspace_bytes(ctx, shape(), 0, 2) == none
    assert B.pg_attention_workspace_bytes(ctx, shape(), B.PG_BF16, False) == 0                    # a tile of states: nothing to split
    assert B.pg_attention_workspace_bytes(ctx, shape(), B.PG_BF16, True) == 4 * 128               # 72 floats of dy . y in whole 256 bytes
    long = shape(memory=4096, rows=1, heads=16, kv_heads=4, width=128)
    assert B.pg_attention_workspace_bytes(ctx, long, B.PG_BF16, False) > 0


def test_attention_kernels_have_their_kinds_and_registers():
    """Own rows and results of every width up to 128 fit the registers of a lane, but for the 96 bytes that two wavefronts a SIMD are worth."""
    import code_objects
    import re
    from paper_2008_01425_amd.rocprof_summary import kernel_kind
    assert kernel_kind("pg::attention_kernel<1, 128, 4>") == kernel_kind("pg::attention_join_kernel<1>") == "attention"
    assert kernel_kind("pg::attention_dq_kernel<1, 128, 4>") == kernel_kind("pg::attention_delta_kernel<0>") == "attention_dq"
    assert kernel_kind("pg::attention_dkv_kernel<1, 128, 3>") == kernel_kind("pg::attention_sum_kernel<0>") == "attention_dkv"
    found = 0
    for name, kernel in code_objects.kernels(B.LIB_PATH).items():
        m = re.match(r"pg::attention_(|dq_|dkv_)kernel<1, (\d+), ", name)
        if m and int(m.group(2)) <= 128:
            assert kernel[".private_segment_fixed_size"] <= 96, name
            found += 1
    assert found >= 12
