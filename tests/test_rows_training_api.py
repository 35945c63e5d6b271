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
