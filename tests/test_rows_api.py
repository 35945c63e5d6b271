"""What the C entry points on rows of activations refuse, without a GPU: every refusal comes before any HIP call, so the addresses here are only numbers."""
import numpy as np
import pytest

from paper_2008_01425_amd import binding as B
from paper_2008_01425_amd import workloads as W

AT = 1 << 20          # an address nothing is read from
N, P, Q, T = 3, 6, 5, 4
WORKERS = [AT] * N


@pytest.fixture
def ctx():
    # 0: weights, 1: bias, 2: gain, 3: a gain too long, 4: another matrix
    shapes = [(P, Q), (P, 1), (Q, 1), (16385, 1), (4, 4)]
    c = B.pg_init(N, W.ring_edges(N), np.full((N,), 0.3, np.float32), [s[0] for s in shapes], [s[1] for s in shapes], 1, 1)
    yield c
    B.pg_destroy(c)


def rows(width, data=AT, row=None, worker=None):
    row = width if row is None else row
    return B.pg_rows(data, row, T * row if worker is None else worker)


def refused(call, *args):
    with pytest.raises(B.PGError) as e:
        call(*args)
    assert e.value.status == B.PG_ERR_ARG


LINEAR = dict(params=WORKERS, layer=0, bias=1, rows=T, counts=None, type=B.PG_F32, x=rows(Q), x8=None, act=B.PG_ACT_GELU, residual=rows(P),
              y=rows(P), z8=AT, ws=AT)
BACKWARD = dict(params=WORKERS, grads=WORKERS, layer=0, bias=1, rows=T, counts=None, type=B.PG_F32, dz=rows(P), x=rows(Q), x8=None,
                act=B.PG_ACT_SILU, z8=AT, residual=rows(Q), dx=rows(Q), accumulate=0, ws=AT)
NORM = dict(params=WORKERS, layer=2, rows=T, counts=None, type=B.PG_F32, eps=1e-6, x=rows(Q), residual=rows(Q), sum=rows(Q), y=rows(Q), y8=AT,
            rstd=AT)
NORM_BACKWARD = dict(params=WORKERS, grads=WORKERS, layer=2, rows=T, counts=None, type=B.PG_F32, dy=rows(Q), sum=rows(Q), rstd=AT,
                     residual=rows(Q), dx=rows(Q), accumulate=0, ws=AT)
STORE = dict(rows=T, cols=Q, counts=None, type=B.PG_F32, x=rows(Q), kept=AT)
LOAD = dict(rows=T, cols=Q, counts=None, type=B.PG_F32, kept=AT, x=rows(Q))
BACK = dict(rows=T, cols=Q, counts=None, type=B.PG_F32, act=B.PG_ACT_RELU, dy=rows(Q), z8=AT, dz=rows(Q))

ANY = [dict(rows=-1), dict(rows=1 << 30), dict(type=2), dict(type=-1), dict(counts=AT + 2)]
LAYER = ANY + [dict(layer=-1), dict(layer=5), dict(params=[AT, 0, AT]), dict(params=[AT, AT + 4, AT])]


def bad_rows(name, width, output, needed):
    out = [dict([(name, r)]) for r in (rows(width, AT + 2), rows(width, row=-1), rows(width, row=(1 << 21) + 1), rows(width, worker=-1),
                                       rows(width, worker=(1 << 40) + 1))]
    if output:      # rows, or workers, that meet
        out += [dict([(name, r)]) for r in (rows(width, row=0), rows(width, row=width - 1), rows(width, worker=0), rows(width, worker=T * width - 1),
                                            B.pg_rows(AT, 2 * width, width))]
    if needed:
        out += [dict([(name, None)]), dict([(name, rows(width, 0))])]
    return out


CASES = [
    (B.pg_linear, LINEAR, LAYER + [dict(layer=4), dict(bias=-2), dict(bias=2), dict(bias=0), dict(bias=5), dict(act=4), dict(act=-1), dict(x=None),
                                   dict(x8=AT), dict(x8=AT + 8, x=None), dict(z8=AT + 8), dict(x=None, x8=AT), dict(ws=AT + 128)]
     + bad_rows("x", Q, False, True) + bad_rows("residual", P, False, False) + bad_rows("y", P, True, True)),
    (B.pg_linear_backward, BACKWARD, LAYER + [dict(layer=4), dict(bias=-2), dict(bias=2), dict(act=4), dict(act=-1), dict(x=None), dict(x8=AT),
                                              dict(x8=AT + 8, x=None), dict(z8=None), dict(z8=AT + 8), dict(act=B.PG_ACT_NONE), dict(accumulate=2),
                                              dict(grads=None, dx=None), dict(grads=[0, AT, AT]), dict(grads=[AT, AT, AT + 8]), dict(ws=AT + 128)]
     + bad_rows("dz", P, False, True) + bad_rows("x", Q, False, True) + bad_rows("residual", Q, False, False) + bad_rows("dx", Q, True, False)),
    (B.pg_norm, NORM, LAYER + [dict(layer=0), dict(layer=3), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")),
                               dict(y=None, y8=None), dict(y8=AT + 8), dict(rstd=AT + 2)]
     + bad_rows("x", Q, False, True) + bad_rows("residual", Q, False, False) + bad_rows("sum", Q, True, False) + bad_rows("y", Q, True, False)),
    (B.pg_norm_backward, NORM_BACKWARD, LAYER + [dict(layer=0), dict(layer=3), dict(accumulate=-1), dict(rstd=None), dict(rstd=AT + 2), dict(ws=None),
                                                 dict(ws=AT + 64), dict(grads=[0, AT, AT])]
     + bad_rows("dy", Q, False, True) + bad_rows("sum", Q, False, True) + bad_rows("residual", Q, False, False) + bad_rows("dx", Q, True, True)),
    (B.pg_checkpoint_store, STORE, ANY + [dict(cols=0), dict(cols=(1 << 21) + 1), dict(kept=None), dict(kept=AT + 8)] + bad_rows("x", Q, False, True)),
    (B.pg_checkpoint_load, LOAD, ANY + [dict(cols=0), dict(kept=None), dict(kept=AT + 8)] + bad_rows("x", Q, True, True)),
    (B.pg_activation_backward, BACK, ANY + [dict(cols=0), dict(act=B.PG_ACT_NONE), dict(act=4), dict(z8=None), dict(z8=AT + 8)]
     + bad_rows("dy", Q, False, True) + bad_rows("dz", Q, True, True)),
]


@pytest.mark.parametrize("call,good,bad", CASES, ids=[c[0].__name__ for c in CASES])
def test_bad_arguments_are_refused(ctx, call, good, bad):
    for change in bad:
        assert set(change) <= set(good), change
        if call is B.pg_linear and change == dict(x=None, x8=AT):
            change = dict(x=None, x8=AT, z8=AT)         # kept where it is read from
        refused(call, ctx, *{**good, **change}.values())
    refused(call, None, *good.values())


def test_sizes(ctx):
    none = (1 << 64) - 1
    assert B.pg_checkpoint_bytes(ctx, T, Q) == 512 + N * T            # 12 rows of 32 codes up to 512, a scale each
    assert B.pg_checkpoint_bytes(ctx, 0, Q) == 0
    assert B.pg_checkpoint_bytes(ctx, 100, 65) == 300 * 96 + 128 + 300 * 3
    for bad in ((-1, 5), (5, 0), (1 << 30, 5), (5, (1 << 21) + 1)):
        assert B.pg_checkpoint_bytes(ctx, *bad) == none
    assert B.pg_norm_workspace_bytes(ctx, 2, T) > 0
    for bad in ((0, T), (3, T), (9, T), (-1, T), (2, -1)):
        assert B.pg_norm_workspace_bytes(ctx, *bad) == none
    for bad in ((9, T, 0), (-1, T, 0), (0, -1, 0), (0, T, 2)):
        assert B.pg_linear_workspace_bytes(ctx, *bad) == none
    assert B.pg_linear_workspace_bytes(ctx, 0, T, B.PG_BF16) != none
    assert B.pg_checkpoint_bytes(None, T, Q) == B.pg_norm_workspace_bytes(None, 2, T) == B.pg_linear_workspace_bytes(None, 0, T, 0) == none


def test_kernels_have_their_kinds_and_registers():
    """Profile summaries name every kernel; none of them needs scratch memory beyond a few spilled addresses, tiles and norms keep two wavefronts per SIMD."""
    import code_objects
    from paper_2008_01425_amd.rocprof_summary import kernel_kind
    assert kernel_kind("pg::linear_kernel<0, 1, true, false, 256, 256, 64, 2, 4>") == "linear"
    assert kernel_kind("pg::linear_kernel<1, 0, false, false, 32, 128, 32, 1, 4>") == "linear_dx"
    assert kernel_kind("pg::linear_join_kernel<2, 1, 64, 128, 2, 2>") == kernel_kind("pg::linear_kernel<2, 0, true, false, 64, 128, 32, 2, 2>") == "linear_dw"
    assert kernel_kind("pg::norm_kernel<1, 256, 1>") == "norm"
    assert kernel_kind("pg::norm_backward_kernel<1, 256, 1>") == kernel_kind("pg::norm_join_kernel") == "norm_backward"
    assert kernel_kind("pg::kept_kernel<0, 0>") == kernel_kind("pg::kept_kernel<1, 1>") == "checkpoint"
    assert kernel_kind("pg::kept_kernel<1, 2>") == "activation"
    found = dict.fromkeys(("linear_kernel<", "linear_join_kernel<", "norm_kernel<", "norm_backward_kernel<", "kept_kernel<"), 0)
    for name, kernel in code_objects.kernels(B.LIB_PATH).items():
        for stem in found:
            if name.startswith("pg::" + stem):
                used = (kernel[".vgpr_count"] + kernel.get(".agpr_count", 0) + 7) // 8 * 8
                assert 512 // used >= 2, (name, used)
                assert kernel[".private_segment_fixed_size"] <= 16, name
                found[stem] += 1
    assert found["linear_kernel<"] >= 40 and all(found.values()), found
