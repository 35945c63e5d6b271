"""More of what the C entry points on rows of activations refuse, without a GPU: each call here differs in one thing from one that is not refused."""
import numpy as np
import pytest
import torch

from paper_2008_01425_amd import binding as B
from paper_2008_01425_amd import workloads as W

AT = 1 << 20          # an address nothing is read from
N, T, P = 3, 4, 6


def context(shapes, n=N):
    edges = W.ring_edges(n)
    return B.pg_init(n, edges, np.full((len(edges),), 0.3, np.float32), [s[0] for s in shapes], [s[1] for s in shapes], 1, 1)


def table(base, n=N, apart=1 << 16):
    return [base + i * apart for i in range(n)]


def rows(width, t=T):
    return B.pg_rows(AT, width, t * width)


def status(call, *args):
    """PG_OK or what the call raised.  The addresses are only numbers: where there is a GPU, a call that is not refused must not be made."""
    try:
        call(*args)
    except B.PGError as e:
        return e.status
    return B.PG_OK


def accepted(call, *args):
    """Past all checks of arguments: without a GPU the first HIP call fails."""
    if torch.cuda.is_available():
        pytest.skip("addresses that are only numbers")
    return status(call, *args) not in (B.PG_OK, B.PG_ERR_ARG)


def test_gradients_of_a_vector_and_its_bias_are_two_layers():
    """A p x 1 layer may be its own bias; its two gradients have one place only, and would be written there by different threads."""
    c = context([(P, 1), (P, 1)])
    params, grads = table(AT), table(2 * AT)

    def backward(bias, g):
        return (c, params, g, 0, bias, T, None, B.PG_F32, rows(P), rows(1), None, B.PG_ACT_NONE, None, None, rows(1), 0, AT)
    assert status(B.pg_linear_backward, *backward(0, grads)) == B.PG_ERR_ARG
    assert accepted(B.pg_linear_backward, *backward(1, grads))
    assert accepted(B.pg_linear_backward, *backward(-1, grads))
    assert accepted(B.pg_linear_backward, *backward(0, None))
    assert accepted(B.pg_linear, c, params, 0, 0, T, None, B.PG_F32, rows(1), None, B.PG_ACT_NONE, None, rows(P), None, AT)
    B.pg_destroy(c)


@pytest.mark.parametrize("n", [2, 3, 17])
def test_gradient_buffers_that_meet(n):
    """Two workers' gradients in one buffer, or in overlapping ones, would be written by different work-groups.  Reading from one is fine."""
    shapes = [(P, 5), (P, 1), (5, 1)]
    c = context(shapes, n)
    size = 4 * B.pg_param_floats(c)
    params = [AT] * n

    def linear(g):
        return status(B.pg_linear_backward, c, params, g, 0, 1, T, None, B.PG_F32, rows(P), rows(5), None, B.PG_ACT_NONE, None, None, rows(5), 0, AT)

    def norm(g):
        return status(B.pg_norm_backward, c, params, g, 2, T, None, B.PG_F32, rows(5), rows(5), AT, None, rows(5), 0, AT)
    apart = table(2 * AT, n, size)
    for call in (linear, norm):
        same, near, before = list(apart), list(apart), list(reversed(apart))
        same[n - 1] = same[0]
        near[n - 1] = near[0] + size - 16
        before[0] = before[n - 1] - size + 16
        for bad in (same, near, before):
            assert call(bad) == B.PG_ERR_ARG
        if not torch.cuda.is_available():
            assert call(apart) != B.PG_ERR_ARG and call(list(reversed(apart))) != B.PG_ERR_ARG
    B.pg_destroy(c)


def test_the_cases_of_refusals_differ_from_calls_that_are_taken():
    """The calls that test_rows_api.py changes in one argument, with a gradient buffer for each worker: taken as they are, refused with each change."""
    from test_rows_api import CASES, P as p, Q as q
    c = context([(p, q), (p, 1), (q, 1), (16385, 1), (4, 4)])
    for call, good, bad in CASES:
        good = dict(good)
        if "grads" in good:
            good["grads"] = table(2 * AT, N, 1 << 20)
        for change in bad:
            if call is B.pg_linear and change == dict(x=None, x8=AT):
                change = dict(x=None, x8=AT, z8=AT)
            if call is B.pg_linear_backward and change in (dict(grads=[AT, AT, AT + 8]),):
                change = dict(grads=[2 * AT, 3 * AT, 4 * AT + 8])
            assert status(call, c, *{**good, **change}.values()) == B.PG_ERR_ARG, (call.__name__, change)
        assert torch.cuda.is_available() or accepted(call, c, *good.values()), call.__name__
    B.pg_destroy(c)


@pytest.mark.parametrize("tile", [32, 64, 128])
def test_more_forced_tiles_than_a_launch_takes(tile):
    """No tile of the forced size makes a launch of at most 2^22: the call is refused, rather than taken and nothing computed.  The same rows by the estimate are fine."""
    from parity_util import env_settings
    many = (1 << 22) * tile + 1
    assert many <= 1 << 30
    for forced in (True, False):
        with env_settings(dict(PG_LINEAR_TILE=tile) if forced else {}):
            c = context([(P, 5), (P, 1)], 1)
        x, y = B.pg_rows(AT, 5, 0), B.pg_rows(AT, P, 0)
        forward = (c, [AT], 0, 1, many, None, B.PG_BF16, x, None, B.PG_ACT_NONE, None, y, None, AT)
        backward = (c, [AT], None, 0, 1, many, None, B.PG_BF16, y, x, None, B.PG_ACT_NONE, None, None, x, 0, AT)
        if forced:
            assert status(B.pg_linear, *forward) == status(B.pg_linear_backward, *backward) == B.PG_ERR_ARG
        elif not torch.cuda.is_available():
            assert accepted(B.pg_linear, *forward) and accepted(B.pg_linear_backward, *backward)
        B.pg_destroy(c)


def test_rows_up_to_two_to_the_thirty():
    """2^30 rows over all workers are refused, one less is not."""
    none = (1 << 64) - 1
    for n in (1, 4):
        c = context([(P, 5), (P, 1), (5, 1)], n)
        first = (1 << 30) // n
        assert B.pg_checkpoint_bytes(c, first, 5) == none and B.pg_checkpoint_bytes(c, first - 1, 5) != none
        assert B.pg_linear_workspace_bytes(c, 0, first, B.PG_BF16) == none and B.pg_linear_workspace_bytes(c, 0, first - 1, B.PG_BF16) != none
        assert B.pg_norm_workspace_bytes(c, 2, first) == none and B.pg_norm_workspace_bytes(c, 2, first - 1) != none
        x = B.pg_rows(AT, 5, 1 << 40)
        assert status(B.pg_norm, c, [AT] * n, 2, first, None, B.PG_F32, 1e-6, x, None, None, x, None, None) == B.PG_ERR_ARG
        assert status(B.pg_checkpoint_store, c, first, 5, None, B.PG_F32, x, AT) == B.PG_ERR_ARG
        if not torch.cuda.is_available():
            assert accepted(B.pg_norm, c, [AT] * n, 2, first - 1, None, B.PG_F32, 1e-6, x, None, None, x, None, None)
            assert accepted(B.pg_checkpoint_store, c, first - 1, 5, None, B.PG_F32, x, AT)
        B.pg_destroy(c)
