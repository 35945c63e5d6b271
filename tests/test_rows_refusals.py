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
