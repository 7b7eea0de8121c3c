"""Sizes past what a call takes are refused on the host before anything is launched (there is no GPU here: a launch would
report POLYQ_ERR_DEVICE).  No device pointer is dereferenced."""
import ctypes

import pytest

import paper_2607_14618_amd as pq

P = ctypes.c_void_p(1 << 20)
CAPACITY = 5
HUGE = 1 << 60    # a workspace that is never too small


def call(name, *args):
    return getattr(pq.lib(), name)(*args)


# a launch's work-items have to stay below 2^32
@pytest.mark.parametrize("t", [0, 1, 2])
@pytest.mark.parametrize("rows,k", [(1 << 24, 8192), (1 << 24, 1 << 20), ((1 << 18) - 15, 1 << 19)])
def test_quantization_of_too_many_records(rows, k, t):
    assert call("polyq_mx_quantize", P, t, rows, k, P, None) == CAPACITY
    assert call("polyq_mx_dequantize", P, rows, k, P, t, None) == CAPACITY


@pytest.mark.parametrize("m,n,k,xt", [(1 << 24, 1 << 24, 32, 3), (1 << 24, 1 << 24, 32, 0), (1 << 18, 1 << 24, 32, 3),
                                      (1 << 18, 1 << 24, 32, 2), (1 << 24, 1 << 18, 1000, 1), (1 << 24, 64, 1 << 20, 2)])
def test_products_of_too_many_tiles(m, n, k, xt):
    assert call("polyq_mx_linear", P, xt, m, P, n, k, P, 2, P, HUGE, None) == CAPACITY
    assert call("polyq_mx_gated", P, xt, m, P, P, n, k, 0, P, 2, P, HUGE, None) == CAPACITY


@pytest.mark.parametrize("xt", [2, 3])
@pytest.mark.parametrize("m,n,dx,dw", [(1 << 21, 64, P, None), (64, 1 << 21, None, P), (1 << 21, 64, None, P)])
def test_gradients_of_too_many_tiles(m, n, dx, dw, xt):
    """dx of 2^21 x 2^20, dW of as many, and an x of that many to transpose."""
    k = 1 << 20
    assert call("polyq_mx_linear_backward", P, 2, P, xt, m, P, n, k, dx, dw, 2, P, HUGE, None) == CAPACITY
    assert call("polyq_mx_gated_backward", P, 2, P, xt, m, P, P, n, k, 0, dx, dw, dw, 2, P, HUGE, None) == CAPACITY


def test_gated_gradients_of_too_many_tokens_and_rows():
    m = 1 << 21     # g and u of 2^21 x 2^21
    assert call("polyq_mx_gated_backward", P, 2, P, 3, m, P, P, m, 32, 0, P, None, None, 2, P, HUGE, None) == CAPACITY
