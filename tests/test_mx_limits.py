"""Sizes past what a call takes are refused on the host before anything is launched (there is no GPU here: a launch would
report POLYQ_ERR_DEVICE).  No device pointer is dereferenced."""
import ctypes

import pytest
import torch

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


@pytest.mark.parametrize("rows,k", [((1 << 32) + 16, 64), (16, (1 << 32) + 64), ((1 << 24) + 1, 64), (16, (1 << 20) + 1)])
def test_sizes_past_32_bits_are_not_cut_to_them(rows, k):
    """A size of 2^32 + 16 is not 16: the binding refuses what the library's 32-bit arguments cannot hold."""
    room = torch.zeros(1280, dtype=torch.uint8)
    with pytest.raises(ValueError, match="packed matrix"):
        pq.MXMatrix(rows, k, room)


def test_more_rows_than_32_bits_hold_are_not_cut_to_them():
    w = pq.MXMatrix(16, 64, torch.zeros(1280, dtype=torch.uint8))
    rows = (1 << 32) + 16
    x, d = torch.zeros(1).expand(rows, 64), torch.zeros(1).expand(rows, 16)
    for call_ in (lambda: pq.mx_quantize(x), lambda: pq.mx_linear(x, w), lambda: pq.mx_gated(x, w, w),
                  lambda: pq.mx_linear_backward(d, x, w), lambda: pq.mx_linear_backward(d, None, w, need_dw=False),
                  lambda: pq.mx_gated_backward(d, x, w, w)):
        with pytest.raises(ValueError, match="rows"):
            call_()


def test_a_gradient_is_not_lost_without_a_word():
    """An x that requires a gradient is refused where autograd records; what refuses it elsewhere is that it is on the CPU."""
    w = pq.MXMatrix(16, 64, torch.zeros(1280, dtype=torch.uint8))
    x = torch.zeros((4, 64), requires_grad=True)
    for product in (lambda v: pq.mx_linear(v, w), lambda v: pq.mx_gated(v, w, w)):
        for v in (x, x * 2):
            with pytest.raises(ValueError, match="requires a gradient"):
                product(v)
        with pytest.raises(ValueError, match="GPU tensors"):
            product(x.detach())
        with torch.no_grad(), pytest.raises(ValueError, match="GPU tensors"):
            product(x)
