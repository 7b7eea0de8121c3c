"""Values at the ends of their range through the microscaled 4-bit operators.  Tolerances as derived at the head of
test_gpu_mx.py."""
import pytest
import torch

import paper_2607_14618_amd as pq
from gpu_util import dev
from test_gpu_mx import F, HALF, TERM, out_tol

pytestmark = pytest.mark.gpu

TOP = [2.0 ** 128 - 2.0 ** 104, 2.0 ** 128 - 2.0 ** 119, 2.0 ** 128 - 2.0 ** 119 - 2.0 ** 104, 2.0 ** 128 - 2.0 ** 120,
       2.0 ** 128 - 2.0 ** 111, 2.0 ** 128 - 2.0 ** 111 - 2.0 ** 104, 2.0 ** 128 - 2.0 ** 112 + 2.0 ** 104, 2.0 ** 127 + 2.0 ** 104]


def test_gradients_next_to_the_largest_value_are_exact():
    """dy = +- the fp32 values from 2^128 - 2^119 on, which round to an infinity in bf16: one W or x^ of a power of two
    in every sum, so that fp32 gradients are the products themselves."""
    size = 64
    dy = torch.randn((size, size), generator=torch.Generator().manual_seed(1)) * 2.0 ** 100
    for i, v in enumerate(TOP):
        dy[i, ::2], dy[i, 1::2] = v, -v
        dy[8:, 8 + i] = v
    power = torch.tensor([1.0, 0.5, -1.0, 2.0 ** -20])[torch.arange(size) % 4]
    one = pq.mx_quantize(torch.diag(power).to(dev()))
    dx, dw = pq.mx_linear_backward(dy.to(dev()), torch.diag(power).to(dev()), one)
    assert torch.equal(dx.cpu(), dy * power)
    assert torch.equal(dw.cpu(), dy.T * power)


@pytest.mark.parametrize("gt", ["bf16", "fp16"])
def test_narrow_gradients_of_the_largest_values_are_finite(gt):
    """The same dy with gradients in 16 bits: W brings the products into their range."""
    typ, size = F[gt], 64
    dy = torch.randn((size, size), generator=torch.Generator().manual_seed(1)) * 2.0 ** 100
    for i, v in enumerate(TOP):
        dy[i, ::2], dy[i, 1::2] = v, -v
    w = torch.eye(size) * 2.0 ** -114
    dx, _ = pq.mx_linear_backward(dy.to(dev()), None, pq.mx_quantize(w.to(dev())), dtype=typ, need_dw=False)
    want = dy.double() * 2.0 ** -114
    got = dx.cpu().double()
    assert bool(torch.isfinite(got).all())
    # one bf16 value below the largest instead of rounding up to an infinity: off by a whole step (2^-8 of 2^128) there
    term = TERM[typ] * (2 if gt == "bf16" else 1)
    assert bool(((got - want).abs() <= term * want.abs() + HALF[typ] * want.abs() * (1 + term) + out_tol(0 * want, typ)).all())


def test_gated_gradients_next_to_the_largest_value_are_exact():
    """g = 64 makes silu's slope 1 to the last bit and u = 1: dg is dh."""
    m, n, k = 8, 8, 32
    x, gate, up = torch.zeros((m, k)), torch.zeros((n, k)), torch.zeros((n, k))
    x[:, 0], gate[:, 0], up[:, 0] = 1.0, 64.0, 1.0
    dh = torch.diag(torch.tensor(TOP))
    _, dgate, _ = pq.mx_gated_backward(dh.to(dev()), x.to(dev()), pq.mx_quantize(gate.to(dev())), pq.mx_quantize(up.to(dev())))
    want = torch.zeros((n, k))
    want[:, 0] = torch.tensor(TOP)
    assert torch.equal(dgate.cpu(), want)
