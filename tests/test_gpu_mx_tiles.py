"""The microscaled 4-bit gated block and the gradients on every tile that a training batch takes, against a plain
implementation in 64 bits.  mx_shapes.py says which kernels a shape reaches, tests/test_mx_plan.py that it does.
Tolerances as derived at the head of test_gpu_mx.py."""
import pytest
import torch

import paper_2607_14618_amd as pq
from gpu_util import dev
from mx_shapes import GATED, LINEAR
from test_gpu_mx import F, HALF, TERM, act64, act_tol, device_linear, out_tol, sum_tol

pytestmark = pytest.mark.gpu

ACTS = ("silu", "gelu", "gelu_tanh")
TERMS = {"bf16": 1, "fp16": 2, "fp32": 3}


def inputs(m, n, k, mats, t):
    g = torch.Generator(device=dev()).manual_seed(m + n)
    x = torch.randn((m, k), generator=g, device=dev()).to(F[t])
    ws = [torch.randn((n, k), generator=g, device=dev()) * 0.05 for _ in range(mats)]
    return x, ws, torch.randn((m, n), generator=g, device=dev()).to(F[t])


def product_tol(mag, err, terms, length):
    """err: what the incoming factor is off by, in the product; the fp32 sums of `terms` products over `length`."""
    return err + 2.0 ** -23 * (terms * (length // 32 + 2) + 40) * (mag + err)


def inside(got, want, tol, typ, what):
    off = (got.double() - want).abs() - (tol * (1 + HALF[typ]) + out_tol(want, typ))
    assert bool(torch.isfinite(got).all()), what
    assert bool((off <= 0).all()), (what, float(off.max()))


@pytest.mark.parametrize("t", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", list(GATED))
def test_gated(shape, t):
    m, n, k = shape
    act = ACTS[(m + k) % 3]
    x, (gate, up), _ = inputs(m, n, k, 2, t)
    _, _, g, gm = device_linear(x, gate)
    _, _, u, um = device_linear(x, up)
    a = act64(act, g)[0]
    ea, eu, want = 1.2 * sum_tol(gm, k) + act_tol(g, a), sum_tol(um, k), a * u
    tol = ea * u.abs() + (a.abs() + ea) * eu + 2.0 ** -23 * want.abs()
    inside(pq.mx_gated(x, pq.mx_quantize(gate), pq.mx_quantize(up), act=act), want, tol, F[t], (shape, t, act))


@pytest.mark.parametrize("t", list(TERMS))
@pytest.mark.parametrize("shape", list(GATED))
def test_gated_backward(shape, t):
    m, n, k = shape
    typ, act = F[t], ACTS[(m + n + k) % 3]
    x, (gate, up), d = inputs(m, n, k, 2, t)
    got = pq.mx_gated_backward(d, x, pq.mx_quantize(gate), pq.mx_quantize(up), act=act)
    xv, gv, g, gm = device_linear(x, gate)
    _, uv, u, um = device_linear(x, up)
    (a, da), eg, eu, d = act64(act, g), sum_tol(gm, k), sum_tol(um, k), d.double()
    dg, du = d * u * da, d * a
    curve = 1.2 * eg + act_tol(g, da) + act_tol(g, a)
    e_dg = d.abs() * (curve * (u.abs() + eu) + eu * da.abs()) + (TERM[typ] + 2.0 ** -22) * dg.abs()
    e_du = d.abs() * (1.2 * eg + act_tol(g, a)) + (TERM[typ] + 2.0 ** -22) * du.abs()
    del gm, um, curve
    for what, out, want, mag, err, length in (
            ("dx", got[0], dg @ gv + du @ uv, dg.abs() @ gv.abs() + du.abs() @ uv.abs(), e_dg @ gv.abs() + e_du @ uv.abs(), 2 * n),
            ("dgate", got[1], dg.T @ xv, dg.abs().T @ xv.abs(), e_dg.T @ xv.abs(), m),
            ("dup", got[2], du.T @ xv, du.abs().T @ xv.abs(), e_du.T @ xv.abs(), m)):
        inside(out, want, product_tol(mag, err, TERMS[t], length), typ, (what, shape, t, act))


@pytest.mark.parametrize("t", list(TERMS))
@pytest.mark.parametrize("shape", list(LINEAR))
def test_linear_backward(shape, t):
    m, n, k = shape
    x, (w,), dy = inputs(m, n, k, 1, t)
    got = pq.mx_linear_backward(dy, x, pq.mx_quantize(w))
    xv, wv, _, _ = device_linear(x, w)
    d = dy.double()
    for what, out, want, mag, length in (("dx", got[0], d @ wv, d.abs() @ wv.abs(), n),
                                         ("dw", got[1], d.T @ xv, d.abs().T @ xv.abs(), m)):
        inside(out, want, product_tol(mag, 0 * mag, TERMS[t], length), F[t], (what, shape, t))
