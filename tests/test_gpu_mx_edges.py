"""Values at the ends of their range through the microscaled 4-bit operators: infinities and NaN in every path, scale
bytes at both ends, gradients next to the largest fp32 value.  Every entry that has to be infinite or NaN is, and no
other.  Tolerances as derived at the head of test_gpu_mx.py."""
import numpy as np
import pytest
import torch

import paper_2607_14618_amd as pq
from gpu_util import dev
from test_gpu_mx import F, GRID, HALF, TERM, act64, activations, out_tol, quantized, sum_tol, weights

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
# tokens, channels: quantized inside the product's launch, a packed x of few tokens, K split over waves, the tiled kernel
PLACES = [(1, 40, 700), (2, 40, 700), (4, 40, 700), (16, 40, 700), (40, 40, 700), (700, 901, 1100), (2000, 641, 1101)]


def nans(t):
    return torch.isnan(t.detach().cpu())


def rows_cols(shape, rows, cols):
    want = torch.zeros(shape, dtype=torch.bool)
    want[list(rows), :] = True
    want[:, list(cols)] = True
    return want


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("m,n,k", PLACES)
def test_products_carry_nan_and_only_there(m, n, k, packed):
    x, gate, up = activations(m, k, "bf16", 5), weights(n, k, 6), weights(n, k, 7)
    last = m - 1
    x[last, k - 1] = NAN if n % 2 else INF
    gate[7, 10], up[31, 300] = INF, NAN
    gq, uq = pq.mx_quantize(gate.to(dev())), pq.mx_quantize(up.to(dev()))
    xd = pq.mx_quantize(x.to(dev())) if packed else x.to(dev())
    assert torch.equal(nans(pq.mx_linear(xd, gq)), rows_cols((m, n), [last], [7]))
    for act in ("silu", "gelu", "gelu_tanh"):
        h = pq.mx_gated(xd, gq, uq, act=act)
        assert torch.equal(nans(h), rows_cols((m, n), [last], [7, 31])), act
        assert not bool(torch.isinf(h).any())


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("t", list(F))
@pytest.mark.parametrize("m,n,k", [(1, 40, 700), (40, 100, 1100), (2000, 641, 1101), (2200, 640, 4352)])
def test_linear_backward_carries_nan_and_infinities_and_only_there(m, n, k, t, packed):
    x, w = activations(m, k, t, 5), weights(n, k, 6)
    dy = torch.randn((m, n), generator=torch.Generator().manual_seed(9)).to(F[t])
    last = m - 1
    x[last, 40], w[7, 69] = NAN, INF             # blocks 32 .. 63 of x's last row, 64 .. 95 of w's row 7
    wq = pq.mx_quantize(w.to(dev()))
    xd = pq.mx_quantize(x.to(dev())) if packed else x.to(dev())
    dx, dw = pq.mx_linear_backward(dy.to(dev()), xd, wq)
    assert torch.equal(nans(dx), rows_cols((m, k), [], range(64, 96)))
    assert torch.equal(nans(dw), rows_cols((n, k), [], range(32, 64)))
    assert not bool(torch.isinf(dx).any()) and not bool(torch.isinf(dw).any())
    dy[last, 3], dy[0, 11] = INF, NAN
    dx, dw = pq.mx_linear_backward(dy.to(dev()), xd, wq)
    xv, wv = pq.mx_dequantize(pq.mx_quantize(x.to(dev()))).cpu().double(), pq.mx_dequantize(wq).cpu().double()
    # an infinity times a weight of 0 is NaN and else an infinity of the product's sign
    want = rows_cols((m, k), [0], range(64, 96))
    want[last] |= (wv[3] == 0) | torch.isnan(wv[3])
    assert torch.equal(nans(dx), want)
    if m > 1:
        inf = dx[last].cpu().double()
        assert torch.equal(inf[~want[last]], (INF * wv[3])[~want[last]])
    want = rows_cols((n, k), [11], range(32, 64))
    want[3] |= (xv[last] == 0) | torch.isnan(xv[last])
    assert torch.equal(nans(dw), want)
    inf = dw[3].cpu().double()
    assert torch.equal(inf[~want[3]], (INF * xv[last])[~want[3]])


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("t", list(F))
@pytest.mark.parametrize("m,n,k", [(1, 40, 700), (40, 100, 1100), (300, 2050, 384), (2000, 641, 1101), (2200, 640, 4352)])
def test_gated_backward_carries_nan_and_only_there(m, n, k, t, packed):
    g = torch.Generator().manual_seed(9)
    d = torch.randn((m, n), generator=g).to(F[t])
    d = torch.where(d == 0, torch.ones_like(d), d)

    def masks(put):
        """What of dx, dgate, dup is NaN with one place of x, gate, up or dh spoiled."""
        v = {"x": activations(m, k, t, 5), "gate": weights(n, k, 6), "up": weights(n, k, 7), "d": d.clone()}
        which, row, col, value = put
        v[which][row, col] = value
        x = pq.mx_quantize(v["x"].to(dev())) if packed else v["x"].to(dev())
        out = pq.mx_gated_backward(v["d"].to(dev()), x, pq.mx_quantize(v["gate"].to(dev())), pq.mx_quantize(v["up"].to(dev())))
        assert not any(bool(torch.isinf(o).any()) for o in out)
        return [nans(o) for o in out]

    last, everywhere = m - 1, range(k)
    # x's last row: g and u of that token, and so all of the weights' gradients
    for got, want in zip(masks(("x", last, k - 1, NAN)), (rows_cols((m, k), [last], []), *[rows_cols((n, k), [], everywhere)] * 2)):
        assert torch.equal(got, want)
    # a row of gate: g of that row for every token, and so all of dx
    for got, want in zip(masks(("gate", n - 1, 3, INF)), (rows_cols((m, k), [], everywhere), *[rows_cols((n, k), [n - 1], [])] * 2)):
        assert torch.equal(got, want)
    # a row of up: its u, which du does not hold
    for got, want in zip(masks(("up", 5, k - 1, NAN)), (rows_cols((m, k), [], everywhere), rows_cols((n, k), [5], []), rows_cols((n, k), [], []))):
        assert torch.equal(got, want)
    # one value of dh
    for got, want in zip(masks(("d", last, 7, NAN)), (rows_cols((m, k), [last], []), *[rows_cols((n, k), [7], [])] * 2)):
        assert torch.equal(got, want)


def coded(rows, k, low, high, codes, seed):
    """A packed matrix with scale bytes low .. high and magnitudes of the given codes, and its values in 64 bits."""
    g = np.random.default_rng(seed)
    c = g.choice(codes, (rows, k)).astype(np.uint8)
    sign = g.integers(0, 2, (rows, k)).astype(np.uint8)
    scale = g.integers(low, high + 1, (rows, k // 32)).astype(np.uint8)
    full = c + 8 * sign
    packed = pq.mx_pack(torch.from_numpy(full[:, 0::2] + 16 * full[:, 1::2]).to(dev()), torch.from_numpy(scale).to(dev()), k)
    val = GRID[c] * np.where(sign == 1, -1.0, 1.0) * np.exp2(np.repeat(scale.astype(np.float64), 32, 1) - 127)
    return packed, torch.from_numpy(val)


# Scale bytes, the codes whose values a float holds there, and the power of two of the other factor.
ENDS = [(0, 0, range(8), 100), (0, 1, range(8), 100), (1, 3, range(8), 100), (252, 252, range(8), -100),
        (253, 253, range(6), -100), (254, 254, range(4), -100)]


@pytest.mark.parametrize("t", ["fp32", "bf16"])
@pytest.mark.parametrize("low,high,codes,power", ENDS)
def test_scales_at_both_ends(low, high, codes, power, t):
    """Values down to 2^-128 (subnormal in bf16 and fp32) and up to the largest, times something that brings the result
    to an ordinary size: exact factors, so the usual bounds hold."""
    m, n, k = 40, 70, 256
    w, wv = coded(n, k, low, high, list(codes), 1)
    assert torch.equal(pq.mx_dequantize(w).cpu().double(), wv)
    x = (activations(m, k, "fp32", 2).double() * 2.0 ** power).float().to(F[t])
    xv = quantized(x)[0]
    want, mag = xv @ wv.T, xv.abs() @ wv.abs().T
    for tokens in (1, 4, m):   # every kernel of few tokens
        y = pq.mx_linear(x[:tokens].to(dev()), w, dtype=torch.float32).cpu().double()
        assert bool(((y - want[:tokens]).abs() <= sum_tol(mag[:tokens], k) + out_tol(want[:tokens], torch.float32)).all())
    dy = (torch.randn((m, n), generator=torch.Generator().manual_seed(3)).double() * 2.0 ** power).float().to(F[t])
    xq, xqv = coded(m, k, low, high, list(codes), 4)
    dx, dw = pq.mx_linear_backward(dy.to(dev()), xq, w)
    d = dy.double()
    terms = {"fp32": 3, "bf16": 1}[t]
    for got, want, mag, length in ((dx, d @ wv, d.abs() @ wv.abs(), n), (dw, d.T @ xqv, d.abs().T @ xqv.abs(), m)):
        tol = 2.0 ** -23 * (terms * (length // 32 + 2) + 40) * mag + out_tol(want, F[t])
        got = got.cpu().double()
        assert bool(torch.isfinite(got).all())
        assert bool(((got - want).abs() <= tol).all()), (low, high, t, float(((got - want).abs() - tol).max()))


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


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gated_gradients_are_finite_where_dh_u_alone_is_not(act):
    """dh u = 2^140 lies past the largest float, dh u act'(-64) does not (gelu: 0).  Every sum has two products at most;
    act and its slope are within 2^-24 (16 + 4 x 120) of themselves (act_tol of test_gpu_mx.py at its largest)."""
    m, n, k = 4, 4, 32
    x, gate, up = torch.zeros((m, k)), torch.zeros((n, k)), torch.zeros((n, k))
    x[:, 0], gate[:, 0], up[:, 0] = 1.0, -64.0, 2.0 ** 40
    dh = torch.eye(m) * 2.0 ** 100
    got = pq.mx_gated_backward(dh.to(dev()), x.to(dev()), pq.mx_quantize(gate.to(dev())), pq.mx_quantize(up.to(dev())), act=act)
    a, da = act64(act, torch.full((m, n), -64.0, dtype=torch.float64))
    dg, du = dh.double() * 2.0 ** 40 * da, dh.double() * a
    for out, parts in ((got[0], (dg @ gate.double(), du @ up.double())), (got[1], (dg.T @ x.double(),)), (got[2], (du.T @ x.double(),))):
        want, mag = sum(parts), sum(p.abs() for p in parts)
        off = (out.cpu().double() - want).abs()
        assert bool(torch.isfinite(out).all())
        assert bool((off <= (2.0 ** -24 * (16 + 4 * 120) + 2.0 ** -20) * mag + 1e-30).all()), (act, float(off.max()), float(mag.max()))
