"""What the microscaled 4-bit entry points refuse, on the host: no device pointer is touched (the ones
passed are never dereferenced) and nothing is launched, so none of this needs a GPU."""
import ctypes

import pytest
import torch

import paper_2607_14618_amd as pq

P = ctypes.c_void_p(1 << 20)       # 256-byte aligned
ODD = ctypes.c_void_p((1 << 20) + 1)
NULL = None
ARG, SHAPE, CAPACITY = 1, 4, 5
BIG = 1 << 40


def call(name, *args):
    return getattr(pq.lib(), name)(*args)


def test_sizes():
    assert call("polyq_mx_bytes", 1, 1) == 256 + 1024
    assert call("polyq_mx_bytes", 16, 512) == 4352
    assert call("polyq_mx_bytes", 17, 513) == 2 * (4352 + 1280)
    assert call("polyq_mx_bytes", 5120, 13824) == 320 * (27 * 4352)
    for rows, k in ((0, 1), (1, 0), (-1, 5), (5, -1), ((1 << 24) + 1, 8), (1, (1 << 20) + 1)):
        assert call("polyq_mx_bytes", rows, k) == 0
    for op in ("linear", "gated"):
        assert call(f"polyq_mx_{op}_workspace_bytes", 17, 513, 2) == call("polyq_mx_bytes", 17, 513)
        assert call(f"polyq_mx_{op}_workspace_bytes", 17, 513, 3) == 0
        assert call(f"polyq_mx_{op}_workspace_bytes", 1, 513, 0) == 0
        assert call(f"polyq_mx_{op}_workspace_bytes", 0, 513, 0) == 0
    assert call("polyq_mx_linear_backward_workspace_bytes", 0, 1, 1, 0, 0, 1, 1) == 0
    assert call("polyq_mx_gated_backward_workspace_bytes", 1, 1, 1, 0, 7, 1, 1) == 0
    assert call("polyq_mx_bytes", 1 << 24, 1 << 20) > 1 << 43     # no overflow


@pytest.mark.parametrize("x,t,rows,k,packed,want", [
    (NULL, 0, 1, 32, P, ARG), (P, 0, 1, 32, NULL, ARG), (P, 3, 1, 32, P, ARG), (P, -1, 1, 32, P, ARG),
    (ODD, 1, 1, 32, P, ARG), (P, 0, 1, 32, ODD, ARG), (P, 0, 0, 32, P, SHAPE), (P, 0, 1, 0, P, SHAPE),
    (P, 0, 1, (1 << 20) + 1, P, SHAPE), (P, 0, (1 << 24) + 1, 32, P, SHAPE)])
def test_quantize_refusals(x, t, rows, k, packed, want):
    assert call("polyq_mx_quantize", x, t, rows, k, packed, None) == want
    assert call("polyq_mx_dequantize", packed, rows, k, x, t, None) == want


@pytest.mark.parametrize("codes,scales,rows,k,packed,want", [
    (NULL, P, 1, 32, P, ARG), (P, NULL, 1, 32, P, ARG), (P, P, 1, 32, NULL, ARG), (P, P, 1, 32, ODD, ARG),
    (P, P, 0, 32, P, SHAPE), (P, P, 1, -3, P, SHAPE)])
def test_pack_refusals(codes, scales, rows, k, packed, want):
    assert call("polyq_mx_pack", codes, scales, rows, k, packed, None) == want
    assert call("polyq_mx_unpack", packed, rows, k, codes, scales, None) == want


GOOD = dict(x=P, xt=2, m=20, w=P, n=16, k=64, y=P, yt=2, ws=P, wsb=BIG)
BAD = [(dict(x=NULL), ARG), (dict(w=NULL), ARG), (dict(y=NULL), ARG), (dict(xt=4), ARG), (dict(yt=3), ARG),
       (dict(m=0), ARG), (dict(m=-1), ARG), (dict(n=0), SHAPE), (dict(k=0), SHAPE), (dict(n=(1 << 24) + 1), SHAPE),
       (dict(k=(1 << 20) + 1), SHAPE), (dict(w=ODD), ARG), (dict(x=ODD), ARG), (dict(y=ODD), ARG),
       (dict(ws=NULL), CAPACITY), (dict(wsb=10), CAPACITY), (dict(ws=ODD), ARG), (dict(x=ODD, xt=3), ARG)]


@pytest.mark.parametrize("change,want", BAD)
def test_product_refusals(change, want):
    a = dict(GOOD, **change)
    assert call("polyq_mx_linear", a["x"], a["xt"], a["m"], a["w"], a["n"], a["k"], a["y"], a["yt"], a["ws"], a["wsb"],
                None) == want
    for gate, up in ((a["w"], P), (P, a["w"])):
        if "w" in change or gate is P:
            assert call("polyq_mx_gated", a["x"], a["xt"], a["m"], gate, up, a["n"], a["k"], 0, a["y"], a["yt"], a["ws"],
                        a["wsb"], None) == want


@pytest.mark.parametrize("act", [-1, 3])
def test_unknown_activations_are_refused(act):
    assert call("polyq_mx_gated", P, 2, 2, P, P, 16, 64, act, P, 2, P, BIG, None) == ARG
    assert call("polyq_mx_gated_backward", P, 2, P, 2, 2, P, P, 16, 64, act, P, P, P, 2, P, BIG, None) == ARG


BACK_GOOD = dict(d=P, dt=2, x=P, xt=2, m=2, w=P, n=16, k=64, dx=P, dw=P, gt=2, ws=P, wsb=BIG)
BACK_BAD = [(dict(d=NULL), ARG), (dict(x=NULL), ARG), (dict(w=NULL), ARG), (dict(dt=3), ARG), (dict(xt=5), ARG),
            (dict(gt=3), ARG), (dict(m=0), ARG), (dict(n=0), SHAPE), (dict(k=0), SHAPE), (dict(dx=NULL, dw=NULL), ARG),
            (dict(d=ODD), ARG), (dict(dx=ODD), ARG), (dict(dw=ODD), ARG), (dict(w=ODD), ARG), (dict(x=ODD), ARG),
            (dict(ws=NULL), CAPACITY), (dict(wsb=100), CAPACITY), (dict(ws=ODD), ARG),
            (dict(m=(1 << 21) + 1), CAPACITY), (dict(n=(1 << 21) + 1), CAPACITY)]


@pytest.mark.parametrize("change,want", BACK_BAD)
def test_backward_refusals(change, want):
    a = dict(BACK_GOOD, **change)
    assert call("polyq_mx_linear_backward", a["d"], a["dt"], a["x"], a["xt"], a["m"], a["w"], a["n"], a["k"], a["dx"],
                a["dw"], a["gt"], a["ws"], a["wsb"], None) == want
    assert call("polyq_mx_gated_backward", a["d"], a["dt"], a["x"], a["xt"], a["m"], a["w"], P, a["n"], a["k"], 0, a["dx"],
                a["dw"], a["dw"], a["gt"], a["ws"], a["wsb"], None) == want


def test_gated_backward_takes_both_weight_gradients_or_none():
    for dg, du in ((P, NULL), (NULL, P)):
        assert call("polyq_mx_gated_backward", P, 2, P, 2, 2, P, P, 16, 64, 0, P, dg, du, 2, P, BIG, None) == ARG


def test_binding_refusals():
    """What the binding refuses before the library is called: wrong types, shapes and places."""
    cpu = torch.zeros((4, 64))
    w = pq.MXMatrix(16, 64, torch.zeros(1280, dtype=torch.uint8))
    with pytest.raises(ValueError, match="GPU tensors"):
        pq.mx_quantize(cpu)
    with pytest.raises(ValueError, match="fp32, fp16 or bf16"):
        pq.mx_quantize(cpu.double())
    with pytest.raises(ValueError, match="rows"):
        pq.mx_quantize(torch.zeros((2, 3, 4)))
    with pytest.raises(ValueError, match="channels"):
        pq.mx_linear(torch.zeros((4, 63)), w)
    with pytest.raises(ValueError, match="packed"):
        pq.mx_linear(cpu, cpu)
    for bad in (None, cpu):
        with pytest.raises(ValueError, match="packed"):
            pq.mx_gated(cpu, w, bad)
        with pytest.raises(ValueError, match="packed"):
            pq.mx_gated_backward(torch.zeros((4, 16)), cpu, w, bad)
    with pytest.raises(ValueError, match="GPU tensors"):
        pq.mx_linear(cpu, w)
    with pytest.raises(ValueError, match="act must be"):
        pq.mx_gated(cpu, w, w, act="relu")
    with pytest.raises(ValueError, match="same shape"):
        pq.mx_gated(cpu, w, pq.MXMatrix(15, 64, w.packed))
    for rows, k, packed in ((17, 64, w.packed), (16, 129, w.packed), (16, 64, w.packed.int()), (16, 64, w.packed[:1279]),
                            (0, 64, w.packed), (16, 64, torch.zeros((2560,), dtype=torch.uint8)[::2])):
        with pytest.raises(ValueError, match="packed matrix"):
            pq.MXMatrix(rows, k, packed)
    with pytest.raises(ValueError, match=r"dh must be"):
        pq.mx_gated_backward(torch.zeros((4, 15)), cpu, w, w)
    with pytest.raises(ValueError, match="dw needs x"):
        pq.mx_linear_backward(torch.zeros((4, 16)), None, w)
    with pytest.raises(ValueError, match="neither"):
        pq.mx_linear_backward(torch.zeros((4, 16)), cpu, w, need_dx=False, need_dw=False)
    with pytest.raises(ValueError, match="neither"):
        pq.mx_gated_backward(torch.zeros((4, 16)), cpu, w, w, need_dx=False, need_dw=False)
    with pytest.raises(ValueError, match="GPU tensors"):
        pq.mx_pack(torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8), 64)
