"""Microscaled 4-bit floating point (MXFP4) on one GPU: quantization, the linear layer,
the gated feed-forward block and their gradients (marshalling around the C ABI).
Gradients are computed by the ``_backward`` functions; nothing is recorded for autograd, and a
product of an x that asks for it is refused."""
from __future__ import annotations

from typing import Optional, Tuple, Union

import torch

from . import _lib
from ._lib import _aligned_empty, _check, _need_cuda, _ptr, lib

BLOCK = 32
TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
PACKED = 3
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2}
MAX_ROWS, MAX_K = 1 << 24, 1 << 20  # POLYQ_MAX_N, POLYQ_MAX_K; a larger size could not even be handed over (32 bits)


# torch's own lookups of the current stream and device build objects around them (2 us of a call's 7).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(dev: torch.device) -> int:
    return _lib._stream(dev) if _raw_stream is None else _raw_stream(dev.index)


def _launch(name: str, dev: torch.device, *args) -> None:
    """Calls the library on the tensors' device, whatever the current one is, and its current stream."""
    fn = getattr(lib(), name)
    if dev.index == _current():
        status = fn(*args, _stream(dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _stream(dev))
    if status != 0:
        _check(status, name)


def _packed_bytes(rows: int, k: int) -> int:
    """Bytes of a packed matrix; 0 if it cannot be packed."""
    return int(lib().polyq_mx_bytes(rows, k)) if 0 < rows <= MAX_ROWS and 0 < k <= MAX_K else 0


class MXMatrix:
    """A packed matrix [rows][k] in microscaled 4-bit floating point (polyq.h), as
    ``mx_quantize`` and ``mx_pack`` make it."""

    __slots__ = ("rows", "k", "packed")

    def __init__(self, rows: int, k: int, packed: torch.Tensor):
        nbytes = _packed_bytes(rows, k)
        if nbytes == 0 or packed.dtype != torch.uint8 or not packed.is_contiguous() or packed.numel() < nbytes:
            raise ValueError(f"a packed matrix of {rows} rows x {k} channels is {nbytes} contiguous bytes (uint8)")
        self.rows, self.k, self.packed = rows, k, packed

    @property
    def shape(self) -> Tuple[int, int]:
        return self.rows, self.k

    @property
    def device(self) -> torch.device:
        return self.packed.device

    def __repr__(self):
        return f"MXMatrix(rows={self.rows}, k={self.k}, device={self.device})"


def _bytes(nbytes: int, dev: torch.device) -> torch.Tensor:
    """Device memory on 256 bytes, as torch's allocator hands it out."""
    t = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    return t if t.data_ptr() % 256 == 0 else _aligned_empty(nbytes, dev)


def _type(t: torch.dtype, what: str) -> int:
    if t not in TYPES:
        raise ValueError(f"{what} must be fp32, fp16 or bf16, got {t}")
    return TYPES[t]


def _two(x: torch.Tensor, what: str) -> torch.Tensor:
    if x.dim() not in (1, 2):
        raise ValueError(f"{what} must be [rows][columns] or one row")
    if x.dim() == 1:
        return x.reshape(1, -1)
    if x.shape[0] > MAX_ROWS:
        raise ValueError(f"{what} has {x.shape[0]} rows, at most {MAX_ROWS} are taken")
    return x


def _empty_matrix(rows: int, k: int, dev: torch.device) -> MXMatrix:
    nbytes = _packed_bytes(rows, k)
    if nbytes == 0:
        raise ValueError(f"a matrix of {rows} rows x {k} channels cannot be packed")
    q = MXMatrix.__new__(MXMatrix)
    q.rows, q.k, q.packed = rows, k, _bytes(nbytes, dev)
    return q


def mx_quantize(x: torch.Tensor) -> MXMatrix:
    """x [rows][k] (fp32, fp16 or bf16; one row as [k]) in microscaled 4 bits."""
    t = _type(x.dtype, "x")
    x2 = _two(x, "x")
    dev = _need_cuda(x2)
    out = _empty_matrix(*x2.shape, dev)
    _launch("polyq_mx_quantize", dev, x2.data_ptr(), t, out.rows, out.k, out.packed.data_ptr())
    return out


def mx_dequantize(q: MXMatrix, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """The values of a packed matrix, [rows][k]."""
    t = _type(dtype, "dtype")
    dev = _need_cuda(q.packed)
    out = torch.empty((q.rows, q.k), dtype=dtype, device=dev)
    _launch("polyq_mx_dequantize", dev, q.packed.data_ptr(), q.rows, q.k, out.data_ptr(), t)
    return out


def mx_pack(codes: torch.Tensor, scales: torch.Tensor, k: int) -> MXMatrix:
    """A checkpoint's codes uint8 [rows][ceil(k / 2)] (even channels in the low halves) and
    scale bytes uint8 [rows][ceil(k / 32)] as a packed matrix."""
    dev = _need_cuda(codes, scales)
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.dim() != 2:
        raise ValueError("codes and scales must be uint8 [rows][..]")
    if tuple(codes.shape) != (codes.shape[0], (k + 1) // 2):
        raise ValueError(f"codes shape {tuple(codes.shape)} is not [rows][{(k + 1) // 2}]")
    if tuple(scales.shape) != (codes.shape[0], -(-k // BLOCK)):
        raise ValueError(f"scales shape {tuple(scales.shape)} is not [{codes.shape[0]}][{-(-k // BLOCK)}]")
    out = _empty_matrix(codes.shape[0], int(k), dev)
    _launch("polyq_mx_pack", dev, _ptr(codes), _ptr(scales), out.rows, out.k, _ptr(out.packed))
    return out


def mx_unpack(q: MXMatrix) -> Tuple[torch.Tensor, torch.Tensor]:
    """(codes, scales) of a packed matrix, as ``mx_pack`` takes them."""
    dev = _need_cuda(q.packed)
    codes = torch.empty((q.rows, (q.k + 1) // 2), dtype=torch.uint8, device=dev)
    scales = torch.empty((q.rows, -(-q.k // BLOCK)), dtype=torch.uint8, device=dev)
    _launch("polyq_mx_unpack", dev, _ptr(q.packed), q.rows, q.k, _ptr(codes), _ptr(scales))
    return codes, scales


Activations = Union[torch.Tensor, MXMatrix]


def _input(x: Activations, w: MXMatrix, up: Optional[MXMatrix] = None):
    """(x's tensor, its type, tokens, the default output type) with the weights' shapes checked."""
    if not isinstance(w, MXMatrix) or not (up is None or isinstance(up, MXMatrix)):
        raise ValueError("weights must be packed (mx_quantize or mx_pack)")
    if up is not None and (up.rows != w.rows or up.k != w.k):
        raise ValueError(f"gate {w.shape} and up {up.shape} must have the same shape")
    if isinstance(x, MXMatrix):
        t, m, k, out, held = PACKED, x.rows, x.k, torch.bfloat16, x.packed
    else:
        t, held, out = _type(x.dtype, "x"), _two(x, "x"), x.dtype
        m, k = held.shape
    if k != w.k:
        raise ValueError(f"x has {k} channels, the weights have {w.k}")
    return held, t, m, out


def _output(y: Optional[torch.Tensor], shape, dtype: torch.dtype, dev: torch.device, what: str) -> torch.Tensor:
    if y is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    if tuple(y.shape) != tuple(shape) or y.dtype != dtype:
        raise ValueError(f"{what} must be {dtype} {tuple(shape)}, got {y.dtype} {tuple(y.shape)}")
    return y


def _scratch(workspace: Optional[torch.Tensor], nbytes: int, dev: torch.device):
    """(pointer, bytes, tensor): the caller's, or memory of this call alone (torch hands it out in the
    stream's order, so that neither two streams nor two captured graphs share it)."""
    if workspace is None and nbytes:
        workspace = _bytes(nbytes, dev)
    if workspace is None:
        return None, 0, None
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def _product(x: Activations, w: MXMatrix, up: Optional[MXMatrix], act: int, dtype, y, workspace):
    held, t, m, out = _input(x, w, up)
    if held.requires_grad and torch.is_grad_enabled():
        raise ValueError("x requires a gradient, which is not recorded here: call this in the forward of a "
                         "torch.autograd.Function (or without gradients) and the _backward function in its backward")
    dev = _need_cuda(held, w.packed, None if up is None else up.packed, y, workspace)
    dtype = y.dtype if dtype is None and y is not None else out if dtype is None else dtype
    ot = _type(dtype, "the output")
    y = _output(y, (m, w.rows), dtype, dev, "the output")
    if t == PACKED:
        need = 0
    elif up is None:
        need = lib().polyq_mx_linear_workspace_bytes(m, w.k, t)
    else:
        need = lib().polyq_mx_gated_workspace_bytes(m, w.k, t)
    ptr, nbytes, _keep = _scratch(workspace, need, dev)
    if up is None:
        _launch("polyq_mx_linear", dev, held.data_ptr(), t, m, w.packed.data_ptr(), w.rows, w.k, y.data_ptr(), ot, ptr,
                nbytes)
    else:
        _launch("polyq_mx_gated", dev, held.data_ptr(), t, m, w.packed.data_ptr(), up.packed.data_ptr(), w.rows, w.k,
                act, y.data_ptr(), ot, ptr, nbytes)
    return y


def mx_linear(x: Activations, w: MXMatrix, dtype: Optional[torch.dtype] = None, y: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [m][n] = q(x) W^T, q(x) the microscaled 4-bit form of x.  x is [m][k] (fp32,
    fp16 or bf16; one row as [k]) or a packed matrix, which several products can share;
    y has x's type (bf16 for a packed x) unless ``dtype`` or ``y`` says otherwise.  An x that
    requires a gradient is taken where none is recorded (torch.no_grad, the forward of an
    autograd.Function) and refused elsewhere."""
    return _product(x, w, None, 0, dtype, y, workspace)


def mx_gated(x: Activations, gate: MXMatrix, up: MXMatrix, act: str = "silu", dtype: Optional[torch.dtype] = None,
             y: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """h [m][n] = act(q(x) gate^T) * (q(x) up^T); act: "silu", "gelu" or "gelu_tanh".  One
    launch, and one before it that quantizes more than two tokens of an x that is not packed.
    x, dtype and y as for ``mx_linear``."""
    a = _act(act)
    if up is None:
        raise ValueError("weights must be packed (mx_quantize or mx_pack)")
    return _product(x, gate, up, a, dtype, y, workspace)


def _act(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {tuple(ACTIVATIONS)}, got {act!r}")
    return ACTIVATIONS[act]


def _incoming(d: torch.Tensor, m: int, n: int, what: str):
    d2 = _two(d, what)
    if tuple(d2.shape) != (m, n):
        raise ValueError(f"{what} must be [{m}][{n}], got {tuple(d2.shape)}")
    return d2, _type(d.dtype, what)


def mx_linear_backward(dy: torch.Tensor, x: Optional[Activations], w: MXMatrix, dtype: Optional[torch.dtype] = None,
                       need_dx: bool = True, need_dw: bool = True, workspace: Optional[torch.Tensor] = None
                       ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx [m][k], dw [n][k]) of ``mx_linear``, None for one that is not asked for: dx = dy W,
    dw = dy^T q(x), the rounding to 4 bits passed by as the identity.  The gradients
    have ``dtype`` (dy's type by default), and that says how dy enters the products: as one
    bf16 value (2^-8) for bf16, to 2^-17 for fp16, exactly for fp32.  x may be None where dw
    is not asked for."""
    if not isinstance(w, MXMatrix):
        raise ValueError("weights must be packed (mx_quantize or mx_pack)")
    if not (need_dx or need_dw):
        raise ValueError("neither dx nor dw is asked for")
    if need_dw:
        if x is None:
            raise ValueError("dw needs x")
        held, t, m, _ = _input(x, w)
    else:
        held, t, m = None, PACKED, _two(dy, "dy").shape[0]
    d, dt = _incoming(dy, m, w.rows, "dy")
    dev = _need_cuda(d, held, w.packed, workspace)
    dtype = dy.dtype if dtype is None else dtype
    gt = _type(dtype, "dtype")
    dx = torch.empty((m, w.k), dtype=dtype, device=dev) if need_dx else None
    dw = torch.empty((w.rows, w.k), dtype=dtype, device=dev) if need_dw else None
    need = int(lib().polyq_mx_linear_backward_workspace_bytes(m, w.rows, w.k, t, gt, need_dx, need_dw))
    ptr, nbytes, _keep = _scratch(workspace, need, dev)
    _launch("polyq_mx_linear_backward", dev, _ptr(d), dt, _ptr(held), t, m, _ptr(w.packed), w.rows, w.k, _ptr(dx), _ptr(dw),
            gt, ptr, nbytes)
    return dx, dw


def mx_gated_backward(dh: torch.Tensor, x: Activations, gate: MXMatrix, up: MXMatrix, act: str = "silu",
                      dtype: Optional[torch.dtype] = None, need_dx: bool = True, need_dw: bool = True,
                      workspace: Optional[torch.Tensor] = None):
    """(dx [m][k], dgate [n][k], dup [n][k]) of ``mx_gated``, None for those not asked for;
    g and u are computed again, so that the forward pass keeps nothing but x.  The
    gradients have ``dtype`` (dh's type by default), and that says how the gradients of g and u
    enter the products, as dy in ``mx_linear_backward``: for bf16 each is rounded to one bf16
    value, which makes the result's error 1.4 times that of its own rounding; fp32 keeps them
    whole, at 2.6 times the time."""
    a = _act(act)
    if not (need_dx or need_dw):
        raise ValueError("neither dx nor the weights' gradients are asked for")
    if up is None:
        raise ValueError("weights must be packed (mx_quantize or mx_pack)")
    held, t, m, _ = _input(x, gate, up)
    n, k = gate.shape
    d, dt = _incoming(dh, m, n, "dh")
    dev = _need_cuda(d, held, gate.packed, up.packed, workspace)
    dtype = dh.dtype if dtype is None else dtype
    gt = _type(dtype, "dtype")
    dx = torch.empty((m, k), dtype=dtype, device=dev) if need_dx else None
    dg, du = (torch.empty((n, k), dtype=dtype, device=dev) if need_dw else None for _ in range(2))
    need = int(lib().polyq_mx_gated_backward_workspace_bytes(m, n, k, t, gt, need_dx, need_dw))
    ptr, nbytes, _keep = _scratch(workspace, need, dev)
    _launch("polyq_mx_gated_backward", dev, _ptr(d), dt, _ptr(held), t, m, _ptr(gate.packed), _ptr(up.packed), n, k, a,
            _ptr(dx), _ptr(dg), _ptr(du), gt, ptr, nbytes)
    return dx, dg, du
