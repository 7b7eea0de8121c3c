"""MI355X (gfx950) mixed-bit linear layer: PolyQ's decode GEMV and prefill GEMM; and linear layers, the gated
block and their gradients in microscaled 4-bit floating point (mx_*).

Python binding of libpolyq.so (include/polyq.h).  The functions take torch
tensors for device memory and run on torch's current HIP stream.
"""
from ._lib import (Block, Layout, PolyQError, EXPORTS, LIB_PATH, lib, plan, pack, pack_rows, unpack,  # noqa
                   permute, gemv, gemv_batch, gemm, gemm_batch, gemv_workspace_bytes, gemm_workspace_bytes,
                   PreparedBatch, read_probe, channel_error, waterfill, quanta_match, cluster, allocate, bit_scaling,
                   SCALE_GRID)
from .mx import (MXMatrix, mx_quantize, mx_dequantize, mx_pack, mx_unpack, mx_linear, mx_linear_backward,  # noqa: F401
                 mx_gated, mx_gated_backward)
from .layer import PackedLinear, decode_batch, prefill_batch, group_index, device_perm  # noqa: F401
