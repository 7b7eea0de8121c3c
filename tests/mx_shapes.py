"""Shapes of the microscaled 4-bit operators' tests, by the kernels that they reach (tests/test_mx_plan.py holds them
to it on the host)."""

# (m, n, k) of the gated block and of its backward pass: the kernel of g and u; for one, two and three bf16 terms (bf16,
# fp16, fp32 gradients) the tile of dx and its splits, and the tile of the weights' gradients and its splits.
GATED = {
    (2048, 2048, 4096): ("gemm 4", [("256x256", 2)] * 3, [("256x256", 1)] * 3),   # whole tiles
    (2300, 2500, 4099): ("gemm 3", [("256x256", 3), ("256x256", 5), ("256x256", 5)],
                         [("256x256", 1), ("256x256", 3), ("256x256", 3)]),       # ragged, splits inside a matrix
    (2048, 3000, 4200): ("gemm 2", [("256x256", 3), ("256x256", 5), ("256x256", 5)], [("256x256", 1)] * 3),
    (2200, 640, 4352): ("gemm 2", [("256x256", 1), ("256x256", 1), ("256x256", 3)], [("256x64", 1)] * 3),
    (700, 901, 6001): ("gemm 1", [("256x64", 1)] * 3, [("256x256", 1)] * 3),       # ragged
    (1000, 1024, 1536): ("gemm 1", [("256x64", 4)] * 3, [("256x64", 1), ("256x64", 2), ("256x64", 2)]),
    (2000, 641, 1101): ("gemm 2", [("256x64", 2)] * 3, [("256x64", 4)] * 3),       # ragged
    (2000, 5001, 1201): ("gemm 4", [("256x64", 3)] * 3, [("256x256", 1)] * 3),     # ragged
    (2048, 320, 8192): ("gemm 1", [("256x256", 1)] * 3, [("256x256", 2)] * 3),
    (40, 100, 1100): ("split 1", [("128x64", 1)] * 3, [("256x64", 1)] * 3),
    (60, 1000, 1100): ("split 1", [("128x64", 4)] * 3, [("256x64", 1)] * 3),
    (300, 2050, 384): ("split 2", [("128x64", 8)] * 3, [("256x64", 1)] * 3),
}
# The same of the linear layer's backward pass, without g and u.
LINEAR = {
    (2300, 2500, 4099): ([("256x256", 1), ("256x256", 3), ("256x256", 3)], [("256x256", 1), ("256x256", 3), ("256x256", 3)]),
    (2048, 4096, 4096): ([("256x256", 2)] * 3, [("256x256", 1)] * 3),
}
