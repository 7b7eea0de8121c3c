"""Microscaled 4-bit calls of more elements than one launch has work-items for (2^32), as much of the card's memory
as they need.  Skipped where that is not free."""
import pytest
import torch

import paper_2607_14618_amd as pq
from gpu_util import dev

pytestmark = [pytest.mark.gpu, pytest.mark.slow]


@pytest.fixture
def need():
    """need(gib): nothing of other tests in the way, or a skip; nothing is left behind."""
    def check(gib):
        torch.cuda.empty_cache()
        free = torch.cuda.mem_get_info()[0] >> 30
        if free < gib:
            pytest.skip(f"{free} GiB of {gib} are free")
    yield check
    torch.cuda.empty_cache()


def test_gradients_of_two_to_the_34_incoming_values(need):
    """dy [131072][131072] is 0 but for four rows: dx is 0 but for those, dW comes from those alone."""
    need(90)
    m = n = 131072
    k = 32
    g = torch.Generator(device=dev()).manual_seed(1)
    rows = torch.tensor([0, 65535, m - 2, m - 1], device=dev())
    dy = torch.zeros((m, n), dtype=torch.bfloat16, device=dev())
    dy[rows] = torch.randn((len(rows), n), generator=g, device=dev()).bfloat16()
    x = torch.randn((m, k), generator=g, device=dev()).bfloat16()
    wq = pq.mx_quantize(torch.randn((n, k), generator=g, device=dev()) * 0.05)
    dx, dw = pq.mx_linear_backward(dy, x, wq)
    d, wv, xv = dy[rows].double(), pq.mx_dequantize(wq).double(), pq.mx_dequantize(pq.mx_quantize(x)).double()[rows]
    # dy is exact in bf16: what rounds are the fp32 sums, at most 2^-23 of the magnitudes' sum for each 16 of a reduction,
    # and the result, 2^-8 of it
    for got, want, mag, length in ((dx[rows], d @ wv, d.abs() @ wv.abs(), n), (dw, d.T @ xv, d.abs().T @ xv.abs(), m)):
        tol = 2.0 ** -23 * (length // 16 + 8) * mag
        assert bool(((got.double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all())
    dx[rows] = 0
    assert not bool(dx.any())


def test_pack_and_unpack_more_blocks_than_work_items(need):
    """2^32 blocks and some: the first, middle and last rows are where they belong, and come back."""
    need(170)
    rows, k = 131072 + 16, 1 << 20
    g = torch.Generator(device=dev()).manual_seed(2)
    codes = torch.zeros((rows, k // 2), dtype=torch.uint8, device=dev())
    scales = torch.full((rows, k // 32), 127, dtype=torch.uint8, device=dev())
    tiles = [0, 4001, rows // 16 - 2, rows // 16 - 1]
    some = {t: (torch.randint(0, 256, (16, k // 2), generator=g, device=dev(), dtype=torch.uint8),
                torch.randint(0, 255, (16, k // 32), generator=g, device=dev(), dtype=torch.uint8)) for t in tiles}
    for t, (c, s) in some.items():
        codes[16 * t:16 * t + 16], scales[16 * t:16 * t + 16] = c, s
    w = pq.mx_pack(codes, scales, k)
    size = w.packed.numel() // (rows // 16)
    none = pq.mx_pack(torch.zeros((16, k // 2), dtype=torch.uint8, device=dev()),
                      torch.full((16, k // 32), 127, dtype=torch.uint8, device=dev()), k).packed[:size]
    for t, (c, s) in some.items():
        assert torch.equal(w.packed[t * size:(t + 1) * size], pq.mx_pack(c, s, k).packed[:size]), t
    for t in (1, 4000, 4096, rows // 16 - 3):
        assert torch.equal(w.packed[t * size:(t + 1) * size], none), t
    del codes, scales
    codes, scales = pq.mx_unpack(w)
    for t, (c, s) in some.items():
        assert torch.equal(codes[16 * t:16 * t + 16], c) and torch.equal(scales[16 * t:16 * t + 16], s)
        codes[16 * t:16 * t + 16], scales[16 * t:16 * t + 16] = 0, 127
    for at in range(0, rows, 4096):
        assert not bool(codes[at:at + 4096].any()) and bool((scales[at:at + 4096] == 127).all())
