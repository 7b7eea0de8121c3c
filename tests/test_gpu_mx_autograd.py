"""The microscaled 4-bit operators inside torch.autograd.Function, as a training program uses them: a feed-forward
block whose gradients for x and for the weights it was quantized from come from the _backward functions."""
import pytest
import torch

import paper_2607_14618_amd as pq
from gpu_util import dev

pytestmark = pytest.mark.gpu


class Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        wq = pq.mx_quantize(w)
        ctx.save_for_backward(x)
        ctx.wq = wq
        return pq.mx_linear(x, wq)

    @staticmethod
    def backward(ctx, dy):
        return pq.mx_linear_backward(dy.contiguous(), ctx.saved_tensors[0], ctx.wq)


class Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, up):
        ctx.qs = pq.mx_quantize(gate), pq.mx_quantize(up)
        ctx.save_for_backward(x)
        return pq.mx_gated(x, *ctx.qs, act="gelu")

    @staticmethod
    def backward(ctx, dh):
        return pq.mx_gated_backward(dh.contiguous(), ctx.saved_tensors[0], *ctx.qs, act="gelu")


@pytest.mark.parametrize("t", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m", [1, 3, 50])
def test_feed_forward_block_under_autograd(m, t):
    k, n = 384, 300
    g = torch.Generator().manual_seed(m)
    x = torch.randn((m, k), generator=g).to(t).to(dev()).requires_grad_()
    gate, up, down = ((torch.randn(s, generator=g) * 0.05).to(t).to(dev()).requires_grad_() for s in ((n, k), (n, k), (k, n)))
    y = Linear.apply(Gated.apply(x, gate, up), down)
    dy = torch.randn((m, k), generator=g).to(t).to(dev())
    got = torch.autograd.grad(y, (x, gate, up, down), dy)
    with torch.no_grad():
        gq, uq, dq = (pq.mx_quantize(w) for w in (gate, up, down))
        h = pq.mx_gated(x, gq, uq, act="gelu")
        assert torch.equal(y, pq.mx_linear(h, dq))
        dh, ddown = pq.mx_linear_backward(dy, h, dq)
        want = (*pq.mx_gated_backward(dh, x, gq, uq, act="gelu"), ddown)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(ValueError, match="requires a gradient"):
        pq.mx_linear(x, gq)
