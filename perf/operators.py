"""The microscaled 4-bit operators and the workloads they are timed on.

A matrix in microscaled 4-bit floating point (MXFP4) holds every 32 consecutive
values of a row as sign, two exponent bits and one mantissa bit each (0, 0.5, 1,
1.5, 2, 3, 4, 6 and their negatives) with one power of two in common, the block's
scale 2^(byte - 127).  Quantizing a block takes 2^(floor(log2(largest)) - 2) as its
scale and rounds to the nearest value, ties to the even code, at most 6.  With q(x)
the values that x has then, Wq, Gq, Uq the values of quantized weights:

    quantize         q(x)
    linear           y = q(x) Wq^T
    linear_backward  dx = dy Wq, dW = dy^T q(x)
    gated            h = act(g) * u, g = q(x) Gq^T, u = q(x) Uq^T
    gated_backward   dg = dh u act'(g), du = dh act(g),
                     dx = dg Gq + du Uq, dG = dg^T q(x), dU = du^T q(x)

(the gradients pass the rounding by as if it were the identity).  Fields of a case:
``op``; ``m`` rows of x (tokens); ``k`` input channels; ``n`` output channels of
each weight; ``type`` of x, of the incoming gradient and of what comes out; ``act``
of the gated block.  Where ``own`` is false the operators are computed in their plain
form, in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 32
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def _case(name, op, m, k, n=0, type="bf16", act=""):
    return {"name": name, "op": op, "m": m, "k": k, "n": n, "type": type, "act": act}


def listed():
    return [
        # one token's activations: launch and latency bound
        _case("quantize_token", "quantize", 1, 5120, type="fp16"),
        # the hidden activations of a long prompt, or a matrix of weights at load time
        _case("quantize_prompt", "quantize", 4096, 13824),
        # one token through a square projection: the smallest product of a decode step
        _case("linear_token", "linear", 1, 5120, 5120, type="fp16"),
        # a short ragged prompt
        _case("linear_ragged_m77", "linear", 77, 2976, 1357, type="fp32"),
        # a long prompt through the down projection
        _case("linear_down_m2000", "linear", 2000, 13824, 5120),
        # a small fine-tuning batch through a square projection
        _case("linear_backward_m64", "linear_backward", 64, 5120, 5120, type="fp16"),
        # a training batch through the down projection
        _case("linear_backward_m2000", "linear_backward", 2000, 13824, 5120),
        # one token of a chat session through a layer's gate and up
        _case("gated_token", "gated", 1, 5120, 13824, type="fp16", act="silu"),
        # sixteen concurrent sessions, the widest gate and up
        _case("gated_m16", "gated", 16, 5120, 25600, act="silu"),
        # a long prompt
        _case("gated_m2000", "gated", 2000, 5120, 13824, act="silu"),
        # a ragged small batch with gradients in 32 bits
        _case("gated_backward_m77", "gated_backward", 77, 2976, 1357, type="fp32", act="gelu"),
        # a training batch
        _case("gated_backward_m2000", "gated_backward", 2000, 5120, 13824, act="silu"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["quantize", "linear", "linear", "linear_backward", "gated", "gated", "gated_backward"])
        m = _log_int(rng, 1, rng.choice([16, 256, 4096]))
        k = _log_int(rng, 500, 26000)
        n = _log_int(rng, 300, 26000)
        if rng.random() < 0.6:  # the widths of most models
            k, n = max(1, k // 256) * 256, max(1, n // 64) * 64
        c = _case("", op, m, k, 0 if op == "quantize" else n, rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                  rng.choice(["silu", "silu", "gelu", "gelu_tanh"]) if op.startswith("gated") else "")
        del c["name"]
        if _cost(c) <= top:
            return c


# --------------------------------------------------------------------------- inputs
def _weights(case):
    return {"quantize": 0, "linear": 1, "linear_backward": 1, "gated": 2, "gated_backward": 2}[case["op"]]


def _inputs(case, seed):
    """x: N(0, 1) with 1 % of the channels 20 times larger; weights N(0, 0.02^2) in 32 bits;
    the incoming gradient N(0, 1)."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000003 * int(seed) + 17)
    m, k, n, t = case["m"], case["k"], case["n"], TYPES[case["type"]]
    x = torch.randn((m, k), generator=gen, device=DEV)
    x[:, torch.randperm(k, generator=gen, device=DEV)[: max(1, k // 100)]] *= 20
    ws = [torch.randn((n, k), generator=gen, device=DEV) * 0.02 for _ in range(_weights(case))]
    d = torch.randn((m, n), generator=gen, device=DEV).to(t) if case["op"].endswith("backward") else None
    return x.to(t), ws, d


def prepare(case, seed):
    """The activations, the incoming gradient and the quantized weights, as a checkpoint holds them
    (two codes a byte and a byte per block) or laid out for the kernels."""
    x, ws, d = _inputs(case, seed)
    ws = [_checkpoint(w) for w in ws]
    if own:
        import paper_2607_14618_amd as pq
        ws = [pq.mx_pack(codes, scales, case["k"]) for codes, scales in ws]
    return {"op": case["op"], "x": x, "d": d, "w": ws, "k": case["k"], "act": case["act"]}


# --------------------------------------------------------------------------- plain form
def _split(x):
    """The values of x over their block's scale, rounded, as [rows][blocks][32] in 32 bits, and the
    scales' exponents [rows][blocks][1]."""
    rows, k = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -k % BLOCK)).view(rows, -1, BLOCK)
    e = (torch.frexp(v.abs().amax(2, keepdim=True)).exponent - 3).clamp(min=-127)
    v = torch.ldexp(v, -e)
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign((torch.round(a / step) * step).clamp(max=6), v), e


def _quantized(x):
    v, e = _split(x)
    return torch.ldexp(v, e).view(x.shape[0], -1)[:, : x.shape[1]]


def _checkpoint(w):
    """(codes uint8 [n][ceil(k / 2)], low half first; scales uint8 [n][ceil(k / 32)])."""
    v, e = _split(w)
    a = v.abs()
    c = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * (v < 0).to(torch.uint8)
    c = c.view(w.shape[0], -1)[:, : (w.shape[1] + 1) // 2 * 2]
    return (c[:, 0::2] + 16 * c[:, 1::2]).contiguous(), (e.squeeze(2) + 127).to(torch.uint8)


def _values(w, k):
    """The 32-bit values of a checkpoint's matrix."""
    codes, scales = w
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    c = torch.stack((codes & 15, codes >> 4), 2).view(codes.shape[0], -1)[:, :k]
    e = (scales.int() - 127).repeat_interleave(BLOCK, 1)[:, :k]
    return torch.ldexp(table[c.int()], e)


def _act(g, act):
    """act(g) and act'(g)."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if act == "gelu":
        p = 0.5 * torch.erfc(-g * math.sqrt(0.5))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    a, b = math.sqrt(2 / math.pi), 0.044715
    p = 1 / (1 + torch.exp(-2 * a * (g + b * g * g * g)))
    return g * p, p + g * p * (1 - p) * 2 * a * (1 + 3 * b * g * g)


def _plain(s):
    op, x, t = s["op"], s["x"], s["x"].dtype
    if op == "quantize":
        return _quantized(x).to(t)
    w = [_values(v, s["k"]) for v in s["w"]]
    d = None if s["d"] is None else s["d"].float()
    xq = _quantized(x)
    if op == "linear":
        return (xq @ w[0].T).to(t)
    if op == "linear_backward":
        return (d @ w[0]).to(t), (d.T @ xq).to(t)
    g, u = xq @ w[0].T, xq @ w[1].T
    a, da = _act(g, s["act"])
    if op == "gated":
        return (a * u).to(t)
    dg, du = d * u * da, d * a
    return (dg @ w[0] + du @ w[1]).to(t), (dg.T @ xq).to(t), (du.T @ xq).to(t)


def _own(s):
    import paper_2607_14618_amd as pq
    op, x, w = s["op"], s["x"], s["w"]
    if op == "quantize":
        return pq.mx_dequantize(pq.mx_quantize(x), dtype=x.dtype)
    if op == "linear":
        return pq.mx_linear(x, w[0])
    if op == "linear_backward":
        return pq.mx_linear_backward(s["d"], x, w[0])
    if op == "gated":
        return pq.mx_gated(x, w[0], w[1], act=s["act"])
    return pq.mx_gated_backward(s["d"], x, w[0], w[1], act=s["act"])


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------------------------- what a pass costs and gives
def work(case):
    m, k, n, size = case["m"], case["k"], case["n"], TYPES[case["type"]].itemsize
    weight = n * (-(-k // 2) + -(-k // BLOCK))
    x = m * k * size
    return {"quantize": {"bytes": 2 * x + m * (-(-k // 2) + -(-k // BLOCK)), "flops": 0},
            "linear": {"bytes": x + weight + m * n * size, "flops": 2 * m * n * k},
            "linear_backward": {"bytes": 2 * x + weight + (m * n + n * k) * size, "flops": 4 * m * n * k},
            "gated": {"bytes": x + 2 * weight + m * n * size, "flops": 4 * m * n * k},
            "gated_backward": {"bytes": 2 * x + 2 * weight + (m * n + 2 * n * k) * size, "flops": 12 * m * n * k},
            }[case["op"]]


def _cost(case):
    """Seconds of a pass at the card's nominal rates, about."""
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 1e15


# --------------------------------------------------------------------------- in 64 bits
def _exact_quantized(x):
    rows, k = x.shape
    v = torch.zeros((rows, -(-k // BLOCK) * BLOCK), dtype=torch.float64, device=DEV)
    v[:, :k] = x.double()
    v = v.view(rows, -1, BLOCK)
    top = v.abs().max(dim=2, keepdim=True).values
    scale = torch.exp2(torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top)))) - 2)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)
    middle = (grid[1:] + grid[:-1]) / 2
    a = v.abs() / scale
    low = torch.searchsorted(middle, a.contiguous(), right=False)  # middles below a: at a middle the lower neighbour
    high = torch.searchsorted(middle, a.contiguous(), right=True)
    q = grid[torch.where(low % 2 == 0, low, high)]
    return (torch.sign(v) * q * scale).view(rows, -1)[:, :k]


def exact(case, seed):
    x, ws, d = _inputs(case, seed)
    xq = _exact_quantized(x)
    w = [_exact_quantized(v) for v in ws]
    op, act = case["op"], case["act"]
    if op == "quantize":
        return xq
    if op == "linear":
        return torch.matmul(xq, w[0].transpose(0, 1))
    if op == "linear_backward":
        d = d.double()
        return torch.matmul(d, w[0]), torch.matmul(d.transpose(0, 1), xq)
    g, u = (torch.matmul(xq, v.transpose(0, 1)) for v in w)
    if act == "silu":
        value, slope = g * torch.sigmoid(g), torch.sigmoid(g) + g * torch.sigmoid(g) * torch.sigmoid(-g)
    elif act == "gelu":
        normal = (1 + torch.erf(g / math.sqrt(2))) / 2
        value, slope = g * normal, normal + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    else:
        z = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        value = 0.5 * g * (1 + torch.tanh(z))
        slope = 0.5 * (1 + torch.tanh(z)) + 0.5 * g / torch.cosh(z) ** 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)
    if op == "gated":
        return value * u
    d = d.double()
    dg, du = d * u * slope, d * value
    return (torch.matmul(dg, w[0]) + torch.matmul(du, w[1]), torch.matmul(dg.transpose(0, 1), xq),
            torch.matmul(du.transpose(0, 1), xq))
