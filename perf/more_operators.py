"""Products in 8-bit integers and the gated feed-forward block, as cases to be measured.

Seven kinds of pass (``case["op"]``):

  token8          y = q(x) W8^T with weights that are kept in 8 bits, for a few tokens
  forward8        y = q(x) q(W)^T of a linear layer, both operands quantized along the contraction in the call
  backward8       dx = q(dy) q(W^T)^T and dW = q(dy^T) q(x^T)^T, the gradients of that layer (dy rounded stochastically)
  gated           h = act(x Wg^T) * (x Wu^T) in 16 bits, for an answer: nothing else is kept
  gated_train     the same, with both projections kept for the backward pass
  gated_backward  dx, dWg and dWu from dh and what was kept
  gated8          h = act(q(x) Wg8^T) * (q(x) Wu8^T) with weights that are kept in 8 bits

The 8-bit format: a row of a matrix (a token, a channel) has one scale.  With a = max(max |x|, 2^-100) over the row,
r the largest float32 with r a <= 127, and scale = a / 127 (rounded to float32), a code is x r rounded to the nearest
whole number (ties to even), and stands for code * scale.  Stochastic: (floor(16384 x r) + u) >> 14, u the upper 14 of
the 16 bits that (seed, node, row, column) give.  A row that holds a NaN or an infinity has codes 0 and scale NaN.
"""
import math

import torch

own = False

ACTS = ("silu", "gelu", "gelu_tanh", "relu", "sigmoid")


# --------------------------------------------------------------------------- sizes
def listed():
    return [
        # a classifier layer answering one token from 8-bit weights: the call's latency is what a user sees
        {"name": "token8 1", "op": "token8", "t": 1, "i": 2048, "o": 1000},
        # a wide layer answering a small batch of tokens
        {"name": "token8 16", "op": "token8", "t": 16, "i": 4096, "o": 16384},
        # a layer of odd sizes in training, forward, from float32
        {"name": "forward8 odd", "op": "forward8", "t": 777, "i": 1083, "o": 515, "dtype": "float32"},
        # a wide layer over a full batch, forward: the largest 8-bit product
        {"name": "forward8 wide", "op": "forward8", "t": 8192, "i": 4096, "o": 16384, "dtype": "bfloat16"},
        # both gradients of a square layer
        {"name": "backward8 square", "op": "backward8", "t": 8192, "i": 4096, "o": 4096, "dtype": "bfloat16"},
        # a gated block answering one token: the weights' way from memory
        {"name": "gated token", "op": "gated", "t": 1, "i": 4096, "f": 8192, "dtype": "bfloat16", "act": "silu"},
        # a training batch of odd sizes in half precision
        {"name": "gated odd", "op": "gated_train", "t": 333, "i": 515, "f": 1027, "dtype": "float16", "act": "gelu"},
        # a full batch in training, forward
        {"name": "gated wide", "op": "gated_train", "t": 8192, "i": 4096, "f": 8192, "dtype": "bfloat16", "act": "silu"},
        # all gradients of a block of odd sizes
        {"name": "gated backward odd", "op": "gated_backward", "t": 777, "i": 515, "f": 1029, "dtype": "bfloat16", "act": "gelu_tanh"},
        # all gradients over a full batch: the largest pass
        {"name": "gated backward wide", "op": "gated_backward", "t": 8192, "i": 4096, "f": 8192, "dtype": "bfloat16", "act": "silu"},
        # 8-bit weights answering a small batch of tokens
        {"name": "gated8 16", "op": "gated8", "t": 16, "i": 4096, "f": 8192, "dtype": "bfloat16", "act": "silu"},
        # 8-bit weights reading a long prompt
        {"name": "gated8 prompt", "op": "gated8", "t": 2048, "i": 4096, "f": 8192, "dtype": "bfloat16", "act": "silu"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["token8", "forward8", "backward8", "gated", "gated_train", "gated_backward", "gated8"])
    if op == "token8":
        return {"op": op, "t": _log(rng, 1, 64), "i": _log(rng, 64, 8192), "o": _log(rng, 64, 16384)}
    if op in ("forward8", "backward8"):
        return {"op": op, "t": _log(rng, 65, 8192), "i": _log(rng, 33, 4096), "o": _log(rng, 33, 4096),
                "dtype": rng.choice(["float32", "bfloat16", "float16"])}
    case = {"op": op, "t": _log(rng, 65, 8192), "i": _log(rng, 33, 4096), "f": _log(rng, 33, 8192),
            "dtype": rng.choice(["bfloat16", "float16"]), "act": rng.choice(ACTS),
            "pad": rng.choice([0, 0, 8, 5])}      # the tokens' rows are a part of wider ones
    if op in ("gated", "gated8"):
        case["t"] = _log(rng, 1, 4096)
    return case


def work(case):
    op, t, i = case["op"], case["t"], case["i"]
    size = 4 if case.get("dtype") == "float32" else 2
    if op == "token8":
        o = case["o"]
        return {"bytes": o * (i + 4) + 2 * t * (i + o), "flops": 2 * t * i * o}
    if op == "forward8":
        o = case["o"]
        return {"bytes": size * (t * i + o * i) + 2 * t * o, "flops": 2 * t * i * o}
    if op == "backward8":
        o = case["o"]
        return {"bytes": size * (t * i + o * i + t * o) + 2 * t * i + 4 * o * i, "flops": 4 * t * i * o}
    f = case["f"]
    if op == "gated":
        return {"bytes": 2 * (t * i + 2 * f * i + t * f), "flops": 4 * t * i * f}
    if op == "gated_train":
        return {"bytes": 2 * (t * i + 2 * f * i + 3 * t * f), "flops": 4 * t * i * f}
    if op == "gated8":
        return {"bytes": 2 * f * (i + 4) + 2 * (t * i + t * f), "flops": 4 * t * i * f}
    return {"bytes": 2 * (3 * t * f + 2 * t * i + 4 * f * i), "flops": 8 * t * i * f}


# --------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _activations(g, t, i, dtype, pad=0):
    """Unit-variance activations with a few channels ten times as large, as trained networks show."""
    loud = 1 + 9 * (torch.rand((i + pad,), generator=g, device="cuda") < 0.01)
    return (_randn(g, t, i + pad) * loud).to(dtype)[:, :i]


def _gradients(g, t, o, dtype, size=1e-4):
    """Gradients whose tokens differ by two orders of magnitude."""
    return (size * _randn(g, t, o) * 10 ** (-2 * torch.rand((t, 1), generator=g, device="cuda"))).to(dtype)


def _kept(g, o, i):
    """Weights as a program keeps them in 8 bits: (codes [o, ceil(i / 16) * 16], scales [o])."""
    code, scale = _quantized(_randn(g, o, i) / math.sqrt(i))
    return torch.nn.functional.pad(code, (0, -i % 16)).to(torch.int8), scale


def prepare(case, seed):
    g = _gen(seed)
    op, t, i = case["op"], case["t"], case["i"]
    dtype = getattr(torch, case.get("dtype", "bfloat16"))
    s = {"case": case, "seed": int(seed) & 0xFFFFFFFF, "x": _activations(g, t, i, dtype, case.get("pad", 0))}
    if op == "token8":
        s["w"] = _kept(g, case["o"], i)
    elif op == "gated8":
        s["wg"], s["wu"] = _kept(g, case["f"], i), _kept(g, case["f"], i)
    elif op in ("forward8", "backward8"):
        s["w"] = (_randn(g, case["o"], i) / math.sqrt(i)).to(dtype)
        if op == "backward8":
            s["dy"] = _gradients(g, t, case["o"], dtype)
    else:
        s["wg"], s["wu"] = ((_randn(g, case["f"], i) / math.sqrt(i)).to(dtype) for _ in range(2))
        if op == "gated_backward":
            # (half precision is trained with a scaled loss: gradients are kept off its smallest values)
            s["dh"] = _gradients(g, t, case["f"], dtype, 1e-4 if dtype == torch.bfloat16 else 1.0)
            x = s["x"].float()
            s["g"], s["u"] = (x @ s["wg"].float().T).to(dtype), (x @ s["wu"].float().T).to(dtype)
    return s


# --------------------------------------------------------------------------- plain forms: 8-bit integers
def _mix(z):
    z = z ^ ((z >> 30) & 0x3FFFFFFFF)
    z = z * (0xBF58476D1CE4E5B9 - (1 << 64))
    z = z ^ ((z >> 27) & 0x1FFFFFFFFF)
    z = z * (0x94D049BB133111EB - (1 << 64))
    return z ^ ((z >> 31) & 0x1FFFFFFFF)


def _u14(seed, rows, cols):
    """The 14-bit random numbers of [rows, cols] entries of node 0: one 32-bit word for two columns."""
    h = torch.tensor((seed + 0x9E3779B97F4A7C15) % (1 << 64) - (1 << 63), device="cuda") + (-1 << 63)
    i = torch.arange(1, rows + 1, device="cuda")
    h = _mix(_mix(h) ^ (i * (0xD1B54A32D192ED03 - (1 << 64))))[:, None]
    j = torch.arange(1, (cols + 1) // 2 + 1, device="cuda")
    x = ((h >> 32) & 0xFFFFFFFF) ^ (((h & 0xFFFFFFFF) + 0x9E3779B9 * j) & 0xFFFFFFFF)
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & 0xFFFFFFFF
    x = x ^ (x >> 16)
    return torch.stack((x & 0xFFFF, x >> 16), 2).view(rows, -1)[:, :cols] >> 2


def _quantized(x, seed=None):
    """(codes as float32 [rows, cols], scales float32 [rows]); stochastic where a seed is given."""
    x = x.float()
    a = x.abs().amax(1, keepdim=True)
    fine = torch.isfinite(x).all(1, keepdim=True)
    a = torch.where(fine, a, torch.ones_like(a)).clamp_min(2.0 ** -100)
    top = torch.full_like(a, 127)      # (a tensor: a division by a number may be a product with its reciprocal)
    r = top / a
    r = torch.where(r.double() * a.double() > 127, torch.nextafter(r, torch.zeros_like(r)), r)
    v = torch.where(fine, x, torch.zeros_like(x)).double() * r.double()      # exact: a rounding's border lies in it
    if seed is None:
        code = v.round()
    else:
        code = (((v * 16384).floor().to(torch.int64) + _u14(seed, *x.shape)) >> 14)
    return code.float(), torch.where(fine, a / top, torch.full_like(a, float("nan")))[:, 0]


def _product(a, b):
    """a b^T of what two quantized operands stand for, in float32."""
    return (a[0] @ b[0].T) * a[1][:, None] * b[1]


def _of_kept(w, i):
    return w[0][:, :i].float(), w[1]


def _act(name, g):
    if name == "relu":
        return g.clamp_min(0)
    if name == "gelu":
        return 0.5 * g * (1 + torch.erf(g * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
    s = 1 / (1 + torch.exp(-g))
    return s if name == "sigmoid" else g * s


def _slope(name, g):
    """The activation's derivative."""
    if name == "relu":
        return (g > 0).to(g.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        th = torch.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * c * (1 + 3 * 0.044715 * g * g)
    s = 1 / (1 + torch.exp(-g))
    return s * (1 - s) if name == "sigmoid" else s * (1 + g * (1 - s))


def _plain(s):
    case, x = s["case"], s["x"]
    op, i, bf16 = case["op"], case["i"], torch.bfloat16
    if op == "token8":
        return {"y": _product(_quantized(x), _of_kept(s["w"], i)).to(bf16)}
    if op == "forward8":
        return {"y": _product(_quantized(x), _quantized(s["w"])).to(bf16)}
    if op == "backward8":
        dy, seed = s["dy"], s["seed"]
        return {"dx": _product(_quantized(dy, seed), _quantized(s["w"].T)).to(bf16),
                "dw": _product(_quantized(dy.T, seed), _quantized(x.T))}
    act, dtype = case["act"], x.dtype
    if op == "gated8":
        q = _quantized(x)
        g, u = _product(q, _of_kept(s["wg"], i)), _product(q, _of_kept(s["wu"], i))
        return {"h": (_act(act, g) * u).to(dtype)}
    x, wg, wu = x.float(), s["wg"].float(), s["wu"].float()
    if op != "gated_backward":
        g, u = x @ wg.T, x @ wu.T
        h = (_act(act, g) * u).to(dtype)
        return {"h": h} if op == "gated" else {"h": h, "g": g.to(dtype), "u": u.to(dtype)}
    g, u, dh = s["g"].float(), s["u"].float(), s["dh"].float()
    dg, du = dh * u * _slope(act, g), dh * _act(act, g)
    return {"dx": (dg @ wg + du @ wu).to(dtype), "dwg": (dg.T @ x).to(dtype), "dwu": (du.T @ x).to(dtype)}


# --------------------------------------------------------------------------- the library's calls
_made = []    # the context, as a program keeps it


def _context():
    if not _made:
        from paper_1811_03617_b200 import gvq
        _made.append(gvq.Context(gvq.HostLayout(4, 4, [0], [4])))
    return _made[0]


def _own(s):
    from paper_1811_03617_b200 import gvq
    ctx, case, x = _context(), s["case"], s["x"]
    op, t, i = case["op"], case["t"], case["i"]

    def empty(rows, cols, dtype=x.dtype):
        return torch.empty((rows, cols), device="cuda", dtype=dtype)
    if op in ("token8", "forward8"):
        w = gvq.I8(case["o"], i, *s["w"]) if op == "token8" else ctx.i8_quantize(s["w"])
        return {"y": ctx.i8_matmul(ctx.i8_quantize(x), w, empty(t, case["o"], torch.bfloat16))}
    if op == "backward8":
        dy, dy_t = ctx.i8_quantize_both(s["dy"], stochastic=True, seed=s["seed"])
        dx = ctx.i8_matmul(dy, ctx.i8_quantize_transposed(s["w"]), empty(t, i, torch.bfloat16))
        return {"dx": dx, "dw": ctx.i8_matmul(dy_t, ctx.i8_quantize_transposed(x), empty(case["o"], i, torch.float32))}
    f, act = case["f"], case["act"]
    if op == "gated8":
        wg, wu = gvq.I8(f, i, *s["wg"]), gvq.I8(f, i, *s["wu"])
        return {"h": ctx.i8_gated(ctx.i8_quantize(x), wg, wu, empty(t, f), act=act)}
    if op == "gated":
        return {"h": ctx.gated_forward(x, s["wg"], s["wu"], empty(t, f), act=act)}
    if op == "gated_train":
        out = {"h": empty(t, f), "g": empty(t, f), "u": empty(t, f)}
        ctx.gated_forward(x, s["wg"], s["wu"], out["h"], act=act, gate=out["g"], up=out["u"])
        return out
    out = {"dx": empty(t, i), "dwg": empty(f, i), "dwu": empty(f, i)}
    ctx.gated_backward(s["dh"], s["g"], s["u"], x, s["wg"], s["wu"], act=act, dx=out["dx"], dw_gate=out["dwg"], dw_up=out["dwu"])
    return out


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# --------------------------------------------------------------------------- 64 bits, written apart
def _exact_values(x, seed=None):
    """float64 values of x [r, c] after quantization along its rows."""
    top = x.double().abs().max(1).values.clamp_min(2.0 ** -100)
    most = torch.full_like(top, 127)
    # the largest float32 not above 127 / top: its pattern, and one below where rounding went up
    r = (most / top).to(torch.float32)
    r = torch.where(r.double() * top > 127.0, (r.view(torch.int32) - 1).view(torch.float32), r).double()
    at = x.double() * r[:, None]
    lo = torch.floor(at)
    if seed is None:
        part = at - lo
        code = torch.where((part > 0.5) | ((part == 0.5) & (torch.remainder(lo, 2) == 1)), lo + 1, lo)
    else:
        level = torch.floor((at - lo) * 16384)
        code = torch.where(level + _u14(seed, *x.shape) >= 16384, lo + 1, lo)
    return code * (top / most).to(torch.float32).double()[:, None]


def _exact_kept(w, i):
    return w[0].double()[:, :i] * w[1].double()[:, None]


def _exact_act(name, g):
    """(activation, derivative) in 64 bits."""
    if name == "relu":
        return torch.where(g > 0, g, torch.zeros_like(g)), torch.where(g > 0, torch.ones_like(g), torch.zeros_like(g))
    if name == "gelu":
        cdf = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":      # (1 + tanh z) / 2 is the logistic function of 2 z
        c = 2 * math.sqrt(2 / math.pi)
        s = torch.sigmoid(c * (g + 0.044715 * g * g * g))
        return g * s, s + g * s * (1 - s) * c * (1 + 0.134145 * g * g)
    s = torch.sigmoid(g)
    if name == "sigmoid":
        return s, s * torch.sigmoid(-g)
    return g * s, s + g * s * torch.sigmoid(-g)


def exact(case, seed):
    s = prepare(case, seed)
    op, i, x = case["op"], case["i"], s["x"]
    if op == "token8":
        return {"y": _exact_values(x) @ _exact_kept(s["w"], i).T}
    if op == "forward8":
        return {"y": _exact_values(x) @ _exact_values(s["w"]).T}
    if op == "backward8":
        dy = s["dy"]
        return {"dx": _exact_values(dy, s["seed"]) @ _exact_values(s["w"].T).T,
                "dw": _exact_values(dy.T, s["seed"]) @ _exact_values(x.T).T}
    if op == "gated8":
        q = _exact_values(x)
        g, u = q @ _exact_kept(s["wg"], i).T, q @ _exact_kept(s["wu"], i).T
        return {"h": _exact_act(case["act"], g)[0] * u}
    x, wg, wu = x.double(), s["wg"].double(), s["wu"].double()
    if op != "gated_backward":
        g, u = x @ wg.T, x @ wu.T
        h = _exact_act(case["act"], g)[0] * u
        return {"h": h} if op == "gated" else {"h": h, "g": g, "u": u}
    value, slope = _exact_act(case["act"], s["g"].double())
    dg, du = s["dh"].double() * s["u"].double() * slope, s["dh"].double() * value
    return {"dx": torch.cat((dg, du), 1) @ torch.cat((wg, wu)), "dwg": dg.T @ x, "dwu": du.T @ x}
