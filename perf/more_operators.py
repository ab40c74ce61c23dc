"""The operators in front of a transformer block's projections, and the work that their speed is judged by.

The sparse-attention layer stands in a block of a video transformer.  In front of each of the block's products there is a
layer norm, whose factor and offset come from the timestep (a row of them for each batch entry or frame) or are plain weights;
the products themselves run on quantised operands.  The operators here are

  norm         y = (x - mean) / sqrt(variance + eps) * s + b over the rows of B groups; s is w or 1 + w, w and b belong to all
               rows, to a group each, or are not there
  norm_bwd     its gradients: of x, w and b
  quantize     8-bit floating point (E4M3) with one power of two for each block of 128 along the contracted axis, or for each
               128 x 128 values ("square", for weights: X and its transpose then hold the same values); of X, of its transpose,
               or of both; and the values back
  product      C = A B^T + bias of two such operands
  linear       a projection: quantize the activations, product with kept weights
  norm_linear  norm, its result as an operand without a rounding in between, product with kept weights
  linear_bwd   gradients of a projection: dX = dY W and dW = dY^T X, every operand quantised along the axis that the product
               contracts

Plain forms below; `own` switches to the library.  Storage of a quantised operand of R rows and K columns, Kp = K rounded up
to 128: codes [R, Kp] bytes; scales [Kp/512 rounded up, R, 4] bytes, the exponent + 127 of block b of row r at
[b // 4, r, b % 4], zeros behind the last block.
"""
from __future__ import annotations

import math

import torch

own = False

_EPS = 1e-6


# ---------------------------------------------------------------- cases

def _norm(name, kind, dtype, y_dtype, B, N, D, weights, one_plus):
    """weights: "shared" [D], "group" [B,D] (rows of a wider table of modulations), "none"."""
    return {"name": name, "kind": kind, "dtype": dtype, "y_dtype": y_dtype, "B": B, "N": N, "D": D, "weights": weights,
            "one_plus": one_plus}


def _quant(name, dtype, M, G, Kg, heads_first, what, square):
    """what: "rows" (the operand of X), "transposed" (of X^T), "both"."""
    return {"name": name, "kind": "quantize", "dtype": dtype, "M": M, "G": G, "Kg": Kg, "heads_first": heads_first, "what": what,
            "square": square}


def _mm(name, kind, dtype, M, N, K, bias, B=1):
    """B: groups of rows of a norm_linear, M rows in all."""
    return {"name": name, "kind": kind, "dtype": dtype, "M": M, "N": N, "K": K, "bias": bias, "B": B}


def listed():
    return [
        # the norm of one row: latency is all of it
        _norm("norm_token", "norm", "bf16", "bf16", 1, 1, 5120, "shared", False),
        # the modulated norm of a Wan-like layer's hidden states
        _norm("norm_video", "norm", "bf16", "bf16", 1, 75600, 5120, "group", True),
        # a ragged batch of short clips, hidden states kept in fp32, odd channels
        _norm("norm_ragged", "norm", "f32", "bf16", 3, 1078, 777, "group", True),
        # training steps: two clips of 8192 tokens, modulated; an fp32 one with plain weights
        _norm("norm_bwd_clip", "norm_bwd", "bf16", "bf16", 2, 8192, 5120, "group", True),
        _norm("norm_bwd_ragged", "norm_bwd", "f32", "f32", 3, 333, 777, "shared", False),
        # a training step's activations, which the forward product contracts along their channels and the weight's gradient along their tokens
        _quant("quantize_clip", "bf16", 16384, 1, 5120, False, "both", False),
        # the weights of a Wan-like projection to Q, K and V, after the optimiser's step
        _quant("quantize_weights", "bf16", 15360, 1, 5120, False, "both", True),
        # norm and projection of a Wan-like layer; of a ragged batch of short clips
        _mm("norm_linear_video", "norm_linear", "bf16", 75600, 5120, 5120, True),
        _mm("norm_linear_ragged", "norm_linear", "bf16", 2156, 1537, 1000, True, B=2),
        # one token's modulation vector; odd sizes of short clips
        _mm("linear_token", "linear", "bf16", 1, 15360, 5120, True),
        _mm("product_ragged", "product", "f32", 1021, 1537, 1000, True),
        # gradients of a projection over the Small configuration's tokens
        _mm("linear_bwd_clip", "linear_bwd", "bf16", 16384, 1536, 1536, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "norm_bwd", "quantize", "norm_linear", "linear", "product", "linear_bwd"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("norm", "norm_bwd"):
        top = 5120 * (75600 if kind == "norm" else 16384) // (2 if dtype == "f32" else 1)
        while True:
            B, N, D = rng.choice((1, 1, 2, 3, 21)), _log(rng, 1, 75600), _log(rng, 64, 8192)
            if B * N * D <= top:
                break
        weights = rng.choice(("shared", "group", "group", "none"))
        return _norm(None, kind, dtype, rng.choice(("bf16", dtype)), B, N, D, weights, weights == "group")
    if kind == "quantize":
        while True:
            heads_first = rng.random() < 0.3
            M, G, Kg = _log(rng, 1, 75600), (_log(rng, 1, 40) if heads_first else 1), (rng.choice((64, 128)) if heads_first else _log(rng, 32, 8192))
            if M * G * Kg <= 16384 * 5120 // (2 if dtype == "f32" else 1):
                break
        return _quant(None, dtype, M, G, Kg, heads_first, rng.choice(("rows", "transposed", "both")), rng.random() < 0.3)
    while True:
        M, N, K = _log(rng, 1, 75600), _log(rng, 64, 20480), _log(rng, 64, 8192)
        if M * N * K <= 75600 * 5120 * 5120 // (2 if kind == "linear_bwd" else 1) and M * max(N, K) <= 75600 * 5120:
            break
    if kind == "norm_linear":
        B = rng.choice((1, 2, 3))
        return _mm(None, kind, "bf16", -(-M // B) * B, N, K, rng.random() < 0.7, B)
    return _mm(None, kind, dtype, M, N, K, kind != "linear_bwd" and rng.random() < 0.7)


def _size(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_bwd"):
        e, sets = case["B"] * case["N"] * case["D"], {"none": 0, "shared": 1, "group": case["B"]}[case["weights"]]
        xs, ys, w = _size(case["dtype"]), _size(case["y_dtype"]), 4 * sets * case["D"]
        if kind == "norm":
            return {"bytes": e * (xs + ys) + 2 * w, "flops": 8 * e}
        return {"bytes": e * (2 * xs + ys) + 3 * w, "flops": 16 * e}
    if kind == "quantize":
        e, results = case["M"] * case["G"] * case["Kg"], 2 if case["what"] == "both" else 1
        return {"bytes": e * _size(case["dtype"]) * (1 + results) + results * (e + e // 128), "flops": 4 * e * results}
    M, N, K, es = case["M"], case["N"], case["K"], _size(case["dtype"])
    q = lambda rows, cols: rows * (cols + -(-cols // 128))      # noqa: E731  bytes of a quantised operand
    if kind == "product":
        return {"bytes": q(M, K) + q(N, K) + M * N * es, "flops": 2 * M * N * K}
    if kind in ("linear", "norm_linear"):
        return {"bytes": M * K * es + q(N, K) + M * N * es, "flops": 2 * M * N * K}
    return {"bytes": (M * N + 2 * M * K) * es + q(K, N) + 4 * N * K, "flops": 4 * M * N * K}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _activations(M, K, g, dtype):
    """Unit noise times a spread of channel sizes, with the few large channels that hidden states have, and a mean of its own for
    each row."""
    channel = torch.exp(0.5 * torch.randn((K,), generator=g, device="cuda"))
    channel = channel * torch.where(torch.rand((K,), generator=g, device="cuda") < 0.01, 20.0, 1.0)
    mean = 0.3 * torch.randn((M, 1), generator=g, device="cuda")
    return (torch.randn((M, K), generator=g, device="cuda") * channel + mean).to(dtype)


def _modulation(B, D, weights, g):
    """w and b: plain weights around 1 and 0, or two rows of each group's table of six."""
    if weights == "none":
        return None, None
    if weights == "shared":
        return (1.0 + 0.2 * torch.randn((D,), generator=g, device="cuda")), 0.2 * torch.randn((D,), generator=g, device="cuda")
    table = 0.3 * torch.randn((B, 6, D), generator=g, device="cuda")
    return table[:, 1], table[:, 0]


def prepare(case, seed):
    g = _gen(seed)
    kind, dtype = case["kind"], _dtype(case["dtype"])
    st = {"case": case}
    if kind in ("norm", "norm_bwd"):
        B, N, D = case["B"], case["N"], case["D"]
        st["x"] = _activations(B * N, D, g, dtype).view(B, N, D)
        st["w"], st["b"] = _modulation(B, D, case["weights"], g)
        if kind == "norm_bwd":
            st["dy"] = torch.randn((B, N, D), generator=g, device="cuda").to(_dtype(case["y_dtype"]))
        return st
    if kind == "quantize":
        M, G, Kg = case["M"], case["G"], case["Kg"]
        x = _activations(M, G * Kg, g, dtype).view(M, G, Kg)
        st["x"] = x.transpose(0, 1).contiguous().transpose(0, 1) if case["heads_first"] else x
        return st
    M, N, K = case["M"], case["N"], case["K"]
    w = (torch.randn((N, K), generator=g, device="cuda") / math.sqrt(K)).to(dtype)
    if kind == "linear_bwd":
        st["x"], st["dy"] = _activations(M, K, g, dtype), torch.randn((M, N), generator=g, device="cuda").to(dtype)
        st["weight"] = _pack(*_quantize(w.t().float(), True))
        return st
    st["weight"] = _pack(*_quantize(w.float(), True))
    st["bias"] = torch.randn((N,), generator=g, device="cuda") if case["bias"] else None
    x = _activations(M, K, g, dtype)
    if kind == "product":
        st["a"] = _pack(*_quantize(x.float(), False))
    elif kind == "linear":
        st["x"] = x
    else:
        st["x"] = x.view(case["B"], M // case["B"], K)
        st["w"], st["b"] = _modulation(case["B"], K, "group", g)
    return st


# ---------------------------------------------------------------- plain forms

def _times_power(x, e):
    """x * 2^e, in two steps so that neither power leaves fp32's range."""
    h = torch.div(e, 2, rounding_mode="floor")
    power = lambda k: ((k + 127) << 23).to(torch.int32).view(torch.float32)     # noqa: E731
    return x * power(h) * power(e - h)


def _e4m3(y):
    """fp32 values up to 448 in size -> the nearest E4M3 numbers, ties to the even one: steps of 1/8 of their power of two, of 2^-9 below
    2^-6."""
    p = (torch.frexp(y).exponent - 1).clamp(min=-6)
    return _times_power(torch.round(_times_power(y, 3 - p)), p - 3)


def _quantize(x, square):
    """fp32 [R,K] -> E4M3 values [R, Kp/128, 128] and exponents [R, Kp/128, 1]."""
    R, K = x.shape
    x = torch.nn.functional.pad(x, (0, -K % 128)).view(R, -1, 128)
    amax = x.abs().amax(2, keepdim=True)
    if square:
        amax = torch.nn.functional.pad(amax, (0, 0, 0, 0, 0, -R % 128))
        amax = amax.view(-1, 128, amax.shape[1], 1).amax(1, keepdim=True).expand(-1, 128, -1, -1).reshape(-1, amax.shape[1], 1)[:R]
    m, e = torch.frexp(amax)
    e = (e - 9 + (m > 0.875).to(torch.int32)).clamp(min=-127)       # 448 = 0.875 * 2^9
    e = torch.where(amax == 0, torch.full_like(e, -127), e)
    return _e4m3(_times_power(x, -e)), e


def _pack(v, e):
    R, n = v.shape[:2]
    codes = v.view(R, -1).to(torch.float8_e4m3fn).view(torch.uint8).contiguous()
    scales = torch.nn.functional.pad((e[:, :, 0] + 127).to(torch.uint8), (0, -n % 4))
    return codes, scales.view(R, -1, 4).transpose(0, 1).contiguous()


def _unpack(codes, scales):
    """codes, scales -> fp32 [R,Kp]"""
    R, Kp = codes.shape
    e = scales.transpose(0, 1).reshape(R, -1, 1)[:, :Kp // 128].int() - 127
    return _times_power(codes.view(torch.float8_e4m3fn).float().view(R, -1, 128), e).view(R, Kp)


def _dequantized(x, square=False):
    v, e = _quantize(x, square)
    return _times_power(v, e).view(x.shape[0], -1)


def _factor(st, w):
    w = w.float() if w.dim() == 1 else w.float()[:, None, :]
    return 1.0 + w if st["case"].get("one_plus", True) else w


def _offset(b):
    return b.float() if b.dim() == 1 else b.float()[:, None, :]


def _plain_norm(st):
    x = st["x"].float()
    x = x - x.mean(-1, keepdim=True)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
    if st["w"] is not None:
        y = y * _factor(st, st["w"]) + _offset(st["b"])
    return y


def _plain_norm_bwd(st):
    x, dy = st["x"].float(), st["dy"].float()
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
    n = x * r
    g = dy if st["w"] is None else dy * _factor(st, st["w"])
    dx = r * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
    out = [dx.to(st["x"].dtype)]
    if st["w"] is not None:
        over = (0, 1) if st["w"].dim() == 1 else (1,)
        out += [(dy * n).sum(over, dtype=torch.float64).float(), dy.sum(over, dtype=torch.float64).float()]
    return out


def _plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "norm":
        return _plain_norm(st).to(_dtype(case["y_dtype"]))
    if kind == "norm_bwd":
        return _plain_norm_bwd(st)
    dtype = _dtype(case["dtype"])
    if kind == "quantize":
        x, out = st["x"].flatten(1).float(), []
        if case["what"] != "transposed":
            out.append(_dequantized(x, case["square"])[:, :x.shape[1]].to(dtype))
        if case["what"] != "rows":
            out.append(_dequantized(x.t(), case["square"])[:, :x.shape[0]].to(dtype))
        return out
    if kind == "linear_bwd":
        dy, x, w = st["dy"].float(), st["x"].float(), _unpack(*st["weight"])
        return [torch.matmul(_dequantized(dy), w.t()).to(dtype), torch.matmul(_dequantized(dy.t()), _dequantized(x.t()).t())]
    a = _unpack(*st["a"]) if kind == "product" else _dequantized(st["x"].float() if kind == "linear" else _plain_norm(st).flatten(0, 1))
    c = torch.matmul(a, _unpack(*st["weight"]).t())
    if st["bias"] is not None:
        c = c + st["bias"]
    return c.to(dtype)


# ---------------------------------------------------------------- the library's calls

def _own(st):
    import paper_2505_18875_amd as svg2
    case = st["case"]
    kind = case["kind"]
    if kind == "norm":
        return svg2.svg2_layer_norm(st["x"], st["w"], st["b"], eps=_EPS, one_plus=case["one_plus"], out_dtype=_dtype(case["y_dtype"]))
    if kind == "norm_bwd":
        res = svg2.svg2_layer_norm_backward(st["dy"], st["x"], st["w"], st["b"], eps=_EPS, one_plus=case["one_plus"])
        return [res.grad] + ([] if st["w"] is None else [res.dweight, res.dbias])
    dtype = _dtype(case["dtype"])
    if kind == "quantize":
        x = st["x"] if case["G"] > 1 else st["x"][:, 0]
        M, K = case["M"], case["G"] * case["Kg"]
        if case["what"] == "both":
            pairs = svg2.svg2_quantize_fp8_blocks(x, transposed="both", square=case["square"])
        else:
            pairs = [svg2.svg2_quantize_fp8_blocks(x, transposed=case["what"] == "transposed", square=case["square"])]
        columns = {"rows": (K,), "transposed": (M,), "both": (K, M)}[case["what"]]
        return [svg2.svg2_dequantize_fp8_blocks(*p, n, dtype=dtype) for p, n in zip(pairs, columns)]
    if kind == "linear_bwd":
        dy, dy_t = svg2.svg2_quantize_fp8_blocks(st["dy"], transposed="both")
        dx = svg2.svg2_matmul_fp8_blocks(*dy, *st["weight"], out_dtype=dtype)
        dw = svg2.svg2_matmul_fp8_blocks(*dy_t, *svg2.svg2_quantize_fp8_blocks(st["x"], transposed=True), out_dtype=torch.float32)
        return [dx, dw]
    if kind == "product":
        a = st["a"]
    elif kind == "linear":
        a = svg2.svg2_quantize_fp8_blocks(st["x"])
    else:
        a = svg2.svg2_layer_norm_fp8(st["x"], st["w"], st["b"], eps=_EPS, one_plus=True)
    return svg2.svg2_matmul_fp8_blocks(*a, *st["weight"], bias=st["bias"], out_dtype=dtype)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- 64 bits, from the definitions

def _exact_norm(st):
    """rows [B,N,D] -> deviation over standard deviation, and 1 / standard deviation"""
    x = st["x"].double()
    variance, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
    inv = (variance + _EPS) ** -0.5
    return (x - mean) * inv, inv


def _exact_modulated(st, n):
    w, b = st["w"], st["b"]
    if w is None:
        return n
    w, b = (t.double() if t.dim() == 1 else t.double().unsqueeze(1) for t in (w, b))
    return n + n * w + b if st["case"].get("one_plus", True) else n * w + b


def _exact_power(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_table(device):
    """The 127 finite magnitudes of E4M3 by their codes."""
    code = torch.arange(127, device=device)
    exponent, mantissa = code // 8, (code % 8).double()
    return torch.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * _exact_power(exponent - 10))


def _exact_values(x, square=False):
    """The values that quantising the rows of x (64 bits) leaves: nearest of the E4M3 numbers times the block's scale, ties to the even
    code."""
    R, K = x.shape
    tall = -(-R // 128) * 128 if square else R
    full = torch.zeros((tall, (K + 127) // 128 * 128), dtype=torch.float64, device=x.device)
    full[:R, :K] = x
    rows = 128 if square else 1
    blocks = full.view(tall // rows, rows, -1, 128)
    top = blocks.abs().amax((1, 3), keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).clamp(-127, 127)
    e = torch.where(top > 448 * _exact_power(e), e + 1, torch.where(top <= 448 * _exact_power((e - 1).clamp(min=-127)), (e - 1).clamp(min=-127), e))
    scale = _exact_power(e)
    table = _exact_table(x.device)
    a = blocks.abs() / scale
    border = (table[1:] + table[:-1]) / 2
    low, high = torch.bucketize(a, border), torch.bucketize(a, border, right=True)
    value = table[torch.where((low != high) & (low % 2 == 1), high, low)]
    return (torch.sign(blocks) * value * scale).view(tall, -1)[:R, :K]


def _exact_stored(codes, scales, K):
    k = torch.arange(K, device=codes.device)
    code = codes[:, k].to(torch.int64)
    value = _exact_table(codes.device)[(code % 128).clamp(max=126)] * torch.where(code >= 128, -1.0, 1.0).double()
    b = k // 128
    return value * _exact_power(scales[b // 4, :, b % 4].t().to(torch.int64) - 127)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _exact_modulated(st, _exact_norm(st)[0])
    if kind == "norm_bwd":
        n, inv = _exact_norm(st)
        dy, w = st["dy"].double(), st["w"]
        g = dy
        if w is not None:
            w = (w.double() if w.dim() == 1 else w.double().unsqueeze(1)) + (1.0 if case["one_plus"] else 0.0)
            g = dy * w
        D = case["D"]
        dx = inv * (g - (g.sum(-1, keepdim=True) + n * (g * n).sum(-1, keepdim=True)) / D)
        if w is None:
            return [dx]
        shared = st["w"].dim() == 1
        dw, db = (dy * n).sum(1), dy.sum(1)
        return [dx, dw.sum(0) if shared else dw, db.sum(0) if shared else db]
    if kind == "quantize":
        x = st["x"].double().reshape(case["M"], -1)
        out = [] if case["what"] == "transposed" else [_exact_values(x, case["square"])]
        return out if case["what"] == "rows" else out + [_exact_values(x.t().contiguous(), case["square"])]
    M, N, K = case["M"], case["N"], case["K"]
    if kind == "linear_bwd":
        dy, x = st["dy"].double(), st["x"].double()
        return [_exact_values(dy) @ _exact_stored(*st["weight"], N).t(),
                _exact_values(dy.t().contiguous()) @ _exact_values(x.t().contiguous()).t()]
    if kind == "product":
        a = _exact_stored(*st["a"], K)
    elif kind == "linear":
        a = _exact_values(st["x"].double())
    else:
        a = _exact_values(_exact_modulated(st, _exact_norm(st)[0]).view(M, K))
    c = a @ _exact_stored(*st["weight"], K).t()
    return c if st["bias"] is None else c + st["bias"].double()
