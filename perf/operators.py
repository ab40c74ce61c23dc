"""The operators around the sparse-attention layer, and the work that their speed is judged by.

The layer takes Q, K and V per head, [H,N,d].  A video transformer has hidden states, one row per token, and gets from the
one to the other by a projection, a normalisation of Q and K, rotary positions over (time, height, width) and the move from
token order to head order; the attention's output goes back through a second projection.  The operators here are

  rope       RMS normalisation of Q and K (over the head or over all heads of the token), rotary positions over several
             axes, token order -> head order; for Q, K and V of one packed projection in one call
  rope_bwd   its gradients: of Q, K, V and of the norms' weights
  quantize   microscaled 4-bit floating point (blocks of 32 along the contracted axis: one power-of-two scale, E2M1
             elements), rows of any strides, or transposed; and the values back
  product    C = A B^T + bias of two such operands
  linear     a projection: quantize the activations, product with kept weights
  linear_bwd its gradients dX = dY W and dW = dY^T X, every operand quantised along the axis that the product contracts

Plain forms below; `own` switches to the library.  Storage of a quantised operand of R rows and K columns, Kp = K rounded up
to 128: codes [R, Kp/2] bytes, element 2j in the low half of byte j; scales [Kp/128, R, 4] bytes, the exponent + 127 of block
b of row r at [b // 4, r, b % 4].
"""
from __future__ import annotations

import math

import torch

own = False

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_THETA = 10000.0


# ---------------------------------------------------------------- cases

def _rope(name, kind, dtype, B, grid, text, H, d, norm, pairing, first):
    return {"name": name, "kind": kind, "dtype": dtype, "B": B, "T": grid[0], "Y": grid[1], "X": grid[2], "text": text,
            "H": H, "d": d, "norm": norm, "pairing": pairing, "first": first}


def _quant(name, dtype, M, G, Kg, transposed, heads_first):
    return {"name": name, "kind": "quantize", "dtype": dtype, "M": M, "G": G, "Kg": Kg, "transposed": transposed,
            "heads_first": heads_first}


def _mm(name, kind, dtype, M, N, K, bias):
    return {"name": name, "kind": kind, "dtype": dtype, "M": M, "N": N, "K": K, "bias": bias}


def listed():
    return [
        # one token of 40 heads far into a stream: latency is all of it
        _rope("rope_token", "rope", "bf16", 1, (1, 1, 1), 0, 40, 128, "token", "adjacent", 1000003),
        # the fp32 head of the Tiny configuration's grid
        _rope("rope_tiny_f32", "rope", "f32", 1, (16, 16, 16), 0, 1, 64, "none", "adjacent", 0),
        # a ragged batch of short clips, text tokens behind the video's, norm per head, halves paired
        _rope("rope_ragged", "rope", "bf16", 2, (7, 13, 11), 77, 5, 64, "head", "halves", 3),
        # Q, K and V of a Wan-like layer
        _rope("rope_video", "rope", "bf16", 1, (21, 45, 80), 0, 40, 128, "token", "adjacent", 0),
        # a training step on the Small configuration's grid, and a ragged fp32 one
        _rope("rope_bwd_clip", "rope_bwd", "bf16", 1, (16, 32, 32), 0, 40, 128, "token", "adjacent", 0),
        _rope("rope_bwd_ragged", "rope_bwd", "f32", 3, (3, 9, 11), 36, 7, 64, "head", "halves", 0),
        # the attention's output, in head order, as the rows of the second projection (Wan-like)
        _quant("quantize_video", "bf16", 75600, 40, 128, False, True),
        # odd rows and columns, transposed: the operand of a weight gradient
        _quant("quantize_ragged_t", "f32", 1021, 1, 777, True, False),
        # the second projection of a Wan-like layer, one token's modulation vector, odd sizes of short clips
        _mm("linear_video", "linear", "bf16", 75600, 5120, 5120, True),
        _mm("linear_token", "linear", "bf16", 1, 15360, 5120, True),
        _mm("product_ragged", "product", "f32", 1021, 1537, 1000, True),
        # gradients of a projection over the Small configuration's tokens
        _mm("linear_bwd_clip", "linear_bwd", "bf16", 16384, 1536, 1536, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "rope", "rope_bwd", "quantize", "linear", "linear", "product", "linear_bwd"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if kind in ("rope", "rope_bwd"):
        top = 40 * 128 * (75600 if kind == "rope" else 16384) // (2 if dtype == "f32" else 1)
        while True:
            grid = (_log(rng, 1, 33), _log(rng, 1, 48), _log(rng, 1, 80))
            B, H, d, text = rng.choice((1, 1, 2, 3)), _log(rng, 1, 40), rng.choice((64, 128)), rng.choice((0, 0, rng.randint(1, 256)))
            if B * H * d * (grid[0] * grid[1] * grid[2] + text) <= top:
                break
        return _rope(None, kind, dtype, B, grid, text, H, d, rng.choice(("none", "head", "token")),
                     rng.choice(("adjacent", "halves")), rng.choice((0, 0, _log(rng, 1, 1000000))))
    if kind == "quantize":
        while True:
            heads_first = rng.random() < 0.5
            M, G, Kg = _log(rng, 1, 75600), (_log(rng, 1, 40) if heads_first else 1), (rng.choice((64, 128)) if heads_first else _log(rng, 32, 5120))
            if M * G * Kg <= 75600 * 5120 // (2 if dtype == "f32" else 1):
                break
        return _quant(None, dtype, M, G, Kg, rng.random() < 0.4, heads_first)
    while True:
        M, N, K = _log(rng, 1, 75600), _log(rng, 64, 20480), _log(rng, 64, 8192)
        if M * N * K <= 75600 * 5120 * 5120 // (2 if kind == "linear_bwd" else 1) and M * max(N, K) <= 75600 * 5120:
            break
    return _mm(None, kind, dtype, M, N, K, kind != "linear_bwd" and rng.random() < 0.7)


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] in ("rope", "rope_bwd"):
        n = case["B"] * (case["T"] * case["Y"] * case["X"] + case["text"])
        e = 3 * n * case["H"] * case["d"]               # elements of Q, K and V
        normed = case["norm"] != "none"
        if case["kind"] == "rope":
            return {"bytes": 2 * e * es + 12 * n, "flops": (2 * e // 3) * (3 + (4 if normed else 0))}
        # the gradients come in and go out; Q and K are read again only where they are normalised
        return {"bytes": (2 * e + (2 * e // 3 if normed else 0)) * es + 12 * n,
                "flops": (2 * e // 3) * (3 + (12 if normed else 0))}
    if case["kind"] == "quantize":
        e = case["M"] * case["G"] * case["Kg"]
        return {"bytes": 2 * e * es + e // 2 + e // 32, "flops": 4 * e}
    M, N, K = case["M"], case["N"], case["K"]
    q = lambda rows, cols: rows * (cols // 2 + cols // 32)      # noqa: E731  bytes of a quantised operand
    if case["kind"] == "product":
        return {"bytes": q(M, K) + q(N, K) + M * N * es, "flops": 2 * M * N * K}
    if case["kind"] == "linear":
        return {"bytes": M * K * es + q(N, K) + M * N * es, "flops": 2 * M * N * K}
    return {"bytes": (M * N + 2 * M * K) * es + q(K, N) + 4 * N * K, "flops": 4 * M * N * K}


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, g, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _activations(M, K, g, dtype):
    """Unit noise times a spread of channel sizes, with the few large channels that hidden states have."""
    channel = torch.exp(0.5 * torch.randn((K,), generator=g, device="cuda"))
    channel = channel * torch.where(torch.rand((K,), generator=g, device="cuda") < 0.01, 20.0, 1.0)
    return (torch.randn((M, K), generator=g, device="cuda") * channel).to(dtype)


def _axis_pairs(d):
    side = 2 * (d // 6)                                  # height and width get a third of the head each, rounded down
    return ((d - 2 * side) // 2, side // 2, side // 2)


def _frequencies(d):
    out = []
    for n in _axis_pairs(d):
        out += [_THETA ** (-i / n) for i in range(n)]
    return torch.tensor(out, dtype=torch.float64)


def _positions(case):
    """(time, height, width) of every token, int32 [N,3]; text tokens behind the video's keep position 0."""
    T, Y, X = case["T"], case["Y"], case["X"]
    t, y, x = torch.meshgrid(torch.arange(T) + case["first"], torch.arange(Y), torch.arange(X), indexing="ij")
    video = torch.stack([t.reshape(-1), y.reshape(-1), x.reshape(-1)], 1)
    return torch.cat([video, torch.zeros((case["text"], 3), dtype=video.dtype)]).to(torch.int32)


def prepare(case, seed):
    g = _gen(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    st = {"case": case}
    if case["kind"] in ("rope", "rope_bwd"):
        B, H, d = case["B"], case["H"], case["d"]
        pos = _positions(case)
        N = pos.shape[0]
        st["pos"], st["freq"] = pos.cuda(), _frequencies(d).cuda()
        st["packed"] = _randn((B, N, 3, H, d), g, dtype)        # what one projection to Q, K and V leaves
        if case["norm"] != "none":
            shape = (d,) if case["norm"] == "head" else (H, d)
            st["weights"] = [1.0 + 0.2 * torch.randn(shape, generator=g, device="cuda") for _ in range(2)] + [None]
        else:
            st["weights"] = None
        if case["kind"] == "rope_bwd":
            st["grads"] = [_randn((B * H, N, d), g, dtype) for _ in range(3)]
        return st
    if case["kind"] == "quantize":
        M, G, Kg = case["M"], case["G"], case["Kg"]
        x = _activations(M, G * Kg, g, dtype).view(M, G, Kg)
        st["x"] = x.transpose(0, 1).contiguous().transpose(0, 1) if case["heads_first"] else x
        return st
    M, N, K = case["M"], case["N"], case["K"]
    w = (torch.randn((N, K), generator=g, device="cuda") / math.sqrt(K)).to(dtype)
    if case["kind"] == "linear_bwd":
        st["x"], st["dy"] = _activations(M, K, g, dtype), _randn((M, N), g, dtype)
        st["w"] = _pack(*_quantize(w.t().float()))
        return st
    st["w"] = _pack(*_quantize(w.float()))
    st["bias"] = torch.randn((N,), generator=g, device="cuda") if case["bias"] else None
    x = _activations(M, K, g, dtype)
    if case["kind"] == "linear":
        st["x"] = x
    else:
        st["a"] = _pack(*_quantize(x.float()))
    return st


# ---------------------------------------------------------------- plain forms

def _times_power(x, e):
    """x * 2^e, in two steps so that neither power leaves fp32's range."""
    h = torch.div(e, 2, rounding_mode="floor")
    power = lambda k: ((k + 127) << 23).to(torch.int32).view(torch.float32)     # noqa: E731
    return x * power(h) * power(e - h)


def _quantize(x):
    """fp32 [R,K] -> signed E2M1 values and their exponents, [R, Kp/32, 32] and [R, Kp/32, 1]."""
    R, K = x.shape
    x = torch.nn.functional.pad(x, (0, -K % 128)).view(R, -1, 32)
    amax = x.abs().amax(2, keepdim=True)
    e = (torch.frexp(amax).exponent - 3).clamp(-127, 125)       # the largest of a block lands in [4, 8)
    e = torch.where(amax == 0, torch.full_like(e, -127), e)
    y = _times_power(x, -e)
    a = y.abs()
    a = torch.where(a < 2, torch.round(2 * a) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2))).clamp(max=6)
    return torch.copysign(a, y), e


def _pack(v, e):
    R = v.shape[0]
    a = v.abs()
    code = torch.where(a <= 2, 2 * a, torch.where(a <= 4, a + 2, a + 1)).to(torch.uint8) + 8 * torch.signbit(v).to(torch.uint8)
    code = code.view(R, -1, 2)
    codes = (code[:, :, 0] + 16 * code[:, :, 1]).contiguous()
    scales = (e + 127).to(torch.uint8).view(R, -1, 4).transpose(0, 1).contiguous()
    return codes, scales


def _unpack(codes, scales):
    """codes, scales -> fp32 [R,Kp]"""
    R = codes.shape[0]
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], 2).view(R, -1, 32)
    e = scales.transpose(0, 1).reshape(R, -1, 1).int() - 127
    return _times_power(v, e).view(R, -1)


def _dequantized(x):
    v, e = _quantize(x)
    return _times_power(v, e).view(x.shape[0], -1)


def _angles(st):
    pos = st["pos"].double()
    axis = torch.repeat_interleave(torch.arange(3, device=pos.device), torch.tensor(_axis_pairs(st["case"]["d"]), device=pos.device))
    a = pos[:, axis] * st["freq"]                                # [N, d/2], in 64 bits: positions are far
    return a.cos().float()[:, None, :], a.sin().float()[:, None, :]


def _pairs(x, pairing):
    return (x[..., 0::2], x[..., 1::2]) if pairing == "adjacent" else x.chunk(2, dim=-1)


def _unpairs(a, b, pairing):
    return torch.stack([a, b], -1).flatten(-2) if pairing == "adjacent" else torch.cat([a, b], -1)


def _norm_dims(case):
    return (-1,) if case["norm"] == "head" else (-2, -1)


def _plain_rope(st):
    case, out = st["case"], []
    cos, sin = _angles(st)
    for i in range(3):
        x = st["packed"][:, :, i].float()                        # [B,N,H,d]
        if i < 2:
            if st["weights"] is not None:
                x = x * torch.rsqrt((x * x).mean(_norm_dims(case), keepdim=True) + 1e-6) * st["weights"][i]
            a, b = _pairs(x, case["pairing"])
            x = _unpairs(a * cos - b * sin, a * sin + b * cos, case["pairing"])
        out.append(x.to(st["packed"].dtype).transpose(1, 2).flatten(0, 1).contiguous())
    return out


def _plain_rope_bwd(st):
    case = st["case"]
    B, N, _, H, d = st["packed"].shape
    cos, sin = _angles(st)
    dx, dw = torch.empty_like(st["packed"]), []
    for i in range(3):
        g = st["grads"][i].view(B, H, N, d).transpose(1, 2).float()
        if i < 2:
            a, b = _pairs(g, case["pairing"])
            g = _unpairs(a * cos + b * sin, b * cos - a * sin, case["pairing"])
            if st["weights"] is not None:
                x = st["packed"][:, :, i].float()
                dims = _norm_dims(case)
                r = torch.rsqrt((x * x).mean(dims, keepdim=True) + 1e-6)
                xn = x * r
                dw.append((g * xn).sum((0, 1, 2) if case["norm"] == "head" else (0, 1), dtype=torch.float64).float())
                g = g * st["weights"][i]
                g = r * (g - xn * (g * xn).mean(dims, keepdim=True))
        dx[:, :, i] = g.to(dx.dtype)
    return [dx] + dw


def _plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "rope":
        return _plain_rope(st)
    if kind == "rope_bwd":
        return _plain_rope_bwd(st)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    if kind == "quantize":
        x = st["x"].flatten(1).float()
        x = x.t() if case["transposed"] else x
        return _dequantized(x)[:, :x.shape[1]].to(dtype)
    if kind == "linear_bwd":
        dy, x, w = st["dy"].float(), st["x"].float(), _unpack(*st["w"])
        return [torch.matmul(_dequantized(dy), w.t()).to(dtype), torch.matmul(_dequantized(dy.t()), _dequantized(x.t()).t())]
    a = _dequantized(st["x"].float()) if kind == "linear" else _unpack(*st["a"])
    c = torch.matmul(a, _unpack(*st["w"]).t())
    if st["bias"] is not None:
        c = c + st["bias"]
    return c.to(dtype)


# ---------------------------------------------------------------- the library's calls

def _own(st):
    import paper_2505_18875_amd as svg2
    case = st["case"]
    kind = case["kind"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    if kind in ("rope", "rope_bwd"):
        qkv = [st["packed"][:, :, i] for i in range(3)]
        kw = dict(axis_pairs=_axis_pairs(case["d"]), rotate=(True, True, False), norm_weights=st["weights"],
                  norm_scope=case["norm"] if st["weights"] is not None else "head", eps=1e-6, pairing=case["pairing"])
        if kind == "rope":
            return svg2.svg2_rope(qkv, st["pos"], st["freq"], **kw)
        dx = torch.empty_like(st["packed"])
        res = svg2.svg2_rope_backward(st["grads"], qkv, st["pos"], st["freq"], outs=[dx[:, :, i] for i in range(3)], **kw)
        return [dx] + [w for w in res.dweights if w is not None]
    if kind == "quantize":
        x = st["x"] if case["G"] > 1 else st["x"][:, 0]
        codes, scales = svg2.svg2_quantize_mxfp4(x, transposed=case["transposed"])
        return svg2.svg2_dequantize_mxfp4(codes, scales, case["M"] if case["transposed"] else case["G"] * case["Kg"], dtype=dtype)
    if kind == "linear_bwd":
        dx = svg2.svg2_matmul_mxfp4(*svg2.svg2_quantize_mxfp4(st["dy"]), *st["w"], out_dtype=dtype)
        dw = svg2.svg2_matmul_mxfp4(*svg2.svg2_quantize_mxfp4(st["dy"], transposed=True),
                                    *svg2.svg2_quantize_mxfp4(st["x"], transposed=True), out_dtype=torch.float32)
        return [dx, dw]
    a = svg2.svg2_quantize_mxfp4(st["x"]) if kind == "linear" else st["a"]
    return svg2.svg2_matmul_mxfp4(*a, *st["w"], bias=st["bias"], out_dtype=dtype)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- 64 bits, from the definitions

def _exact_power(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(x):
    """The values that quantising the rows of x (64 bits) leaves: nearest of the E2M1 numbers times the block's scale, ties to
    the even code."""
    R, K = x.shape
    full = torch.zeros((R, (K + 31) // 32 * 32), dtype=torch.float64, device=x.device)
    full[:, :K] = x
    blocks = full.view(R, -1, 32)
    top = blocks.abs().max(dim=2, keepdim=True).values
    scale = _exact_power((torch.frexp(top).exponent - 3).clamp(-127, 125))
    a = blocks.abs() / scale
    code = torch.zeros(a.shape, dtype=torch.int64, device=x.device)
    for border, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if up else (a > border)
    value = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)[code]
    return (torch.sign(blocks) * value * scale).view(R, -1)[:, :K]


def _exact_stored(codes, scales, K):
    R = codes.shape[0]
    k = torch.arange(K, device=codes.device)
    byte = codes[:, k // 2].to(torch.int64)
    code = torch.where(k % 2 == 0, byte % 16, byte // 16)
    value = torch.tensor(_E2M1, dtype=torch.float64, device=codes.device)[code % 8] * torch.where(code >= 8, -1.0, 1.0).double()
    b = k // 32
    return value * _exact_power(scales[b // 4, :, b % 4].t().to(torch.int64) - 127)


def _exact_turn(x, angle, pairing, sense):
    """The pairs of x [..., N, H, d] turned by sense * angle [N, d/2]."""
    d = x.shape[-1]
    p = torch.arange(d // 2, device=x.device)
    i, j = (2 * p, 2 * p + 1) if pairing == "adjacent" else (p, p + d // 2)
    z = torch.complex(x[..., i], x[..., j]) * torch.polar(torch.ones_like(angle), sense * angle)[:, None, :]
    out = torch.empty_like(x)
    out[..., i], out[..., j] = z.real, z.imag
    return out


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rope", "rope_bwd"):
        B, N, _, H, d = st["packed"].shape
        n = _axis_pairs(d)
        angle = torch.cat([st["pos"][:, i:i + 1].double() * st["freq"][sum(n[:i]):sum(n[:i + 1])] for i in range(3)], 1)
        outs, dws = [], []
        for i in range(3):
            x = st["packed"][:, :, i].double()
            normed = i < 2 and st["weights"] is not None
            if normed:
                w = st["weights"][i].double()
                ms = x.pow(2).mean(-1, keepdim=True)
                if case["norm"] == "token":
                    ms = ms.mean(-2, keepdim=True)
                inv = (ms + 1e-6) ** -0.5
            if kind == "rope":
                x = x * inv * w if normed else x
                x = _exact_turn(x, angle, case["pairing"], 1.0) if i < 2 else x
                outs.append(x.permute(0, 2, 1, 3).reshape(B * H, N, d))
                continue
            g = st["grads"][i].double().view(B, H, N, d).permute(0, 2, 1, 3)
            g = _exact_turn(g.contiguous(), angle, case["pairing"], -1.0) if i < 2 else g
            if normed:
                prod = g * x * inv
                dws.append(prod.sum((0, 1)).sum(0) if case["norm"] == "head" else prod.sum((0, 1)))
                inner = (prod * w).mean(-1, keepdim=True)
                if case["norm"] == "token":
                    inner = inner.mean(-2, keepdim=True)
                g = inv * g * w - inv.pow(2) * x * inner
            outs.append(g)
        return outs if kind == "rope" else [torch.stack(outs, 2)] + dws
    if kind == "quantize":
        x = st["x"].double().reshape(case["M"], -1)
        return _exact_values(x.t().contiguous() if case["transposed"] else x)
    M, N, K = case["M"], case["N"], case["K"]
    if kind == "linear_bwd":
        dy, x = st["dy"].double(), st["x"].double()
        return [_exact_values(dy) @ _exact_stored(*st["w"], N).t(),
                _exact_values(dy.t().contiguous()) @ _exact_values(x.t().contiguous()).t()]
    a = _exact_values(st["x"].double()) if kind == "linear" else _exact_stored(*st["a"], K)
    c = a @ _exact_stored(*st["w"], K).t()
    return c if st["bias"] is None else c + st["bias"].double()
