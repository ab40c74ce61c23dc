"""Plain 64-bit forms of the operators around the layer (norm + rotary positions, microscaled 4-bit operands), on the CPU."""
import numpy as np
import torch

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -24


# ---------------------------------------------------------------- norm + rotary positions
def pair_index(d, pairing):
    p = np.arange(d // 2)
    return (2 * p, 2 * p + 1) if pairing == "adjacent" else (p, p + d // 2)


def angles(pos, freq, axis_pairs):
    """[.., N, axes] int, [d/2] -> [.., N, d/2]"""
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    return pos[..., axis].astype(np.float64) * freq


def turn(x, a, pairing, sense=1.0):
    """x [B,N,H,d], a [B or 1,N,d/2]"""
    i, j = pair_index(x.shape[-1], pairing)
    c, s = np.cos(a)[..., None, :], sense * np.sin(a)[..., None, :]
    y = np.empty_like(x)
    y[..., i] = x[..., i] * c - x[..., j] * s
    y[..., j] = x[..., i] * s + x[..., j] * c
    return y


def pair_norm(x, pairing):
    """sqrt(x_i^2 + x_j^2) in both places of a pair"""
    i, j = pair_index(x.shape[-1], pairing)
    y = np.empty_like(x)
    y[..., i] = y[..., j] = np.hypot(x[..., i], x[..., j])
    return y


def scope_axes(scope):
    return (-1,) if scope == "head" else (-2, -1)


def sum_steps(H, d):
    """Additions in a row (8 values per lane and step of 512 / d heads), then across 64 lanes, that a sum over a token takes."""
    return 8 * -(-H // (512 // d)) + 6


def rope(x, w, a, scope, eps, pairing):
    """x [B,N,H,d] float64; w or None; a or None -> y, and the bound of a result formed in fp32 (without its last rounding).

    fp32 error: the sum of squares is off by sum_steps * U relative, its root by half of that; mean, root, quotient and the two
    products by one U each; cosine and sine by 2 U each (argument rounded to fp32 below pi / 4: U / 2; polynomial), the rotation by
    2 more of the pair's norm per term.  In all (sum_steps / 2 + 12) U of the pair's norm."""
    steps = 0
    if w is not None:
        steps = sum_steps(*x.shape[-2:])
        x = x / np.sqrt((x * x).mean(scope_axes(scope), keepdims=True) + eps) * w
    bound = (steps / 2 + 12) * U * pair_norm(x, pairing)
    return (x if a is None else turn(x, a, pairing)), bound


def rope_backward(g, x, w, a, scope, eps, pairing):
    """-> dx, bound of dx, dw, bound of dw (without the last roundings).

    dx = r (g w - xn m), xn = x r, m = mean(g w xn): g is off by 6 U of its pair's norm, r by (s/2 + 4) U, m by (s + s/2 + 12) U
    of the mean of magnitudes; products 4 more.  dw: summands off by (s/2 + 12) U, at most 64 additions in a row where the
    test has at most 64 tokens per wavefront times steps, and 8 across wavefronts and lanes."""
    if a is not None:
        gn = pair_norm(g, pairing)
        g = turn(g, a, pairing, -1.0)
    else:
        gn = np.abs(g)
    if w is None:
        return g, 12 * U * gn, None, None
    axes, s = scope_axes(scope), sum_steps(*x.shape[-2:])
    r = 1.0 / np.sqrt((x * x).mean(axes, keepdims=True) + eps)
    xn = x * r
    m = (g * w * xn).mean(axes, keepdims=True)
    m_abs = (gn * np.abs(w * xn)).mean(axes, keepdims=True)
    dx = r * (g * w - xn * m)
    bound = U * r * ((s / 2 + 14) * gn * np.abs(w) + (2 * s + 20) * np.abs(xn) * m_abs)
    over = (0, 1, 2) if scope == "head" else (0, 1)
    dw = (g * xn).sum(over)
    dw_bound = (s / 2 + 12 + 72) * U * (gn * np.abs(xn)).sum(over)
    return dx, bound, dw, dw_bound


# ---------------------------------------------------------------- MXFP4
def quantize(x):
    """float64 [R,K] (fp32 or bf16 numbers) -> codes [R,Kp/2], scales [Kp/128,R,4] uint8"""
    R, K = x.shape
    nk = -(-K // 128)
    full = np.zeros((R, nk * 128))
    full[:, :K] = x
    b = full.reshape(R, nk * 4, 32)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    top = np.abs(b).max(-1)
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -127)
    e = np.clip(e, -127, 125)
    a = np.abs(np.ldexp(b, -e[..., None]))
    # nearest of the E2M1 numbers; a tie goes to the even code
    code = np.zeros(a.shape, dtype=np.int64)
    for k in range(7):
        mid = (E2M1[k] + E2M1[k + 1]) / 2
        code += (a > mid) | ((a == mid) & (k % 2 == 1))
    code = (code + 8 * np.signbit(b)).reshape(R, -1, 2)
    codes = (code[..., 0] + 16 * code[..., 1]).astype(np.uint8)
    scales = np.where(bad, 255, e + 127).astype(np.uint8).reshape(R, nk, 4).transpose(1, 0, 2)
    return codes, np.ascontiguousarray(scales)


def values(codes, scales):
    """-> float64 [R,Kp]"""
    R = codes.shape[0]
    c = np.stack([codes & 15, codes >> 4], -1).reshape(R, -1, 32).astype(np.int64)
    s = scales.transpose(1, 0, 2).reshape(R, -1, 1).astype(np.int64)
    v = np.where(c >= 8, -1.0, 1.0) * E2M1[c % 8]
    v = np.ldexp(v, s - 127)
    return np.where(s == 255, np.nan, v).reshape(R, -1)


def product(a, b, bias=None):
    """a [M,Kp], b [N,Kp] values -> C and the bound of a sum formed in fp32, without its last rounding: Kp / 64 sums of 64 products
    one after another, each step off by at most 2^-23 of the magnitudes (the matrix cores may cut off instead of rounding), the
    products themselves exact, and as much for parts of the sum that are joined."""
    c = a @ b.T
    mags = np.abs(a) @ np.abs(b).T
    steps = a.shape[1] / 64 + 64
    if bias is not None:
        c, mags = c + bias, mags + np.abs(bias)
    return c, steps * 2.0 ** -23 * mags


def assert_within(got, ref, bound, dtype, what=""):
    got = got.double().cpu().numpy()
    tol = bound + HALF_STEP[dtype] * (np.abs(ref) + bound) + 1e-37
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), "%s: %d of %d outside, worst at %.3g of its bound" % (
        what, bad.sum(), bad.size, np.nanmax(np.abs(got - ref) / tol))
