"""Plain 64-bit forms of the layer norm and of E4M3 operands with a scale for each block of 128, on the CPU."""
import numpy as np

from _operators import U

E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127])


# ---------------------------------------------------------------- layer norm
# Additions in a row that a sum over a row takes: 24 values of a thread at most, 6 steps over a wavefront, 16 wavefronts, and two roundings
# more for the quotient by D.
STEPS = 48


def _rows(t):
    """[D] or [B,D] -> something that a [B,N,D] tensor takes"""
    return t if t is None or t.ndim == 1 else t[:, None, :]


def _stats(x, eps):
    """x [B,N,D] float64 -> n, r, and how far n may be off in fp32, relative error of r.

    The mean is off by STEPS U of the mean magnitude A, a deviation d by that and U |d|.  The sum of squares: STEPS U relative for the sum,
    2 U for a square, 2 U for the deviations' own rounding, and the mean's error times 2 / sigma (Cauchy-Schwarz: mean |d| <= sigma); r has half
    of that, and 3 U for mean, root and quotient."""
    mean = x.mean(-1, keepdims=True)
    d = x - mean
    r = 1.0 / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    off_mean = STEPS * U * np.abs(x).mean(-1, keepdims=True)
    off_r = (STEPS + 4) / 2 * U + off_mean * r + 3 * U
    n = d * r
    return n, r, r * off_mean + np.abs(n) * (off_r + 2 * U), off_r


def layer_norm(x, w, b, eps, one_plus):
    """-> y, and the bound of a result formed in fp32 (without its last rounding)"""
    n, r, off, _ = _stats(x, eps)
    w, b = _rows(w), _rows(b)
    s = 1.0 if w is None else w + 1.0 if one_plus else w
    y = n * s + (0.0 if b is None else b)
    return y, off * np.abs(s) + U * (2 * np.abs(n * s) + np.abs(y) + (0.0 if b is None else np.abs(b)))


def layer_norm_backward(dy, x, w, eps, one_plus):
    """-> dx, its bound, and (dw, bound, db, bound) of every group [B,D] (without the last roundings; to be added up where groups share).

    dw and db: a share of the rows is added up one after another, at most 8 and a 128th of all rows of them."""
    n, r, off_n, off_r = _stats(x, eps)
    s = 1.0 if w is None else _rows(w) + 1.0 if one_plus else _rows(w)
    g = dy * s
    mean = lambda t: t.mean(-1, keepdims=True)          # noqa: E731
    mg, mgn = mean(g), mean(g * n)
    dx = r * (g - mg - n * mgn)
    off_mg = (STEPS + 3) * U * mean(np.abs(g))
    off_mgn = (STEPS + 6) * U * mean(np.abs(g * n)) + mean(np.abs(g) * off_n) + np.abs(mgn) * off_r
    bound = r * (2 * U * np.abs(g) + off_mg + np.abs(n) * off_mgn + off_n * np.abs(mgn)
                 + 4 * U * (np.abs(g) + np.abs(mg) + np.abs(n * mgn))) + np.abs(dx) * off_r
    share = 8 + x.shape[0] * x.shape[1] / 128
    dw, dw_bound = (dy * n).sum(1), (np.abs(dy) * off_n + (share + 2) * U * np.abs(dy * n)).sum(1)
    return dx, bound, dw, dw_bound, dy.sum(1), share * U * np.abs(dy).sum(1)


# ---------------------------------------------------------------- E4M3, a power of two for each block of 128
def quantize(x, square=False):
    """float64 [R,K] (fp32 or bf16 numbers) -> codes [R,Kp], scales [ceil(Kp/512),R,4] uint8"""
    R, K = x.shape
    nk, nr = -(-K // 128), -(-R // 128)
    full = np.zeros((nr * 128 if square else R, nk * 128))
    full[:R, :K] = x
    rows = 128 if square else 1
    b = full.reshape(-1, rows, nk, 128)
    bad = ~np.isfinite(b).all((1, 3), keepdims=True)
    b = np.where(bad, 0.0, b)
    top = np.abs(b).max((1, 3), keepdims=True)
    m, e = np.frexp(top)
    e = np.where(top > 0, e - 9 + (m > 0.875), -127)    # 448 = 0.875 * 2^9
    e = np.maximum(e, -127)
    a = np.ldexp(np.abs(b), -e)
    assert a.max() <= 448.0
    mid = (E4M3[1:] + E4M3[:-1]) / 2
    low, high = np.searchsorted(mid, a, "left"), np.searchsorted(mid, a, "right")
    code = np.where((low != high) & (low % 2 == 1), high, low) + 128 * np.signbit(b)
    codes = code.astype(np.uint8).reshape(-1, nk * 128)[:R]
    scales = np.where(bad, 255, e + 127).astype(np.uint8)[:, 0, :, 0].repeat(rows, 0)[:R]
    scales = np.pad(scales, ((0, 0), (0, -nk % 4)))
    return codes, np.ascontiguousarray(scales.reshape(R, -1, 4).transpose(1, 0, 2))


def values(codes, scales):
    """-> float64 [R,Kp]"""
    R, Kp = codes.shape
    s = scales.transpose(1, 0, 2).reshape(R, -1, 1)[:, :Kp // 128].astype(np.int64)
    c = codes.reshape(R, -1, 128).astype(np.int64)
    v = np.where(c >= 128, -1.0, 1.0) * np.append(E4M3, np.nan)[c % 128]
    return np.where(s == 255, np.nan, np.ldexp(v, s - 127)).reshape(R, Kp)


def product(a, b, bias=None, exact=True):
    """a [M,Kp], b [N,Kp] values -> C and the bound of a sum formed in fp32, without its last rounding.

    exact (fp32 results): Kp / 16 sums of 16 products one after another, each off by at most 2^-23 of the magnitudes, the products
    themselves exact, and 64 more for parts of the sum that are joined (as many as there are operations in a wavefront's and a workgroup's).
    Else (bf16 results) the matrix cores' E4M3 sums: of eight neighbouring products, seven may lose less than 2^-13 of the power of two of the largest."""
    c = a @ b.T
    mags = np.abs(a) @ np.abs(b).T
    bound = (a.shape[1] / 16 + 64) * 2.0 ** -23 * mags
    if not exact:
        largest = mags
        if a.shape[0] * b.shape[0] * a.shape[1] <= 1 << 27:      # the sum of the largest of each eight; more than that is too long here
            largest = np.zeros_like(mags)
            for k in range(0, a.shape[1], 8):
                largest += (np.abs(a[:, None, k:k + 8]) * np.abs(b[None, :, k:k + 8])).max(-1)
        bound = bound + 7 * 2.0 ** -13 * largest
    if bias is not None:
        c, bound = c + bias, bound + 2.0 ** -23 * (mags + np.abs(bias))
    return c, bound
