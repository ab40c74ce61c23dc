"""The layer norm's rows one by one: what all lanes of a row decide together, sums at the end of fp32."""
import numpy as np
import pytest
import torch

import _block_operators as ops
from _operators import assert_within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-6
# rows of a sixteenth, a half and a whole wavefront, of one, two and three steps, of workgroups of two and four steps, whole and with an end
LENGTHS = [100, 128, 200, 300, 512, 777, 1024, 1300, 1536, 1999, 2048, 5120, 5119, 8192, 10000, 16384]


@pytest.fixture(scope="module")
def svg2():
    import paper_2505_18875_amd as pkg
    pkg.load_library()
    assert torch.cuda.is_available()
    return pkg


def _np(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", LENGTHS)
def test_every_lane_of_a_row_has_the_same_sums(svg2, D, dtype):
    """Columns of equal values have equal results, bit for bit, within the 512 neighbouring columns of a wavefront (whose values are taken relative to a
    mean of its own): every lane has the same mean, root and, for gradients, means of g and g n."""
    N = 200
    r = np.random.default_rng(D)
    x, dy = (torch.from_numpy(r.standard_normal((N, D))).to(dtype) for _ in range(2))
    same = slice(3, None, 8)
    x[:, same], dy[:, same] = 0.7, -0.4
    x, dy = x.cuda(), dy.cuda()
    y = svg2.svg2_layer_norm(x, eps=EPS, out_dtype=F32)
    dx = svg2.svg2_layer_norm_backward(dy, x, eps=EPS).grad
    for t in (y, dx):
        for k in range(0, D, 512):
            part = t[:, k:k + 512][:, same]
            assert bool((part == part[:, :1]).all()), k


@pytest.mark.parametrize("D", LENGTHS)
def test_squares_that_just_reach_the_largest_number(svg2, D):
    """Rows whose squares add up to the largest fp32 number, a few roundings more or less, so that it depends on the order of the sum whether they have
    to be taken again, every third an ordinary one: all within the bound, and the ordinary ones as in a call of their own."""
    N = 3000
    r = np.random.default_rng(D)
    x = r.standard_normal((N, D))
    x -= x.mean(-1, keepdims=True)
    far = np.arange(N) % 3 != 0
    top = float(np.finfo(np.float32).max) * (1 + r.uniform(-8, 8, (N, 1)) * 2.0 ** -24)
    x[far] *= np.sqrt(top / (x * x).sum(-1, keepdims=True))[far]
    x = torch.from_numpy(x).float().cuda()
    w, b, dy = (torch.from_numpy(r.standard_normal(s)).float().cuda() for s in (D, D, (N, D)))
    y = svg2.svg2_layer_norm(x, w, b, eps=EPS)
    codes, scales = svg2.svg2_layer_norm_fp8(x, w, b, eps=EPS)
    res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=EPS)
    rows = torch.from_numpy(~far).cuda()
    alone = svg2.svg2_layer_norm_fp8(x[rows], w, b, eps=EPS)
    assert torch.equal(svg2.svg2_layer_norm(x[rows], w, b, eps=EPS), y[rows])
    assert torch.equal(alone[0], codes[rows]) and torch.equal(alone[1], scales[:, rows]) and bool((scales < 255).all())
    assert torch.equal(svg2.svg2_layer_norm_backward(dy[rows], x[rows], w, b, eps=EPS).grad, res.grad[rows])
    few = slice(0, 200)
    ref, bound = ops.layer_norm(_np(x[None, few]), _np(w), _np(b), EPS, False)
    assert_within(y[None, few], ref, bound, F32)
    dx, bound = ops.layer_norm_backward(_np(dy[None, few]), _np(x[None, few]), _np(w), EPS, False)[:2]
    assert_within(res.grad[None, few], dx, bound, F32)
    *_, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(dy)[None], _np(x)[None], _np(w), EPS, False)
    assert_within(res.dweight[None], dw, dw_bound, F32)
    assert_within(res.dbias[None], db, db_bound, F32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [1, 5, 64, *LENGTHS])
def test_constant_rows_of_large_numbers(svg2, D, dtype):
    """Finite rows of one number have no variance, also where their sum is past fp32 or off by a rounding that is: as rows of zeros, forward, to FP8
    and in every gradient, the sums over all rows among them."""
    N, large = 120, [1e35, -1e35, 2.0 ** 123, -2.0 ** 123, torch.finfo(dtype).max, torch.finfo(dtype).min, 3e30, -1.1e37]
    r = np.random.default_rng(D)
    x = torch.from_numpy(r.standard_normal((N, D))).to(dtype)
    rows = torch.arange(len(large)) * 13 + 2
    x[rows] = 0.0
    zeros = x.cuda()
    x[rows] = torch.tensor(large, dtype=torch.float64).to(dtype)[:, None]
    x = x.cuda()
    w, b = (torch.from_numpy(r.standard_normal(D)).float().cuda() for _ in range(2))
    dy = torch.from_numpy(r.standard_normal((N, D))).to(dtype).cuda()
    y = svg2.svg2_layer_norm(x, w, b, eps=EPS, out_dtype=F32)
    assert bool((y[rows] == b).all())
    assert torch.equal(y, svg2.svg2_layer_norm(zeros, w, b, eps=EPS, out_dtype=F32))
    for got, want in zip(svg2.svg2_layer_norm_fp8(x, w, b, eps=EPS), svg2.svg2_layer_norm_fp8(zeros, w, b, eps=EPS)):
        assert torch.equal(got, want)
    res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=EPS)
    dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(dy)[None], _np(zeros)[None], _np(w), EPS, False)
    assert_within(res.grad[None], dx, bound, dtype)
    assert_within(res.dweight[None], dw, dw_bound, F32)
    assert_within(res.dbias[None], db, db_bound, F32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, *LENGTHS])
def test_rows_that_are_nearly_constant_or_not_finite(svg2, D, dtype):
    """One number next to the others', first, last or between: finite, and the others of a row alike.  Rows of infinities or NaN: NaN."""
    top = torch.tensor(2.0 ** 123, dtype=dtype)
    near = (top.double() * (1 - torch.finfo(dtype).eps / 2)).to(dtype)
    assert near != top
    x = top.repeat(6, D)
    at = [0, D - 1, D // 2]
    for row, k in enumerate(at):
        x[row, k] = near
    for row, v in enumerate((float("inf"), -float("inf"), float("nan"))):
        x[3 + row] = v
    x = x.cuda()
    dy = torch.from_numpy(np.random.default_rng(D).standard_normal((6, D))).to(dtype).cuda()
    y = svg2.svg2_layer_norm(x, eps=EPS, out_dtype=F32)
    codes, scales = svg2.svg2_layer_norm_fp8(x, eps=EPS)
    dx = svg2.svg2_layer_norm_backward(dy, x, eps=EPS).grad
    nk = -(-D // 128)
    flat = scales.transpose(0, 1).reshape(6, -1)[:, :nk]
    assert bool(y[:3].isfinite().all()) and bool((flat[:3] < 255).all()) and bool(dx[:3].isfinite().all())
    for row, k in enumerate(at):
        assert bool((y[row, k] < y[row, [j for j in range(D) if j != k]]).all())
    assert bool(y[3:].isnan().all()) and bool((flat[3:] == 255).all()) and bool((codes[3:] == 0).all()) and bool(dx[3:].isnan().all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, *LENGTHS])
def test_rows_of_zeros_but_for_large_numbers_at_an_end(svg2, D, dtype):
    """As many large columns as may stand behind the last whole eight, at either end: taken again, but not rows of one number."""
    x = torch.zeros((14, D), dtype=dtype)
    for n in range(1, 8):
        x[n - 1, D - n:], x[6 + n, :n] = 2.0 ** 100, -2.0 ** 100
    x = x.cuda()
    r = np.random.default_rng(D)
    w, b = (torch.from_numpy(r.standard_normal(D)).float().cuda() for _ in range(2))
    dy = torch.from_numpy(r.standard_normal(x.shape)).to(dtype).cuda()
    y, bound = ops.layer_norm(_np(x)[None], _np(w), _np(b), EPS, False)
    assert_within(svg2.svg2_layer_norm(x, w, b, eps=EPS, out_dtype=F32)[None], y, bound, F32)
    res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=EPS)
    dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(dy)[None], _np(x)[None], _np(w), EPS, False)
    assert_within(res.grad[None], dx, bound, dtype)
    assert_within(res.dweight[None], dw, dw_bound, F32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [10000, 16384])
def test_an_eps_that_large_rows_feel(svg2, D, dtype):
    """The largest eps beside rows whose squares are past fp32 by little: some 2^-15 of their variance."""
    N, eps = 12, 9e29
    r = np.random.default_rng(D)
    x = r.standard_normal((N, D))
    x *= np.sqrt(float(np.finfo(np.float32).max) * r.uniform(0.8, 1.6, (N, 1)) / (x * x).sum(-1, keepdims=True))
    x = torch.from_numpy(x).to(dtype).cuda()
    w, b = (torch.from_numpy(r.standard_normal(D)).float().cuda() for _ in range(2))
    dy = torch.from_numpy(r.standard_normal((N, D))).to(dtype).cuda()
    y, bound = ops.layer_norm(_np(x)[None], _np(w), _np(b), eps, False)
    assert_within(svg2.svg2_layer_norm(x, w, b, eps=eps, out_dtype=F32)[None], y, bound, F32)
    res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=eps)
    dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(dy)[None], _np(x)[None], _np(w), eps, False)
    assert_within(res.grad[None], dx, bound, dtype)
    assert_within(res.dweight[None], dw, dw_bound, F32)


@pytest.mark.parametrize("D", [5, 300, 2048, 5119, 10000])
def test_the_smallest_eps(svg2, D):
    """Rows without variance, by the smallest number that fp32 has and the smallest normal one."""
    x = torch.tensor([7.0, 0.0, -3.0, 2.0 ** 123], device="cuda")[:, None].repeat(1, D)
    g = torch.Generator(device="cuda").manual_seed(D)
    w, b, dy = (torch.randn(s, generator=g, device="cuda") for s in (D, D, (4, D)))
    for eps in (2.0 ** -149, 2.0 ** -126):
        assert bool((svg2.svg2_layer_norm(x, w, b, eps=eps) == b).all())
        res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=eps)
        zeros = np.zeros((1, 4, D))
        dx, bound, dw, dw_bound, _, _ = ops.layer_norm_backward(_np(dy)[None], zeros, _np(w), eps, False)
        assert_within(res.grad[None], dx, bound, F32)
        assert_within(res.dweight[None], dw, dw_bound, F32)


@pytest.mark.parametrize("D", [100, 777, 1536, 5120])
def test_a_factor_of_all_rows_with_an_offset_of_each_group(svg2, D):
    """Forward and to FP8, either way round; the gradients of such a pair are refused."""
    from paper_2505_18875_amd.binding import Svg2Error
    B, N = 3, 11
    g = torch.Generator(device="cuda").manual_seed(D)
    x, w, b = (torch.randn(s, generator=g, device="cuda") for s in ((B, N, D), (B, D), (B, D)))
    for ww, bb in ((w[0].clone(), b), (w, b[0].clone())):
        y = svg2.svg2_layer_norm(x, ww, bb, eps=EPS)
        ref, bound = ops.layer_norm(_np(x), _np(ww), _np(bb), EPS, False)
        assert_within(y, ref, bound, F32)
        codes, scales = svg2.svg2_layer_norm_fp8(x, ww, bb, eps=EPS)
        c, s = svg2.svg2_quantize_fp8_blocks(y.view(B * N, D))
        assert torch.equal(codes, c) and torch.equal(scales, s)
        with pytest.raises(Svg2Error, match="both"):
            svg2.svg2_layer_norm_backward(x, x, ww, bb, eps=EPS)
