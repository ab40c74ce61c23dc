"""The layer norm, its result as an FP8 operand and its gradients, against 64 bits."""
import numpy as np
import pytest
import torch

import _block_operators as ops
from _operators import HALF_STEP, assert_within

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
EPS = 1e-6


@pytest.fixture(scope="module")
def svg2():
    import paper_2505_18875_amd as pkg
    pkg.load_library()
    assert torch.cuda.is_available()
    return pkg


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _inputs(B, N, D, dtype, weights, seed=0):
    """Rows with means and sizes of their own; weights around 1, or a small modulation of each group."""
    r = np.random.default_rng(seed + B * N + D)
    x = r.standard_normal((B, N, D)) * 2.0 ** r.integers(-4, 5, size=(B, N, 1)) + r.standard_normal((B, N, 1))
    x = torch.from_numpy(x).to(dtype).cuda()
    shape = {"none": None, "shared": (D,), "group": (B, D)}[weights]
    if shape is None:
        return x, None, None
    w, b = (torch.from_numpy(0.3 * r.standard_normal(shape)).float().cuda() for _ in range(2))
    return x, (w if weights == "group" else 1 + w), b


# lengths of one piece of a thread, of a wavefront, of each kind of workgroup, one on each side of the borders
LENGTHS = [1, 2, 7, 8, 9, 100, 127, 128, 129, 255, 256, 257, 500, 512, 513, 777, 1024, 1025, 1280, 1301, 1535, 1536, 1537, 2048, 2049, 4096, 4100, 5120, 6144, 6145, 8192, 8200, 12289,
           16384]


@pytest.mark.parametrize("x_dtype,y_dtype", [(BF16, BF16), (F32, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("D", LENGTHS)
def test_layer_norm_matches_64_bits(svg2, D, x_dtype, y_dtype):
    for B, N, weights in ((1, 1, "shared"), (2, 3, "group"), (3, 21, "none")):
        x, w, b = _inputs(B, N, D, x_dtype, weights)
        y = svg2.svg2_layer_norm(x, w, b, eps=EPS, one_plus=weights == "group", out_dtype=y_dtype)
        ref, bound = ops.layer_norm(_np(x), _np(w), _np(b), EPS, weights == "group")
        assert y.shape == x.shape and y.dtype == y_dtype
        assert_within(y, ref, bound, y_dtype, "%s %s" % (weights, (B, N)))


@pytest.mark.parametrize("x_dtype,y_dtype", [(BF16, BF16), (F32, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("D", LENGTHS)
def test_gradients_match_64_bits(svg2, D, x_dtype, y_dtype):
    for B, N, weights in ((1, 1, "shared"), (2, 3, "group"), (3, 21, "none"), (3, 50, "group"), (2, 37, "shared")):
        x, w, b = _inputs(B, N, D, x_dtype, weights)
        dy = torch.from_numpy(np.random.default_rng(D).standard_normal((B, N, D))).to(y_dtype).cuda()
        one = weights == "group"
        res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=EPS, one_plus=one)
        dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(dy), _np(x), _np(w), EPS, one)
        assert_within(res.grad, dx, bound, x_dtype, "dx %s" % weights)
        if weights == "none":
            assert res.dweight is None and res.dbias is None
            continue
        if weights == "shared":
            dw, dw_bound, db, db_bound = (t.sum(0) for t in (dw, dw_bound, db, db_bound))
        assert_within(res.dweight, dw, dw_bound, F32, "dw %s" % weights)
        assert_within(res.dbias, db, db_bound, F32, "db %s" % weights)


@pytest.mark.parametrize("D", [5, 777, 2049])
def test_weight_without_bias_and_bias_without_weight(svg2, D):
    x, w, b = _inputs(2, 9, D, F32, "group")
    dy = torch.randn(x.shape, generator=torch.Generator().manual_seed(D)).cuda()
    for ww, bb in ((w, None), (None, b), (w[0].clone(), None), (None, b[1].clone())):
        y = svg2.svg2_layer_norm(x, ww, bb, eps=EPS)
        ref, bound = ops.layer_norm(_np(x), _np(ww), _np(bb), EPS, False)
        assert_within(y, ref, bound, F32)
        res = svg2.svg2_layer_norm_backward(dy, x, ww, bb, eps=EPS)
        dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(dy), _np(x), _np(ww), EPS, False)
        assert_within(res.grad, dx, bound, F32)
        assert (res.dweight is None) == (ww is None) and (res.dbias is None) == (bb is None)
        for got, t, g, gb in ((res.dweight, ww, dw, dw_bound), (res.dbias, bb, db, db_bound)):
            if t is not None:
                assert_within(got, g if t.dim() == 2 else g.sum(0), gb if t.dim() == 2 else gb.sum(0), F32)


def test_gradients_against_differences_of_the_kernel(svg2):
    """The forward kernel's own differences, in fp32: with steps h of 2^-7 and outputs of size 1, off by 2^-24 / h from rounding and h^2 from
    the step, some 2^-13 for a sum of 66 products of size 1; 2^-8 is asked for."""
    B, N, D, h = 2, 3, 11, 2.0 ** -7
    x, w, b = _inputs(B, N, D, F32, "group")
    x = x / x.std(-1, keepdim=True)
    dy = torch.randn(x.shape, generator=torch.Generator().manual_seed(1)).cuda()
    res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=EPS, one_plus=True)
    for k, grad in enumerate((res.grad, res.dweight, res.dbias)):
        for i in np.ndindex(*grad.shape):
            loss = []
            for sign in (1.0, -1.0):
                args = [t.clone() for t in (x, w, b)]
                args[k][i] += sign * h
                loss.append((svg2.svg2_layer_norm(*args, eps=EPS, one_plus=True).double() * dy.double()).sum().item())
            assert abs((loss[0] - loss[1]) / (2 * h) - grad[i].item()) < 2.0 ** -8 * max(1.0, abs(grad[i].item())), (k, i)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [100, 777, 2560])
def test_views_of_any_strides(svg2, D, dtype):
    """Rows that are slices of a wider tensor at odd addresses, groups in reverse order, gradients into a slice, in place; what is beside the
    slices stays."""
    B, N = 3, 10
    x, w, b = _inputs(B, N, D, dtype, "group")
    table = torch.zeros((B, 6, D + 3), device="cuda")
    table[:, 1, 1:D + 1], table[:, 4, 3:] = w, b
    w_view, b_view = table[:, 1, 1:D + 1], table[:, 4, 3:]
    ref = svg2.svg2_layer_norm(x, w, b, eps=EPS, one_plus=True)
    wide = torch.full((N, B, D + 5), 3.0, dtype=dtype, device="cuda")
    view = wide[:, :, 3:3 + D].transpose(0, 1)
    view.copy_(x)
    assert torch.equal(svg2.svg2_layer_norm(view, w_view, b_view, eps=EPS, one_plus=True), ref)
    out = torch.full_like(wide, 5.0)
    o_view = out[:, :, 1:1 + D].transpose(0, 1)
    svg2.svg2_layer_norm(view, w_view, b_view, eps=EPS, one_plus=True, out=o_view)
    assert torch.equal(o_view, ref) and bool((out[:, :, 0] == 5).all()) and bool((out[:, :, 1 + D:] == 5).all())

    dy = torch.from_numpy(np.random.default_rng(D).standard_normal((B, N, D))).to(dtype).cuda()
    want = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=EPS, one_plus=True)
    out.fill_(5.0)
    got = svg2.svg2_layer_norm_backward(dy, view, w_view, b_view, eps=EPS, one_plus=True, out=o_view)
    assert torch.equal(o_view, want.grad) and torch.equal(got.dweight, want.dweight) and torch.equal(got.dbias, want.dbias)
    assert bool((out[:, :, 0] == 5).all()) and bool((out[:, :, 1 + D:] == 5).all())
    one = dy[:1, :1].expand(B, N, D)                             # a broadcast gradient: strides of 0
    got = svg2.svg2_layer_norm_backward(one, x, w, b, eps=EPS, one_plus=True)
    want = svg2.svg2_layer_norm_backward(one.contiguous(), x, w, b, eps=EPS, one_plus=True)
    assert torch.equal(got.grad, want.grad) and torch.equal(got.dweight, want.dweight)
    # in place: the result over x, the gradient over dy
    svg2.svg2_layer_norm(view, w, b, eps=EPS, one_plus=True, out=view)
    assert torch.equal(view, ref) and bool((wide[:, :, :3] == 3).all()) and bool((wide[:, :, 3 + D:] == 3).all())
    d = one.contiguous()
    svg2.svg2_layer_norm_backward(d, x, w, b, eps=EPS, one_plus=True, out=d)
    assert torch.equal(d, want.grad)


def test_rows_that_are_special(svg2):
    """Constant rows (no variance), zeros, an infinity or a NaN, which stays in its row, numbers near the ends of fp32."""
    D = 600
    x = torch.randn((8, D), generator=torch.Generator().manual_seed(3))
    x[1], x[2] = 7.0, 0.0
    x[3, 5], x[4, 9] = float("inf"), float("nan")
    x[5] *= 2.0 ** 60
    x[6] *= 2.0 ** -80
    w, b = 1 + torch.arange(D) / D, torch.arange(D) / 7.0
    y = _np(svg2.svg2_layer_norm(x.cuda(), w.cuda(), b.cuda(), eps=EPS))
    assert np.array_equal(y[1], _np(b)) and np.array_equal(y[2], _np(b))
    assert np.isnan(y[3]).all() and np.isnan(y[4]).all()
    fine = [0, 1, 2, 5, 6, 7]
    ref, bound = ops.layer_norm(_np(x)[None, fine], _np(w), _np(b), EPS, False)
    assert_within(torch.from_numpy(y[fine])[None], ref, bound, F32)
    codes, scales = svg2.svg2_layer_norm_fp8(x.cuda(), w.cuda(), b.cuda(), eps=EPS)
    assert bool((codes[3:5] == 0).all()) and bool((scales[0, 3:5] == 255).all()) and bool((scales[1, 3:5, 0] == 255).all())
    assert bool((scales[1, :, 1:] == 0).all()) and bool((scales[:, fine] < 255).all())
    res = svg2.svg2_layer_norm_backward(torch.ones_like(x).cuda(), x.cuda(), w.cuda(), eps=EPS)
    dx = _np(res.grad)
    assert np.isnan(dx[3:5]).all() and np.isfinite(dx[fine]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [1, 100, 128, 129, 256, 300, 512, 777, 1024, 1280, 1500, 1536, 2048, 2500, 4096, 5120, 6000, 7000, 8192, 10000, 16384])
def test_fp8_result(svg2, D, dtype):
    """A value that the norm leaves within its fp32 bound of y is one of the E4M3 numbers next to it times the scale, or their neighbour where
    the bound reaches over a border: the operand is that of some value within the bound.  The scale is that of the block's largest
    magnitude, which the bound may put on the other side of 448 times a power of two."""
    B, N = 2, 19
    x, w, b = _inputs(B, N, D, dtype, "group")
    codes, scales = svg2.svg2_layer_norm_fp8(x, w, b, eps=EPS, one_plus=True)
    ref, bound = ops.layer_norm(_np(x), _np(w), _np(b), EPS, True)
    ref, bound = ref.reshape(B * N, D), bound.reshape(B * N, D)
    nk = -(-D // 128)
    assert codes.shape == (B * N, nk * 128) and scales.shape == (-(-nk // 4), B * N, 4)
    assert bool((codes[:, D:] == 0).all())
    flat = scales.transpose(0, 1).reshape(B * N, -1)
    assert bool((flat[:, nk:] == 0).all())
    pad = np.zeros((B * N, nk * 128 - D))
    mag = np.concatenate([np.abs(ref), pad], 1).reshape(B * N, nk, 128)
    off = np.concatenate([bound, pad], 1).reshape(B * N, nk, 128)
    up = lambda t: np.maximum(np.ceil(np.log2(np.maximum(t, 1e-300) / 448)), -127) + 127      # noqa: E731
    got = _np(flat)[:, :nk]
    assert (got >= up((mag - off).max(2))).all() and (got <= up((mag + off).max(2))).all()
    v = ops.values(codes.cpu().numpy(), scales.cpu().numpy())[:, :D]
    scale = 2.0 ** (got.repeat(128, 1)[:, :D] - 127)
    step = np.maximum(2.0 ** -4 * (np.abs(ref) + bound), 2.0 ** -10 * scale)                # half a step of E4M3
    assert (np.abs(v - ref) <= bound + step).all()
    again = svg2.svg2_layer_norm_fp8(x, w, b, eps=EPS, one_plus=True)
    assert torch.equal(again[0], codes) and torch.equal(again[1], scales)
    if dtype is F32:                                            # the same as quantising the fp32 result
        q = svg2.svg2_quantize_fp8_blocks(svg2.svg2_layer_norm(x, w, b, eps=EPS, one_plus=True).view(B * N, D))
        assert torch.equal(q[0], codes) and torch.equal(q[1], scales)


@pytest.mark.parametrize("B,N,D,weights", [(1, 5000, 640, "shared"), (1, 9000, 64, "shared"), (700, 3, 200, "group"), (3, 2000, 1000, "group"),
                                           (40, 100, 128, "shared"), (1500, 1, 300, "group")])
def test_sums_over_many_rows_and_groups(svg2, B, N, D, weights):
    x, w, b = _inputs(B, N, D, BF16, weights)
    dy = torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").to(BF16)
    res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=EPS, one_plus=True)
    dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(dy), _np(x), _np(w), EPS, True)
    if weights == "shared":
        dw, dw_bound, db, db_bound = (t.sum(0) for t in (dw, dw_bound, db, db_bound))
    assert_within(res.grad, dx, bound, BF16)
    assert_within(res.dweight, dw, dw_bound, F32)
    assert_within(res.dbias, db, db_bound, F32)
    again = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=EPS, one_plus=True)
    assert torch.equal(again.grad, res.grad) and torch.equal(again.dweight, res.dweight) and torch.equal(again.dbias, res.dbias)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [1300, 1536, 2048, 5120])
def test_rows_taken_again_among_others(svg2, D, dtype):
    """Rows whose squares leave fp32's range between ordinary ones that the same threads take, many to a place: each as if it were alone."""
    N = 9000
    x = torch.randn((N, D), generator=torch.Generator(device="cuda").manual_seed(D), device="cuda")
    x[::7] *= 2.0 ** 62
    x[::11] *= 2.0 ** -70
    x[5::1000, 3] = float("inf")
    x = x.to(dtype)
    w, b = (torch.randn(D, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda") for k in (1, 2))
    dy = torch.randn((N, D), generator=torch.Generator(device="cuda").manual_seed(7), device="cuda").to(dtype)
    rows = torch.tensor([0, 1, 5, 7, 11, 77, 1005, 4998, 8998, 8999], device="cuda")
    few = x[rows].contiguous()
    y, alone = svg2.svg2_layer_norm(x, w, b), svg2.svg2_layer_norm(few, w, b)
    assert torch.equal(y[rows].nan_to_num(7.0), alone.nan_to_num(7.0)) and bool(y[5].isnan().all()) and bool(y[4].isfinite().all())
    codes, scales = svg2.svg2_layer_norm_fp8(x, w, b)
    c, s = svg2.svg2_layer_norm_fp8(few, w, b)
    assert torch.equal(codes[rows], c) and torch.equal(scales[:, rows], s)
    dx = svg2.svg2_layer_norm_backward(dy, x, w, b).grad
    alone = svg2.svg2_layer_norm_backward(dy[rows].contiguous(), few, w, b).grad
    assert torch.equal(dx[rows].nan_to_num(7.0), alone.nan_to_num(7.0)) and bool(dx[5].isnan().all()) and bool(dx[4].isfinite().all())
    ref, bound = ops.layer_norm(_np(few[[0, 1, 3, 4, 5, 8]])[None], _np(w), _np(b), EPS, False)
    assert_within(svg2.svg2_layer_norm(few[[0, 1, 3, 4, 5, 8]].contiguous(), w, b)[None], ref, bound, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [5, 9, 127, 255, 510, 1021, 1301, 2047, 5119, 9001])
def test_in_place_with_rows_taken_again(svg2, D, dtype):
    """The end of a row is loaded with columns of the thread in front, and a row that is taken again is read twice: neither may see results that are
    written over x, or over dy."""
    x = torch.randn((700, D), generator=torch.Generator(device="cuda").manual_seed(D), device="cuda")
    x[::3] *= 2.0 ** 62
    x = x.to(dtype)
    w, b, dy = (torch.randn(s, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda") for k, s in ((1, D), (2, D), (3, (700, D))))
    dy = dy.to(dtype)
    want = svg2.svg2_layer_norm_backward(dy, x, w, b)
    again = dy.clone()
    got = svg2.svg2_layer_norm_backward(again, x, w, b, out=again)
    assert torch.equal(again, want.grad) and torch.equal(got.dweight, want.dweight) and torch.equal(got.dbias, want.dbias)
    y = svg2.svg2_layer_norm(x, w, b)
    assert bool(y.isfinite().all())
    svg2.svg2_layer_norm(x, w, b, out=x)
    assert torch.equal(x, y)


def test_a_row_does_not_depend_on_the_others(svg2):
    x, w, b = _inputs(1, 300, 1000, BF16, "shared")
    y = svg2.svg2_layer_norm(x[0], w, b)
    assert torch.equal(svg2.svg2_layer_norm(x[0, 77:78], w, b), y[77:78])
    assert HALF_STEP[BF16] == 2.0 ** -8


def test_refusals_of_the_binding(svg2):
    x = torch.zeros((2, 3, 64), device="cuda")
    w = torch.ones((64,), device="cuda")
    for bad, error in ((dict(weight=w[:32]), ValueError), (dict(weight=w.bfloat16()), TypeError), (dict(weight=w.cpu()), ValueError),
                       (dict(bias=torch.zeros((3, 64), device="cuda")), ValueError), (dict(weight=torch.ones((128,), device="cuda")[::2]), ValueError),
                       (dict(out=x[0]), ValueError), (dict(out=x.half()), TypeError)):
        with pytest.raises(error):
            svg2.svg2_layer_norm(x, **bad)
    with pytest.raises(ValueError):
        svg2.svg2_layer_norm(x[0, 0])
    with pytest.raises(ValueError):
        svg2.svg2_layer_norm(x.transpose(1, 2))
    with pytest.raises(ValueError):
        svg2.svg2_layer_norm_backward(x, x, w.expand(2, 64))
    with pytest.raises(ValueError):
        svg2.svg2_layer_norm_backward(x[:1], x)
    from paper_2505_18875_amd.binding import Svg2Error
    for call in (lambda: svg2.svg2_layer_norm(x[:, :0]), lambda: svg2.svg2_layer_norm(torch.zeros((1, 16385), device="cuda")),
                 lambda: svg2.svg2_layer_norm(x, eps=0.0), lambda: svg2.svg2_layer_norm_backward(x, x, w, torch.zeros((2, 64), device="cuda"))):
        with pytest.raises(Svg2Error):
            call()
