"""The FP8 product on every path of its plan, bit for bit, the norm's gradients at the edges of theirs, and all of them at the sizes where 32
bits end."""
import numpy as np
import pytest
import torch

import _block_operators as ops
from _operators import assert_within
from test_gpu_fp8_blocks import small_codes

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def svg2():
    import paper_2505_18875_amd as pkg
    pkg.load_library()
    assert torch.cuda.is_available()
    yield pkg
    torch.cuda.empty_cache()


def _values(svg2, codes, scales):
    return svg2.svg2_dequantize_fp8_blocks(codes, scales, dtype=F32).double()


# few rows on either side of that kernel's borders (8 rows, 8192 columns, 5 and 10 times 2^24 weights); small, medium and large tiles, the last rows
# by others, several tiles to a workgroup; parts whose last is shorter
@pytest.mark.parametrize("M,N,nk", [(1, 15360, 40), (3, 100, 64), (4, 20480, 64), (4, 20496, 64), (5, 20480, 32), (8, 20480, 32), (8, 20496, 32), (9, 500, 5),
                                    (8, 4096, 64), (8, 4096, 65), (300, 1100, 17), (700, 1300, 12), (2048, 2048, 16), (1700, 5120, 4), (3400, 5120, 32),
                                    (4200, 4100, 40), (8192, 2048, 6), (1536, 1536, 128), (100, 90, 160), (520, 500, 149)])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_product_of_integers_on_every_path(svg2, M, N, nk, out_dtype):
    """Sums of multiples of 1/4 below 2^2 * 49 * 128 * 160 < 2^22: exact in fp32, in any order; a bf16 result is the exact one, rounded."""
    (a, sa), (b, sb) = small_codes(M, nk, 1), small_codes(N, nk, 2)
    bias = torch.randint(-50, 51, (N,), generator=torch.Generator().manual_seed(3)).float().cuda()
    ref = torch.matmul(_values(svg2, a, sa), _values(svg2, b, sb).t().contiguous())
    for bb in (None, bias):
        got = svg2.svg2_matmul_fp8_blocks(a, sa, b, sb, bias=bb, out_dtype=out_dtype)
        want = (ref if bb is None else ref + bb.double()).float().to(out_dtype)
        assert torch.equal(got, want)
    # rows of a wider result, and nothing behind the last row
    wide = torch.full((M + 2, N + 8), 7.0, dtype=out_dtype, device="cuda")
    svg2.svg2_matmul_fp8_blocks(a, sa, b, sb, bias=bias, out=wide[:M, 4:4 + N])
    assert torch.equal(wide[:M, 4:4 + N], want) and bool((wide[M:] == 7).all()) and bool((wide[:, :4] == 7).all()) and bool((wide[:, 4 + N:] == 7).all())


@pytest.mark.parametrize("M,N,nk", [(70001, 31999, 1), (1048600, 70, 33)])
def test_product_of_far_results_and_far_operands(svg2, M, N, nk):
    """A result of more than 2^31 elements, and an operand of more than 2^32 bytes: the first, middle and last rows against 64 bits."""
    assert M * N > 2 ** 31 or M * nk * 128 > 2 ** 32
    (a, sa), (b, sb) = small_codes(M, nk, 1), small_codes(N, nk, 2)
    got = svg2.svg2_matmul_fp8_blocks(a, sa, b, sb, out_dtype=F32)
    vb = _values(svg2, b, sb).t().contiguous()
    for r0 in (0, M // 2, M - 300):
        va = _values(svg2, a[r0:r0 + 300], sa[:, r0:r0 + 300].clone())
        assert bool((got[r0:r0 + 300] == torch.matmul(va, vb)).all()), r0


@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("H,d", [(40, 128), (1, 5123)])
def test_quantize_more_than_2_31_elements(svg2, H, d, square):
    """From head order, the heads far apart, and of odd rows: the last rows as in a call of their own, and their values."""
    N, last = 420001, 417                   # 420,001 - 417 = 3278 * 128: the blocks of the last rows are the same
    o = torch.randn((H, N, d), generator=torch.Generator(device="cuda").manual_seed(3), dtype=BF16, device="cuda")
    assert o.numel() > 2 ** 31
    x = o.transpose(0, 1) if H > 1 else o[0]
    rows, cols = svg2.svg2_quantize_fp8_blocks(x, transposed="both", square=square)
    r, c = svg2.svg2_quantize_fp8_blocks(x[-last:].contiguous(), transposed="both", square=square)
    assert torch.equal(rows[0][-last:], r[0]) and torch.equal(rows[1][:, -last:], r[1])
    assert torch.equal(cols[0][:, -c[0].shape[1]:], c[0])
    first = (N - last) // 128               # block of the first of them; words of four blocks do not begin where the others' do
    flat = lambda s: s.transpose(0, 1).reshape(s.shape[1], -1)       # noqa: E731
    assert torch.equal(flat(cols[1])[:, first:first + 4], flat(c[1])[:, :4])
    single = svg2.svg2_quantize_fp8_blocks(x, square=square)
    assert torch.equal(single[0], rows[0]) and torch.equal(single[1], rows[1])
    del cols
    values = svg2.svg2_dequantize_fp8_blocks(*rows, H * d)
    assert values.numel() > 2 ** 31 and torch.equal(values[-last:], svg2.svg2_dequantize_fp8_blocks(*r, H * d))


def test_norm_of_more_than_2_31_elements(svg2):
    """420,000 rows of 5120: the last as in a call of their own, the weights' gradients against 64 bits."""
    N, D, eps, last = 420000, 5120, 1e-6, 600
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn((N, D), generator=g, dtype=BF16, device="cuda") for _ in range(2))
    assert x.numel() > 2 ** 31
    w, b = 1 + 0.3 * torch.randn((D,), generator=g, device="cuda"), torch.randn((D,), generator=g, device="cuda")
    y = svg2.svg2_layer_norm(x, w, b, eps=eps)
    assert torch.equal(y[-last:], svg2.svg2_layer_norm(x[-last:], w, b, eps=eps))
    del y
    codes, scales = svg2.svg2_layer_norm_fp8(x, w, b, eps=eps)
    c, s = svg2.svg2_layer_norm_fp8(x[-last:], w, b, eps=eps)
    assert torch.equal(codes[-last:], c) and torch.equal(scales[:, -last:], s)
    del codes
    res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=eps)
    end = svg2.svg2_layer_norm_backward(dy[-last:], x[-last:], w, b, eps=eps)
    assert torch.equal(res.grad[-last:], end.grad)
    dw, db, mags, mags_b = (torch.zeros((D,), dtype=torch.float64, device="cuda") for _ in range(4))
    for n in range(0, N, 10000):
        xs, gs = x[n:n + 10000].double(), dy[n:n + 10000].double()
        var, mean = torch.var_mean(xs, -1, correction=0, keepdim=True)
        xn = (xs - mean) * (var + eps).rsqrt()
        dw += (gs * xn).sum(0)
        db += gs.sum(0)
        mags += (gs * xn).abs().sum(0)
        mags_b += gs.abs().sum(0)
    # a share is added up one row after another (ops.layer_norm_backward); a row's own error of xn is at most STEPS U (A r + |xn|), A r < 1 and some
    # values of xn below 1, so it is counted against the mean magnitudes, of which |dy| is one
    share = 8 + N / 128
    assert_within(res.dweight, dw.cpu().numpy(), (ops.U * ((share + ops.STEPS) * mags + 2 * ops.STEPS * mags_b)).cpu().numpy(), F32)
    assert_within(res.dbias, db.cpu().numpy(), (share * ops.U * mags_b).cpu().numpy(), F32)


@pytest.mark.parametrize("D", [5, 24])
def test_norm_of_as_many_rows_as_it_takes(svg2, D):
    """2^26 rows, four different ones over and over, in place: each comes out as in a call of four, and the rows behind the last stay."""
    N, behind = 2 ** 26, 8
    g = torch.Generator().manual_seed(1)
    four = torch.randn((4, D), generator=g).to(BF16).cuda()
    w, b = torch.randn((D,), generator=g).cuda(), torch.randn((D,), generator=g).cuda()
    ref = svg2.svg2_layer_norm(four, w, b)
    x = four.repeat((N + behind) // 4, 1)
    codes, scales = svg2.svg2_layer_norm_fp8(x[:N], w, b)
    c, s = svg2.svg2_layer_norm_fp8(four, w, b)
    for r0 in range(0, N, 2 ** 24):
        assert bool((codes[r0:r0 + 2 ** 24].view(-1, 4, 128) == c).all()) and bool((scales[0, r0:r0 + 2 ** 24].view(-1, 4, 4) == s[0]).all())
    del codes
    svg2.svg2_layer_norm(x[:N], w, b, out=x[:N])
    for r0 in range(0, N, 2 ** 24):
        assert bool((x[r0:r0 + 2 ** 24].view(-1, 4, D) == ref).all())
    assert torch.equal(x[N:], four.repeat(2, 1))
    # four different gradients likewise, of powers of two: every sum of theirs is exact
    dy = (2.0 ** torch.arange(4, device="cuda"))[:, None].expand(4, D).to(BF16).repeat(N // 4, 1)
    res = svg2.svg2_layer_norm_backward(dy, x[:N], w, b, out=dy)
    end = svg2.svg2_layer_norm_backward((2.0 ** torch.arange(4, device="cuda"))[:, None].expand(4, D).to(BF16).contiguous(), ref, w, b)
    for r0 in range(0, N, 2 ** 24):
        assert bool((dy[r0:r0 + 2 ** 24].view(-1, 4, D) == end.grad).all())
    assert bool((res.dbias == 15.0 * (N // 4)).all())


@pytest.mark.parametrize("B", [1, 70000])
def test_a_group_for_every_row(svg2, B):
    """Modulations of each row, more of them than a grid dimension has."""
    D, eps = 48, 1e-6
    g = torch.Generator(device="cuda").manual_seed(B)
    x, dy = (torch.randn((B, 1, D), generator=g, device="cuda") for _ in range(2))
    table = torch.randn((B, 6, D), generator=g, device="cuda")
    w, b = table[:, 1], table[:, 0]
    up = lambda t: t.double().cpu().numpy()     # noqa: E731
    y, bound = ops.layer_norm(up(x), up(w), up(b), eps, True)
    assert_within(svg2.svg2_layer_norm(x, w, b, eps=eps, one_plus=True), y, bound, F32)
    res = svg2.svg2_layer_norm_backward(dy, x, w, b, eps=eps, one_plus=True)
    dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(up(dy), up(x), up(w), eps, True)
    assert_within(res.grad, dx, bound, F32)
    assert_within(res.dweight, dw, dw_bound, F32)
    assert np.array_equal(up(res.dbias), db)


@pytest.mark.parametrize("M,K", [(1031, 1543), (129, 2047), (5000, 130), (1, 1025)])
@pytest.mark.parametrize("square", [False, True])
def test_tiles_of_rows_that_share_lines(svg2, M, K, square):
    """Rows that are not whole lines of memory have their tiles in another order: the same operands, both ways, as from rows that are."""
    x = torch.randn((M, K), generator=torch.Generator(device="cuda").manual_seed(M + K), device="cuda").bfloat16()
    lines = torch.zeros((M, -(-K // 64) * 64), dtype=x.dtype, device="cuda")[:, :K]
    lines.copy_(x)
    assert lines.stride(0) * 2 % 128 == 0 and x.stride(0) * 2 % 128 != 0
    for transposed in (True, "both"):
        got, want = (svg2.svg2_quantize_fp8_blocks(t, transposed=transposed, square=square) for t in (x, lines))
        for g, w in zip(got, want):
            for a, b in zip(g, w) if transposed == "both" else ((g, w),):
                assert torch.equal(a, b)
