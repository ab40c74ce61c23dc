"""Block scales at their ends in products of either result type, and quantisation past the caches."""
import numpy as np
import pytest
import torch

import _block_operators as ops

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def svg2():
    import paper_2505_18875_amd as pkg
    pkg.load_library()
    assert torch.cuda.is_available()
    yield pkg
    torch.cuda.empty_cache()


def _operand(R, K, seed):
    r = np.random.default_rng(seed)
    x = r.standard_normal((R, K)) * 2.0 ** r.integers(-6, 7, size=(R, 1))
    return ops.quantize(x.astype(np.float32).astype(np.float64))


# few rows, small, medium and large tiles, and parts of a contraction that are joined
SIZES = [(5, 70, 640), (200, 300, 640), (2048, 2048, 640), (4100, 4200, 384), (130, 140, 16384)]


def _chosen(M, N, K):
    from paper_2505_18875_amd import binding
    return binding._fp8_blocks_workspace_size(M, N, K)


def _run(svg2, a, b, out_dtype):
    up = lambda t: torch.from_numpy(t).cuda()           # noqa: E731
    return svg2.svg2_matmul_fp8_blocks(*map(up, a), *map(up, b), out_dtype=out_dtype).double().cpu().numpy()


def _check(got, va, vb, out_dtype, nan):
    """Against 64 bits.  An fp32 result is formed from the values as bf16: one below 2^-126 is off by at most itself, which its factors multiply; a sum
    below that may be lost at each of K / 64 steps, less than the other side's magnitudes add up to.  A sum that may leave fp32 on its way, where the
    magnitudes do, is not compared (two infinite parts of it may be NaN together); a bf16 result is rounded from fp32, to infinity above 2^128 (1 - 2^-9)."""
    with np.errstate(invalid="ignore"):
        va, vb = np.where(np.isnan(va), 0.0, va), np.where(np.isnan(vb), 0.0, vb)
    ref, bound = ops.product(va, vb, None, out_dtype is F32)
    bound += 2.0 ** -126 * (np.abs(va).sum(1)[:, None] + np.abs(vb).sum(1)[None, :]) + 2.0 ** -149
    far = np.abs(va) @ np.abs(vb).T > np.finfo(np.float32).max * (1 - 2.0 ** -8)
    assert np.array_equal(np.isnan(got)[~far | nan], nan[~far | nan])
    fine = ~nan & ~far
    assert fine.sum() >= 0.5 * fine.size
    with np.errstate(invalid="ignore"):
        off = np.abs(got - ref)
    # half a step of the result, at least that of the smallest normal numbers
    assert (off[fine] <= (bound + HALF_STEP[out_dtype] * np.maximum(np.abs(ref) + bound, 2.0 ** -126))[fine]).all()


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_nan_blocks_beside_others_of_their_word(svg2, M, N, K, out_dtype):
    """A block of scale 255 makes its row of C, or column, NaN, in each of the four places of a word of scales, and nothing else."""
    nk = K // 128
    (ac, sa), (bc, sb) = _operand(M, K, 5), _operand(N, K, 6)
    nan = np.zeros((M, N), dtype=bool)
    for block in range(min(nk, 5)):
        col = (7 * block + 3) % N
        sb[block // 4, col, block % 4] = 255
        nan[:, col] = True
        if M > 5 or block == 1:
            sa[block // 4, block, block % 4] = 255
            nan[block] = True
    _check(_run(svg2, (ac, sa), (bc, sb), out_dtype), ops.values(ac, sa), ops.values(bc, sb), out_dtype, nan)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_far_scales(svg2, M, N, K, out_dtype):
    """Rows whose scales are 2^-126 and 2^110, one block apart from its word's others by as much, and single NaN codes."""
    (ac, sa), (bc, sb) = _operand(M, K, 5), _operand(N, K, 6)
    sa[:, 2] = 1
    sb[:, 7] = 237
    sa[0, 3, 1], sb[0, 9, 2] = 3, 1
    ac[4, 5], bc[11, 200] = 127, 255                    # E4M3's NaN
    nan = np.zeros((M, N), dtype=bool)
    nan[4], nan[:, 11] = True, True
    with np.errstate(invalid="ignore"):
        _check(_run(svg2, (ac, sa), (bc, sb), out_dtype), ops.values(ac, sa), ops.values(bc, sb), out_dtype, nan)


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_blocks_of_zeros(svg2, M, N, K, out_dtype):
    """Scale byte 0, which blocks of zeros get: whole rows, single blocks of either side, opposite blocks of large scale, and both sides at once."""
    r = np.random.default_rng(M)
    xa, xb = (r.standard_normal((R, K)).astype(np.float32).astype(np.float64) for R in (M, N))
    xb[:, 256:384] *= 2.0 ** 100                        # opposite A's zeros and numbers
    xa[1] = 0.0                                         # a row of zeros
    xa[2:5, 256:384] = 0.0
    xb[5, :128], xa[2, :128] = 0.0, 0.0
    xb[6] = 0.0
    a, b = ops.quantize(xa), ops.quantize(xb)
    assert (a[1][:, 1] == 0).all() and (b[1][:, 6] == 0).all() and a[1][0, 2, 2] == 0
    got = _run(svg2, a, b, out_dtype)
    assert (got[1] == 0).all() and (got[:, 6] == 0).all()
    _check(got, ops.values(*a), ops.values(*b), out_dtype, np.zeros((M, N), dtype=bool))


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("M,N", [(5, 70), (200, 300)])
def test_one_large_channel_among_small_ones(svg2, M, N, out_dtype):
    """Where eight neighbouring products differ by 2^12 and cancel, a bf16 result's error is relative to the largest of them, not to the result: within
    the documented 7 * 2^-13 of the sum over eights of the largest product, and fp32 results exact to their own rounding."""
    K = 512
    r = np.random.default_rng(N)
    xa, xb = r.standard_normal((M, K)), r.standard_normal((N, K))
    xa[:, ::16] *= 300.0
    xa[:, 1::16] = -xa[:, ::16]
    xb[:, 1::16] = xb[:, ::16]                          # large products that cancel
    a, b = (ops.quantize(x.astype(np.float32).astype(np.float64)) for x in (xa, xb))
    _check(_run(svg2, a, b, out_dtype), ops.values(*a), ops.values(*b), out_dtype, np.zeros((M, N), dtype=bool))


def test_the_sizes_take_different_ways(svg2):
    assert _chosen(5, 70, 640) == 256 and _chosen(200, 300, 640) == 256 and _chosen(130, 140, 16384) > 256


# X of whole lines, bf16 and fp32, on either side of the sizes from which it is read (64 to 256 MB) and its values are written (128 or 256 MB) past the caches
@pytest.mark.parametrize("dtype,M,K", [(BF16, 4095, 8192), (BF16, 4096, 8192), (BF16, 8191, 8192), (BF16, 8192, 8192), (BF16, 16380, 8128), (F32, 2047, 8192), (F32, 2048, 8192),
                                       (F32, 8191, 8160), (F32, 8192, 8192)])
@pytest.mark.parametrize("square", [False, True])
def test_quantize_past_the_caches(svg2, dtype, M, K, square):
    """The same operands as from rows that are not whole lines of memory, which stay in the caches; and the values back."""
    x = torch.randn((M, K), generator=torch.Generator(device="cuda").manual_seed(M), device="cuda")
    x = (x * torch.exp2(torch.randint(-8, 9, (M, 1), generator=torch.Generator(device="cuda").manual_seed(K), device="cuda").float())).to(dtype)
    es = x.element_size()
    apart = torch.empty((M, K + 5), dtype=dtype, device="cuda")[:, 3:3 + K]
    apart.copy_(x)
    assert x.stride(0) * es % 128 == 0 and x.data_ptr() % 128 == 0 and apart.stride(0) * es % 128 != 0
    for transposed in (False, True, "both"):
        got, want = (svg2.svg2_quantize_fp8_blocks(t, transposed=transposed, square=square) for t in (x, apart))
        pairs = [(got, want)] if transposed != "both" else list(zip(got, want))
        for g, w in pairs:
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])
        if transposed == "both":
            (rows, cols), n = got, 300                  # the last rows' values, and the whole result into lines and past them
            values = svg2.svg2_dequantize_fp8_blocks(*rows, K, dtype=dtype)
            into = torch.empty((M, K + 5), dtype=dtype, device="cuda")[:, 3:3 + K]
            assert torch.equal(svg2.svg2_dequantize_fp8_blocks(*rows, K, out=into), values)
            if not square:
                codes, scales = ops.quantize(x[-n:].double().cpu().numpy())
                assert np.array_equal(rows[0][-n:].cpu().numpy(), codes) and np.array_equal(rows[1][:, -n:].cpu().numpy(), scales)
                assert np.array_equal(values[-n:].double().cpu().numpy(), ops.values(codes, scales)[:, :K])
