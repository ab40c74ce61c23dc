"""MXFP4 operands and their product: codes and scales bit for bit against the definition, products against 64 bits."""
import numpy as np
import pytest
import torch

import _operators as ops
from _operators import assert_within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def svg2():
    import paper_2505_18875_amd as pkg
    pkg.load_library()
    assert torch.cuda.is_available()
    return pkg


def _np(t):
    return t.double().cpu().numpy()


def _spread(shape, seed, dtype):
    """Noise over many binary orders, with zeros, halves of steps and whole blocks of zeros."""
    r = np.random.default_rng(seed)
    x = r.standard_normal(shape) * 2.0 ** r.integers(-6, 7, size=shape[:-1] + (1,))
    x[r.random(shape) < 0.05] = 0.0
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0])
    pick = r.random(shape) < 0.2
    x[pick] = (r.choice(ties, size=shape) * r.choice([-1.0, 1.0], size=shape))[pick]
    x.reshape(-1)[: min(64, x.size // 3)] = 0.0
    return torch.from_numpy(x).to(dtype).cuda()


def _check(codes, scales, x64):
    c, s = ops.quantize(x64)
    assert codes.shape == c.shape and scales.shape == s.shape
    assert np.array_equal(scales.cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), c)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 32), (3, 127), (17, 128), (16, 129), (31, 1000), (130, 640), (65, 37), (515, 264)])
def test_quantize_matches_the_definition_bit_for_bit(svg2, M, K, dtype):
    x = _spread((M, K), 10 * M + K, dtype)
    _check(*svg2.svg2_quantize_mxfp4(x), _np(x))
    _check(*svg2.svg2_quantize_mxfp4(x, transposed=True), _np(x).T)
    # rows apart, and at an address that no 16-byte load can take
    wide = torch.full((M, K + 9), 3.0, dtype=dtype, device="cuda")
    wide[:, 5:5 + K] = x
    _check(*svg2.svg2_quantize_mxfp4(wide[:, 5:5 + K]), _np(x))
    _check(*svg2.svg2_quantize_mxfp4(wide[:, 5:5 + K], transposed=True), _np(x).T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,N,d", [(3, 37, 64), (5, 130, 128), (2, 9, 20)])
def test_quantize_head_order(svg2, H, N, d, dtype):
    """The layer's O [H,N,d] as rows of H d columns (d of 20: blocks that run across heads)."""
    o = _spread((H, N, d), H * N, dtype)
    x = _np(o).transpose(1, 0, 2).reshape(N, H * d)
    _check(*svg2.svg2_quantize_mxfp4(o.transpose(0, 1)), x)
    _check(*svg2.svg2_quantize_mxfp4(o.transpose(0, 1), transposed=True), x.T)


@pytest.mark.parametrize("dtype,M,K", [(torch.bfloat16, 33000, 4160), (torch.float32, 16500, 4128), (torch.bfloat16, 33001, 4131)])
def test_quantize_past_the_caches(svg2, dtype, M, K):
    """Operands of more than 256 MB take loads and stores of their own: the same bits as their parts."""
    x = torch.randn((M, K), generator=torch.Generator(device="cuda").manual_seed(M), device="cuda").to(dtype)
    assert x.numel() * x.element_size() >= 1 << 28
    codes, scales = svg2.svg2_quantize_mxfp4(x)
    tc, ts = svg2.svg2_quantize_mxfp4(x, transposed=True)
    back = svg2.svg2_dequantize_mxfp4(codes, scales, K, dtype=dtype)
    for r0 in range(0, M, 11008):
        c, s = svg2.svg2_quantize_mxfp4(x[r0:r0 + 11008])
        assert torch.equal(codes[r0:r0 + 11008], c) and torch.equal(scales[:, r0:r0 + 11008], s)
        assert torch.equal(back[r0:r0 + 11008], svg2.svg2_dequantize_mxfp4(c, s, K, dtype=dtype))
    for c0 in range(0, K, 1368):
        c, s = svg2.svg2_quantize_mxfp4(x[:, c0:c0 + 1368], transposed=True)
        assert torch.equal(tc[c0:c0 + 1368], c) and torch.equal(ts[:, c0:c0 + 1368], s)


def test_quantize_extremes(svg2):
    """Subnormals, the largest numbers, blocks of one value, negative zeros; an infinity or a NaN makes its block NaN."""
    fi = torch.finfo(torch.float32)
    x = torch.zeros((9, 96), dtype=torch.float32)
    x[0, :32] = fi.max
    x[1, :32] = fi.smallest_normal
    x[2, 5] = 2.0 ** -149
    x[3] = -fi.max
    x[4, 40] = float("inf")
    x[5, 70] = float("nan")
    x[6] = -0.0
    x[7, 3], x[7, 4] = 2.0 ** 127, 2.0 ** -149
    x[8] = 2.0 ** -126 * torch.arange(96)
    with np.errstate(invalid="ignore"):
        ref = ops.quantize(x.double().numpy())
    for t in (False, True):
        src = x.t().contiguous().cuda() if t else x.cuda()
        codes, scales = svg2.svg2_quantize_mxfp4(src, transposed=t)
        assert np.array_equal(scales.cpu().numpy(), ref[1])
        assert np.array_equal(codes.cpu().numpy(), ref[0])
        for dtype in (torch.float32, torch.bfloat16):
            back = svg2.svg2_dequantize_mxfp4(codes, scales, 96, dtype=dtype).double().cpu().numpy()
            v = ops.values(*ref)[:, :96]
            assert np.array_equal(np.isnan(back), np.isnan(v)) and np.array_equal(back[~np.isnan(v)], v[~np.isnan(v)])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,K", [(1, 1), (5, 131), (33, 256), (100, 1000)])
def test_dequantize_gives_the_values(svg2, R, K, dtype):
    r = np.random.default_rng(R + K)
    nk = -(-K // 128)
    codes = r.integers(0, 256, size=(R, nk * 64)).astype(np.uint8)
    scales = r.integers(0, 253, size=(nk, R, 4)).astype(np.uint8)       # all that quantising can leave
    back = svg2.svg2_dequantize_mxfp4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K, dtype=dtype)
    assert np.array_equal(_np(back), ops.values(codes, scales)[:, :K])
    wide = torch.full((R, K + 3), 7.0, dtype=dtype, device="cuda")
    svg2.svg2_dequantize_mxfp4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), K, out=wide[:, 1:K + 1])
    assert torch.equal(wide[:, 1:K + 1], back)
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, K + 1:] == 7).all())


def _operand(R, K, seed, exps=(-6, 7)):
    r = np.random.default_rng(seed)
    x = r.standard_normal((R, K)) * 2.0 ** r.integers(exps[0], exps[1], size=(R, 1))
    c, s = ops.quantize(x.astype(np.float32).astype(np.float64))
    return c, s, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()


# rows of a few tokens, of half a tile and across tiles; columns of one block of 128 up to a long sum (even and odd numbers of them:
# a stage is two)
PRODUCTS = [(1, 1, 1), (1, 64, 128), (1, 513, 640), (2, 96, 300), (7, 1000, 1000), (16, 130, 4224), (15, 33, 17000), (17, 255, 256),
            (33, 65, 129), (64, 512, 2048), (65, 127, 384), (128, 128, 128), (129, 257, 512), (255, 300, 1280), (256, 256, 256),
            (300, 1023, 777), (513, 640, 1000), (1000, 77, 64),
            # few tiles and a long contraction: in parts, the last of them shorter, with 128 columns more
            (70, 60, 20000), (130, 260, 16384), (129, 100, 33000), (300, 520, 24704),
            # more tiles of 64 x 64 than fit at once, and more than one of 128 x 128 or 256 x 256 for a workgroup; one to five stages
            (2049, 2177, 100), (2000, 2100, 513), (4129, 4225, 300), (4095, 4090, 513), (8190, 4093, 300), (4090, 8100, 1100)]


@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product_matches_64_bits(svg2, M, N, K, out_dtype):
    ac, as_, a, sa = _operand(M, K, 1 + M)
    bc, bs, b, sb = _operand(N, K, 2 + N)
    bias = torch.randn((N,), generator=torch.Generator().manual_seed(K)).cuda()
    va, vb = ops.values(ac, as_), ops.values(bc, bs)
    for bb in (None, bias):
        ref, bound = ops.product(va, vb, None if bb is None else _np(bb))
        got = svg2.svg2_matmul_mxfp4(a, sa, b, sb, bias=bb, out_dtype=out_dtype)
        assert got.shape == (M, N) and got.dtype == out_dtype
        assert_within(got, ref, bound, out_dtype, "%s" % (bb is not None))
    # a slice of a wider result, at an address of its own
    wide = torch.full((M, N + 7), 5.0, dtype=out_dtype, device="cuda")
    svg2.svg2_matmul_mxfp4(a, sa, b, sb, bias=bias, out=wide[:, 3:3 + N])
    assert torch.equal(wide[:, 3:3 + N], got)
    assert bool((wide[:, :3] == 5).all()) and bool((wide[:, 3 + N:] == 5).all())


@pytest.mark.parametrize("M,N,K", [(3, 40, 256), (100, 150, 384), (300, 520, 512)])
def test_product_of_small_integers_is_exact(svg2, M, N, K):
    """Random codes, block scales of 1/2, 1 and 2: every sum is a multiple of 2^-4 below 2^4 * 36 * K < 2^19, exact in fp32.  Any
    mistake in which scale or element goes where shows."""
    r = np.random.default_rng(M)
    nk = K // 128
    ac, bc = (r.integers(0, 256, size=(R, K // 2)).astype(np.uint8) for R in (M, N))
    as_, bs = (r.integers(126, 129, size=(nk, R, 4)).astype(np.uint8) for R in (M, N))
    up = lambda t: torch.from_numpy(t).cuda()       # noqa: E731
    got = svg2.svg2_matmul_mxfp4(up(ac), up(as_), up(bc), up(bs), out_dtype=torch.float32)
    assert np.array_equal(_np(got), ops.values(ac, as_) @ ops.values(bc, bs).T)


def test_product_of_few_rows_and_many_columns(svg2):
    """Five rows times 20,992 x 4096 codes go through tiles, half of them through the kernel for few rows: sums of multiples of 1/4 of
    size 10^3, exact in fp32, so the same bits."""
    M, N, K = 5, 20992, 4096
    g = torch.Generator(device="cuda").manual_seed(4)
    a, b = (torch.randint(0, 256, (R, K // 2), dtype=torch.uint8, device="cuda", generator=g) for R in (M, N))
    one = lambda R: torch.full((K // 128, R, 4), 127, dtype=torch.uint8, device="cuda")     # noqa: E731
    whole = svg2.svg2_matmul_mxfp4(a, one(M), b, one(N), out_dtype=torch.float32)
    for h in (0, 1):
        part = svg2.svg2_matmul_mxfp4(a, one(M), b[h * N // 2:(h + 1) * N // 2], one(N // 2), out_dtype=torch.float32)
        assert torch.equal(whole[:, h * N // 2:(h + 1) * N // 2], part)
    ref = torch.matmul(svg2.svg2_dequantize_mxfp4(a, one(M), dtype=torch.float32).double(),
                       svg2.svg2_dequantize_mxfp4(b, one(N), dtype=torch.float32).double().t())
    assert torch.equal(whole.double(), ref)


@pytest.mark.parametrize("M,N", [(5, 70), (200, 300)])
def test_product_keeps_nan_blocks_and_far_scales_apart(svg2, M, N):
    K = 512
    ac, as_, a, sa = _operand(M, K, 5)
    bc, bs, b, sb = _operand(N, K, 6)
    sa[2, 1, 3] = 255                       # one block of row 1 of A, one of row 4 of B
    sb[0, 4, 0] = 255
    sa[:, 2] = 1                            # row 2 of A at 2^-126, row 7 of B at 2^120: a small and a large result
    sb[:, 7] = 247
    got = _np(svg2.svg2_matmul_mxfp4(a, sa, b, sb, out_dtype=torch.float32))
    va, vb = ops.values(ac, sa.cpu().numpy()), ops.values(bc, sb.cpu().numpy())
    nan = np.zeros((M, N), dtype=bool)
    nan[1], nan[:, 4] = True, True
    assert np.array_equal(np.isnan(got), nan)
    ref, bound = ops.product(np.nan_to_num(va), np.nan_to_num(vb))
    near = ~nan
    near[2], near[:, 7] = False, False
    assert np.all(np.abs(got - ref)[near] <= (bound + 2.0 ** -24 * np.abs(ref))[near])
    assert abs(got[2, 7] - ref[2, 7]) <= bound[2, 7] + 2.0 ** -24 * abs(ref[2, 7])


def test_linear_and_its_gradients(svg2):
    """Y = X W^T + b as a user runs it, and dX = dY W, dW = dY^T X on operands quantised along the contracted axis."""
    M, N, K = 203, 192, 160
    g = torch.Generator().manual_seed(1)
    x, w, dy = (torch.randn(s, generator=g).to(torch.bfloat16).cuda() for s in ((M, K), (N, K), (M, N)))
    bias = torch.randn((N,), generator=g).cuda()
    y = svg2.svg2_matmul_mxfp4(*svg2.svg2_quantize_mxfp4(x), *svg2.svg2_quantize_mxfp4(w), bias=bias)
    q = lambda t: ops.values(*ops.quantize(t))      # noqa: E731
    X, W, DY = _np(x), _np(w), _np(dy)
    assert_within(y, *ops.product(q(X), q(W), _np(bias)), torch.bfloat16, "y")
    dx = svg2.svg2_matmul_mxfp4(*svg2.svg2_quantize_mxfp4(dy), *svg2.svg2_quantize_mxfp4(w, transposed=True))
    assert_within(dx, *ops.product(q(DY), q(W.T)), torch.bfloat16, "dx")
    dw = svg2.svg2_matmul_mxfp4(*svg2.svg2_quantize_mxfp4(dy, transposed=True), *svg2.svg2_quantize_mxfp4(x, transposed=True),
                                out_dtype=torch.float32)
    assert_within(dw, *ops.product(q(DY.T), q(X.T)), torch.float32, "dw")


@pytest.mark.parametrize("M,N,K", [(1, 520, 2176), (130, 520, 2176), (2060, 2050, 2176), (100, 200, 20000)])
def test_product_in_a_graph_beside_another(svg2, M, N, K):
    """Two captured graphs, each with a workspace of its own (the last shape uses it), replayed with eager calls between them, then the
    same two products at once on two streams."""
    sets = []
    for seed in (1, 2):
        _, _, a, sa = _operand(M, K, seed)
        _, _, b, sb = _operand(N, K, 10 + seed)
        ref = svg2.svg2_matmul_mxfp4(a, sa, b, sb)
        ws = torch.empty(svg2.load_library().svg2_matmul_mxfp4_workspace_size(M, N, K), dtype=torch.uint8, device="cuda")
        sets.append((a, sa, b, sb, ref, torch.empty_like(ref), ws))
    graphs = []
    for a, sa, b, sb, ref, out, ws in sets:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            svg2.svg2_matmul_mxfp4(a, sa, b, sb, out=out, ws=ws)
        graphs.append(g)
    for rep in range(4):
        for (a, sa, b, sb, ref, out, ws), g in zip(sets, graphs):
            out.zero_()
            ws.random_(0, 256)
            g.replay()
            again = svg2.svg2_matmul_mxfp4(a, sa, b, sb)
            torch.cuda.synchronize()
            assert torch.equal(out, ref) and torch.equal(again, ref)
    streams = [torch.cuda.Stream() for _ in sets]
    for s in sets:
        s[5].zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for (a, sa, b, sb, ref, out, ws), s in zip(sets, streams):
            with torch.cuda.stream(s):
                svg2.svg2_matmul_mxfp4(a, sa, b, sb, out=out, ws=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(s[5], s[4]) for s in sets)


def test_block_from_hidden_states_to_hidden_states(svg2):
    """The operators together, as a block of a video transformer runs them around the layer: hidden states -> MXFP4 projection to
    Q, K and V -> norm, rotary positions, head order -> svg2_forward (every key selected) -> MXFP4 projection of O out of head
    order.  Each stage is checked against 64 bits on what the stage before left."""
    grid, text, H, d = (3, 8, 9), 11, 4, 64
    N, D = 3 * 8 * 9 + text, H * d
    g = torch.Generator().manual_seed(3)
    hidden = torch.randn((N, D), generator=g).to(torch.bfloat16).cuda()
    w_qkv, w_out = (torch.randn(s, generator=g).cuda() / D ** 0.5 for s in ((3 * D, D), (D, D)))
    b_qkv, b_out = torch.randn((3 * D,), generator=g).cuda(), torch.randn((D,), generator=g).cuda()
    nw = [1 + 0.1 * torch.randn((H, d), generator=g) for _ in range(2)]
    share = (12, 10, 10)
    pos, freq = svg2.svg2_grid_positions(grid, extra=text), svg2.svg2_rope_frequencies(share)
    q_in, q_qkv, q_out = (svg2.svg2_quantize_mxfp4(t) for t in (hidden, w_qkv, w_out))
    qkv = svg2.svg2_matmul_mxfp4(*q_in, *q_qkv, bias=b_qkv)
    packed = qkv.view(N, 3, H, d)
    Q, K, V = svg2.svg2_rope([packed[:, i] for i in range(3)], pos, freq, axis_pairs=share, rotate=(True, True, False),
                             norm_weights=[nw[0].cuda(), nw[1].cuda(), None], norm_scope="token")
    C = 8
    cq, ck = Q[:, :C].float().contiguous(), K[:, :C].float().contiguous()
    O = svg2.svg2_forward(Q, K, V, cq, ck, 1.0, 2).O
    q_o = svg2.svg2_quantize_mxfp4(O.transpose(0, 1))
    out = svg2.svg2_matmul_mxfp4(*q_o, *q_out, bias=b_out)
    torch.cuda.synchronize()

    val = lambda t: ops.values(*ops.quantize(t))    # noqa: E731
    assert_within(qkv, *ops.product(val(_np(hidden)), val(_np(w_qkv)), _np(b_qkv)), torch.bfloat16, "qkv")
    a = ops.angles(_np(pos).astype(np.int64)[None], _np(freq), share)
    for i, t in enumerate((Q, K)):
        ref, bound = ops.rope(_np(packed[:, i])[None], _np(nw[i]), a, "token", 1e-6, "adjacent")
        assert_within(t.transpose(0, 1)[None], ref, bound, torch.bfloat16, "rope %d" % i)
    assert torch.equal(V, packed[:, 2].transpose(0, 1))
    s = _np(Q) @ _np(K).transpose(0, 2, 1) / d ** 0.5
    p = np.exp(s - s.max(-1, keepdims=True))
    p = p / p.sum(-1, keepdims=True)
    # a probability goes into the second product as bf16: off by 2^-8 of itself.  A score is off by at most 64 * 2^-24 of its sum of
    # magnitudes, here below 2^6 (64 products of numbers of size one, over 8): 2^-12 of the probability.  The result is rounded by
    # assert_within.
    assert (np.abs(_np(Q)) @ np.abs(_np(K)).transpose(0, 2, 1)).max() / d ** 0.5 < 2 ** 6
    assert_within(O, p @ _np(V), (2.0 ** -8 + 2.0 ** -12) * (1 + 2.0 ** -7) * (p @ np.abs(_np(V))), torch.bfloat16, "attention")
    assert_within(out, *ops.product(val(_np(O).transpose(1, 0, 2).reshape(N, D)), val(_np(w_out)), _np(b_out)), torch.bfloat16, "out")


def test_the_block_diagnostic_runs(svg2, capsys):
    from types import SimpleNamespace
    from paper_2505_18875_amd import diagnostics
    diagnostics.block(SimpleNamespace(workload="small", heads=2))
    rows = [l for l in capsys.readouterr().out.splitlines() if l.startswith(("| fp32", "| bf16", "| mxfp4"))]
    assert len(rows) == 3 and all("nan" not in r for r in rows)
