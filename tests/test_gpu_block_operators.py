"""Norm, FP8 operands and their product as a block uses them: one behind the other with the rotary call and the sparse layer, the way back, in
graphs, on streams of their own."""
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
    return t.double().cpu().numpy()


def _rand(shape, seed, dtype=F32, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()


def _product_within(svg2, got, a, b, bias=None):
    ref, bound = ops.product(ops.values(*(t.cpu().numpy() for t in a)), ops.values(*(t.cpu().numpy() for t in b)),
                             None if bias is None else _np(bias), got.dtype is F32)
    assert_within(got, ref, bound, got.dtype)


def test_a_block_forward(svg2):
    """Norm -> FP8 operand -> projection to Q, K, V -> rotary positions and head order -> sparse layer -> its output from head order as an FP8 operand ->
    second projection; each product against 64 bits on its own operands."""
    H, d, grid, eps = 2, 128, (2, 9, 15), EPS
    N, D = grid[0] * grid[1] * grid[2], H * d
    x, w, b = _rand((1, N, D), 1, BF16), _rand((1, D), 2, scale=0.3), _rand((1, D), 3, scale=0.3)
    w_qkv = svg2.svg2_quantize_fp8_blocks(_rand((3 * D, D), 4, BF16, D ** -0.5), square=True)
    w_out = svg2.svg2_quantize_fp8_blocks(_rand((D, D), 5, BF16, D ** -0.5), square=True)
    b_qkv, b_out = _rand((3 * D,), 6), _rand((D,), 7)
    operand = svg2.svg2_layer_norm_fp8(x, w, b, eps=eps, one_plus=True)
    qkv = svg2.svg2_matmul_fp8_blocks(*operand, *w_qkv, bias=b_qkv)
    _product_within(svg2, qkv, operand, w_qkv, b_qkv)
    side = 2 * (d // 6)
    pairs = ((d - 2 * side) // 2, side // 2, side // 2)
    p = qkv.view(N, 3, H, d)
    q, k, v = svg2.svg2_rope([p[:, i] for i in range(3)], svg2.svg2_grid_positions(grid), svg2.svg2_rope_frequencies(pairs), axis_pairs=pairs,
                             rotate=(True, True, False), norm_weights=[torch.ones((H, d), device="cuda")] * 2 + [None], norm_scope="token")
    at = torch.arange(0, N, N // 8, device="cuda")[:8]
    O = svg2.svg2_forward(q, k, v, q[:, at].float().contiguous(), k[:, at].float().contiguous(), 0.9, 2).O
    assert bool(torch.isfinite(O.float()).all())
    o = svg2.svg2_quantize_fp8_blocks(O.transpose(0, 1))
    same = svg2.svg2_quantize_fp8_blocks(O.transpose(0, 1).reshape(N, D))
    assert torch.equal(o[0], same[0]) and torch.equal(o[1], same[1])
    out = svg2.svg2_matmul_fp8_blocks(*o, *w_out, bias=b_out)
    _product_within(svg2, out, o, w_out, b_out)
    # the block's result against the same without quantisation: E4M3 numbers are off by at most 2^-4 of themselves, two operands in a row, so
    # 2^-3 of the products' magnitudes (each sum of D products of independent signs: sqrt(D) of them stand against D)
    y = svg2.svg2_layer_norm(x, w, b, eps=eps, one_plus=True, out_dtype=F32)[0].double()
    ref = y @ svg2.svg2_dequantize_fp8_blocks(*w_qkv, D, dtype=F32).double().t() + b_qkv.double()
    mags = y.abs() @ svg2.svg2_dequantize_fp8_blocks(*w_qkv, D, dtype=F32).double().abs().t()
    assert bool(((qkv.double() - ref).abs() <= 2.0 ** -4 * mags + 2.0 ** -8 * (ref.abs() + mags)).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_block_backward(svg2, dtype):
    """The gradients of norm and projection: dX of the product from dY and W^T, dW from dY^T and X^T, then the norm's."""
    B, N, D, E = 2, 150, 200, 330
    x, w, b = _rand((B, N, D), 1, dtype), _rand((B, D), 2, scale=0.3), _rand((B, D), 3, scale=0.3)
    weight, dy = _rand((E, D), 4, dtype, D ** -0.5), _rand((B * N, E), 5, dtype)
    rows, cols = svg2.svg2_quantize_fp8_blocks(weight, transposed="both", square=True)
    # W and W^T stand for the same values
    assert torch.equal(svg2.svg2_dequantize_fp8_blocks(*rows, D, dtype=F32), svg2.svg2_dequantize_fp8_blocks(*cols, E, dtype=F32).t())
    y = svg2.svg2_layer_norm(x, w, b, eps=EPS, one_plus=True).view(B * N, D)
    out = svg2.svg2_matmul_fp8_blocks(*svg2.svg2_quantize_fp8_blocks(y), *rows, out_dtype=dtype)
    _product_within(svg2, out, svg2.svg2_quantize_fp8_blocks(y), rows)
    g, g_t = svg2.svg2_quantize_fp8_blocks(dy, transposed="both")
    y_t = svg2.svg2_quantize_fp8_blocks(y, transposed=True)
    d_in = svg2.svg2_matmul_fp8_blocks(*g, *cols, out_dtype=dtype)
    d_weight = svg2.svg2_matmul_fp8_blocks(*g_t, *y_t, out_dtype=F32)
    _product_within(svg2, d_in, g, cols)
    _product_within(svg2, d_weight, g_t, y_t)
    res = svg2.svg2_layer_norm_backward(d_in.view(B, N, D), x, w, b, eps=EPS, one_plus=True)
    dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(d_in).reshape(B, N, D), _np(x), _np(w), EPS, True)
    assert_within(res.grad, dx, bound, dtype)
    assert_within(res.dweight, dw, dw_bound, F32)
    assert_within(res.dbias, db, db_bound, F32)


def _step(svg2, st, ws):
    """A training step's calls on buffers that stay; ws: one workspace for all of them."""
    B, N, D = st["x"].shape
    y = svg2.svg2_layer_norm(st["x"], st["w"], st["b"], one_plus=True).view(B * N, D)
    a = svg2.svg2_layer_norm_fp8(st["x"], st["w"], st["b"], one_plus=True)
    out = svg2.svg2_matmul_fp8_blocks(*a, *st["rows"], bias=st["bias"])
    g, g_t = svg2.svg2_quantize_fp8_blocks(st["dy"], transposed="both")
    d_in = svg2.svg2_matmul_fp8_blocks(*g, *st["cols"], ws=ws)
    d_weight = svg2.svg2_matmul_fp8_blocks(*g_t, *svg2.svg2_quantize_fp8_blocks(y, transposed=True), out_dtype=F32, ws=ws)
    res = svg2.svg2_layer_norm_backward(d_in.view(B, N, D), st["x"], st["w"], st["b"], one_plus=True, ws=ws)
    return [y, *a, out, *g, *g_t, d_in, d_weight, res.grad, res.dweight, res.dbias]


def _state(svg2, B, N, D, E, seed):
    st = dict(x=_rand((B, N, D), seed, BF16), w=_rand((B, D), seed + 1, scale=0.3), b=_rand((B, D), seed + 2, scale=0.3),
              dy=_rand((B * N, E), seed + 3, BF16), bias=_rand((E,), seed + 4))
    st["rows"], st["cols"] = svg2.svg2_quantize_fp8_blocks(_rand((E, D), seed + 5, BF16, D ** -0.5), transposed="both", square=True)
    return st


def test_two_graphs_that_share_a_workspace(svg2):
    """Captured steps replayed in turn on changed inputs, with eager work and a scribbled-over workspace between: as the eager calls, bit for bit."""
    from paper_2505_18875_amd import binding
    shapes = [(2, 1100, 264, 200), (1, 2177, 136, 328)]
    need = max(max(binding._fp8_blocks_workspace_size(E, D, -(-B * N // 128) * 128), binding._fp8_blocks_workspace_size(B * N, D, -(-E // 128) * 128))
               for B, N, D, E in shapes) + (1 << 23)
    assert max(binding._fp8_blocks_workspace_size(E, D, -(-B * N // 128) * 128) for B, N, D, E in shapes) > 256         # in parts
    ws = torch.empty((need,), dtype=torch.uint8, device="cuda")
    states = [_state(svg2, *s, 10 * k) for k, s in enumerate(shapes)]
    graphs = []
    for st in states:
        for _ in range(2):
            _step(svg2, st, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = _step(svg2, st, ws)
        graphs.append((g, outs))
    for turn in range(4):
        for k, (st, (g, outs)) in enumerate(zip(states, graphs)):
            new = _state(svg2, *shapes[k], 100 + 10 * turn + k)
            for name in ("x", "w", "b", "dy", "bias"):
                st[name].copy_(new[name])
            for t, n in zip((*st["rows"], *st["cols"]), (*new["rows"], *new["cols"])):
                t.copy_(n)
            ws.fill_(255)
            g.replay()
        torch.cuda.synchronize()
        for st, (g, outs) in zip(states, graphs):
            for got, want in zip(outs, _step(svg2, st, ws)):
                assert torch.equal(got, want)
        g.replay()                          # once more on the same inputs
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, _step(svg2, st, ws)))


def test_streams_of_their_own(svg2):
    """Two steps at once on two streams that are not the default, inputs made on them: as one after the other."""
    want = [_step(svg2, _state(svg2, 2, 500, 300, 260, s), None) for s in (0, 50)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for s, seed in zip(streams, (0, 50)):
            with torch.cuda.stream(s):
                got.append(_step(svg2, _state(svg2, 2, 500, 300, 260, seed), None))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_an_operand_times_itself_and_one_tensor_twice(svg2):
    x = _rand((300, 700), 1, BF16)
    a = svg2.svg2_quantize_fp8_blocks(x)
    got = svg2.svg2_matmul_fp8_blocks(*a, *a, out_dtype=F32)
    _product_within(svg2, got, a, a)
    assert torch.equal(got, got.t())
    # the same tensor as weight and bias, as gradient and input
    w = _rand((700,), 2)
    y, bound = ops.layer_norm(_np(x)[None], _np(w), _np(w), EPS, False)
    assert_within(svg2.svg2_layer_norm(x, w, w, eps=EPS), y[0], bound[0], BF16)
    res = svg2.svg2_layer_norm_backward(x, x, w, w, eps=EPS)
    dx, bound, dw, dw_bound, db, db_bound = ops.layer_norm_backward(_np(x)[None], _np(x)[None], _np(w), EPS, False)
    assert_within(res.grad, dx[0], bound[0], BF16)
    assert_within(res.dweight, dw[0], dw_bound[0], F32)
    assert_within(res.dbias, db[0], db_bound[0], F32)
    assert HALF_STEP[BF16] == 2.0 ** -8 and np.isfinite(dx).all()


@pytest.mark.parametrize("normed", [False, True])
def test_the_block_diagnostic_has_them(svg2, capsys, normed):
    from types import SimpleNamespace
    from paper_2505_18875_amd import diagnostics
    diagnostics.block(SimpleNamespace(workload="small", heads=2, norm=normed))
    rows = [l for l in capsys.readouterr().out.splitlines() if l.startswith(("| fp32", "| bf16", "| fp8", "| mxfp4"))]
    assert len(rows) == 4 and all("nan" not in r and r.count("|") == (11 if normed else 10) for r in rows)
