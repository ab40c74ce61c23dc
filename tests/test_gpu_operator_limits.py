"""The operators around the layer at the sizes where 32 bits end: launches of 2^32 threads, tensors of more than 2^31 elements."""
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
    yield pkg
    torch.cuda.empty_cache()


# one token of a wavefront: 2^26 of them are 2^32 threads; five more than 2^25 leave a second row of workgroups almost empty
@pytest.mark.parametrize("N", [2 ** 25 + 5, 2 ** 26])
def test_rope_of_as_many_tokens_as_it_takes(svg2, N):
    """Four different rows at four positions over and over, in place: each has to come out as in a call of four tokens, once, and the
    rows behind the last stay."""
    H, d, behind, eps = 5, 64, 8, 1e-6
    g = torch.Generator().manual_seed(1)
    four = torch.randn((4, H, d), generator=g).to(torch.bfloat16)
    w = 1 + 0.3 * torch.randn((d,), generator=g)
    freq = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))
    kw = dict(axis_pairs=(d // 2,), norm_weights=[w.cuda()])
    pos = (7 + torch.arange(N, dtype=torch.int32, device="cuda") % 4)[:, None].contiguous()
    ref, = svg2.svg2_rope([four.cuda()], pos[:4], freq.cuda(), **kw)
    ref = ref.transpose(0, 1).contiguous()
    a = ops.angles(pos[:4].cpu().numpy()[None], freq.numpy(), (d // 2,))
    y, bound = ops.rope(four.double().numpy()[None], w.double().numpy(), a, "head", eps, "adjacent")
    assert_within(ref[None], y, bound + 2.0 ** -51 * 10 * ops.pair_norm(y, "adjacent"), torch.bfloat16)

    x = four.cuda().repeat((N + behind + 3) // 4, 1, 1)[:N + behind]
    svg2.svg2_rope([x[:N]], pos, freq.cuda(), eps=eps, outs=[x[:N]], **kw)
    whole, step = N // 4 * 4, 2 ** 20
    for r0 in range(0, whole, step):
        part = x[r0:min(whole, r0 + step)].view(-1, 4, H, d)
        assert bool((part == ref).all()), "tokens from %d" % r0
    assert torch.equal(x[whole:N], ref[:N - whole])
    assert all(torch.equal(x[r].cpu(), four[r % 4]) for r in range(N, N + behind))


def test_gradients_of_more_than_2_31_elements(svg2):
    """420,000 tokens of 40 heads of 128: the last tokens as in a call of their own, and the weights' gradient against 64 bits.  A
    workgroup holds one of 512 shares of the tokens and adds them up one after another: 821 additions more than ops.rope_backward counts."""
    N, H, d, eps = 420000, 40, 128, 1e-6
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dy = (torch.randn((N, H, d), generator=g, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert x.numel() > 2 ** 31
    w = 1 + 0.3 * torch.randn((H, d), generator=g, device="cuda")
    pos = torch.randint(0, 200, (N, 1), generator=g, dtype=torch.int32, device="cuda")
    freq = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64, device="cuda") / (d // 2))
    kw = dict(axis_pairs=(d // 2,), norm_weights=[w], norm_scope="token", eps=eps)
    res = svg2.svg2_rope_backward([dy[None]], [x], pos, freq, **kw)
    end = svg2.svg2_rope_backward([dy[None, -600:]], [x[-600:]], pos[-600:], freq, **kw)
    assert torch.equal(res.grads[0][:, -600:], end.grads[0])
    dw = torch.zeros((H, d), dtype=torch.float64, device="cuda")
    mags = torch.zeros_like(dw)
    for n in range(0, N, 10000):
        a = (pos[n:n + 10000].double() * freq)[:, None, :]
        xs, gs = x[n:n + 10000].double(), dy[n:n + 10000].double()
        xn = xs * (xs.pow(2).mean((1, 2), keepdim=True) + eps).rsqrt()
        gi, gj = gs[..., 0::2], gs[..., 1::2]
        back = torch.stack([gi * a.cos() + gj * a.sin(), gj * a.cos() - gi * a.sin()], -1).flatten(-2)
        dw += (back * xn).sum(0)
        size = torch.hypot(gi, gj)
        mags += (torch.stack([size, size], -1).flatten(-2) * xn.abs()).sum(0)
    steps = ops.sum_steps(H, d) / 2 + 12 + 72 + 821
    assert_within(res.dweights[0], dw.cpu().numpy(), steps * ops.U * mags.cpu().numpy(), torch.float32)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("H,d", [(40, 128), (1, 5123)])
def test_quantize_more_than_2_31_elements(svg2, H, d, transposed):
    """An operand from head order, its heads far apart, and one of odd rows: the last rows as in a call of their own, and their values."""
    N, last = 420001, 417                   # 420,001 - 417 = 3278 * 128: the blocks of the transposed operand are the same
    o = torch.randn((H, N, d), generator=torch.Generator(device="cuda").manual_seed(3), dtype=torch.bfloat16, device="cuda")
    assert o.numel() > 2 ** 31
    x = o.transpose(0, 1) if H > 1 else o[0]
    codes, scales = svg2.svg2_quantize_mxfp4(x, transposed=transposed)
    c, s = svg2.svg2_quantize_mxfp4(x[-last:].contiguous(), transposed=transposed)
    if transposed:
        assert torch.equal(codes[:, -c.shape[1]:], c) and torch.equal(scales[-s.shape[0]:], s)
    else:
        assert torch.equal(codes[-last:], c) and torch.equal(scales[:, -last:], s)
    K = N if transposed else H * d
    values = svg2.svg2_dequantize_mxfp4(codes, scales, K)
    assert values.numel() > 2 ** 31
    part = svg2.svg2_dequantize_mxfp4(c, s, last if transposed else K)
    assert torch.equal(values[:, -last:] if transposed else values[-last:], part)


@pytest.mark.parametrize("M,N,nk", [(70001, 31999, 1), (1048600, 70, 65)])
def test_product_of_far_results_and_far_operands(svg2, M, N, nk):
    """A result of more than 2^31 elements, and an operand of more than 2^32 bytes: the last rows and columns, and the first, against 64
    bits (sums of at most 8320 products, exact in fp32: see test_gpu_mxfp4_paths.py)."""
    from test_gpu_mxfp4_paths import small_operand
    assert M * N > 2 ** 31 or M * nk * 64 > 2 ** 32
    a, sa = small_operand(M, nk, 1)
    b, sb = small_operand(N, nk, 2)
    got = svg2.svg2_matmul_mxfp4(a, sa, b, sb, out_dtype=torch.float32)
    vb = svg2.svg2_dequantize_mxfp4(b, sb, dtype=torch.float32).double().t().contiguous()
    for r0 in (0, M // 2, M - 300):
        va = svg2.svg2_dequantize_mxfp4(a[r0:r0 + 300], sa[:, r0:r0 + 300].clone(), dtype=torch.float32).double()
        assert bool((got[r0:r0 + 300] == torch.matmul(va, vb)).all()), r0
