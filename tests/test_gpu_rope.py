"""svg2_rope and svg2_rope_backward against the formulas in 64 bits; gradients against differences too."""
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


def _case(dtype, B, N, H, d, scope, seed, n_axes=3, far=False, layout="packed"):
    g = torch.Generator().manual_seed(seed)
    if layout == "packed":
        qkv = torch.randn((B, N, 3, H, d), generator=g).to(dtype).cuda()
        x = [qkv[:, :, i] for i in range(3)]
    elif layout == "head_order":
        x = [torch.randn((B, H, N, d), generator=g).to(dtype).cuda().transpose(1, 2) for _ in range(3)]
    else:
        x = [torch.randn((B, N, H, d), generator=g).to(dtype).cuda() for _ in range(3)]
    top = 2 ** 31 - 1 if far else 97
    pos = torch.randint(-top if far else 0, top, (N, n_axes), generator=g, dtype=torch.int32)
    share = [d // 2 // n_axes] * n_axes
    share[0] += d // 2 - sum(share)
    freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in share])
    w = None
    if scope != "none":
        w = [1 + 0.3 * torch.randn((d,) if scope == "head" else (H, d), generator=g) for _ in range(2)]
    return x, pos, freq, share, w


def _kw(share, w, scope, pairing, **more):
    return dict(axis_pairs=share, rotate=(True, True, False), norm_weights=None if w is None else [w[0].cuda(), w[1].cuda(), None],
                norm_scope="head" if scope == "none" else scope, pairing=pairing, **more)


def _np(t):
    return t.double().cpu().numpy()


# lengths around one wavefront per token and four per workgroup; heads around a step (4 of 128, 8 of 64) and around ten steps
FORWARD = [
    # dtype, B, N, H, d, scope, pairing, axes, far
    (torch.bfloat16, 1, 1, 1, 64, "none", "adjacent", 1, False),
    (torch.float32, 1, 1, 1, 128, "head", "halves", 3, False),
    (torch.bfloat16, 2, 37, 5, 64, "head", "halves", 3, False),
    (torch.bfloat16, 1, 33, 40, 128, "token", "adjacent", 3, False),
    (torch.bfloat16, 1, 18, 41, 128, "token", "halves", 2, False),
    (torch.bfloat16, 1, 8201, 17, 64, "token", "adjacent", 3, False),       # many tokens of more than two steps, a wavefront each
    (torch.float32, 1, 8195, 9, 128, "head", "halves", 3, False),
    (torch.float32, 3, 7, 9, 64, "token", "halves", 4, True),
    (torch.float32, 1, 66, 3, 128, "none", "adjacent", 3, True),
    (torch.bfloat16, 2, 5, 81, 64, "token", "adjacent", 3, False),
    (torch.bfloat16, 2, 7, 97, 64, "token", "halves", 3, False),            # a token that takes two rounds of a wavefront
    (torch.float32, 1, 6, 131, 128, "head", "adjacent", 3, False),
    # long tokens, a workgroup each
    (torch.bfloat16, 1, 1, 40, 128, "token", "adjacent", 3, True),
    (torch.float32, 2, 3, 17, 64, "token", "halves", 3, False),
    (torch.bfloat16, 2, 128, 32, 64, "head", "adjacent", 3, False),
    (torch.bfloat16, 1, 257, 33, 64, "head", "halves", 3, False),
    (torch.float32, 1, 5, 48, 128, "none", "halves", 2, False),
    (torch.bfloat16, 1, 3, 49, 128, "token", "adjacent", 3, False),
    # tokens of 8, 16 and 32 lanes, several in a wavefront
    (torch.float32, 2, 45, 1, 64, "token", "adjacent", 3, False),
    (torch.bfloat16, 1, 67, 1, 128, "head", "halves", 3, False),
    (torch.bfloat16, 1, 70, 2, 64, "token", "halves", 3, False),
    (torch.float32, 1, 35, 3, 64, "token", "adjacent", 3, False),
    (torch.bfloat16, 1, 19, 4, 64, "head", "adjacent", 3, False),
    (torch.float32, 1, 13, 2, 128, "token", "halves", 3, False),
    (torch.float32, 1, 9, 83, 64, "head", "adjacent", 1, False),
    (torch.bfloat16, 1, 4099, 2, 128, "head", "adjacent", 3, True),
]


@pytest.mark.parametrize("dtype,B,N,H,d,scope,pairing,axes,far", FORWARD)
def test_rope_matches_the_formula(svg2, dtype, B, N, H, d, scope, pairing, axes, far):
    x, pos, freq, share, w = _case(dtype, B, N, H, d, scope, 1000 + N, axes, far)
    out = svg2.svg2_rope(x, pos.cuda(), freq.cuda(), **_kw(share, w, scope, pairing))
    a = ops.angles(pos.numpy()[None], freq.numpy(), share)
    for i in range(3):
        assert out[i].shape == (B * H, N, d) and out[i].is_contiguous()
        got = out[i].view(B, H, N, d).transpose(1, 2)
        if i == 2:
            assert torch.equal(got, x[2])               # V is moved, bit for bit
            continue
        ref, bound = ops.rope(_np(x[i]), None if w is None else _np(w[i]), a, scope, 1e-6, pairing)
        # the angle itself is one 64-bit product: 2^-53 of it, and as much from taking off the quarter turns
        bound = bound + 2.0 ** -51 * np.abs(a).max() * ops.pair_norm(ref, pairing)
        assert_within(got, ref, bound, dtype, "tensor %d" % i)


@pytest.mark.parametrize("layout", ["head_order", "token_order"])
def test_rope_strides_in_place_and_positions_per_batch(svg2, layout):
    B, N, H, d = 2, 21, 6, 64
    x, _, freq, share, w = _case(torch.bfloat16, B, N, H, d, "head", 5, layout=layout)
    pos = torch.randint(0, 50, (B, N, 3), dtype=torch.int32, generator=torch.Generator().manual_seed(6))
    kw = _kw(share, w, "head", "adjacent")
    before = [_np(t) for t in x]
    plain = svg2.svg2_rope(x, pos.cuda(), freq.cuda(), **kw)
    same = svg2.svg2_rope(x, pos.cuda(), freq.cuda(), outs=x, **kw)
    a = ops.angles(pos.numpy(), freq.numpy(), share)
    for i in range(3):
        assert same[i] is x[i]
        assert torch.equal(x[i], plain[i].view(B, H, N, d).transpose(1, 2))
        if i < 2:
            ref, bound = ops.rope(before[i], _np(w[i]), a, "head", 1e-6, "adjacent")
            assert_within(x[i], ref, bound, torch.bfloat16)


def test_rope_writes_only_its_rows(svg2):
    B, N, H, d = 1, 13, 3, 64
    x, pos, freq, share, w = _case(torch.bfloat16, B, N, H, d, "token", 7)
    big = torch.full((N + 5, 3, H + 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
    outs = [big[2:2 + N, i, 1:1 + H] for i in range(3)]
    kw = _kw(share, w, "token", "halves")
    ref = svg2.svg2_rope(x, pos.cuda(), freq.cuda(), **kw)
    svg2.svg2_rope(x, pos.cuda(), freq.cuda(), outs=outs, **kw)
    for i in range(3):
        assert torch.equal(outs[i].transpose(0, 1), ref[i])
        outs[i].fill_(7.0)
    assert bool((big == 7.0).all())


def test_rope_position_zero_zero_rows_and_special_values(svg2):
    N, H, d = 6, 2, 64
    x = torch.randn((N, H, d), generator=torch.Generator().manual_seed(8)).cuda()
    pos = torch.zeros((N, 3), dtype=torch.int32)
    pos[3] = torch.tensor([5, 1, 2])
    share = [12, 10, 10]
    freq = svg2.svg2_rope_frequencies(share)
    y, = svg2.svg2_rope([x], pos.cuda(), freq, axis_pairs=share)
    still = [0, 1, 2, 4, 5]
    assert torch.equal(y[:, still], x[still].transpose(0, 1))       # position 0: the same bits
    assert not torch.equal(y[:, 3], x[3])
    # a zero row under a norm is zero; a NaN stays in its scope; infinities do not spread to other tokens
    x[0] = 0.0
    x[1, 0, 3] = float("nan")
    x[2, 1, 9] = float("inf")
    w = torch.ones((d,), device="cuda")
    y, = svg2.svg2_rope([x], pos.cuda(), freq, axis_pairs=share, norm_weights=[w])
    assert bool((y[:, 0] == 0).all())
    assert bool(y[0, 1].isnan().all()) and not bool(y[1, 1].isnan().any())
    assert not bool(y[0, 2].isnan().any()) and bool(y[:, 3:].isfinite().all())
    xb = x.to(torch.bfloat16)
    yb, = svg2.svg2_rope([xb], pos.cuda(), freq, axis_pairs=share, norm_weights=[w])
    assert bool(yb[0, 1].isnan().all()) and not bool(yb[1, 1].isnan().any())


BACKWARD = [
    (torch.float32, 1, 1, 1, 64, "token", "adjacent"),
    (torch.float32, 2, 19, 7, 64, "head", "halves"),
    (torch.float32, 1, 13, 16, 128, "token", "halves"),         # the longest token that a wavefront holds
    (torch.float32, 1, 14, 17, 128, "token", "adjacent"),       # one head more: a workgroup holds it
    (torch.bfloat16, 1, 21, 128, 64, "token", "halves"),        # the longest that a workgroup holds, and the next
    (torch.float32, 2, 11, 64, 128, "token", "adjacent"),
    (torch.float32, 1, 10, 65, 128, "token", "halves"),
    (torch.bfloat16, 1, 1031, 40, 128, "token", "adjacent"),    # more tokens than workgroups
    (torch.bfloat16, 1, 9, 40, 128, "token", "adjacent"),
    (torch.bfloat16, 1, 10, 41, 128, "token", "halves"),
    (torch.bfloat16, 3, 31, 5, 128, "head", "adjacent"),
    (torch.bfloat16, 1, 17, 12, 64, "none", "halves"),
    (torch.bfloat16, 1, 5309, 3, 64, "token", "adjacent"),      # more groups of tokens than workgroups
    (torch.float32, 1, 2111, 2, 64, "head", "adjacent"),
    # several tokens in a wavefront; token and head norms of one step
    (torch.bfloat16, 2, 41, 1, 64, "token", "halves"),
    (torch.float32, 1, 47, 1, 128, "head", "adjacent"),
    (torch.float32, 1, 39, 2, 64, "token", "adjacent"),
    (torch.bfloat16, 1, 43, 3, 64, "token", "halves"),
    (torch.float32, 1, 37, 4, 64, "head", "halves"),
    (torch.bfloat16, 1, 29, 4, 128, "token", "adjacent"),
    (torch.float32, 1, 31, 7, 64, "token", "adjacent"),
    (torch.bfloat16, 1, 33, 9, 64, "token", "adjacent"),
    (torch.bfloat16, 1, 35, 1, 64, "none", "adjacent"),
    (torch.float32, 1, 27, 20, 128, "none", "halves"),
    (torch.float32, 1, 301, 131, 64, "token", "adjacent"),      # long tokens, more groups of them than slices
]


@pytest.mark.parametrize("dtype,B,N,H,d,scope,pairing", BACKWARD)
def test_rope_backward_matches_the_formula(svg2, dtype, B, N, H, d, scope, pairing):
    x, pos, freq, share, w = _case(dtype, B, N, H, d, scope, 2000 + N)
    gen = torch.Generator().manual_seed(3000 + N)
    grads = [torch.randn((B * H, N, d), generator=gen).to(dtype).cuda() for _ in range(3)]
    res = svg2.svg2_rope_backward(grads, x, pos.cuda(), freq.cuda(), **_kw(share, w, scope, pairing))
    a = ops.angles(pos.numpy()[None], freq.numpy(), share)
    for i in range(3):
        g = grads[i].view(B, H, N, d).transpose(1, 2)
        if i == 2:
            assert torch.equal(res.grads[2], g) and res.dweights[2] is None
            continue
        dx, bound, dw, dw_bound = ops.rope_backward(_np(g), _np(x[i]), None if w is None else _np(w[i]), a, scope, 1e-6, pairing)
        assert_within(res.grads[i], dx, bound, dtype, "dx %d" % i)
        if w is not None:
            assert res.dweights[i].dtype == torch.float32
            assert_within(res.dweights[i], dw, dw_bound, torch.float32, "dw %d" % i)


@pytest.mark.parametrize("scope", ["head", "token"])
def test_rope_backward_is_the_slope_of_the_forward(svg2, scope):
    """Central differences of sum(y * g) along random directions, fp32.  With step h the difference is off by h^2 / 6 times a
    third derivative (of order one here, times 2^-12: below 1e-4 of the terms' root sum of squares) and by the rounding of two sums
    of 2 * N * H * d fp32 results, 2^-22 of each, over 2 h = 2^-5."""
    B, N, H, d = 1, 7, 3, 64
    x, pos, freq, share, w = _case(torch.float32, B, N, H, d, scope, 11)
    gen = torch.Generator().manual_seed(12)
    grads = [torch.randn((H, N, d), generator=gen).cuda() for _ in range(3)]
    kw = _kw(share, w, scope, "adjacent")
    res = svg2.svg2_rope_backward(grads, x, pos.cuda(), freq.cuda(), **kw)

    def value(xs, ws):
        k = dict(kw, norm_weights=[ws[0], ws[1], None])
        out = svg2.svg2_rope(xs, pos.cuda(), freq.cuda(), **k)
        return sum(float((o.double() * g.double()).sum()) for o, g in zip(out, grads))

    h = 2.0 ** -6
    ws = kw["norm_weights"]
    for trial in range(3):
        dirs = [torch.randn((B, N, H, d), generator=gen).cuda() for _ in range(3)]
        wdirs = [torch.randn(ws[0].shape, generator=gen).cuda() for _ in range(2)]
        plus = value([t + h * v for t, v in zip(x, dirs)], [ws[i] + h * wdirs[i] for i in range(2)])
        minus = value([t - h * v for t, v in zip(x, dirs)], [ws[i] - h * wdirs[i] for i in range(2)])
        terms = [r.double() * v.double() for r, v in zip(res.grads, dirs)] + [res.dweights[i].double() * wdirs[i].double() for i in range(2)]
        want = sum(float(t.sum()) for t in terms)
        size = sum(float((t * t).sum()) for t in terms) ** 0.5
        assert abs((plus - minus) / (2 * h) - want) <= 2e-2 * size, (plus, minus, want, size)


def test_rope_backward_strides_expanded_gradient_and_repeat(svg2):
    B, N, H, d = 2, 15, 4, 128
    x, pos, freq, share, w = _case(torch.bfloat16, B, N, H, d, "token", 13)
    kw = _kw(share, w, "token", "adjacent")
    one = torch.randn((1, 1, H, d), generator=torch.Generator().manual_seed(14)).to(torch.bfloat16).cuda()
    dense = [one.expand(B, N, H, d).contiguous() for _ in range(3)]
    ref = svg2.svg2_rope_backward(dense, x, pos.cuda(), freq.cuda(), **kw)
    packed = torch.zeros((B, N + 2, 3, H, d), dtype=torch.bfloat16, device="cuda")
    outs = [packed[:, 1:N + 1, i] for i in range(3)]
    ws = torch.randint(0, 256, (1 << 20,), dtype=torch.uint8, device="cuda")
    res = svg2.svg2_rope_backward([one.expand(B, N, H, d)] * 3, x, pos.cuda(), freq.cuda(), outs=outs, ws=ws, **kw)
    for i in range(3):
        assert torch.equal(outs[i], ref.grads[i])
    for i in range(2):
        assert torch.equal(res.dweights[i], ref.dweights[i])            # a fixed order of summation
    assert bool((packed[:, 0] == 0).all()) and bool((packed[:, -1] == 0).all())


def test_rope_in_a_graph_and_on_another_stream(svg2):
    B, N, H, d = 1, 70, 5, 128
    x, pos, freq, share, w = _case(torch.bfloat16, B, N, H, d, "token", 15)
    x2, _, _, _, _ = _case(torch.bfloat16, B, N, H, d, "token", 16)
    pos, freq = pos.cuda(), freq.cuda()
    kw = _kw(share, w, "token", "halves")
    outs = [torch.empty((B, N, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    grads = [torch.randn((H, N, d), generator=torch.Generator().manual_seed(17)).to(torch.bfloat16).cuda() for _ in range(3)]
    static = [t.clone() for t in x]
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def both(xs):
        svg2.svg2_rope(xs, pos, freq, outs=outs, **kw)
        return svg2.svg2_rope_backward(grads, xs, pos, freq, ws=ws, **kw)
    refs = []
    for xs in (x, x2):
        r = both([t.contiguous() for t in xs])
        torch.cuda.synchronize()
        refs.append(([o.clone() for o in outs], r))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = both(static)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, refs[0][0])) and torch.equal(r.dweights[0], refs[0][1].dweights[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r = both(static)
    for rep in range(4):
        xs, ref = (x, refs[0]) if rep % 2 == 0 else (x2, refs[1])
        for s, t in zip(static, xs):
            s.copy_(t)
        for o in outs:
            o.zero_()
        ws.random_(0, 256)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, ref[0]))
        assert all(torch.equal(a, b) for a, b in zip(r.grads, ref[1].grads))
        assert all(torch.equal(r.dweights[i], ref[1].dweights[i]) for i in range(2))


def test_rope_helpers(svg2):
    pos = svg2.svg2_grid_positions((2, 3, 2), first=(4, 0, 1), extra=2)
    assert pos.dtype == torch.int32 and pos.shape == (14, 3)
    assert pos[0].tolist() == [4, 0, 1] and pos[5].tolist() == [4, 2, 2] and pos[11].tolist() == [5, 2, 2] and pos[13].tolist() == [0, 0, 0]
    f = svg2.svg2_rope_frequencies((22, 21, 21))
    assert f.dtype == torch.float64 and f.shape == (64,)
    assert f[0] == 1 and f[22] == 1 and abs(float(f[23]) - 10000.0 ** (-1 / 21)) < 1e-15
