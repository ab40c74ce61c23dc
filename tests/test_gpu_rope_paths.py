"""svg2_rope and svg2_rope_backward: what is not rotated, and the loops that the shapes of test_gpu_rope.py do not go round."""
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


def _bits(t):
    return t.contiguous().view(torch.int16 if t.dtype is torch.bfloat16 else torch.int32)


# a wavefront for several tokens, one token, a workgroup for one token
@pytest.mark.parametrize("H", [1, 9, 40])
@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_is_not_rotated_keeps_its_bits(svg2, dtype, pairing, H):
    """Tokens at position 0 and pairs of frequency 0 come out as they went in: negative zeros, and numbers whose partner is an
    infinity or a NaN, among them.  Forward, and turned back."""
    N, d = 7, 64
    g = torch.Generator().manual_seed(H)
    x = torch.randn((N, H, d), generator=g).to(dtype)
    i, j = ops.pair_index(d, pairing)
    for k, v in ((0, float("inf")), (3, -float("inf")), (5, float("nan")), (6, -0.0), (20, 0.0), (31, float("inf"))):
        x[:, :, int(i[k])] = v
    x[:, :, int(j[3])] = -0.0
    x[:, :, int(j[9])] = float("nan")
    x = x.cuda()
    pos = torch.zeros((N, 2), dtype=torch.int32)
    pos[2], pos[6] = torch.tensor([3, 5]), torch.tensor([-4, 1])
    still_token = [0, 1, 3, 4, 5]
    freq = 100.0 ** (-torch.arange(d // 2, dtype=torch.float64) / 16)
    still_pair = [3, 5, 6, 9, 20, 31]
    freq[still_pair] = 0.0
    kw = dict(axis_pairs=(20, 12), pairing=pairing)
    y, = svg2.svg2_rope([x], pos.cuda(), freq.cuda(), **kw)
    back = svg2.svg2_rope_backward([x[None]], [x[None]], pos.cuda(), freq.cuda(), **kw).grads[0][0]
    columns = torch.from_numpy(np.concatenate([i[still_pair], j[still_pair]])).cuda()
    moving = np.setdiff1d(np.arange(d // 2), still_pair + [0])
    moving = np.concatenate([i[moving], j[moving]])
    a = ops.angles(pos.numpy()[None], freq.numpy(), (20, 12))
    for got, sense in ((y.transpose(0, 1), 1.0), (back, -1.0)):
        assert torch.equal(_bits(got[still_token]), _bits(x[still_token]))
        assert torch.equal(_bits(got[:, :, columns]), _bits(x[:, :, columns]))
        # the others are rotated: each angle, of size 20 at most, is one 64-bit product, and the rest as in ops.rope
        x64 = x.double().cpu().numpy()[None]
        with np.errstate(invalid="ignore"):
            ref, size = ops.turn(x64, a, pairing, sense), ops.pair_norm(x64, pairing)
        bound = (12 * ops.U + 2.0 ** -51 * 20) * size
        assert_within(got[:, :, moving][None], ref[..., moving], bound[..., moving], dtype)


# a norm over the head goes through the heads 16 (of 128) or 32 (of 64) at a time: one, two and three rounds, the last of them partial;
# fewer tokens than wavefronts and more
HEADS = [(torch.bfloat16, 1, 37, 40, 128), (torch.float32, 2, 19, 17, 128), (torch.float32, 1, 23, 33, 64), (torch.float32, 1, 1, 67, 64),
         (torch.bfloat16, 1, 2111, 40, 128), (torch.float32, 3, 701, 35, 64), (torch.bfloat16, 2, 5, 32, 64), (torch.float32, 1, 11, 16, 128)]


@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("dtype,B,N,H,d", HEADS)
def test_gradients_of_a_norm_over_many_heads(svg2, dtype, B, N, H, d, pairing):
    g = torch.Generator().manual_seed(N + H)
    qk = torch.randn((B, N, 2, H, d), generator=g).to(dtype).cuda()
    x = [qk[:, :, i] for i in range(2)]
    grads = [torch.randn((B * H, N, d), generator=g).to(dtype).cuda() for _ in range(2)]
    w = [1 + 0.3 * torch.randn((d,), generator=g) for _ in range(2)]
    pos = torch.randint(0, 97, (N, 2), generator=g, dtype=torch.int32)
    share = (d // 2 - 11, 11)
    freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in share])
    res = svg2.svg2_rope_backward(grads, x, pos.cuda(), freq.cuda(), axis_pairs=share, norm_weights=[t.cuda() for t in w], pairing=pairing)
    a = ops.angles(pos.numpy()[None], freq.numpy(), share)
    for i in range(2):
        gi = grads[i].view(B, H, N, d).transpose(1, 2)
        dx, bound, dw, dw_bound = ops.rope_backward(gi.double().cpu().numpy(), x[i].double().cpu().numpy(), w[i].double().numpy(), a, "head",
                                                    1e-6, pairing)
        assert_within(res.grads[i], dx, bound, dtype, "dx %d" % i)
        assert_within(res.dweights[i], dw, dw_bound, torch.float32, "dw %d" % i)


@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("scope,H,d", [("head", 3, 64), ("token", 3, 64), ("head", 33, 64), ("token", 17, 128), ("token", 65, 128)])
def test_gradients_are_the_slope_of_the_formula(svg2, scope, H, d, pairing):
    """The gradients, along random directions, against central differences of the formula in 64 bits.  With steps of h = 2^-17 a difference
    is off by a third of what doubling the step changes (its error goes with h^2), and by the rounding of its two values: 16 operations of 2^-53
    of the sum of magnitudes, over h.  The gradients are off by their bounds and one rounding to fp32."""
    N, eps = 7, 1e-6
    g = torch.Generator().manual_seed(H + d)
    x, dy, dir_x = (torch.randn((1, N, H, d), generator=g) for _ in range(3))
    shape = (d,) if scope == "head" else (H, d)
    w, dir_w = 1 + 0.3 * torch.randn(shape, generator=g), torch.randn(shape, generator=g)
    pos = torch.randint(0, 50, (N, 3), generator=g, dtype=torch.int32)
    share = (d // 2 - 20, 10, 10)
    freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in share])
    res = svg2.svg2_rope_backward([dy.cuda()], [x.cuda()], pos.cuda(), freq.cuda(), axis_pairs=share, norm_weights=[w.cuda()], norm_scope=scope,
                                  eps=eps, pairing=pairing)
    a = ops.angles(pos.numpy()[None], freq.numpy(), share)
    x, dy, dir_x, w, dir_w = (t.double().numpy() for t in (x, dy, dir_x, w, dir_w))

    def slope(h):
        y = [ops.rope(x + s * h * dir_x, w + s * h * dir_w, a, scope, eps, pairing)[0] * dy for s in (1, -1)]
        return (y[0].sum() - y[1].sum()) / (2 * h), 16 * 2.0 ** -53 * np.abs(y[0]).sum() / h

    want, rounding = slope(2.0 ** -17)
    twice, _ = slope(2.0 ** -16)
    _, bound, _, dw_bound = ops.rope_backward(dy, x, w, a, scope, eps, pairing)
    dx, dw = (t.double().cpu().numpy() for t in (res.grads[0], res.dweights[0]))
    tol = ((bound + ops.U * np.abs(dx)) * np.abs(dir_x)).sum() + ((dw_bound + ops.U * np.abs(dw)) * np.abs(dir_w)).sum()
    got = (dx * dir_x).sum() + (dw * dir_w).sum()
    assert abs(got - want) <= tol + rounding + abs(twice - want), (got, want, tol, rounding, twice)


# which tensors have a norm, which are rotated; one to three of them; axes without pairs
MIXED = [((None, "w"), (True, False)), (("w", None), (False, True)), (("w",), (False,)), ((None, None, "w"), (True, False, True)),
         (("w", "w", "w"), (False, False, False)), ((None, None), (False, False))]


@pytest.mark.parametrize("scope,H,d", [("head", 5, 64), ("token", 2, 128), ("token", 9, 128), ("token", 33, 128), ("token", 65, 128)])
@pytest.mark.parametrize("normed,rotate", MIXED)
def test_each_tensor_has_its_own_norm_and_rotation(svg2, normed, rotate, scope, H, d):
    B, N, n = 2, 11, len(normed)
    g = torch.Generator().manual_seed(H + n)
    packed = torch.randn((B, N, n, H, d), generator=g).cuda()
    x = [packed[:, :, i] for i in range(n)]
    dy = [torch.randn((B * H, N, d), generator=g).cuda() for _ in range(n)]
    w = [None if k is None else 1 + 0.3 * torch.randn((d,) if scope == "head" else (H, d), generator=g) for k in normed]
    share = (0, d // 2 - 5, 0, 5)
    pos = torch.randint(-60, 60, (B, N, 4), generator=g, dtype=torch.int32)
    freq = 10.0 ** -torch.rand(d // 2, generator=g, dtype=torch.float64)
    kw = dict(axis_pairs=share, rotate=rotate, norm_weights=[None if t is None else t.cuda() for t in w], norm_scope=scope, pairing="halves")
    place = (pos.cuda(), freq.cuda()) if any(rotate) else (None, None)
    out = svg2.svg2_rope(x, *place, **kw)
    res = svg2.svg2_rope_backward(dy, x, *place, **kw)
    angle = ops.angles(pos.numpy(), freq.numpy(), share)
    for i in range(n):
        heads = lambda t: t.view(B, H, N, d).transpose(1, 2)        # noqa: E731
        if w[i] is None and not rotate[i]:
            assert torch.equal(heads(out[i]), x[i]) and torch.equal(res.grads[i], heads(dy[i])) and res.dweights[i] is None
            continue
        x64, g64 = (t.double().cpu().numpy() for t in (x[i], heads(dy[i])))
        w64 = None if w[i] is None else w[i].double().numpy()
        a = angle if rotate[i] else None
        y, bound = ops.rope(x64, w64, a, scope, 1e-6, "halves")
        far = 2.0 ** -51 * 60                                       # an angle is one 64-bit product
        assert_within(heads(out[i]), y, bound + far * ops.pair_norm(y, "halves"), torch.float32, "y %d" % i)
        dx, bound, dw, dw_bound = ops.rope_backward(g64, x64, w64, a, scope, 1e-6, "halves")
        # without a rotation the gradient's own size stands for its pair's: the bound of a rotation is the larger
        assert_within(res.grads[i], dx, bound + far * ops.pair_norm(np.abs(dx), "halves"), torch.float32, "dx %d" % i)
        if w64 is None:
            assert res.dweights[i] is None
        else:
            assert_within(res.dweights[i], dw, dw_bound, torch.float32, "dw %d" % i)
