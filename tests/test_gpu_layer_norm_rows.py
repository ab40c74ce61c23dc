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
