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
