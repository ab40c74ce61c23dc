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
