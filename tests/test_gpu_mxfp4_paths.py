"""The tiled MXFP4 product on every path that its plan takes: three sizes of tiles, one part of the contraction or several, one tile a
workgroup or more of them, the last stage of 256 columns or 128.  Sums are exact in fp32, so every result is compared bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def svg2():
    import paper_2505_18875_amd as pkg
    pkg.load_library()
    assert torch.cuda.is_available()
    yield pkg
    torch.cuda.empty_cache()


def small_operand(R, nk, seed):
    """Values of 0 to 1.5 in halves, with a sign, at block scales of 1 and 2."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (R, nk * 64), dtype=torch.uint8, device="cuda", generator=g) & 0xBB      # bits 0, 1 and the sign of both halves
    scales = 127 + torch.randint(0, 2, (nk, R, 4), dtype=torch.uint8, device="cuda", generator=g)
    return codes, scales


# M, N, columns; behind it the tiles that product_plan gives it, the parts, and the most tiles that a workgroup goes through
PATHS = [(18, 16, 131),             # 64 x 64
         (17, 17, 70),              # the same, a single stage of 128 columns
         (33227, 151, 132),         # 64 x 64, two tiles for some workgroups
         (35675, 129, 69),
         (75600, 64, 8192),         # the same, 32 stages
         (19, 16, 4769),            # 64 x 64, 4 parts
         (19, 17, 4910),            # 5 parts, the last with 128 columns more
         (20, 17, 5248),            # 5 parts, the last of 128 columns only
         (24900, 17, 17579),        # 64 x 64, 5 parts, two tiles, of different parts for some workgroups
         (24735, 16, 14939),
         (35701, 65, 129),          # 128 x 128
         (33257, 67, 70),
         (22517, 556, 131),         # two tiles
         (39806, 259, 67),
         (65, 3669, 15821),         # 8 parts
         (4109, 65, 12043),         # 7 parts
         (3480, 69, 15974),         # 9 parts
         (2000, 70, 38528),         # 16 parts, the last of 128 columns only
         (35601, 66, 16112),        # 3 parts, two tiles, of different parts for some workgroups
         (34164, 74, 17410),
         (17048, 67, 66971),        # 7 parts, the same
         (28433, 387, 135),         # 256 x 256
         (7809, 1542, 64),
         (17317, 1455, 129),        # two tiles
         (17128, 1410, 66),
         (11530, 136, 23434),       # 5 parts
         (8464, 129, 23046),        # 7 parts
         (8372, 141, 27104),        # 7 parts, the last shorter
         (16520, 393, 33520),       # 3 parts, two tiles, of different parts for some workgroups
         (13210, 530, 29777)]


@pytest.mark.parametrize("M,N,K", PATHS)
def test_product_on_every_path(svg2, M, N, K):
    """Products are multiples of 1/4 of size 9 at most: sums of up to 2^16 of them stay below 2^22 quarters, exact in fp32 in any order."""
    nk = -(-K // 128)
    assert 36 * nk * 128 + 4 * 64 < 2 ** 24
    a, sa = small_operand(M, nk, M)
    b, sb = small_operand(N, nk, N + 1)
    bias = torch.randint(-256, 257, (N,), generator=torch.Generator().manual_seed(K)).cuda().float() / 4
    ref = torch.matmul(svg2.svg2_dequantize_mxfp4(a, sa, dtype=torch.float32).double(),
                       svg2.svg2_dequantize_mxfp4(b, sb, dtype=torch.float32).double().t().contiguous()).float()
    need = svg2.load_library().svg2_matmul_mxfp4_workspace_size(M, N, nk * 128)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")            # NaN, where a part is read before it is written
    got = svg2.svg2_matmul_mxfp4(a, sa, b, sb, out_dtype=torch.float32, ws=ws)
    assert bool((got == ref).all())
    # with a bias and rounded, into a slice of a wider result
    wide = torch.full((M, N + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    svg2.svg2_matmul_mxfp4(a, sa, b, sb, bias=bias, out=wide[:, 2:2 + N], ws=ws)
    assert bool((wide[:, 2:2 + N] == (ref + bias).to(torch.bfloat16)).all())
    assert bool((wide[:, :2] == 7).all()) and bool((wide[:, 2 + N:] == 7).all())
    # a block of NaN in the last columns of one row of A and in the first of one of B: that row and that column, and nothing else
    sa[-1, M // 2, 1] = 255
    sb[0, N // 3, 2] = 255
    svg2.svg2_matmul_mxfp4(a, sa, b, sb, out=got, ws=ws)
    assert bool(got[M // 2].isnan().all()) and bool(got[:, N // 3].isnan().all())
    got[M // 2], got[:, N // 3] = ref[M // 2], ref[:, N // 3]
    assert bool((got == ref).all())


# both sides of the borders of the kernel for few rows: 4 rows and 10 * 2^24 weights, 16 rows and 5 * 2^24, rows of 2^14 and 4096 of them
@pytest.mark.parametrize("M,N,K", [(1, 20480, 8192), (4, 20480, 8192), (4, 20481, 8192), (3, 18431, 5376), (2, 300, 400000), (4, 400, 500000),
                                   (4, 4096, 16512), (4, 4095, 16512), (16, 4095, 16384), (16, 97, 16512),
                                   (5, 16384, 5120), (5, 16385, 5120), (16, 8192, 10240), (16, 8192, 10368), (17, 8192, 2048)])
def test_product_of_few_rows_beside_its_borders(svg2, M, N, K):
    """Rows of ones and of twos, and weights of 0 to 1.5 in halves at scale 1: sums of up to 500,096 halves of at most 6, exact in fp32."""
    nk = -(-K // 128)
    assert 6 * nk * 128 < 2 ** 24
    b, sb = small_operand(N, nk, 5)
    sb.fill_(127)
    a = torch.full((M, nk * 64), 0x22, dtype=torch.uint8, device="cuda")
    sa = torch.full((nk, M, 4), 127, dtype=torch.uint8, device="cuda")
    sa[:, M // 2] = 128
    sums = torch.zeros((N,), dtype=torch.float64, device="cuda")
    for n0 in range(0, N, 2048):
        sums[n0:n0 + 2048] = svg2.svg2_dequantize_mxfp4(b[n0:n0 + 2048], sb[:, n0:n0 + 2048].clone(), dtype=torch.float32).double().sum(1)
    got = svg2.svg2_matmul_mxfp4(a, sa, b, sb, out_dtype=torch.float32)
    for m in range(M):
        assert bool((got[m].double() == (2 if m == M // 2 else 1) * sums).all()), m


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_takes_any_view_with_contiguous_groups(svg2, dtype, transposed):
    """Rows that are one row, a transposed matrix as groups of one column, windows that overlap, one row, one column: as their dense copies."""
    g = torch.Generator().manual_seed(9)
    base = torch.randn((300, 517), generator=g).to(dtype).cuda()
    views = [base[7].expand(130, 517),                              # stride 0
             base.t().unsqueeze(-1),                                # [517, 300, 1]: any matrix, a column a group
             base.as_strided((90, 300), (7, 1), 3),                 # rows that overlap
             base.as_strided((40, 11, 33), (517, 64, 1), 1),        # groups with gaps, off every alignment
             base[:1], base[:, 3:4], base[5:6, 5:6]]
    for v in views:
        dense = v.contiguous().reshape(v.shape[0], -1)
        got, ref = svg2.svg2_quantize_mxfp4(v, transposed=transposed), svg2.svg2_quantize_mxfp4(dense, transposed=transposed)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1]), (v.shape, v.stride())


def test_an_operand_times_itself_and_two_streams(svg2):
    """A and B may be one operand; products on two streams share operands but not workspaces."""
    a, sa = small_operand(300, 160, 3)
    v = svg2.svg2_dequantize_mxfp4(a, sa, dtype=torch.float32).double()
    ref = torch.matmul(v, v.t().contiguous()).float()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(svg2.svg2_matmul_mxfp4(a, sa, a, sa, out_dtype=torch.float32))
    torch.cuda.synchronize()
    assert all(bool((o == ref).all()) for o in outs)
