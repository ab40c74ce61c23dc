"""What svg2_rope* and svg2_*_mxfp4 refuse, before anything is launched (no GPU needed), and what their size queries say."""
import ctypes
import os

import numpy as np
import pytest
import torch

import _operators as ops


@pytest.fixture(scope="module")
def lib():
    from paper_2505_18875_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.load_library()


class _RopeArgs(ctypes.Structure):
    """svg2_rope_args of include/svg2.h"""
    _fields_ = [("n_tensors", ctypes.c_int), ("dtype", ctypes.c_int), ("B", ctypes.c_int), ("N", ctypes.c_int),
                ("H", ctypes.c_int), ("d", ctypes.c_int), ("src", ctypes.c_void_p * 3), ("dst", ctypes.c_void_p * 3),
                ("rotate", ctypes.c_int * 3), ("norm_weight", ctypes.c_void_p * 3), ("src_stride", ctypes.c_int64 * 3),
                ("dst_stride", ctypes.c_int64 * 3), ("pos", ctypes.c_void_p), ("pos_stride_b", ctypes.c_int64),
                ("freq", ctypes.c_void_p), ("n_axes", ctypes.c_int), ("axis_pairs", ctypes.c_int * 4),
                ("pairing", ctypes.c_int), ("norm_scope", ctypes.c_int), ("eps", ctypes.c_float)]


def test_the_binding_packs_the_struct_as_c_does():
    from paper_2505_18875_amd.binding import _ROPE_ARGS
    values = list(range(1, 36))
    packed = _ROPE_ARGS.pack(*values[:-1], 0.5)
    assert len(packed) == ctypes.sizeof(_RopeArgs)
    a = _RopeArgs.from_buffer_copy(packed)
    flat = []
    for name, _ in _RopeArgs._fields_:
        v = getattr(a, name)
        flat += list(v) if hasattr(v, "__len__") else [v]
    assert flat[:-1] == values[:-1] and flat[-1] == 0.5


def _args(**change):
    a = _RopeArgs()
    a.n_tensors, a.dtype, a.B, a.N, a.H, a.d = 2, 1, 2, 8, 4, 64
    a.src = (ctypes.c_void_p * 3)(1 << 20, 2 << 20, 3 << 20)
    a.dst = (ctypes.c_void_p * 3)(4 << 20, 5 << 20, 6 << 20)
    a.rotate = (ctypes.c_int * 3)(1, 1, 0)
    a.src_stride = (ctypes.c_int64 * 3)(8 * 256, 256, 64)
    a.dst_stride = (ctypes.c_int64 * 3)(4 * 8 * 64, 64, 8 * 64)
    a.pos, a.freq, a.n_axes, a.axis_pairs = 256, 256, 3, (ctypes.c_int * 4)(12, 10, 10, 0)
    a.eps = 1e-6
    for k, v in change.items():
        if k == "norm":
            a.norm_weight = (ctypes.c_void_p * 3)(*v)
        elif isinstance(v, (tuple, list)):
            arr = getattr(a, k)
            for i, x in enumerate(v):
                arr[i] = x
        else:
            setattr(a, k, v)
    return a


REFUSED = [
    (dict(n_tensors=0), 1, b"n_tensors"), (dict(n_tensors=4), 1, b"n_tensors"), (dict(dtype=5), 2, b"dtype"), (dict(d=96), 2, b"head dimension"),
    (dict(B=0), 1, b"B = 0"), (dict(N=0), 1, b"N = 0"), (dict(H=0), 1, b"H = 0"), (dict(B=1 << 14, N=1 << 13), 1, b"2^26"),
    (dict(pairing=2), 1, b"pairing"), (dict(norm_scope=-1), 1, b"norm_scope"), (dict(n_axes=0), 1, b"n_axes"), (dict(n_axes=5), 1, b"n_axes"),
    (dict(rotate=(0, 0, 0), n_axes=5), 1, b"n_axes"), (dict(rotate=(0, 0, 0), n_axes=-1), 1, b"n_axes"),
    (dict(axis_pairs=(12, 10, 9)), 1, b"pairs"), (dict(axis_pairs=(42, -10, 0)), 1, b"negative"), (dict(pos=None), 1, b"pos and freq"),
    (dict(freq=None), 1, b"pos and freq"), (dict(src_stride=(2048, 252, 64)), 1, b"src stride"), (dict(pos_stride_b=-1), 1, b"pos_stride_b"),
    (dict(norm=(8, None, None)), 1, b"norm_weight[0]"), (dict(norm=(256, None, None), eps=0.0), 1, b"eps"),
    (dict(norm=(256, None, None), eps=float("nan")), 1, b"eps"), (dict(norm=(256, None, None), eps=float("inf")), 1, b"eps"),
]
FORWARD_ONLY = [
    (dict(dst_stride=(2048, 64, 0)), 1, b"positive"), (dict(dst_stride=(2048, 60, 512)), 1, b"dst stride"), (dict(src=(None,)), 1, b"null"),
    (dict(dst=(None,)), 1, b"null"), (dict(src=((1 << 20) + 8,)), 1, b"16-byte"), (dict(dst=(1 << 20,)), 1, b"other strides"),
    (dict(dst=(2 << 20,)), 1, b"alias"), (dict(dst=(5 << 20,)), 1, b"alias"),
]


@pytest.mark.parametrize("change,code,word", REFUSED + FORWARD_ONLY)
def test_rope_refuses(lib, change, code, word):
    a = _args(**change)
    assert lib.svg2_rope(ctypes.addressof(a), None) == code
    assert word in lib.svg2_last_error(), lib.svg2_last_error()


def _backward(lib, a, dY=(7 << 20, 8 << 20, 9 << 20), dX=(10 << 20, 11 << 20, 12 << 20), dW=(256, 512, None), stride=(2048, 256, 64),
              ws=256, ws_bytes=1 << 40):
    v3 = lambda t: (ctypes.c_void_p * 3)(*t)    # noqa: E731
    return lib.svg2_rope_backward(ctypes.addressof(a), v3(dY), v3(dX), (ctypes.c_int64 * 3)(*stride), v3(dW), ws, ws_bytes, None)


@pytest.mark.parametrize("change,code,word", REFUSED)
def test_rope_backward_refuses(lib, change, code, word):
    a = _args(**change)
    assert _backward(lib, a) == code
    assert word in lib.svg2_last_error(), lib.svg2_last_error()
    assert lib.svg2_rope_backward_workspace_size(ctypes.addressof(a)) == 256


def test_rope_backward_refuses_its_own_arguments(lib):
    normed = dict(norm=(1024, 2048, None))
    a = _args(**normed)
    for kw, code, word in ((dict(dX=(None, 1 << 20, None)), 1, b"null"), (dict(dY=(None, 1 << 20, None)), 1, b"null"),
                           (dict(dX=(8, 1 << 24, None)), 1, b"16-byte"), (dict(dW=(None, 512, None)), 1, b"dW[0]"),
                           (dict(dW=(512, 512, None)), 1, b"alias"), (dict(dX=(10 << 20, 10 << 20, None)), 1, b"alias"),
                           (dict(dX=(7 << 20, 11 << 20, None)), 1, b"alias"), (dict(dX=(2 << 20, 11 << 20, None)), 1, b"alias"),
                           (dict(stride=(2048, 0, 64)), 1, b"positive"), (dict(ws=None), 1, b"workspace"), (dict(ws=8), 1, b"aligned"),
                           (dict(ws_bytes=16), 3, b"workspace")):
        assert _backward(lib, a, **kw) == code, kw
        assert word in lib.svg2_last_error(), (kw, lib.svg2_last_error())
    a = _args(src=(None,), **normed)
    assert _backward(lib, a) == 1 and b"src[0]" in lib.svg2_last_error()
    assert lib.svg2_rope(None, None) == 1


def test_rope_backward_workspace_sizes(lib):
    def size(**kw):
        a = _args(**kw)
        return lib.svg2_rope_backward_workspace_size(ctypes.addressof(a))
    assert size() == 256
    assert size(norm=(256, None, None)) >= 3 * 2 * 64 * 4                       # two groups of tokens, [d] sums
    assert size(norm=(256, None, None), norm_scope=1) >= 3 * 2 * 256 * 4
    long_tokens = size(norm=(256, None, None), norm_scope=1, H=5000)            # stays bounded for long tokens
    assert 3 * 16 * 4 < long_tokens < 1 << 30


def test_quantize_mxfp4_refuses(lib):
    ok = (1 << 20, 1, 4, 1, 64, 64, 64, 0, 2 << 20, 3 << 20, None)
    for at, v, code, word in ((0, None, 1, b"null"), (0, (1 << 20) + 1, 1, b"aligned"), (1, 3, 2, b"dtype"), (2, 0, 1, b"rows"), (3, 0, 1, b"G = 0"),
                              (4, 0, 1, b"Kg = 0"), (4, (1 << 26) + 1, 1, b"columns"), (8, None, 1, b"null"), (9, (3 << 20) + 8, 1, b"16-byte"),
                              (8, 1 << 20, 1, b"alias"), (2, (1 << 26) + 1, 1, b"rows")):
        args = list(ok)
        args[at] = v
        assert lib.svg2_quantize_mxfp4(*args) == code, (at, v)
        assert word in lib.svg2_last_error(), (at, v, lib.svg2_last_error())
    # 65536 groups of 65536 columns: 2^32 columns
    assert lib.svg2_quantize_mxfp4(1 << 20, 1, 4, 65536, 65536, 64, 64, 0, 2 << 20, 3 << 20, None) == 1


def test_dequantize_mxfp4_refuses(lib):
    ok = (1 << 20, 2 << 20, 4, 64, 1, 3 << 20, 64, None)
    for at, v, code, word in ((0, None, 1, b"null"), (1, 8, 1, b"16-byte"), (2, 0, 1, b"rows"), (3, -1, 1, b"columns"), (4, 2, 2, b"dtype"),
                              (5, None, 1, b"null"), (5, (3 << 20) + 1, 1, b"aligned"), (6, 63, 1, b"ldx"), (5, 1 << 20, 1, b"alias")):
        args = list(ok)
        args[at] = v
        assert lib.svg2_dequantize_mxfp4(*args) == code, (at, v)
        assert word in lib.svg2_last_error(), (at, v, lib.svg2_last_error())


def test_matmul_mxfp4_refuses(lib):
    ok = (1 << 20, 2 << 20, 3 << 20, 4 << 20, 128, 256, 512, None, 1, 5 << 20, 256, 256, 1 << 40, None)
    for at, v, code, word in ((0, None, 1, b"A:"), (1, None, 1, b"A:"), (2, 8, 1, b"B:"), (3, None, 1, b"B:"), (4, 0, 1, b"rows"), (5, -3, 1, b"rows"),
                              (6, 0, 1, b"columns"), (6, (1 << 24) + 1, 1, b"2^24"), (7, 2, 1, b"aligned"), (8, 9, 2, b"dtype"), (9, None, 1, b"null"),
                              (9, (5 << 20) + 1, 1, b"aligned"), (10, 255, 1, b"ldc"), (9, 1 << 20, 1, b"alias"), (11, 8, 1, b"aligned"),
                              (12, 16, 3, b"workspace")):
        args = list(ok)
        args[at] = v
        assert lib.svg2_matmul_mxfp4(*args) == code, (at, v)
        assert word in lib.svg2_last_error(), (at, v, lib.svg2_last_error())
    assert lib.svg2_matmul_mxfp4(1 << 20, 2 << 20, 3 << 20, 4 << 20, 1 << 21, 1 << 21, 512, None, 1, 5 << 20, 1 << 21, None, 0, None) == 1
    assert b"tiles" in lib.svg2_last_error()
    # a long contraction of few tiles needs a workspace, an ordinary product none
    size = lib.svg2_matmul_mxfp4_workspace_size
    assert size(75600, 5120, 5120) == 256 and size(1, 15360, 5120) == 256 and size(0, 4, 4) == 256 and size(4, 4, 1 << 25) == 256
    need = size(512, 512, 65536)
    assert need >= 2 * 512 * 512 * 4
    args = [1 << 20, 2 << 20, 3 << 20, 4 << 20, 512, 512, 65536, None, 1, 5 << 20, 512, None, 0, None]
    assert lib.svg2_matmul_mxfp4(*args) == 1 and b"workspace" in lib.svg2_last_error()
    args[11:13] = [6 << 20, need - 1]
    assert lib.svg2_matmul_mxfp4(*args) == 3 and b"workspace" in lib.svg2_last_error()
    args[11:13] = [5 << 20, need]
    assert lib.svg2_matmul_mxfp4(*args) == 1 and b"alias" in lib.svg2_last_error()


def test_bindings_refuse(lib):
    import paper_2505_18875_amd as svg2
    x = torch.zeros((8, 2, 64))
    with pytest.raises(ValueError):
        svg2.svg2_rope([x], torch.zeros((8, 3), dtype=torch.int32), torch.zeros(32, dtype=torch.float64), axis_pairs=(12, 10, 10))
    with pytest.raises(ValueError):
        svg2.svg2_rope([x] * 4)
    with pytest.raises(ValueError):
        svg2.svg2_quantize_mxfp4(torch.zeros((4, 64)))
    with pytest.raises(ValueError):
        svg2.svg2_matmul_mxfp4(torch.zeros((4, 60), dtype=torch.uint8), torch.zeros((1, 4, 4), dtype=torch.uint8),
                               torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((1, 4, 4), dtype=torch.uint8))


def test_plain_forms_agree_with_themselves():
    """The 64-bit forms that the GPU tests measure against: quantising its own values changes nothing, every E2M1 number is kept, and
    a rotation back undoes a rotation."""
    r = np.random.default_rng(0)
    x = r.standard_normal((5, 200)) * 2.0 ** r.integers(-20, 20, size=(5, 1))
    c, s = ops.quantize(x)
    v = ops.values(c, s)
    c2, s2 = ops.quantize(v)
    assert np.array_equal(ops.values(c2, s2), v)
    assert np.abs(v[:, :200] - x).max(1).max() <= np.abs(x).max() / 4
    block = np.concatenate([ops.E2M1, -ops.E2M1, ops.E2M1, -ops.E2M1])[None]
    assert np.array_equal(ops.values(*ops.quantize(block))[:, :32], block)
    q = r.standard_normal((1, 3, 2, 64))
    a = ops.angles(r.integers(-1000, 1000, size=(1, 3, 3)), r.random(32), (12, 10, 10))
    for pairing in ("adjacent", "halves"):
        assert np.allclose(ops.turn(ops.turn(q, a, pairing), a, pairing, -1.0), q, atol=1e-12)
