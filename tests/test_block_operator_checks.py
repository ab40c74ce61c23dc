"""What svg2_layer_norm* and svg2_*_fp8_blocks refuse, before anything is launched (no GPU needed), and what their size queries say."""
import ctypes
import os

import numpy as np
import pytest
import torch

import _block_operators as ops


@pytest.fixture(scope="module")
def lib():
    from paper_2505_18875_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.load_library()


class _NormArgs(ctypes.Structure):
    """svg2_layer_norm_args of include/svg2.h"""
    _fields_ = [("dtype", ctypes.c_int), ("y_dtype", ctypes.c_int), ("B", ctypes.c_int), ("N", ctypes.c_int), ("D", ctypes.c_int),
                ("x", ctypes.c_void_p), ("x_stride", ctypes.c_int64 * 2), ("weight", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("weight_stride", ctypes.c_int64), ("bias_stride", ctypes.c_int64), ("one_plus", ctypes.c_int), ("eps", ctypes.c_float),
                ("y", ctypes.c_void_p), ("y_stride", ctypes.c_int64 * 2)]


def test_the_binding_packs_the_struct_as_c_does():
    from paper_2505_18875_amd.binding import _NORM_ARGS
    values = [*range(1, 14), 0.5, 14, 15, 16]
    packed = _NORM_ARGS.pack(*values)
    assert len(packed) == ctypes.sizeof(_NormArgs)
    a, flat = _NormArgs.from_buffer_copy(packed), []
    for name, _ in _NormArgs._fields_:
        v = getattr(a, name)
        flat += list(v) if hasattr(v, "__len__") else [v]
    assert flat == values


def _args(**change):
    a = _NormArgs(1, 1, 2, 8, 100, 1 << 20, (ctypes.c_int64 * 2)(800, 100), 2 << 20, 3 << 20, 100, 100, 1, 1e-6, 4 << 20,
                  (ctypes.c_int64 * 2)(800, 100))
    for k, v in change.items():
        setattr(a, k, (ctypes.c_int64 * 2)(*v) if isinstance(v, tuple) else v)
    return a


REFUSED = [
    (dict(dtype=5), 2, b"dtype"), (dict(B=0), 1, b"B = 0"), (dict(N=0), 1, b"N = 0"), (dict(N=-1), 1, b"N = -1"), (dict(D=0), 1, b"D = 0"),
    (dict(D=16385), 1, b"16384"), (dict(B=1 << 14, N=1 << 13), 1, b"2^26"), (dict(eps=0.0), 1, b"eps"), (dict(eps=float("nan")), 1, b"eps"),
    (dict(eps=float("inf")), 1, b"eps"), (dict(eps=-1.0), 1, b"eps"), (dict(weight=(2 << 20) + 2), 1, b"aligned"),
    (dict(bias=(3 << 20) + 1), 1, b"aligned"), (dict(x=None), 1, b"null"), (dict(x=(1 << 20) + 1), 1, b"aligned"),
]
FORWARD_ONLY = [
    (dict(y_dtype=2), 2, b"dtype"), (dict(y=None), 1, b"null"), (dict(y=(4 << 20) + 1), 1, b"aligned"), (dict(y=(4 << 20) + 2, y_dtype=0), 1, b"aligned"),
    (dict(y_stride=(0, 100)), 1, b"positive"), (dict(y_stride=(800, -100)), 1, b"positive"), (dict(y=1 << 20, y_stride=(900, 100)), 1, b"other strides"),
    (dict(y=1 << 20, y_dtype=0), 1, b"another type"), (dict(y=2 << 20), 1, b"alias"), (dict(y=3 << 20), 1, b"alias"),
]


@pytest.mark.parametrize("change,code,word", REFUSED + FORWARD_ONLY)
def test_layer_norm_refuses(lib, change, code, word):
    a = _args(**change)
    assert lib.svg2_layer_norm(ctypes.addressof(a), None) == code
    assert word in lib.svg2_last_error(), lib.svg2_last_error()


@pytest.mark.parametrize("change,code,word", REFUSED)
def test_layer_norm_fp8_refuses(lib, change, code, word):
    a = _args(**change)
    assert lib.svg2_layer_norm_fp8(ctypes.addressof(a), 5 << 20, 6 << 20, None) == code
    assert word in lib.svg2_last_error(), lib.svg2_last_error()


def test_layer_norm_fp8_refuses_its_own_arguments(lib):
    a = _args(y=None, y_dtype=7, y_stride=(0, 0))               # ignored
    for codes, scales, word in ((None, 6 << 20, b"null"), (5 << 20, None, b"null"), ((5 << 20) + 8, 6 << 20, b"16-byte"), (5 << 20, 6, b"16-byte"),
                                (5 << 20, 5 << 20, b"alias"), (1 << 20, 6 << 20, b"alias"), (5 << 20, 2 << 20, b"alias"), (3 << 20, 6 << 20, b"alias")):
        assert lib.svg2_layer_norm_fp8(ctypes.addressof(a), codes, scales, None) == 1
        assert word in lib.svg2_last_error(), lib.svg2_last_error()
    assert lib.svg2_layer_norm(None, None) == 1 and lib.svg2_layer_norm_fp8(None, 256, 512, None) == 1


def _backward(lib, a, dY=7 << 20, dX=8 << 20, stride=(800, 100), dW=9 << 20, dB=10 << 20, ws=11 << 20, ws_bytes=1 << 40):
    return lib.svg2_layer_norm_backward(ctypes.addressof(a), dY, dX, (ctypes.c_int64 * 2)(*stride) if stride else None, dW, dB, ws, ws_bytes, None)


@pytest.mark.parametrize("change,code,word", REFUSED + [(dict(y_dtype=2), 2, b"dtype"), (dict(weight=None), 1, b"weight is null"), (dict(bias=None), 1, b"bias"),
                                                        (dict(weight_stride=0), 1, b"both"), (dict(bias_stride=0), 1, b"both")])
def test_layer_norm_backward_refuses(lib, change, code, word):
    a = _args(**change)
    assert _backward(lib, a) == code
    assert word in lib.svg2_last_error(), lib.svg2_last_error()


def test_layer_norm_backward_refuses_its_own_arguments(lib):
    a = _args(B=2, N=4000)
    need = lib.svg2_layer_norm_backward_workspace_size(ctypes.addressof(a))
    assert need > 256
    for kw, code, word in ((dict(dY=None), 1, b"null"), (dict(dX=None), 1, b"null"), (dict(stride=None), 1, b"null"), (dict(dY=3), 1, b"aligned"),
                           (dict(dX=(8 << 20) + 1), 1, b"aligned"), (dict(dW=(9 << 20) + 2), 1, b"aligned"), (dict(dB=2), 1, b"aligned"),
                           (dict(stride=(0, 100)), 1, b"positive"), (dict(dX=1 << 20), 1, b"alias"), (dict(dX=7 << 20, stride=(900, 100)), 1, b"other strides"),
                           (dict(dW=10 << 20), 1, b"alias"), (dict(dB=8 << 20), 1, b"alias"), (dict(dW=2 << 20), 1, b"alias"), (dict(dB=7 << 20), 1, b"alias"),
                           (dict(ws=None), 1, b"workspace"), (dict(ws=8), 1, b"aligned"), (dict(ws_bytes=need - 1), 3, b"workspace"),
                           (dict(ws=8 << 20), 1, b"alias")):
        assert _backward(lib, a, **kw) == code, kw
        assert word in lib.svg2_last_error(), (kw, lib.svg2_last_error())


def test_layer_norm_backward_workspace_sizes(lib):
    def size(**kw):
        a = _args(**kw)
        return lib.svg2_layer_norm_backward_workspace_size(ctypes.addressof(a))
    assert size(B=1, N=1) == 256 and size(B=1000, N=3) == 256 and size(D=0) == 256
    shared = dict(weight_stride=0, bias_stride=0)
    assert size(B=1, N=75600, weight=None, bias=None) == 256    # nothing to add up
    assert size(B=1000, N=3, **shared) > 256                    # 3000 rows that share one sum
    assert 2 * 2 * 100 * 4 < size(B=1, N=75600, D=100) < 1 << 23
    assert size(B=2, N=1 << 24, D=16384) < 1 << 28              # stays bounded


def test_quantize_fp8_blocks_refuses(lib):
    ok = (1 << 20, 1, 4, 1, 64, 64, 64, 0, 2 << 20, 3 << 20, 4 << 20, 5 << 20, None)
    for at, v, code, word in ((0, None, 1, b"null"), (0, (1 << 20) + 1, 1, b"aligned"), (1, 3, 2, b"dtype"), (2, 0, 1, b"rows"), (3, 0, 1, b"G = 0"),
                              (4, 0, 1, b"Kg = 0"), (4, (1 << 26) + 1, 1, b"columns"), (8, None, 1, b"null"), (9, None, 1, b"null"),
                              (9, (3 << 20) + 8, 1, b"16-byte"), (10, None, 1, b"transposed"), (11, None, 1, b"transposed"), (10, 8, 1, b"16-byte"),
                              (8, 1 << 20, 1, b"alias"), (10, 2 << 20, 1, b"alias"), (11, 3 << 20, 1, b"alias"), (2, (1 << 26) + 1, 1, b"rows")):
        args = list(ok)
        args[at] = v
        assert lib.svg2_quantize_fp8_blocks(*args) == code, (at, v)
        assert word in lib.svg2_last_error(), (at, v, lib.svg2_last_error())
    args = list(ok)
    args[8:12] = [None] * 4
    assert lib.svg2_quantize_fp8_blocks(*args) == 1 and b"no result" in lib.svg2_last_error()
    args = list(ok)
    args[2], args[4] = 1 << 20, 1 << 20
    assert lib.svg2_quantize_fp8_blocks(*args) == 1 and b"2^40" in lib.svg2_last_error()


def test_dequantize_fp8_blocks_refuses(lib):
    ok = (1 << 20, 2 << 20, 4, 64, 1, 3 << 20, 64, None)
    for at, v, code, word in ((0, None, 1, b"null"), (1, 8, 1, b"16-byte"), (2, 0, 1, b"rows"), (3, -1, 1, b"columns"), (4, 2, 2, b"dtype"),
                              (5, None, 1, b"null"), (5, (3 << 20) + 1, 1, b"aligned"), (6, 63, 1, b"ldx"), (5, 1 << 20, 1, b"alias")):
        args = list(ok)
        args[at] = v
        assert lib.svg2_dequantize_fp8_blocks(*args) == code, (at, v)
        assert word in lib.svg2_last_error(), (at, v, lib.svg2_last_error())


def test_matmul_fp8_blocks_refuses(lib):
    ok = (1 << 20, 2 << 20, 3 << 20, 4 << 20, 128, 256, 512, None, 1, 5 << 20, 256, 256, 1 << 40, None)
    for at, v, code, word in ((0, None, 1, b"A:"), (1, None, 1, b"A:"), (2, 8, 1, b"B:"), (3, None, 1, b"B:"), (4, 0, 1, b"rows"), (5, -3, 1, b"rows"),
                              (6, 0, 1, b"columns"), (6, (1 << 24) + 1, 1, b"2^24"), (7, 2, 1, b"aligned"), (8, 9, 2, b"dtype"), (9, None, 1, b"null"),
                              (9, (5 << 20) + 1, 1, b"aligned"), (10, 255, 1, b"ldc"), (9, 1 << 20, 1, b"alias"), (11, 8, 1, b"aligned"),
                              (12, 16, 3, b"workspace")):
        args = list(ok)
        args[at] = v
        assert lib.svg2_matmul_fp8_blocks(*args) == code, (at, v)
        assert word in lib.svg2_last_error(), (at, v, lib.svg2_last_error())
    assert lib.svg2_matmul_fp8_blocks(1 << 20, 2 << 20, 3 << 20, 4 << 20, 1 << 21, 1 << 21, 512, None, 1, 5 << 20, 1 << 21, None, 0, None) == 1
    assert b"tiles" in lib.svg2_last_error()
    size = lib.svg2_matmul_fp8_blocks_workspace_size
    assert size(75600, 5120, 5120) == 256 and size(1, 15360, 5120) == 256 and size(0, 4, 4) == 256 and size(4, 4, 1 << 25) == 256


def test_bindings_refuse(lib):
    import paper_2505_18875_amd as svg2
    x = torch.zeros((8, 128))
    for call in (lambda: svg2.svg2_layer_norm(x), lambda: svg2.svg2_layer_norm_fp8(x), lambda: svg2.svg2_layer_norm_backward(x, x),
                 lambda: svg2.svg2_quantize_fp8_blocks(x), lambda: svg2.svg2_dequantize_fp8_blocks(x.byte(), x.byte()),
                 lambda: svg2.svg2_matmul_fp8_blocks(x.byte(), x.byte(), x.byte(), x.byte())):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_plain_forms_agree_with_themselves():
    """The 64-bit forms that the GPU tests measure against: quantising its own values changes nothing, every E4M3 number is kept, square
    blocks commute with transposing; the norm's gradients against differences."""
    r = np.random.default_rng(0)
    x = r.standard_normal((150, 300)) * 2.0 ** r.integers(-20, 20, size=(150, 1))
    for square in (False, True):
        v = ops.values(*ops.quantize(x, square))
        assert np.array_equal(ops.values(*ops.quantize(v, square)), v)
    top = np.abs(x).max(1, keepdims=True)
    v = ops.values(*ops.quantize(x))[:, :300]
    assert (np.abs(v - x) <= np.maximum(2.0 ** -4 * np.abs(x), top * 2.0 ** -17)).all()
    assert np.array_equal(ops.values(*ops.quantize(x.T, True))[:, :150], ops.values(*ops.quantize(x, True))[:, :300].T)
    block = np.zeros((2, 128))
    block[0, :127], block[1, :127] = ops.E4M3, -ops.E4M3
    assert np.array_equal(ops.values(*ops.quantize(block)), block)
    assert np.array_equal(ops.E4M3, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy())

    B, N, D, eps = 2, 3, 7, 1e-3
    x, dy, w = r.standard_normal((B, N, D)), r.standard_normal((B, N, D)), r.standard_normal((B, D))
    b = r.standard_normal((B, D))
    loss = lambda x, w, b: (ops.layer_norm(x, w, b, eps, True)[0] * dy).sum()       # noqa: E731
    dx, _, dw, _, db, _ = ops.layer_norm_backward(dy, x, w, eps, True)
    h = 1e-6
    for grad, k in ((dx, 0), (dw, 1), (db, 2)):
        args = [x, w, b]
        for i in np.ndindex(*args[k].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[k][i] += h
            down[k][i] -= h
            assert abs((loss(*up) - loss(*down)) / (2 * h) - grad[i]) < 1e-6
