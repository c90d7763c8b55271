"""Argument checks of the 8-bit products and of what stands between two blocks: host only, nothing is launched."""
import ctypes

import pytest

P, ODD, HALF, NULL = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0x1008), ctypes.c_void_p(0)   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    from paper_1905_05686_b200 import build
    build.build()
    from paper_1905_05686_b200 import binding
    return binding


def refused(lib, f, good, changes):
    before = lib.launch_count()
    for at, value in changes:
        args = list(good)
        args[at] = value
        assert f(*args) == lib.ERR_INVALID_ARG, (at, value)
    assert lib.launch_count() == before


def test_sizes(lib):
    L = lib.lib()
    assert [L.lrbi_i8_pitch(c) for c in (1, 16, 17, 801, 1 << 17, 0, -3, (1 << 17) + 1)] == [16, 16, 32, 816, 1 << 17, 0, 0, 0]
    for rows, cols in ((0, 1), (1, 4096), (4096, 4096), (10 ** 6, 100), (7, 32768), (2 ** 31 - 4096, 32768)):
        n = L.lrbi_residual_norm_backward_workspace(rows, cols)
        assert n >= 16 and n % 16 == 0
    assert [L.lrbi_residual_norm_backward_workspace(*v) for v in ((-1, 4), (4, 0), (4, 32769), (2 ** 31 - 4095, 4))] == [0] * 4


def test_i8_arguments(lib):
    L = lib.lib()
    lay = lib.Layout(64, 96, 16, 32, 4)
    refused(lib, L.lrbi_i8_quantize, [ctypes.byref(lay), P, P, P, P, P, NULL],
            [(0, None), (0, ctypes.byref(lib.Layout(0, 96, 16, 32, 4))), (0, ctypes.byref(lib.Layout(64, (1 << 17) + 1, 16, 32, 4))),
             (0, ctypes.byref(lib.Layout(64, 96, 0, 32, 4))), (0, ctypes.byref(lib.Layout(64, 96, 16, 32, 0))), (1, NULL), (1, ODD), (2, NULL), (3, NULL), (3, ODD),
             (4, NULL), (4, HALF), (5, NULL), (5, ODD)])
    tokens = [P, 0, 64, 4, 64, -1, P, P, NULL]
    refused(lib, L.lrbi_i8_tokens, tokens, [(0, NULL), (0, ODD), (1, 2), (2, 63), (2, -64), (3, -1), (4, 0), (4, (1 << 17) + 1), (5, -2), (5, 3), (6, NULL), (6, HALF),
                                            (7, NULL), (7, ODD)])
    assert L.lrbi_i8_tokens(NULL, 0, 64, 0, 64, -1, NULL, NULL, NULL) == lib.OK
    gemm = [P, P, 64, 96, P, P, 4, P, 0, NULL]
    refused(lib, L.lrbi_i8_gemm, gemm, [(0, NULL), (0, HALF), (1, NULL), (1, ODD), (2, 0), (3, 0), (3, (1 << 17) + 1), (4, NULL), (4, HALF), (5, NULL), (5, ODD), (6, -1),
                                        (7, NULL), (7, ODD), (8, 2)])
    assert L.lrbi_i8_gemm(P, P, 64, 96, NULL, NULL, 0, NULL, 0, NULL) == lib.OK


def residual(lib, **change):
    v = dict(rows=4, cols=64, kind=0, x_dtype=0, f_dtype=0, param_dtype=1, residual_scale=1.0, eps=1e-5, gamma=0x1000, beta=0x1000, post_gamma=0x1000, post_beta=0x1000,
             gate=0x1000)
    return ctypes.byref(lib.Residual(**(v | change)))


BAD = [dict(rows=-1), dict(cols=0), dict(cols=32769), dict(kind=2), dict(kind=-1), dict(x_dtype=2), dict(f_dtype=-1), dict(param_dtype=2), dict(f_dtype=1), dict(eps=-1.0),
       dict(eps=float("nan")), dict(gamma=0), dict(post_gamma=0), dict(gamma=0x1002), dict(gate=0x1001), dict(post_beta=0x1001)]


def test_residual_arguments(lib):
    L = lib.lib()
    good = [residual(lib), P, 64, P, 64, P, 64, P, 64, NULL, NULL, P, NULL]
    refused(lib, L.lrbi_residual_norm, good, [(0, None)] + [(0, residual(lib, **c)) for c in BAD] + [
        (1, NULL), (1, ODD), (2, 63), (3, NULL), (4, 10), (5, NULL), (6, 0), (7, NULL), (7, ODD), (8, 63), (9, P), (10, P), (11, ODD)])
    tokens = list(good)
    tokens[7], tokens[9], tokens[10] = NULL, P, P
    refused(lib, L.lrbi_residual_norm, tokens, [(7, P), (9, HALF), (10, NULL), (10, ODD), (9, NULL)])
    alone = list(good)
    alone[0] = residual(lib, gamma=0, beta=0)
    refused(lib, L.lrbi_residual_norm, alone, [(11, P)])          # u without gamma
    assert L.lrbi_residual_norm(residual(lib, rows=0), NULL, 64, NULL, 64, NULL, 64, NULL, 64, NULL, NULL, NULL, NULL) == lib.OK
    back = [residual(lib), P, 64, P, 64, P, 64, P, 64, P, P, 64, P, 64, P, P, P, P, P, P, 1 << 20, NULL]
    refused(lib, L.lrbi_residual_norm_backward, back, [(0, None)] + [(0, residual(lib, **c)) for c in BAD] + [
        (1, NULL), (1, ODD), (2, 63), (3, ODD), (4, 63), (5, NULL), (6, 1), (7, NULL), (8, 63), (9, NULL), (9, ODD), (10, NULL), (11, 3), (12, NULL), (13, 3), (14, ODD),
        (15, ODD), (16, ODD), (17, ODD), (18, ODD), (19, NULL), (19, HALF), (20, 64)])
    for change, at in ((dict(beta=0), 15), (dict(post_gamma=0, post_beta=0), 16), (dict(post_beta=0), 17), (dict(gate=0), 18)):
        refused(lib, L.lrbi_residual_norm_backward, back, [(0, residual(lib, **change))])      # a gradient of what is not there
    refused(lib, L.lrbi_residual_norm_backward, back, [(0, residual(lib, gamma=0, beta=0))])    # du without gamma


def test_too_many_rows(lib):
    L, before, most = lib.lib(), lib.launch_count(), 2 ** 31 - 1
    assert L.lrbi_i8_tokens(P, 0, 64, most, 64, -1, P, P, NULL) == lib.ERR_UNSUPPORTED
    assert L.lrbi_i8_gemm(P, P, most, 96, P, P, 4, P, 0, NULL) == lib.ERR_UNSUPPORTED
    assert L.lrbi_i8_gemm(P, P, 64, 96, P, P, most, P, 0, NULL) == lib.ERR_UNSUPPORTED
    assert L.lrbi_i8_quantize(ctypes.byref(lib.Layout(most, 96, 16, 32, 4)), P, NULL, NULL, P, P, NULL) == lib.ERR_UNSUPPORTED
    assert L.lrbi_residual_norm(residual(lib, rows=most), P, 64, P, 64, P, 64, P, 64, NULL, NULL, P, NULL) == lib.ERR_UNSUPPORTED
    assert L.lrbi_residual_norm_backward(residual(lib, rows=most), P, 64, P, 64, P, 64, P, 64, P, P, 64, P, 64, P, P, P, P, P, P, 1 << 40, NULL) == lib.ERR_UNSUPPORTED
    assert lib.launch_count() == before


def test_python_refusals(lib):
    torch = pytest.importorskip("torch")
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        lib.lrbi_i8_tokens(x)                                      # not on a GPU
    with pytest.raises(ValueError):
        lib.lrbi_i8_tokens(x, act="tanh")
    with pytest.raises(TypeError):
        lib.lrbi_residual_norm(x, x, None)
    with pytest.raises(ValueError):
        lib.lrbi_residual_norm(x, x, None, kind="batch")
    with pytest.raises(TypeError):
        lib.lrbi_residual_norm_backward(None, x, None, x, None)
    with pytest.raises(TypeError):
        lib.lrbi_i8_gemm(x, x)
    with pytest.raises(TypeError):
        lib.I8Weights(torch.zeros((4, 64), dtype=torch.int8), torch.zeros(4), 4, 64)
    with pytest.raises(ValueError):
        lib.I8Weights(torch.zeros((4, 64), dtype=torch.int8), torch.zeros(4), 4, (1 << 17) + 1)
