"""Argument checks of the operators around the masked layers: host only, nothing is launched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_1905_05686_b200 import build
    build.build()
    from paper_1905_05686_b200 import binding
    return binding


P, ODD, NULL = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0)   # never dereferenced: the checks fail first


def test_sizes(lib):
    L = lib.lib()
    assert [L.lrbi_checkpoint_pitch(c) for c in (1, 16, 17, 500, 1 << 24)] == [16, 16, 32, 512, 1 << 24]
    assert [L.lrbi_checkpoint_groups(c) for c in (1, 128, 129, 500)] == [1, 1, 2, 4]
    assert [L.lrbi_checkpoint_pitch(c) for c in (0, -5, (1 << 24) + 1)] == [0, 0, 0]
    assert L.lrbi_w4_packed_words(500, 800) == 32 * 13 * 128 and L.lrbi_w4_meta_words(500, 800, 32) == 32 * 25 * 16
    assert L.lrbi_w4_packed_words(0, 800) == 0 and L.lrbi_w4_meta_words(500, 800, 48) == 0
    assert L.lrbi_w4_packed_words(2 ** 31 - 1, 1 << 24) == 2 ** 27 * 2 ** 18 * 128         # beyond 32 bits
    for rows, cols in ((0, 1), (1, 4096), (4096, 4096), (10 ** 6, 100), (7, 1 << 24)):
        n = L.lrbi_layer_norm_backward_workspace(rows, cols)
        assert n >= 8 * cols and n % 32 == 0
    assert L.lrbi_layer_norm_backward_workspace(-1, 4) == 0 and L.lrbi_layer_norm_backward_workspace(4, 0) == 0


def changed(args, at, value):
    a = list(args)
    a[at] = value
    return a


def refused(lib, f, good, changes):
    before = lib.launch_count()
    for at, value in changes:
        assert f(*changed(good, at, value)) == lib.ERR_INVALID_ARG, (at, value)
    assert lib.launch_count() == before


def test_checkpoint_arguments(lib):
    L = lib.lib()
    store = [P, 0, 64, 4, 64, P, P, NULL]
    refused(lib, L.lrbi_checkpoint_store, store, [(0, NULL), (0, ODD), (1, 2), (1, -1), (2, 63), (2, -64), (3, -1), (4, 0), (4, (1 << 24) + 1), (5, NULL), (5, ODD),
                                                  (5, ctypes.c_void_p(0x1008)), (6, NULL), (6, ODD)])
    load = [P, P, 4, 64, P, 1, 64, NULL]
    refused(lib, L.lrbi_checkpoint_load, load, [(0, NULL), (1, NULL), (2, -1), (3, 0), (4, NULL), (4, ctypes.c_void_p(0x1002)), (5, 3), (6, 10)])
    assert L.lrbi_checkpoint_store(*changed(store, 3, 0)) == lib.OK               # no rows: nothing to do
    assert L.lrbi_checkpoint_load(*changed(load, 2, 0)) == lib.OK


def test_layer_norm_arguments(lib):
    L = lib.lib()
    good = [P, 0, 64, 4, 64, P, P, 1, 1e-5, P, 0, 64, P, P, P, P, NULL]
    refused(lib, L.lrbi_layer_norm, good, [(0, NULL), (1, 9), (2, 63), (3, -1), (4, 0), (5, NULL), (5, ODD), (6, ODD), (7, 2), (8, -1.0), (8, float("nan")),
                                           (9, NULL), (10, 2), (11, 1), (12, NULL), (13, NULL), (14, NULL), (15, NULL), (12, ODD)])
    assert L.lrbi_layer_norm(*changed(good, 3, 0)) == lib.OK
    need = L.lrbi_layer_norm_backward_workspace(4, 64)
    back = [P, 0, 64, P, 0, 64, NULL, NULL, 4, 64, P, P, 1, P, P, P, 64, P, 0, 64, P, 64, P, P, P, need, NULL]
    refused(lib, L.lrbi_layer_norm_backward, back, [(0, NULL), (1, 5), (2, 3), (3, NULL), (4, 7), (5, 0), (6, P), (7, P), (8, -1), (9, 0), (10, NULL), (11, ODD),
                                                    (12, 4), (13, NULL), (14, NULL), (15, ODD), (16, 5), (17, NULL), (18, -2), (19, 63), (20, ODD), (21, 63),
                                                    (22, ODD), (23, ODD), (24, NULL), (24, ctypes.c_void_p(0x1004)), (25, need - 1)])
    copied = changed(changed(changed(back, 3, NULL), 6, P), 7, P)
    refused(lib, L.lrbi_layer_norm_backward, copied, [(3, P), (6, NULL), (7, NULL), (6, ctypes.c_void_p(0x1008))])


def test_activation_arguments(lib):
    L = lib.lib()
    good = [P, 0, 64, 4, 64, 1, P, 0, 64, P, P, NULL]
    refused(lib, L.lrbi_activation, good, [(0, NULL), (1, 2), (2, 5), (3, -1), (4, 0), (5, -1), (5, 3), (6, NULL), (6, ODD), (7, 2), (8, 0), (9, NULL), (10, NULL)])
    back = [P, 0, 64, P, 0, 64, NULL, NULL, 4, 64, 2, P, 0, 64, P, 64, NULL]
    refused(lib, L.lrbi_activation_backward, back, [(0, NULL), (1, 2), (2, 5), (3, NULL), (4, 3), (5, 63), (6, P), (8, -1), (9, 0), (10, 3), (11, NULL), (12, 2), (13, 6),
                                                    (14, ODD), (15, 63)])
    assert L.lrbi_activation(*changed(good, 3, 0)) == lib.OK
    assert L.lrbi_activation_backward(*changed(back, 8, 0)) == lib.OK


def test_w4_arguments(lib):
    L = lib.lib()
    lay = lib.Layout(64, 64, 32, 32, 4)
    good = [ctypes.byref(lay), P, P, P, 64, P, P, NULL]
    refused(lib, L.lrbi_w4_quantize, good, [(0, None), (1, NULL), (1, ODD), (2, NULL), (3, NULL), (2, ODD), (4, 0), (4, 96), (5, NULL), (5, ctypes.c_void_p(0x1008)),
                                            (6, NULL), (6, ODD), (0, ctypes.byref(lib.Layout(64, 64, 32, 32, 0))), (0, ctypes.byref(lib.Layout(0, 64, 32, 32, 4)))])
    gemv = [P, P, 64, 64, 64, P, 2, P, 0, NULL]
    refused(lib, L.lrbi_w4_gemv, gemv, [(0, NULL), (0, ctypes.c_void_p(0x1008)), (1, NULL), (2, 0), (3, 0), (4, 16), (5, NULL), (5, ODD), (6, -1), (7, NULL), (7, ODD), (8, 2)])
    assert L.lrbi_w4_gemv(*changed(gemv, 6, 0)) == lib.OK


def test_w4_meta_alignment(lib):
    """Scales and zero points are copied 16 bytes at a time: an array that starts elsewhere is refused, not launched."""
    L = lib.lib()
    lay = lib.Layout(64, 64, 32, 32, 4)
    for at in (0x1004, 0x1008, 0x100C):
        off = ctypes.c_void_p(at)
        refused(lib, L.lrbi_w4_gemv, [P, P, 64, 64, 64, P, 0, P, 0, NULL], [(1, off)])        # no rows of X: nothing could be launched
        refused(lib, L.lrbi_w4_quantize, [ctypes.byref(lay), P, P, P, 64, P, P, NULL], [(6, off)])


def test_rows_far_apart(lib):
    """Rows may be up to 2^32 bytes apart, not more."""
    L = lib.lib()
    for code, size in ((0, 2), (1, 4)):
        most = (1 << 32) // size - 1
        store = [P, code, most, 0, 64, P, P, NULL]
        assert L.lrbi_checkpoint_store(*store) == lib.OK
        refused(lib, L.lrbi_checkpoint_store, store, [(2, most + 1), (2, 1 << 40), (2, (1 << 63) - 1)])
        act = [P, code, most, 0, 64, 1, P, code, most, P, P, NULL]
        assert L.lrbi_activation(*act) == lib.OK
        refused(lib, L.lrbi_activation, act, [(2, most + 1), (8, most + 1)])
        back = [P, code, most, P, code, most, NULL, NULL, 0, 64, 2, P, code, most, P, most, NULL]
        assert L.lrbi_activation_backward(*back) == lib.OK
        refused(lib, L.lrbi_activation_backward, back, [(2, most + 1), (5, most + 1), (13, most + 1), (15, most + 1)])
        norm = [P, code, most, 0, 64, P, P, 1, 1e-5, P, code, most, P, P, P, P, NULL]
        assert L.lrbi_layer_norm(*norm) == lib.OK
        refused(lib, L.lrbi_layer_norm, norm, [(2, most + 1), (11, most + 1)])
