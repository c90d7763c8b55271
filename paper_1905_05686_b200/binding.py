"""Python binding of the lrbi C ABI: argument marshalling only.

Every step of the path (decode, pruning, product) runs in the CUDA library; this module turns
torch CUDA tensors into device pointers and checks return codes.  torch is used for device
memory and streams.  The calls made per layer and per token around the masked layers are marshalled by a small
compiled module (_lrbi_torch-*.so) that calls the same C ABI.  If the library is not built, importing a compute function's first call
raises: there is no CPU fallback.

Calls take `stream`, a torch.cuda.Stream (None: the current one).  A call on another stream does not wait for the current one, so
that the two may overlap: the caller makes that stream wait for whatever writes the inputs (stream.wait_stream), keeps the inputs
until it is through with them (Tensor.record_stream), and makes the current stream wait before the results are used there.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os

import numpy as np
import torch

from .build import calls_path
from .synth import Layer

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblrbi.so")
CALLS_PATH = calls_path()

ALGO_AUTO, ALGO_GENERIC, ALGO_GEMV, ALGO_TENSOR, ALGO_DECODE_BALLOT, ALGO_DECODE_PLANES, ALGO_DECODE_PLANES_WIDE, ALGO_STREAM, ALGO_TENSOR_PAIR, ALGO_TENSOR_PAIR2, ALGO_TENSOR_PAIR192 = range(11)
ALGO_NAMES = {0: "auto", 1: "generic", 2: "gemv", 3: "tensor", 4: "decode_ballot", 5: "decode_planes", 6: "decode_planes_wide", 7: "stream", 8: "tensor_pair", 9: "tensor_pair2", 10: "tensor_pair192"}
Y_BF16, Y_F32 = 0, 1
OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_CUDA, ERR_TIMEOUT, ERR_TOO_LARGE = range(6)
STATIC_SCRATCH_BYTES = 8 * 1024 * 1024


class LrbiError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        super().__init__("%s: %s (status %d, cuda error %d)" % (what, status_string(code), code, lib().lrbi_last_cuda_error()))


class GemmPlan(ctypes.Structure):
    """lrbi_gemm_plan: how lrbi_masked_gemm would run a call."""
    _fields_ = [("algo", ctypes.c_int32), ("batch_tile", ctypes.c_int32), ("cta_pair", ctypes.c_int32),
                ("panel_columns", ctypes.c_int32), ("k_splits", ctypes.c_int32), ("stages", ctypes.c_int32),
                ("scratch_bytes", ctypes.c_uint64)]


class TileRanks(ctypes.Structure):
    """lrbi_tile_ranks: device arrays with one rank and two word offsets per tile."""
    _fields_ = [("ranks", ctypes.c_void_p), ("ip_offset", ctypes.c_void_p), ("iz_offset", ctypes.c_void_p)]


class Layout(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32), ("tile_rows", ctypes.c_int32),
                ("tile_cols", ctypes.c_int32), ("rank", ctypes.c_int32)]

    @classmethod
    def of(cls, layer):
        if isinstance(layer, cls):
            return layer
        if isinstance(layer, Layer):
            return cls(layer.rows, layer.cols, layer.tile_rows, layer.tile_cols, layer.rank)
        return cls(*layer)


_lib = None


def lib():
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("lrbi CUDA library missing: %s (run paper_1905_05686_b200/build.py); "
                               "there is no CPU fallback" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, lp = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(Layout)
        for name in ("lrbi_packed_ip_words", "lrbi_packed_iz_words", "lrbi_mask_words"):
            getattr(L, name).argtypes = [lp]
            getattr(L, name).restype = ctypes.c_size_t
        L.lrbi_decode_mask.argtypes = [lp, vp, vp, vp, i32, vp]
        L.lrbi_decode_mask.restype = i32
        L.lrbi_masked_gemm.argtypes = [lp, vp, vp, vp, vp, i32, vp, i32, i32, vp]
        L.lrbi_masked_gemm.restype = i32
        L.lrbi_masked_gemm_static.argtypes = [lp, vp, vp, vp, vp, i32, vp, i32, vp]
        L.lrbi_masked_gemm_static.restype = i32
        L.lrbi_masked_gemm_static_bytes.argtypes = [lp, i32]
        L.lrbi_masked_gemm_static_bytes.restype = ctypes.c_size_t
        L.lrbi_layer_create.argtypes = [lp, vp, vp, vp, i32, ctypes.POINTER(vp)]
        L.lrbi_layer_create.restype = i32
        L.lrbi_layer_forward_host.argtypes = [vp, vp, i32, vp, i32, i32]
        L.lrbi_layer_forward_host.restype = i32
        L.lrbi_layer_destroy.argtypes = [vp]
        L.lrbi_layer_destroy.restype = i32
        L.lrbi_masked_gemm_choice.argtypes = [lp, i32]
        L.lrbi_masked_gemm_choice.restype = i32
        L.lrbi_masked_gemm_plan.argtypes = [lp, i32, i32, ctypes.POINTER(GemmPlan)]
        L.lrbi_masked_gemm_plan.restype = i32
        L.lrbi_last_device_error.argtypes = []
        L.lrbi_last_device_error.restype = i32
        L.lrbi_selftest_bounded_wait.argtypes = [ctypes.c_uint32, vp]
        L.lrbi_selftest_bounded_wait.restype = i32
        L.lrbi_threshold_pack.argtypes = [lp, vp, vp, vp, vp, vp, vp, vp]
        L.lrbi_threshold_pack.restype = i32
        L.lrbi_index_cost.argtypes = [lp, vp, ctypes.c_float, vp, vp, vp, vp]
        L.lrbi_index_cost.restype = i32
        L.lrbi_decode_mask_ranked.argtypes = [lp, ctypes.POINTER(TileRanks), vp, vp, vp, vp]
        L.lrbi_decode_mask_ranked.restype = i32
        L.lrbi_masked_gemm_ranked.argtypes = [lp, ctypes.POINTER(TileRanks), vp, vp, vp, vp, i32, vp, i32, i32, vp]
        L.lrbi_masked_gemm_ranked.restype = i32
        L.lrbi_decode_mask_batch.argtypes = [i32, lp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), vp]
        L.lrbi_decode_mask_batch.restype = i32
        L.lrbi_transpose_bf16.argtypes = [vp, i32, i32, vp, vp]
        L.lrbi_transpose_bf16.restype = i32
        L.lrbi_masked_gemm_dx.argtypes = [lp, vp, vp, vp, vp, i32, vp, i32, i32, vp]
        L.lrbi_masked_gemm_dx.restype = i32
        L.lrbi_masked_gemm_dw_workspace.argtypes = [lp, i32]
        L.lrbi_masked_gemm_dw_workspace.restype = ctypes.c_size_t
        L.lrbi_masked_gemm_dw.argtypes = [lp, vp, vp, i32, vp, vp, vp, i32, vp, ctypes.c_size_t, vp]
        L.lrbi_masked_gemm_dw.restype = i32
        L.lrbi_nmf_workspace.argtypes = [lp]
        L.lrbi_nmf_workspace.restype = ctypes.c_size_t
        L.lrbi_nmf_update.argtypes = [lp, vp, vp, vp, i32, ctypes.c_float, vp, ctypes.c_size_t, vp]
        L.lrbi_nmf_update.restype = i32
        i64, f32, sz = ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        L.lrbi_checkpoint_pitch.argtypes = [i32]
        L.lrbi_checkpoint_pitch.restype = i32
        L.lrbi_checkpoint_groups.argtypes = [i32]
        L.lrbi_checkpoint_groups.restype = i32
        L.lrbi_checkpoint_store.argtypes = [vp, i32, i64, i32, i32, vp, vp, vp]
        L.lrbi_checkpoint_store.restype = i32
        L.lrbi_checkpoint_load.argtypes = [vp, vp, i32, i32, vp, i32, i64, vp]
        L.lrbi_checkpoint_load.restype = i32
        L.lrbi_layer_norm.argtypes = [vp, i32, i64, i32, i32, vp, vp, i32, f32, vp, i32, i64, vp, vp, vp, vp, vp]
        L.lrbi_layer_norm.restype = i32
        L.lrbi_layer_norm_backward_workspace.argtypes = [i32, i32]
        L.lrbi_layer_norm_backward_workspace.restype = sz
        L.lrbi_layer_norm_backward.argtypes = [vp, i32, i64, vp, i32, i64, vp, vp, i32, i32, vp, vp, i32, vp, vp, vp, i64, vp, i32, i64,
                                               vp, i64, vp, vp, vp, sz, vp]
        L.lrbi_layer_norm_backward.restype = i32
        L.lrbi_activation.argtypes = [vp, i32, i64, i32, i32, i32, vp, i32, i64, vp, vp, vp]
        L.lrbi_activation.restype = i32
        L.lrbi_activation_backward.argtypes = [vp, i32, i64, vp, i32, i64, vp, vp, i32, i32, i32, vp, i32, i64, vp, i64, vp]
        L.lrbi_activation_backward.restype = i32
        L.lrbi_w4_packed_words.argtypes = [i32, i32]
        L.lrbi_w4_packed_words.restype = sz
        L.lrbi_w4_meta_words.argtypes = [i32, i32, i32]
        L.lrbi_w4_meta_words.restype = sz
        L.lrbi_w4_quantize.argtypes = [lp, vp, vp, vp, i32, vp, vp, vp]
        L.lrbi_w4_quantize.restype = i32
        L.lrbi_w4_gemv.argtypes = [vp, vp, i32, i32, i32, vp, i32, vp, i32, vp]
        L.lrbi_w4_gemv.restype = i32
        L.lrbi_launch_count.argtypes = []
        L.lrbi_launch_count.restype = ctypes.c_uint64
        L.lrbi_device_status.argtypes = [i32]
        L.lrbi_device_status.restype = i32
        L.lrbi_status_string.argtypes = [i32]
        L.lrbi_status_string.restype = ctypes.c_char_p
        L.lrbi_last_cuda_error.argtypes = []
        L.lrbi_last_cuda_error.restype = i32
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().lrbi_status_string(code).decode()


def launch_count() -> int:
    return int(lib().lrbi_launch_count())


def device_status(clear: bool = False) -> int:
    return int(lib().lrbi_device_status(1 if clear else 0))


def masked_gemm_choice(layer, batch: int) -> int:
    lay = Layout.of(layer)
    return int(lib().lrbi_masked_gemm_choice(ctypes.byref(lay), batch))


def masked_gemm_plan(layer, batch: int, algo: int = ALGO_AUTO) -> GemmPlan:
    """The kernel instantiation lrbi_masked_gemm would run (nothing is launched)."""
    lay = Layout.of(layer)
    plan = GemmPlan()
    rc = lib().lrbi_masked_gemm_plan(ctypes.byref(lay), batch, algo, ctypes.byref(plan))
    if rc != OK:
        raise LrbiError(rc, "lrbi_masked_gemm_plan")
    return plan


def selftest_bounded_wait(limit_us: int = 1000, stream=None) -> None:
    """Runs the kernel whose bounded wait is meant to give up (leaves 0x600 in the status word)."""
    rc = lib().lrbi_selftest_bounded_wait(limit_us, _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_selftest_bounded_wait")


def _stream_ptr(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _empty(shape, dtype, device, stream) -> torch.Tensor:
    """A new tensor that a call on `stream` writes: out of that stream's pool, since the current stream may still be at work on
    what was freed to its own, and kept until the current stream, which will use it, is through with it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    current = torch.cuda.current_stream(device)
    if not isinstance(stream, torch.cuda.Stream):        # another library's, with the handle in cuda_stream
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(current)
    return t


def _dev(t: torch.Tensor, dtype, what):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise TypeError("%s must be a contiguous CUDA tensor of dtype %s" % (what, dtype))
    return ctypes.c_void_p(t.data_ptr())


def to_device_words(a: np.ndarray, device="cuda") -> torch.Tensor:
    """uint32 numpy words -> int32 CUDA tensor holding the same bits."""
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.uint32).view(np.int32)).to(device)


def to_device_bf16(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """uint16 bf16 bit patterns -> bfloat16 CUDA tensor holding the same bits."""
    return torch.from_numpy(np.ascontiguousarray(bits, dtype=np.uint16).view(np.int16)).to(device).view(torch.bfloat16)


def lrbi_decode_mask(layer, ip: torch.Tensor, iz: torch.Tensor, mask_out: torch.Tensor | None = None,
                     algo: int = ALGO_AUTO, stream=None) -> torch.Tensor:
    """Bit-packed decoded index [rows, ceil(cols/32)] (int32 tensor holding uint32 words)."""
    lay = Layout.of(layer)
    L = lib()
    if ip.numel() != L.lrbi_packed_ip_words(ctypes.byref(lay)) or iz.numel() != L.lrbi_packed_iz_words(ctypes.byref(lay)):
        raise ValueError("packed factor sizes do not match the layout")
    if mask_out is None:
        mask_out = _empty((lay.rows, (lay.cols + 31) // 32), torch.int32, ip.device, stream)
    elif mask_out.numel() != L.lrbi_mask_words(ctypes.byref(lay)):
        raise ValueError("mask_out has the wrong size")
    rc = L.lrbi_decode_mask(ctypes.byref(lay), _dev(ip, torch.int32, "ip"), _dev(iz, torch.int32, "iz"),
                            _dev(mask_out, torch.int32, "mask_out"), algo, _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_decode_mask")
    return mask_out


def _tile_ranks(lay, ranks, ip_off, iz_off):
    tiles = (-(-lay.rows // lay.tile_rows)) * (-(-lay.cols // lay.tile_cols))
    if ranks.numel() != tiles or ip_off.numel() != tiles or iz_off.numel() != tiles:
        raise ValueError("one rank and one pair of offsets per tile")
    return TileRanks(_dev(ranks, torch.int32, "ranks").value, _dev(ip_off, torch.int64, "ip_offset").value,
                     _dev(iz_off, torch.int64, "iz_offset").value)


def lrbi_decode_mask_ranked(layer, ranks, ip_off, iz_off, ip, iz, mask_out=None, stream=None) -> torch.Tensor:
    """lrbi_decode_mask for a ranked layout (one rank per tile; `layer.rank` is the upper bound)."""
    lay = Layout.of(layer)
    tr = _tile_ranks(lay, ranks, ip_off, iz_off)
    if mask_out is None:
        mask_out = _empty((lay.rows, (lay.cols + 31) // 32), torch.int32, ip.device, stream)
    rc = lib().lrbi_decode_mask_ranked(ctypes.byref(lay), ctypes.byref(tr), _dev(ip, torch.int32, "ip"), _dev(iz, torch.int32, "iz"),
                                       _dev(mask_out, torch.int32, "mask_out"), _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_decode_mask_ranked")
    return mask_out


def lrbi_masked_gemm_ranked(layer, ranks, ip_off, iz_off, W, ip, iz, X, Y=None, y_dtype=torch.bfloat16, algo=ALGO_AUTO,
                            stream=None) -> torch.Tensor:
    """lrbi_masked_gemm for a ranked layout."""
    lay = Layout.of(layer)
    tr = _tile_ranks(lay, ranks, ip_off, iz_off)
    if tuple(W.shape) != (lay.rows, lay.cols) or X.dim() != 2 or X.shape[1] != lay.cols:
        raise ValueError("W / X shapes do not match the layout")
    batch = X.shape[0]
    if Y is None:
        Y = _empty((batch, lay.rows), y_dtype, X.device, stream)
    elif tuple(Y.shape) != (batch, lay.rows) or Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y has the wrong shape or dtype")
    rc = lib().lrbi_masked_gemm_ranked(ctypes.byref(lay), ctypes.byref(tr), _dev(W, torch.bfloat16, "W"), _dev(ip, torch.int32, "ip"),
                                       _dev(iz, torch.int32, "iz"), _dev(X, torch.bfloat16, "X"), batch, _dev(Y, Y.dtype, "Y"),
                                       Y_F32 if Y.dtype == torch.float32 else Y_BF16, algo, _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_masked_gemm_ranked")
    return Y


def lrbi_decode_mask_batch(layers, ips, izs, stream=None):
    """Decode the indices of several layers with one launch per 32 layers; returns the list of masks."""
    n = len(layers)
    lays = (Layout * n)(*[Layout.of(l) for l in layers])
    masks = [_empty((l.rows, (l.cols + 31) // 32), torch.int32, ips[0].device, stream) for l in lays]
    arr = lambda ts, what: (ctypes.c_void_p * n)(*[_dev(t, torch.int32, what).value for t in ts])
    rc = lib().lrbi_decode_mask_batch(n, lays, arr(ips, "ip"), arr(izs, "iz"), arr(masks, "mask_out"), _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_decode_mask_batch")
    return masks


def lrbi_transpose_bf16(src: torch.Tensor, dst: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """dst [cols, rows] = src [rows, cols] transposed (bf16)."""
    rows, cols = src.shape
    if dst is None:
        dst = _empty((cols, rows), torch.bfloat16, src.device, stream)
    rc = lib().lrbi_transpose_bf16(_dev(src, torch.bfloat16, "src"), rows, cols, _dev(dst, torch.bfloat16, "dst"), _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_transpose_bf16")
    return dst


def lrbi_masked_gemm_dx(layer, Wt, ip, iz, dY, dX=None, dtype=torch.bfloat16, algo=ALGO_AUTO, stream=None) -> torch.Tensor:
    """dX = dY (W .* Ia): Wt [cols, rows] is W transposed, dY [batch, rows]; returns dX [batch, cols]."""
    lay = Layout.of(layer)
    if tuple(Wt.shape) != (lay.cols, lay.rows) or dY.dim() != 2 or dY.shape[1] != lay.rows:
        raise ValueError("Wt / dY shapes do not match the layout")
    batch = dY.shape[0]
    if dX is None:
        dX = _empty((batch, lay.cols), dtype, dY.device, stream)
    rc = lib().lrbi_masked_gemm_dx(ctypes.byref(lay), _dev(Wt, torch.bfloat16, "Wt"), _dev(ip, torch.int32, "ip"), _dev(iz, torch.int32, "iz"),
                                   _dev(dY, torch.bfloat16, "dY"), batch, _dev(dX, dX.dtype, "dX"),
                                   Y_F32 if dX.dtype == torch.float32 else Y_BF16, algo, _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_masked_gemm_dx")
    return dX


def lrbi_masked_gemm_dw(layer, dY, X, ip, iz, dW=None, dtype=torch.bfloat16, workspace="auto", stream=None) -> torch.Tensor:
    """dW = (dY^T X) .* Ia: dY [batch, rows], X [batch, cols]; returns dW [rows, cols].  workspace: a uint8 CUDA tensor of
    at least masked_gemm_dw_workspace bytes, "auto" (one is made for the call) or None (the slow any-shape kernel)."""
    lay = Layout.of(layer)
    batch = dY.shape[0]
    if tuple(dY.shape) != (batch, lay.rows) or tuple(X.shape) != (batch, lay.cols):
        raise ValueError("dY / X shapes do not match the layout")
    if dW is None:
        dW = _empty((lay.rows, lay.cols), dtype, dY.device, stream)
    need = lib().lrbi_masked_gemm_dw_workspace(ctypes.byref(lay), batch)
    if isinstance(workspace, str):
        workspace = _empty(need, torch.uint8, dY.device, stream)
    wptr, wbytes = (ctypes.c_void_p(workspace.data_ptr()), workspace.numel()) if workspace is not None else (ctypes.c_void_p(0), 0)
    rc = lib().lrbi_masked_gemm_dw(ctypes.byref(lay), _dev(dY, torch.bfloat16, "dY"), _dev(X, torch.bfloat16, "X"), batch,
                                   _dev(ip, torch.int32, "ip"), _dev(iz, torch.int32, "iz"), _dev(dW, dW.dtype, "dW"),
                                   Y_F32 if dW.dtype == torch.float32 else Y_BF16, wptr, wbytes, _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_masked_gemm_dw")
    return dW


def lrbi_nmf_update(layer, W, mp, mz, iterations, eps=1e-9, workspace=None, stream=None):
    """In-place multiplicative NMF updates of (mp, mz) towards |W|, tile by tile; returns (mp, mz)."""
    lay = Layout.of(layer)
    need = lib().lrbi_nmf_workspace(ctypes.byref(lay))
    if workspace is None:
        workspace = _empty(need, torch.uint8, W.device, stream)
    rc = lib().lrbi_nmf_update(ctypes.byref(lay), _dev(W, torch.bfloat16, "W"), _dev(mp, torch.float32, "mp"), _dev(mz, torch.float32, "mz"),
                               iterations, ctypes.c_float(eps), ctypes.c_void_p(workspace.data_ptr()), workspace.numel(), _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_nmf_update")
    return mp, mz


def lrbi_threshold_pack(layer, mp: torch.Tensor, mz: torch.Tensor, tp: torch.Tensor, tz: torch.Tensor, stream=None):
    """Binary conversion of NMF factors into packed (ip, iz): mp [tiles, tm, k], mz [tiles, k, tn] fp32,
    tp, tz [tiles] fp32 thresholds.  Returns the two packed int32 tensors."""
    lay = Layout.of(layer)
    L = lib()
    gr, gc = -(-lay.rows // lay.tile_rows), -(-lay.cols // lay.tile_cols)
    tiles = gr * gc
    if mp.numel() != tiles * lay.tile_rows * lay.rank or mz.numel() != tiles * lay.rank * lay.tile_cols:
        raise ValueError("factor sizes do not match the layout")
    if tp.numel() != tiles or tz.numel() != tiles:
        raise ValueError("one threshold pair per tile")
    ip = _empty(L.lrbi_packed_ip_words(ctypes.byref(lay)), torch.int32, mp.device, stream)
    iz = _empty(L.lrbi_packed_iz_words(ctypes.byref(lay)), torch.int32, mp.device, stream)
    rc = L.lrbi_threshold_pack(ctypes.byref(lay), _dev(mp, torch.float32, "mp"), _dev(mz, torch.float32, "mz"),
                               _dev(tp, torch.float32, "tp"), _dev(tz, torch.float32, "tz"),
                               _dev(ip, torch.int32, "ip"), _dev(iz, torch.int32, "iz"), _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_threshold_pack")
    return ip, iz


def lrbi_index_cost(layer, W: torch.Tensor, theta: float, ip: torch.Tensor, iz: torch.Tensor, out: torch.Tensor | None = None,
                    stream=None) -> torch.Tensor:
    """Per-tile records (kept_i, kept_a, lost as int64 bit patterns, cost as the bits of a double): an int64
    tensor [tiles, 4]; `tile_costs` turns it into numpy arrays."""
    lay = Layout.of(layer)
    L = lib()
    if tuple(W.shape) != (lay.rows, lay.cols):
        raise ValueError("W shape does not match the layout")
    if ip.numel() != L.lrbi_packed_ip_words(ctypes.byref(lay)) or iz.numel() != L.lrbi_packed_iz_words(ctypes.byref(lay)):
        raise ValueError("packed factor sizes do not match the layout")
    tiles = (-(-lay.rows // lay.tile_rows)) * (-(-lay.cols // lay.tile_cols))
    if out is None:
        out = _empty((tiles, 4), torch.int64, W.device, stream)
    elif out.numel() != tiles * 4:
        raise ValueError("out has the wrong size")
    rc = L.lrbi_index_cost(ctypes.byref(lay), _dev(W, torch.bfloat16, "W"), ctypes.c_float(theta), _dev(ip, torch.int32, "ip"),
                           _dev(iz, torch.int32, "iz"), _dev(out, torch.int64, "out"), _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_index_cost")
    return out


def tile_costs(out: torch.Tensor):
    """(kept_i, kept_a, lost, cost) numpy arrays from the records lrbi_index_cost wrote."""
    a = out.cpu().numpy()
    return a[:, 0].copy(), a[:, 1].copy(), a[:, 2].copy(), a[:, 3].copy().view(np.float64)


def lrbi_masked_gemm(layer, W: torch.Tensor, ip: torch.Tensor, iz: torch.Tensor, X: torch.Tensor,
                     Y: torch.Tensor | None = None, y_dtype=torch.bfloat16, algo: int = ALGO_AUTO,
                     stream=None) -> torch.Tensor:
    """Y = X (W .* Ia)^T with the index decoded on the fly; W [rows, cols], X [batch, cols] bf16."""
    lay = Layout.of(layer)
    L = lib()
    if tuple(W.shape) != (lay.rows, lay.cols) or X.dim() != 2 or X.shape[1] != lay.cols:
        raise ValueError("W / X shapes do not match the layout")
    if ip.numel() != L.lrbi_packed_ip_words(ctypes.byref(lay)) or iz.numel() != L.lrbi_packed_iz_words(ctypes.byref(lay)):
        raise ValueError("packed factor sizes do not match the layout")
    batch = X.shape[0]
    if Y is None:
        Y = _empty((batch, lay.rows), y_dtype, X.device, stream)
    if tuple(Y.shape) != (batch, lay.rows) or Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be [batch, rows] bf16 or fp32")
    code = Y_BF16 if Y.dtype == torch.bfloat16 else Y_F32
    rc = L.lrbi_masked_gemm(ctypes.byref(lay), _dev(W, torch.bfloat16, "W"), _dev(ip, torch.int32, "ip"),
                            _dev(iz, torch.int32, "iz"), _dev(X, torch.bfloat16, "X"), batch,
                            _dev(Y, Y.dtype, "Y"), code, algo, _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_masked_gemm")
    return Y


def masked_gemm_static_bytes(layer, batch: int) -> int:
    """Bytes of the fixed scratch array lrbi_masked_gemm_static would use for this call (0 = none)."""
    lay = Layout.of(layer)
    return int(lib().lrbi_masked_gemm_static_bytes(ctypes.byref(lay), batch))


def lrbi_masked_gemm_static(layer, W: torch.Tensor, ip: torch.Tensor, iz: torch.Tensor, X: torch.Tensor,
                            Y: torch.Tensor, stream=None) -> torch.Tensor:
    """lrbi_masked_gemm for callers that may not allocate device memory.

    The library call allocates nothing: its K-split partial sums go to a fixed 8 MiB array inside the
    library.  That is why Y is not optional here: a caller that cannot allocate brings its output.
    Raises LrbiError with code ERR_TOO_LARGE if the fixed array is too small.  Calls share that array:
    keep them on one stream.
    """
    lay = Layout.of(layer)
    L = lib()
    if X.dim() != 2 or tuple(W.shape) != (lay.rows, lay.cols) or X.shape[1] != lay.cols:
        raise ValueError("W / X shapes do not match the layout")
    if ip.numel() != L.lrbi_packed_ip_words(ctypes.byref(lay)) or iz.numel() != L.lrbi_packed_iz_words(ctypes.byref(lay)):
        raise ValueError("packed factor sizes do not match the layout")
    batch = X.shape[0]
    if tuple(Y.shape) != (batch, lay.rows) or Y.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("Y must be [batch, rows] bf16 or fp32")
    code = Y_BF16 if Y.dtype == torch.bfloat16 else Y_F32
    rc = lib().lrbi_masked_gemm_static(ctypes.byref(lay), _dev(W, torch.bfloat16, "W"), _dev(ip, torch.int32, "ip"),
                                       _dev(iz, torch.int32, "iz"), _dev(X, torch.bfloat16, "X"), batch,
                                       _dev(Y, Y.dtype, "Y"), code, _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_masked_gemm_static")
    return Y


# ---------------------------------------------------------------------------------------------
# Around the layers: layer norm, 8-bit copies, the nonlinearity, 4-bit weights
# ---------------------------------------------------------------------------------------------
CHECKPOINT_GROUP = 128
ACTIVATIONS = {"relu": 0, "gelu": 1, "silu": 2}
_calls = None


def _native():
    """The module that checks tensors, allocates outputs and calls the C ABI (csrc/torch_calls.cpp); raises if it has not been built."""
    global _calls
    if _calls is None:
        lib()
        if not os.path.exists(CALLS_PATH):
            raise RuntimeError("lrbi call module missing: %s (run paper_1905_05686_b200/build.py)" % CALLS_PATH)
        spec = importlib.util.spec_from_file_location("_lrbi_torch", CALLS_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.set_error(LrbiError)
        _calls = module
    return _calls


class Checkpoint:
    """A matrix kept in 8 bits: q [rows, pitch] int8, scale [rows, groups] float32 (one per CHECKPOINT_GROUP columns of a row).
    Where a call made it, both lie in one allocation: holding either, or saving it with torch.save, keeps both."""

    __slots__ = ("q", "scale", "rows", "cols")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, rows: int, cols: int):
        pitch, groups = (cols + 15) // 16 * 16, -(-cols // CHECKPOINT_GROUP)
        if q.dtype != torch.int8 or scale.dtype != torch.float32 or not q.is_contiguous() or not scale.is_contiguous():
            raise TypeError("q must be contiguous int8 and scale contiguous float32")
        if q.shape != (rows, pitch) or scale.shape != (rows, groups) or q.device != scale.device or not q.is_cuda:
            raise ValueError("q must be [rows, %d] and scale [rows, %d] on one CUDA device" % (pitch, groups))
        self.q, self.scale, self.rows, self.cols = q, scale, rows, cols

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "Checkpoint":
        q = torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.int8, device=device)
        return cls(q, torch.empty((rows, -(-cols // CHECKPOINT_GROUP)), dtype=torch.float32, device=device), rows, cols)

    @classmethod
    def _of(cls, q, scale, rows, cols):
        kept = object.__new__(cls)
        kept.q, kept.scale, kept.rows, kept.cols = q, scale, rows, cols
        return kept

    @property
    def shape(self):
        return (self.rows, self.cols)

    @property
    def nbytes(self):
        return self.q.numel() + 4 * self.scale.numel()


def _kept_or_rows(x, like, what):
    """(matrix, q, scale): a matrix, or its 8-bit copy."""
    if not isinstance(x, Checkpoint):
        return x, None, None
    if like.dim() != 2 or x.rows != like.shape[0] or x.cols != like.shape[1]:
        raise ValueError("%s must have the shape of the call's input" % what)
    return None, x.q, x.scale


def lrbi_checkpoint_store(x: torch.Tensor, stream=None) -> Checkpoint:
    """The 8-bit copy of x [rows, cols] (bf16 or fp32)."""
    q, scale = _native().checkpoint_store(x, stream)
    return Checkpoint._of(q, scale, *x.shape)


def lrbi_checkpoint_load(kept: Checkpoint, dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """What an 8-bit copy stands for, as a new [rows, cols] tensor of `dtype`."""
    if not isinstance(kept, Checkpoint):
        raise TypeError("kept must be a Checkpoint")
    return _native().checkpoint_load(kept.q, kept.scale, kept.rows, kept.cols, dtype, stream)


def lrbi_layer_norm(x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor | None = None, eps: float = 1e-5, y_dtype=None,
                    checkpoint: bool = False, stream=None):
    """Layer norm over the columns of x [rows, cols].  Returns (y, mean, rstd), and the 8-bit copy of x with checkpoint=True.
    mean and rstd lie in one allocation (clone one to keep or save it by itself)."""
    out = _native().layer_norm(x, gamma, beta, eps, y_dtype, checkpoint, stream)
    return (*out[:3], Checkpoint._of(out[3], out[4], *x.shape)) if checkpoint else out


def lrbi_layer_norm_backward(dy: torch.Tensor, x, gamma: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                             beta: torch.Tensor | None = None, dres: torch.Tensor | None = None, restore: bool = False, dx_dtype=None,
                             stream=None):
    """Gradients of the layer norm: x is the forward input or its Checkpoint.  Returns (dx, dgamma, dbeta), dgamma and dbeta in
    fp32, and the forward result again with restore=True (in dy's type; pass the beta of the forward pass).  dres is added to dx,
    which has x's type, or dy's where x is a Checkpoint, unless dx_dtype says otherwise.  dgamma and dbeta lie in one allocation."""
    return _native().layer_norm_backward(dy, *_kept_or_rows(x, dy, "x"), gamma, mean, rstd, beta, dres, restore, dx_dtype, stream)


def _act(act):
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError("act must be one of %s" % ", ".join(sorted(ACTIVATIONS)))
    return code


def lrbi_activation(h: torch.Tensor, act: str, a_dtype=None, checkpoint: bool = False, stream=None):
    """a = act(h) for act "relu", "gelu" or "silu".  Returns a, or (a, the 8-bit copy of h) with checkpoint=True."""
    out = _native().activation(h, _act(act), a_dtype, checkpoint, stream)
    return (out[0], Checkpoint._of(out[1], out[2], *h.shape)) if checkpoint else out


def lrbi_activation_backward(da: torch.Tensor, h, act: str, restore: bool = False, dh_dtype=None, stream=None):
    """dh = da * act'(h): h is the forward input or its Checkpoint.  Returns dh, or (dh, act(h) in da's type) with restore=True."""
    return _native().activation_backward(da, *_kept_or_rows(h, da, "h"), _act(act), restore, dh_dtype, stream)


class W4Weights:
    """A layer's weights in 4 bits as the library lays them out (lrbi.h): packed and meta are int32 CUDA tensors that start on
    16-byte boundaries (the products refuse others)."""

    __slots__ = ("packed", "meta", "rows", "cols", "group")

    def __init__(self, packed: torch.Tensor, meta: torch.Tensor, rows: int, cols: int, group: int):
        if group not in (32, 64, 128):
            raise ValueError("group must be 32, 64 or 128")
        tiles = -(-rows // 16)
        for t, n, what in ((packed, tiles * -(-cols // 64) * 128, "packed"), (meta, tiles * -(-cols // group) * 16, "meta")):
            _dev(t, torch.int32, what)
            if t.numel() != n or t.device != packed.device:
                raise ValueError("%s must hold %d words on one device" % (what, n))
        self.packed, self.meta, self.rows, self.cols, self.group = packed, meta, rows, cols, group

    @property
    def nbytes(self):
        return 4 * (self.packed.numel() + self.meta.numel())


def lrbi_w4_quantize(layer, W: torch.Tensor, group: int = 128, ip: torch.Tensor | None = None, iz: torch.Tensor | None = None,
                     stream=None) -> W4Weights:
    """Quantises W [rows, cols] bf16 to 4 bits; with the layer's packed factors, pruned weights are exactly zero."""
    lay = Layout.of(layer)
    L = lib()
    if tuple(W.shape) != (lay.rows, lay.cols):
        raise ValueError("W shape does not match the layout")
    if (ip is None) != (iz is None):
        raise ValueError("ip and iz come together")
    if ip is not None and (ip.numel() != L.lrbi_packed_ip_words(ctypes.byref(lay)) or iz.numel() != L.lrbi_packed_iz_words(ctypes.byref(lay))):
        raise ValueError("packed factor sizes do not match the layout")
    if group not in (32, 64, 128):
        raise ValueError("group must be 32, 64 or 128")
    w = _dev(W, torch.bfloat16, "W")
    factors = [None if t is None else _dev(t, torch.int32, what) for t, what in ((ip, "ip"), (iz, "iz"))]
    packed = _empty(L.lrbi_w4_packed_words(lay.rows, lay.cols), torch.int32, W.device, stream)
    meta = _empty(L.lrbi_w4_meta_words(lay.rows, lay.cols, group), torch.int32, W.device, stream)
    rc = L.lrbi_w4_quantize(ctypes.byref(lay), w, *factors, group, packed.data_ptr(), meta.data_ptr(), _stream_ptr(stream))
    if rc != OK:
        raise LrbiError(rc, "lrbi_w4_quantize")
    return W4Weights(packed, meta, lay.rows, lay.cols, group)


def lrbi_w4_gemv(weights: W4Weights, X: torch.Tensor, y_dtype=torch.bfloat16, stream=None) -> torch.Tensor:
    """Y [batch, rows] = X W^T for X [batch, cols] bf16 and 4-bit weights; made for a few rows of X."""
    return _native().w4_gemv(weights.packed, weights.meta, weights.rows, weights.cols, weights.group, X, y_dtype, stream)


class HostLayer:
    """lrbi_layer_* handle: weights and index resident on the device, activations from host memory."""

    def __init__(self, layer, W_bits: np.ndarray, ip_words: np.ndarray, iz_words: np.ndarray, max_batch: int):
        self.layout = Layout.of(layer)
        W_bits = np.ascontiguousarray(W_bits, dtype=np.uint16)
        ip_words = np.ascontiguousarray(ip_words, dtype=np.uint32)
        iz_words = np.ascontiguousarray(iz_words, dtype=np.uint32)
        h = ctypes.c_void_p()
        rc = lib().lrbi_layer_create(ctypes.byref(self.layout), W_bits.ctypes.data, ip_words.ctypes.data,
                                     iz_words.ctypes.data, max_batch, ctypes.byref(h))
        if rc != OK:
            raise LrbiError(rc, "lrbi_layer_create")
        self._h = h

    def forward_host(self, X_host: torch.Tensor, Y_host: torch.Tensor, algo: int = ALGO_AUTO):
        """X_host [batch, cols] bf16 and Y_host [batch, rows] bf16/fp32 are CPU tensors (pinned for overlap)."""
        if X_host.is_cuda or Y_host.is_cuda or not X_host.is_contiguous() or not Y_host.is_contiguous():
            raise TypeError("forward_host takes contiguous CPU tensors")
        if X_host.dtype != torch.bfloat16 or X_host.shape[1] != self.layout.cols:
            raise ValueError("X_host must be [batch, cols] bf16")
        batch = X_host.shape[0]
        if tuple(Y_host.shape) != (batch, self.layout.rows):
            raise ValueError("Y_host must be [batch, rows]")
        code = Y_BF16 if Y_host.dtype == torch.bfloat16 else Y_F32
        rc = lib().lrbi_layer_forward_host(self._h, ctypes.c_void_p(X_host.data_ptr()), batch,
                                           ctypes.c_void_p(Y_host.data_ptr()), code, algo)
        if rc != OK:
            raise LrbiError(rc, "lrbi_layer_forward_host")
        return Y_host

    def close(self):
        if self._h:
            lib().lrbi_layer_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
