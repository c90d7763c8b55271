"""4-bit weights: the quantiser bit for bit against its definition, the product against numpy in 64 bits, through the C ABI.

Tolerance of the product in fp32: weights and activations enter exactly, a group's products are summed by at most eight
tensor-core steps and at most a few hundred fp32 additions follow; 2^-18 of the sum of magnitudes is several times that."""
import numpy as np
import pytest

import oracle
from paper_1905_05686_b200 import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _b():
    from paper_1905_05686_b200 import binding
    return binding


def f32(bits):
    return (np.asarray(bits, dtype=np.uint32) << 16).view(np.float32)


def bf16_bits(v):
    u = np.asarray(v, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint32)


def quantize(W, kept, group):
    """(q, scale bits, z) by the definition; W float32 [rows, cols]."""
    rows, cols = W.shape
    groups = -(-cols // group)
    q, scale, zero = np.zeros((rows, cols), np.int64), np.zeros((rows, groups), np.uint32), np.zeros((rows, groups), np.int64)
    for g in range(groups):
        at = slice(g * group, min(cols, (g + 1) * group))
        w, k = W[:, at], kept[:, at]
        with np.errstate(all="ignore"):
            v = np.where(k, w, np.float32(0))
            bad = ~np.isfinite(v).all(1)
            lo, hi = np.minimum(np.nanmin(v, 1), 0).astype(np.float32), np.maximum(np.nanmax(v, 1), 0).astype(np.float32)
            bits = np.where(bad, 0x7FC0, bf16_bits((hi - lo) / np.float32(15)))
            s = f32(bits)
            fine = ~bad & (s > 0)
            z = np.where(fine, np.clip(np.rint(-lo / s), 0, 15), 8).astype(np.int64)
            each = np.clip(np.rint(w / s[:, None]) + z[:, None], 0, 15)
            q[:, at] = np.where(k & fine[:, None], np.nan_to_num(each), z[:, None]).astype(np.int64)
        scale[:, g], zero[:, g] = bits, z
    return q, scale, zero


def lay_out(q, scale, zero, group):
    """(packed, meta) as lrbi.h words it."""
    rows, cols = q.shape
    tiles, units, groups = -(-rows // 16), -(-cols // 64), -(-cols // group)
    full = np.zeros((tiles * 16, max(units * 64, groups * group)), np.int64)
    full[:rows, :cols] = q
    z = np.zeros((tiles * 16, groups), np.int64)
    z[:rows] = zero
    full[:, cols:groups * group] = np.repeat(z, group, 1)[:, cols:]
    packed = np.zeros((tiles, units, 32, 4), np.uint32)
    for j in range(8):
        i = 2 * (j // 2 & 1) + j // 4
        for lane in range(32):
            g, t = lane // 4, lane % 4
            for s in range(4):
                v = full[g + 8 * (j & 1)::16, 32 * (s // 2) + 8 * t + 4 * (s & 1) + i::64][:, :units]
                packed[:, :, lane, s] |= (v.astype(np.uint32) << np.uint32(4 * j))
    sc = np.zeros((tiles * 16, groups), np.uint32)
    sc[:rows] = scale
    meta = (sc << 16 | z.astype(np.uint32)).reshape(tiles, 16, groups).transpose(0, 2, 1)
    return packed, np.ascontiguousarray(meta)


def weights(b, q, scale, zero, group):
    packed, meta = lay_out(q, scale, zero, group)
    t = lambda a: torch.from_numpy(a.reshape(-1).view(np.int32)).cuda()
    return b.W4Weights(t(packed), t(meta), q.shape[0], q.shape[1], group)


SHAPES = [
    # rows, cols, group, batch
    (1, 1, 32, 1), (3, 5, 128, 2), (16, 64, 64, 8), (17, 65, 32, 9), (16, 128, 128, 16), (40, 129, 128, 7), (33, 192, 128, 3),
    (100, 200, 64, 17), (500, 800, 32, 1), (64, 2056, 128, 5), (48, 8192, 64, 12), (16, 16384, 128, 1), (31, 5001, 32, 8), (200, 75, 128, 40),
    (1040, 1024, 128, 4), (5, 16383, 64, 13),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gemv(shape):
    b = _b()
    rows, cols, group, batch = shape
    rng = np.random.default_rng(rows * cols)
    groups = -(-cols // group)
    q, zero = rng.integers(0, 16, (rows, cols)), rng.integers(0, 16, (rows, groups))
    scale = bf16_bits(rng.uniform(-0.02, 0.02, (rows, groups)))
    X = bf16_bits(rng.standard_normal((batch, cols)))
    w = (q - np.repeat(zero, group, 1)[:, :cols]) * np.repeat(f32(scale).astype(np.float64), group, 1)[:, :cols]
    x = f32(X).astype(np.float64)
    want, size = x @ w.T, np.abs(x) @ np.abs(w).T
    W = weights(b, q, scale, zero, group)
    Xd = torch.from_numpy(X.astype(np.uint16).view(np.int16)).cuda().view(torch.bfloat16)
    got = b.lrbi_w4_gemv(W, Xd, y_dtype=torch.float32)
    assert (np.abs(got.cpu().numpy() - want) <= 2.0 ** -18 * size).all()
    again = b.lrbi_w4_gemv(W, Xd)
    assert again.dtype == torch.bfloat16 and torch.equal(again, got.to(torch.bfloat16))
    assert torch.equal(b.lrbi_w4_gemv(W, Xd, y_dtype=torch.float32), got)
    # each row of the batch by itself gives the bits that it has in the batch
    for i in {0, batch - 1}:
        assert torch.equal(b.lrbi_w4_gemv(W, Xd[i:i + 1].contiguous(), y_dtype=torch.float32)[0], got[i])


def test_gemv_of_no_rows_and_unaligned_rows():
    b = _b()
    rng = np.random.default_rng(3)
    q, zero, scale = rng.integers(0, 16, (20, 72)), rng.integers(0, 16, (20, 1)), bf16_bits(rng.uniform(0, 0.1, (20, 1)))
    W = weights(b, q, scale, zero, 128)
    assert b.lrbi_w4_gemv(W, torch.empty((0, 72), dtype=torch.bfloat16, device="cuda")).shape == (0, 20)
    X = torch.randn((3, 72), device="cuda").bfloat16()
    odd = torch.empty(3 * 72 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(3, 72)
    odd.copy_(X)
    assert torch.equal(b.lrbi_w4_gemv(W, odd), b.lrbi_w4_gemv(W, X))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("cols", [64, 75, 130, 1024])
def test_nothing_is_read_past_the_last_column(group, cols):
    """Activations after the last column, and nibbles of columns that are not there, do not reach the result."""
    b = _b()
    rng = np.random.default_rng(cols)
    groups = -(-cols // group)
    q, zero = rng.integers(0, 16, (24, cols)), rng.integers(0, 16, (24, groups))
    W = weights(b, q, bf16_bits(np.full((24, groups), 0.5)), zero, group)
    flat = torch.full((4 * cols + 64,), float("nan"), dtype=torch.bfloat16, device="cuda")
    flat[:4 * cols] = 1.0
    got = b.lrbi_w4_gemv(W, flat[:4 * cols].view(4, cols), y_dtype=torch.float32)
    want = 0.5 * (q - np.repeat(zero, group, 1)[:, :cols]).sum(1)
    assert (got.cpu().numpy() == want[None]).all()          # whole numbers times 0.5: exact


@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1, 32), (20, 70, 8, 32, 5, 64), (37, 300, 16, 100, 40, 128), (130, 513, 64, 128, 33, 32), (64, 256, 64, 256, 8, 128)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("indexed", [True, False])
def test_quantize(shape, indexed):
    b = _b()
    rows, cols, tm, tn, k, group = shape
    L = synth.Layer("w4", rows, cols, tm, tn, k, 0.4, 0.05)
    Ip, Iz = synth.make_factors(L)
    M = oracle.decode_mask(Ip, Iz, rows, cols).astype(bool) if indexed else np.ones((rows, cols), bool)
    Wb = synth.make_weights(L)
    if indexed:
        Wb = np.where(M, Wb, np.uint16(0x7FC0))             # pruned places hold NaN
    want = lay_out(*quantize(f32(Wb), M, group), group)
    args = (b.to_device_words(synth.pack_ip(Ip)), b.to_device_words(synth.pack_iz(Iz))) if indexed else (None, None)
    got = b.lrbi_w4_quantize(L, b.to_device_bf16(Wb), group, *args)
    meta = got.meta.cpu().numpy().view(np.uint32).reshape(want[1].shape)
    r = np.arange(want[1].shape[0])[:, None, None] * 16 + np.arange(16)[None, None]
    assert (meta[np.broadcast_to(r < rows, meta.shape)] == want[1][np.broadcast_to(r < rows, meta.shape)]).all()
    words = got.packed.cpu().numpy().view(np.uint32).reshape(want[0].shape)
    assert (words[:rows // 16] == want[0][:rows // 16]).all()           # tiles without rows past the last
    # the product with one-hot activations reads every weight back
    eye = torch.eye(cols, device="cuda").bfloat16()
    back = b.lrbi_w4_gemv(got, eye, y_dtype=torch.float32).t().cpu().numpy()
    q, scale, zero = quantize(f32(Wb), M, group)
    stands = (q - np.repeat(zero, group, 1)[:, :cols]) * np.repeat(f32(scale), group, 1)[:, :cols]
    assert (back == stands.astype(np.float32)).all()
    assert not back[~M].any()
    v = np.where(M, f32(Wb), 0)
    step = np.repeat(f32(scale), group, 1)[:, :cols]
    # half a step, and what the scale's rounding to bf16 takes off the range's end (2^-9 of at most 15 steps)
    assert (np.abs(stands - v) <= step * (0.5 + 15 * 2.0 ** -9 + 0.5) + 1e-12).all()


def test_quantize_odd_groups():
    """Groups without a kept weight, of one sign, of equal weights, and with weights that are not finite."""
    b = _b()
    W = np.zeros((16, 128), np.float32)
    W[1] = 0.25
    W[2] = -0.5
    W[3, ::2] = 1e-3
    W[4, 5] = np.nan
    W[5, 6] = np.inf
    W[6] = np.linspace(0.5, 1, 128)
    W[7, 0], W[7, 1] = 3e38, -3e38
    W = f32(bf16_bits(np.nan_to_num(W, nan=0, posinf=0)))
    W[4, 5], W[5, 6] = np.nan, np.inf
    bits = bf16_bits(W)
    bits[4, 5] = 0x7FC0
    q, scale, zero = quantize(W, np.ones_like(W, bool), 64)
    over = 7, 0                                             # a range beyond fp32
    scale[over], zero[over], q[7, :64] = 0x7FC0, 8, 8
    got = b.lrbi_w4_quantize((16, 128, 16, 128, 1), b.to_device_bf16(bits.astype(np.uint16)), 64)
    meta = got.meta.cpu().numpy().view(np.uint32).reshape(1, 2, 16)
    want = lay_out(q, scale, zero, 64)
    assert (meta == want[1]).all()
    assert (got.packed.cpu().numpy().view(np.uint32).reshape(want[0].shape) == want[0]).all()
    y = b.lrbi_w4_gemv(got, torch.ones((1, 128), device="cuda").bfloat16(), y_dtype=torch.float32)[0].cpu().numpy()
    assert np.isnan(y[[4, 5, 7]]).all() and np.isfinite(np.delete(y, [4, 5, 7])).all() and y[0] == 0


def test_refusals():
    b = _b()
    W = torch.zeros((16, 64), dtype=torch.bfloat16, device="cuda")
    ok = b.lrbi_w4_quantize((16, 64, 16, 64, 1), W, 64)
    for bad in (0, 16, 48, 256):
        with pytest.raises(ValueError):
            b.lrbi_w4_quantize((16, 64, 16, 64, 1), W, bad)
        with pytest.raises(ValueError):
            b.W4Weights(ok.packed, ok.meta, 16, 64, bad)
    with pytest.raises(TypeError):
        b.lrbi_w4_quantize((16, 64, 16, 64, 1), W.float(), 64)
    with pytest.raises(ValueError):
        b.lrbi_w4_quantize((16, 65, 16, 65, 1), W, 64)
    with pytest.raises(ValueError):
        b.W4Weights(ok.packed, ok.meta, 17, 64, 64)
    with pytest.raises(ValueError):
        b.lrbi_w4_gemv(ok, torch.zeros((1, 63), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(TypeError):
        b.lrbi_w4_gemv(ok, torch.zeros((1, 64), device="cuda"))
    with pytest.raises(TypeError):
        b.lrbi_w4_gemv(ok, torch.zeros((1, 64), dtype=torch.bfloat16, device="cuda"), y_dtype=torch.float16)
