"""Layer norm, 8-bit copies and the nonlinearity against plain numpy in 64 bits, through the C ABI.

Tolerances.  u = 2^-24.  A row's statistics are sums of fp32 values in a tree, a few u of the largest magnitude X of the row;
the tests allow 16 u (2^-20) of what enters each operation, twice that (and more) where several meet, and add half a step of
bf16 (2^-8 of the value, which also covers the step's upward jump at a power of two) where the output is bf16."""
import math

import numpy as np
import pytest
from scipy.special import ndtr

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32
TOL = 2.0 ** -20


def _b():
    from paper_1905_05686_b200 import binding
    return binding


def half_step(v, dtype):
    return 2.0 ** -8 * np.abs(v) + 1e-38 if dtype == BF16 else 0.0


def np64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def matrix(rows, cols, dtype, pad, seed, scale=1.0, shift=0.0):
    """A [rows, cols] slice of a wider array whose other columns hold NaN."""
    g = torch.Generator().manual_seed(seed)
    wide = torch.full((rows, cols + pad), float("nan"))
    wide[:, :cols] = torch.randn((rows, cols), generator=g) * scale + shift
    return wide.to(dtype).cuda()[:, :cols]


def norm64(x, gamma, beta, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    n = (x - mean) * rstd
    return n * gamma + beta, mean, rstd, n


def back64(dy, n, rstd, gamma):
    g = dy * gamma
    return rstd * (g - g.mean(1, keepdims=True) - n * (g * n).mean(1, keepdims=True)), (dy * n).sum(0), dy.sum(0)


def kept32(x):
    """(q, scale, what they stand for) by the definition, each step one fp32 operation."""
    rows, cols = x.shape
    groups = -(-cols // 128)
    p = np.zeros((rows, groups * 128), np.float32)
    p[:, :cols] = x
    p = p.reshape(rows, groups, 128)
    with np.errstate(all="ignore"):
        top = np.abs(p).max(2, keepdims=True)                    # NaN goes through
        fine, low = np.isfinite(top), top < np.float32(2.0 ** -118)
        q = np.rint(p * (np.float32(127) / top))
        q = np.where(fine & ~low, q, 0)
        scale = np.where(fine, np.where(low, np.float32(0), top / np.float32(127)), np.float32(np.nan)).astype(np.float32)
        stands = (q.astype(np.float32) * scale).reshape(rows, -1)[:, :cols]
    return q.reshape(rows, -1)[:, :cols].astype(np.int8), scale[:, :, 0], stands


NORM_SHAPES = [
    # rows, cols, pad
    (1, 1, 0), (5, 2, 3), (3, 7, 1), (9, 8, 0), (1, 255, 0), (17, 256, 8), (33, 257, 0), (2, 264, 0), (7, 801, 6), (4, 1000, 8),
    (3, 2049, 5), (1, 4096, 0), (600, 512, 0), (5, 8192, 0), (3, 8193, 0), (2, 8200, 0), (3, 12345, 1), (2, 16384, 8), (2, 16385, 0),
    (2, 20000, 0), (300, 129, 2),
    # several rows a block, of the widths at which the backward pass takes another form
    (310, 5123, 3), (450, 8193, 1), (300, 8456, 0), (300, 10248, 8), (310, 10753, 7), (450, 16383, 2), (300, 4104, 8),
]


@pytest.mark.parametrize("shape", NORM_SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,y_dtype,p_dtype", [(BF16, BF16, F32), (F32, F32, F32), (F32, BF16, BF16), (BF16, F32, BF16)],
                         ids=["bf16", "f32", "f32-bf16", "bf16-f32"])
def test_layer_norm(shape, dtype, y_dtype, p_dtype):
    b = _b()
    rows, cols, pad = shape
    x = matrix(rows, cols, dtype, pad, rows + cols, 1.5, 0.7)
    gamma, beta = matrix(1, cols, p_dtype, 0, 1, 0.3, 1.0)[0], matrix(1, cols, p_dtype, 0, 2, 0.3)[0]
    x64, g64, b64 = np64(x), np64(gamma), np64(beta)
    want, mean, rstd, n = norm64(x64, g64, b64, 1e-5)
    top = np.abs(x64).max(1, keepdims=True)
    for with_beta in (True, False):
        y, m, r, kept = b.lrbi_layer_norm(x, gamma, beta if with_beta else None, y_dtype=y_dtype, checkpoint=True)
        w = want if with_beta else n * g64
        # n is off by 2^-20 of X * rstd, and by the relative error of rstd, which is half of the variance's: 2^-20 (X rstd)^2 at most
        off = TOL * ((top * rstd + np.abs(n) * (1 + (top * rstd) ** 2)) * np.abs(g64) + np.abs(w) + np.abs(b64))
        assert y.dtype == y_dtype and (np.abs(np64(y) - w) <= off + half_step(w, y_dtype)).all()
        assert (np.abs(np64(m) - mean[:, 0]) <= TOL * top[:, 0]).all()
        assert (np.abs(np64(r) / rstd[:, 0] - 1) <= TOL * (1 + (top * rstd)[:, 0] ** 2)).all()
        q, scale, _ = kept32(x.float().cpu().numpy())
        assert (kept.q.cpu().numpy()[:, :cols] == q).all() and (kept.scale.cpu().numpy() == scale).all()
        assert not kept.q.cpu().numpy()[:, cols:].any()
    plain = b.lrbi_layer_norm(x, gamma, beta, y_dtype=y_dtype)
    assert len(plain) == 3 and torch.equal(plain[0], b.lrbi_layer_norm(x, gamma, beta, y_dtype=y_dtype, checkpoint=True)[0])


@pytest.mark.parametrize("shape", NORM_SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,dy_dtype,p_dtype", [(BF16, BF16, F32), (F32, F32, F32), (F32, BF16, BF16), (BF16, F32, BF16)],
                         ids=["bf16", "f32", "f32-bf16", "bf16-f32"])
def test_layer_norm_backward(shape, dtype, dy_dtype, p_dtype):
    b = _b()
    rows, cols, pad = shape
    x = matrix(rows, cols, dtype, pad, rows + cols, 1.5, 0.7)
    dy, dres = matrix(rows, cols, dy_dtype, pad, 5), matrix(rows, cols, dtype, pad, 6)
    gamma, beta = matrix(1, cols, p_dtype, 0, 1, 0.3, 1.0)[0], matrix(1, cols, p_dtype, 0, 2, 0.3)[0]
    x64, dy64, g64, b64, r64 = np64(x), np64(dy), np64(gamma), np64(beta), np64(dres)
    _, m, r, kept = b.lrbi_layer_norm(x, gamma, beta, checkpoint=True)
    mean, rstd = np64(m)[:, None], np64(r)[:, None]     # the statistics are inputs of the backward pass
    for copy in (False, True):
        src = kept32(x.float().cpu().numpy())[2].astype(np.float64) if copy else x64
        n = (src - mean) * rstd
        dx, dgamma, dbeta = back64(dy64, n, rstd, g64)
        g, X = np.abs(dy64 * g64), (np.abs(src).max(1, keepdims=True) + np.abs(mean)) * rstd
        along, across = (g * np.abs(n)).mean(1, keepdims=True), g.mean(1, keepdims=True)
        off = 4 * TOL * rstd * (g + across + (np.abs(n) + X) * along + np.abs(n) * X * across)
        got = b.lrbi_layer_norm_backward(dy, kept if copy else x, gamma, m, r, dx_dtype=dtype)
        assert len(got) == 3 and got[0].dtype == dtype and got[1].dtype == got[2].dtype == F32
        assert (np.abs(np64(got[0]) - dx) <= off + half_step(dx, dtype)).all()
        assert (np.abs(np64(got[1]) - dgamma) <= 4 * TOL * (np.abs(dy64) * (np.abs(n) + X)).sum(0)).all()
        assert (np.abs(np64(got[2]) - dbeta) <= 4 * TOL * np.abs(dy64).sum(0)).all()
        more = b.lrbi_layer_norm_backward(dy, kept if copy else x, gamma, m, r, beta=beta, dres=dres, restore=True, dx_dtype=dtype)
        assert torch.equal(more[1], got[1]) and torch.equal(more[2], got[2])        # the same bits again
        assert (np.abs(np64(more[0]) - (dx + r64)) <= off + TOL * np.abs(r64) + half_step(dx + r64, dtype)).all()
        y = n * g64 + b64
        assert more[3].dtype == dy_dtype
        assert (np.abs(np64(more[3]) - y) <= 2 * TOL * ((np.abs(n) + X) * np.abs(g64) + np.abs(b64)) + half_step(y, dy_dtype)).all()


@pytest.mark.parametrize("rows,cols", [(4, 37), (9, 512), (3, 9000)])
def test_layer_norm_gradient_against_differences(rows, cols):
    """<dx, v> + <dgamma, w> + <dbeta, u> against the central difference of <y, dy> in 64 bits along (v, w, u)."""
    b = _b()
    rng = np.random.default_rng(rows)
    x, dy, v = (rng.standard_normal((rows, cols)).astype(np.float32).astype(np.float64) for _ in range(3))
    gamma, beta, w, u = (rng.standard_normal(cols).astype(np.float32).astype(np.float64) for _ in range(4))
    h = 1e-5
    f = lambda s: (norm64(x + s * v, gamma + s * w, beta + s * u, 1e-5)[0] * dy).sum()
    want = (f(h) - f(-h)) / (2 * h)
    t = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    _, m, r = b.lrbi_layer_norm(t(x), t(gamma), t(beta))
    dx, dgamma, dbeta = b.lrbi_layer_norm_backward(t(dy), t(x), t(gamma), m, r)
    got = (np64(dx) * v).sum() + (np64(dgamma) * w).sum() + (np64(dbeta) * u).sum()
    # dx, dgamma and dbeta are off by 2^-18 of terms of order |dy| (|n|^2 + 1); the difference by h^2 of third derivatives
    size = (np.abs(dy) * (np.abs(gamma) * np.abs(v) + np.abs(w) + np.abs(u)) * (1 + x * x)).sum()
    assert abs(got - want) <= 8 * TOL * size + 1e-6 * size


def test_layer_norm_of_no_rows():
    b = _b()
    x = torch.empty((0, 40), dtype=BF16, device="cuda")
    gamma = torch.ones(40, device="cuda")
    y, m, r, kept = b.lrbi_layer_norm(x, gamma, checkpoint=True)
    assert y.shape == (0, 40) and m.numel() == r.numel() == 0 and kept.shape == (0, 40)
    dx, dgamma, dbeta = b.lrbi_layer_norm_backward(x, x, gamma, m, r)
    assert dx.shape == (0, 40) and not dgamma.any() and not dbeta.any() and dgamma.numel() == 40


@pytest.mark.parametrize("cols", [8, 801, 4096, 5121, 8200, 9000, 10241, 16383, 16384, 20000])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_no_rows_of_any_width(cols, dtype):
    b = _b()
    x = torch.empty((0, cols), dtype=dtype, device="cuda")
    gamma = torch.ones(cols, device="cuda")
    y, m, r, kept = b.lrbi_layer_norm(x, gamma, checkpoint=True)
    for src in (x, kept):
        dx, dgamma, dbeta = b.lrbi_layer_norm_backward(x, src, gamma, m, r)
        assert y.shape == dx.shape == (0, cols) and not dgamma.any() and not dbeta.any()
    torch.cuda.synchronize()


@pytest.mark.parametrize("cols", [256, 4096, 9000, 16384])
@pytest.mark.parametrize("pad,off", [(4, 0), (0, 4), (8, 4), (4, 4), (0, 1)])
def test_fp32_rows_at_any_distance_from_a_vector(cols, pad, off):
    """Rows that start on 16-byte boundaries alone, or on none: right, and elementwise results with the bits of packed rows."""
    b = _b()
    rows = 5
    base = torch.randn(rows * (cols + pad) + off, device="cuda", generator=torch.Generator("cuda").manual_seed(cols + pad))
    x = torch.as_strided(base, (rows, cols), (cols + pad, 1), off)
    gamma, beta = matrix(1, cols, F32, 0, 1)[0], matrix(1, cols, F32, 0, 2)[0]
    y, m, r = b.lrbi_layer_norm(x, gamma, beta)
    want, mean, rstd, n = norm64(np64(x), np64(gamma), np64(beta), 1e-5)
    top = np.abs(np64(x)).max(1, keepdims=True)
    off64 = TOL * ((top * rstd + np.abs(n) * (1 + (top * rstd) ** 2)) * np.abs(np64(gamma)) + np.abs(want) + np.abs(np64(beta)))
    assert (np.abs(np64(y) - want) <= off64).all()
    own = x.contiguous()
    a, kept = b.lrbi_activation(x, "gelu", checkpoint=True)
    a1, kept1 = b.lrbi_activation(own, "gelu", checkpoint=True)
    assert torch.equal(a, a1) and torch.equal(kept.q, kept1.q) and torch.equal(kept.scale, kept1.scale)
    assert torch.equal(b.lrbi_activation_backward(x, x, "gelu"), b.lrbi_activation_backward(own, own, "gelu"))
    assert torch.equal(b.lrbi_checkpoint_store(x).q, b.lrbi_checkpoint_store(own).q)


@pytest.mark.parametrize("cols", [800, 801, 9000, 16383])
def test_offsets_past_32_bits(cols):
    """Rows so far apart that the last begin beyond 2^32 bytes: the same bits as side by side."""
    b = _b()
    rows, stride = 18, (1 << 27) - 8
    base = torch.empty(rows * stride, dtype=BF16, device="cuda")
    x = torch.as_strided(base, (rows, cols), (stride, 1))
    own = matrix(rows, cols, BF16, 0, 3)
    x.copy_(own)
    gamma = matrix(1, cols, F32, 0, 1)[0]
    far, near = b.lrbi_layer_norm(x, gamma, checkpoint=True), b.lrbi_layer_norm(own, gamma, checkpoint=True)
    same = [(far[i], near[i]) for i in range(3)] + [(far[3].q, near[3].q)]
    back = [b.lrbi_layer_norm_backward(t, t, gamma, near[1], near[2]) for t in (x, own)]
    act = [b.lrbi_activation(t, "silu", checkpoint=True) for t in (x, own)]
    dact = [b.lrbi_activation_backward(t, k, "silu", restore=True) for t, (_, k) in zip((x, own), act)]
    same += list(zip(*back)) + [(act[0][0], act[1][0]), (act[0][1].q, act[1][1].q)] + list(zip(*dact))
    for u, v in same:
        assert torch.equal(u, v)
    assert not torch.isnan(near[0]).any()


def test_layer_norm_of_equal_values_and_far_offsets():
    """Variance 0 leaves beta and finite gradients; an offset of 2^12 times the spread does not cancel in the variance."""
    b = _b()
    x = torch.full((3, 777), 3.25, device="cuda")
    gamma, beta = torch.ones(777, device="cuda"), torch.full((777,), 0.5, device="cuda")
    y, m, r = b.lrbi_layer_norm(x, gamma, beta)
    assert (y == 0.5).all() and (m == 3.25).all()
    dx, _, _ = b.lrbi_layer_norm_backward(torch.randn_like(x), x, gamma, m, r)
    assert torch.isfinite(dx).all()
    x = matrix(5, 1000, F32, 0, 3) + 4096
    want, mean, rstd, _ = norm64(np64(x), 1.0, 0.0, 1e-5)
    y, m, r = b.lrbi_layer_norm(x, torch.ones(1000, device="cuda"))
    # mean is off by 16 u of 4096; that enters the variance squared, and n once
    assert (np.abs(np64(r) / rstd[:, 0] - 1) <= 1e-5).all()
    assert (np.abs(np64(y) - want) <= TOL * 4097 * rstd + 1e-5 * np.abs(want)).all()


def test_layer_norm_nan_stays_in_its_row():
    b = _b()
    x = matrix(12, 300, F32, 4, 3)
    x[5, 7] = float("nan")
    x[9, 299] = float("inf")
    gamma = torch.ones(300, device="cuda")
    y, m, r, kept = b.lrbi_layer_norm(x, gamma, checkpoint=True)
    bad = torch.zeros(12, dtype=torch.bool, device="cuda")
    bad[[5, 9]] = True
    assert torch.isnan(y[5]).all() and not torch.isfinite(y[9]).any() and torch.isfinite(y[~bad]).all()
    back = b.lrbi_checkpoint_load(kept, F32)
    assert torch.isnan(back[5, :128]).all() and torch.isnan(back[9, 256:]).all()
    back[5, :128] = 0
    back[9, 256:] = 0
    assert torch.isfinite(back).all()


KEEP_SHAPES = [(1, 1, 0), (3, 5, 2), (2, 16, 0), (7, 24, 8), (4, 127, 0), (9, 128, 0), (5, 129, 1), (3, 136, 0), (40, 500, 0), (31, 2056, 8), (6, 2500, 3),
               (2, 16385, 0), (1000, 72, 0), (17, 1157, 3)]


@pytest.mark.parametrize("shape", KEEP_SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_checkpoint(shape, dtype):
    """Bytes and scales are those of the definition, bit for bit; so is what they stand for."""
    b = _b()
    rows, cols, pad = shape
    x = matrix(rows, cols, dtype, pad, rows * cols, 2.0)
    kept = b.lrbi_checkpoint_store(x)
    q, scale, stands = kept32(x.float().cpu().numpy())
    assert (kept.q.cpu().numpy()[:, :cols] == q).all() and not kept.q.cpu().numpy()[:, cols:].any()
    assert (kept.scale.cpu().numpy() == scale).all()
    assert (b.lrbi_checkpoint_load(kept, F32).cpu().numpy() == stands).all()
    assert torch.equal(b.lrbi_checkpoint_load(kept, BF16).cpu(), torch.from_numpy(stands).to(BF16))
    top = np.repeat(np.abs(scale) * 127, 128, 1)[:, :cols]
    assert (np.abs(stands - x.float().cpu().numpy()) <= top / 254 * (1 + 1e-5)).all()


def test_checkpoint_of_hard_groups():
    """Zeros, tiny and huge values, ties, infinities and NaN, one kind to a group."""
    b = _b()
    x = np.zeros((9, 300), np.float32)
    x[1, :128] = np.linspace(-1e-40, 1e-40, 128)             # below 2^-118: zeros
    x[2, :128] = np.float32(2.0 ** -118) * np.linspace(-1, 1, 128)
    x[3] = np.float32(3.4e38) * np.linspace(-1, 1, 300)
    x[4, :256] = np.tile(np.arange(-64, 64), 2) + 0.5        # steps of top / 127: halves tie
    x[4, 0], x[4, 128] = 127, -127
    x[5, 3], x[5, 200] = np.nan, 7
    x[6, 140], x[6, 2] = np.inf, 1
    x[7, 299] = -np.inf
    x[8, 255] = -5                                           # a single value
    q, scale, stands = kept32(x)
    kept = b.lrbi_checkpoint_store(torch.from_numpy(x).cuda())
    assert (kept.q.cpu().numpy()[:, :300] == q).all()
    assert np.array_equal(kept.scale.cpu().numpy(), scale, equal_nan=True)
    assert np.array_equal(b.lrbi_checkpoint_load(kept, F32).cpu().numpy(), stands, equal_nan=True)
    assert np.isnan(scale[5, 0]) and not np.isnan(scale[5, 1]) and np.isnan(scale[6, 1]) and np.isnan(scale[7, 2])


def act64(h, act):
    if act == "relu":
        return np.maximum(h, 0), (h > 0).astype(np.float64)
    if act == "silu":
        s = 1 / (1 + np.exp(-h))
        return h * s, s * (1 + h * (1 - s))
    phi = ndtr(h)
    return h * phi, phi + h * np.exp(-h * h / 2) / math.sqrt(2 * math.pi)


def act_off(h, act):
    """(value's, slope's) allowance: 7.5e-8 for the series of Phi (half its bound on erfc), and the hardware's exp2 and
    reciprocal at 2^-22 each, with the rounding of the exponent's argument (u |argument| log2 e) on top."""
    if act == "relu":
        return 0 * h, 0 * h
    if act == "silu":
        s = 1 / (1 + np.exp(-h))
        e = 4 * 2.0 ** -22 * (1 + np.abs(h))
        return np.abs(h) * s * e, s * e * (2 + np.abs(h))
    e = 2.0 ** -21 * (1 + h * h)
    d = np.exp(-h * h / 2)
    off = 7.5e-8 + e * d + 2.0 ** -23
    return np.abs(h) * off, off + np.abs(h) * d * e


@pytest.mark.parametrize("shape", KEEP_SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype,a_dtype", [(BF16, BF16), (F32, F32), (F32, BF16), (BF16, F32)], ids=["bf16", "f32", "f32-bf16", "bf16-f32"])
def test_activation(shape, act, dtype, a_dtype):
    b = _b()
    rows, cols, pad = shape
    h, da = matrix(rows, cols, dtype, pad, rows + cols, 2.5), matrix(rows, cols, a_dtype, pad, 8)
    h64, da64 = np64(h), np64(da)
    value, slope = act64(h64, act)
    off_v, off_s = act_off(h64, act)
    a, kept = b.lrbi_activation(h, act, a_dtype=a_dtype, checkpoint=True)
    assert a.dtype == a_dtype and (np.abs(np64(a) - value) <= off_v + half_step(value, a_dtype)).all()
    assert torch.equal(a, b.lrbi_activation(h, act, a_dtype=a_dtype))
    q, scale, stands = kept32(h.float().cpu().numpy())
    assert (kept.q.cpu().numpy()[:, :cols] == q).all() and (kept.scale.cpu().numpy() == scale).all()
    for copy in (False, True):
        if copy:
            value, slope = act64(stands.astype(np.float64), act)
            off_v, off_s = act_off(stands.astype(np.float64), act)
        dh, again = b.lrbi_activation_backward(da, kept if copy else h, act, restore=True, dh_dtype=dtype)
        want = da64 * slope
        assert dh.dtype == dtype and (np.abs(np64(dh) - want) <= np.abs(da64) * off_s + 2.0 ** -23 * np.abs(want) + half_step(want, dtype)).all()
        assert again.dtype == a_dtype and (np.abs(np64(again) - value) <= off_v + half_step(value, a_dtype)).all()
        assert torch.equal(dh, b.lrbi_activation_backward(da, kept if copy else h, act, dh_dtype=dtype))


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_activation_gradient_against_differences(act):
    b = _b()
    rng = np.random.default_rng(4)
    h = np.concatenate([rng.uniform(-6, 6, 2000), [-30.0, -12.0, -1e-3, 1e-3, 12.0, 30.0]]).astype(np.float32)[None]
    s = 1e-4
    h64 = h.astype(np.float64)
    d = (act64(h64 + s, act)[0] - act64(h64 - s, act)[0]) / (2 * s)
    got = np64(b.lrbi_activation_backward(torch.ones_like(torch.from_numpy(h)).cuda(), torch.from_numpy(h).cuda(), act))
    away = np.abs(h) > 2 * s if act == "relu" else np.ones_like(h, bool)
    # the difference's own error is s^2 / 6 of a third derivative below 3, and 2^-50 |h| / s
    assert (np.abs(got - d)[away] <= (act_off(h.astype(np.float64), act)[1] + 1e-8 + 1e-10)[away]).all()


def test_activation_far_values():
    b = _b()
    h = torch.tensor([[-200.0, -95.0, -40.0, 0.0, -0.0, 40.0, 200.0, 3e38]], device="cuda")
    for act in ("relu", "gelu", "silu"):
        a = b.lrbi_activation(h, act)[0]
        assert torch.isfinite(a).all() and (a[:3].abs() <= 1e-15).all() and (a[3:5] == 0).all() and torch.equal(a[5:], h[0, 5:])
        dh = b.lrbi_activation_backward(torch.ones_like(h), h, act)[0]
        assert torch.isfinite(dh).all() and (dh[:3].abs() <= 1e-14).all() and (dh[5:] == 1).all()
    nan = torch.full((2, 300), float("nan"), device="cuda")
    for act in ("relu", "gelu", "silu"):
        assert torch.isnan(b.lrbi_activation(nan, act)).all()
        assert torch.isnan(b.lrbi_activation_backward(torch.ones_like(nan), nan, act)).all()
        assert torch.isnan(b.lrbi_activation_backward(torch.ones_like(nan), b.lrbi_checkpoint_store(nan), act)).all()


def test_rows_past_32_bits():
    """Element offsets beyond 2^31: the last rows of a matrix of 2^31 + some elements are treated like the first."""
    b = _b()
    cols, stride = 64, 1 << 20
    rows = 2 ** 11 + 3
    wide = torch.zeros((rows, stride), dtype=BF16, device="cuda")
    x = wide[:, :cols]
    x.copy_(torch.randn((rows, cols), device="cuda"))
    gamma = torch.ones(cols, device="cuda")
    y, m, r, kept = b.lrbi_layer_norm(x, gamma, checkpoint=True)
    y2, _, _, kept2 = b.lrbi_layer_norm(x.contiguous(), gamma, checkpoint=True)
    assert torch.equal(y, y2) and torch.equal(kept.q, kept2.q)
    assert torch.equal(b.lrbi_activation(x, "gelu"), b.lrbi_activation(x.contiguous(), "gelu"))
    dy = torch.randn_like(y)
    for got, want in zip(b.lrbi_layer_norm_backward(dy, x, gamma, m, r), b.lrbi_layer_norm_backward(dy, x.contiguous(), gamma, m, r)):
        assert torch.equal(got, want)


def test_other_streams_and_graphs():
    b = _b()
    x, dy = matrix(300, 1000, BF16, 0, 1), matrix(300, 1000, BF16, 0, 2)
    gamma, beta = torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda")

    def step(stream=None):
        y, m, r, kept = b.lrbi_layer_norm(x, gamma, beta, checkpoint=True, stream=stream)
        a, kept_a = b.lrbi_activation(y, "gelu", checkpoint=True, stream=stream)
        dh, _ = b.lrbi_activation_backward(dy, kept_a, "gelu", restore=True, stream=stream)
        return (a, dh) + b.lrbi_layer_norm_backward(dh, kept, gamma, m, r, stream=stream)

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step(side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for t in held:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(held, want))


def test_refusals():
    b = _b()
    x = torch.zeros((4, 40), device="cuda")
    gamma = torch.ones(40, device="cuda")
    for bad in (x.double(), x.half(), x[0], x.cpu(), None):
        with pytest.raises(TypeError):
            b.lrbi_layer_norm(bad, gamma)
        with pytest.raises(TypeError):
            b.lrbi_checkpoint_store(bad)
        with pytest.raises(TypeError):
            b.lrbi_activation(bad, "relu")
    for bad in (x.t(), x[:, ::2], x[:1].expand(4, 40)):
        with pytest.raises(ValueError):
            b.lrbi_checkpoint_store(bad)
    with pytest.raises(ValueError):
        b.lrbi_layer_norm(x, gamma[:39].contiguous())
    with pytest.raises(ValueError):
        b.lrbi_layer_norm(x, gamma, gamma.bfloat16())
    with pytest.raises(TypeError):
        b.lrbi_layer_norm(x, gamma.double())
    with pytest.raises(b.LrbiError):
        b.lrbi_layer_norm(x, gamma, eps=-1.0)
    with pytest.raises(ValueError):
        b.lrbi_activation(x, "tanh")
    y, m, r, kept = b.lrbi_layer_norm(x, gamma, checkpoint=True)
    with pytest.raises(ValueError):
        b.lrbi_layer_norm_backward(x[:3], kept, gamma, m, r)
    with pytest.raises(TypeError):
        b.lrbi_layer_norm_backward(x, kept, gamma, m[:3], r)
    with pytest.raises(ValueError):
        b.lrbi_layer_norm_backward(x, x, gamma, m, r, dres=x.bfloat16())
    with pytest.raises(ValueError):
        b.lrbi_activation_backward(x[:, :39].contiguous(), kept, "relu")
    with pytest.raises(ValueError):
        b.Checkpoint(kept.q, kept.scale, 4, 60)
