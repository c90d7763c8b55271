"""Values at the edges of the block's operators' range, where a formula meets infinities, zeros and the ends of a type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def _b():
    from paper_1905_05686_b200 import binding
    return binding


@pytest.mark.parametrize("rows,cols,pad", [(5, 512, 0), (3, 16, 8), (7, 301, 0), (4, 256, 3)], ids=lambda v: str(v))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_activation_of_infinities(act, dtype, rows, cols, pad):
    """The formula's own result: +inf for +inf; 0 for relu of -inf, NaN (infinity times zero) for gelu and silu of it."""
    b = _b()
    h = torch.randn((rows, cols + pad), device="cuda").to(dtype)[:, :cols]
    plain = b.lrbi_activation(h.contiguous(), act)
    at = {(0, 0): INF, (1, 7): -INF, (rows - 1, cols - 1): INF, (rows - 1, cols - 2): NAN, (2, 3): -INF, (0, cols // 2): INF}
    for place, v in at.items():
        h[place] = v
    want = {INF: INF, -INF: 0.0 if act == "relu" else NAN}
    a, kept = b.lrbi_activation(h, act, checkpoint=True)
    _, again = b.lrbi_activation_backward(torch.ones_like(h), h, act, restore=True)
    rest = torch.ones((rows, cols), dtype=torch.bool)
    for got in (a, b.lrbi_activation(h, act), again):
        got = got.float().cpu()
        for place, v in at.items():
            w = want.get(v, NAN)
            assert got[place] == w or (np.isnan(w) and torch.isnan(got[place])), (place, v)
            rest[place] = False
        assert torch.equal(got[rest], plain.float().cpu()[rest])
    stands = b.lrbi_checkpoint_load(kept, F32)
    assert all(torch.isnan(stands[place]) for place in at)          # a group with either restores as NaN


def test_gelu_against_64_bits_in_its_tails():
    """Relative to the result, where gelu is small too: lrbi.h's bound 2^-20 (1 + h^2 / 8).  Its parts: the tail's fit 2^-23, its
    evaluation in fp32 with the hardware's reciprocal 3 * 2^-23, exp2 2^-22, and 2^-23 h^2 for the argument of exp2 (three
    roundings of h^2 / 2 each).  Slopes: the same of both terms, and their sum's rounding."""
    from scipy.special import erfcx
    b = _b()
    h = np.concatenate([np.linspace(-13, 13, 400001), -np.logspace(-30, 1, 20000), np.logspace(-30, 1, 20000)]).astype(np.float32)
    h = h[None, : h.size // 8 * 8]
    x = h.astype(np.float64)
    m = np.abs(x)
    phi = np.exp(-x * x / 2) / np.sqrt(2 * np.pi)
    tail = erfcx(m / np.sqrt(2)) * np.exp(-x * x / 2) / 2            # Phi(-|h|), no cancellation
    value, slope = np.where(x > 0, x * (1 - tail), x * tail), np.where(x >= 0, 1 - tail, tail) + x * phi
    rel = 2.0 ** -20 * (1 + x * x / 8)
    t = torch.from_numpy(h).cuda()
    for cols in (h.shape[1], h.shape[1] - 3):                        # whole and ragged rows
        got, again = b.lrbi_activation_backward(torch.ones_like(t[:, :cols]), t[:, :cols], "gelu", restore=True)
        a = b.lrbi_activation(t[:, :cols], "gelu")
        at = np.s_[:, :cols]
        assert torch.equal(a, again)
        off = np.abs(a.cpu().numpy().astype(np.float64) - value[at])
        assert (off <= (m * tail * rel + 2.0 ** -23 * np.where(x > 0, x, 0) + 1e-44)[at]).all()
        off = np.abs(got.cpu().numpy().astype(np.float64) - slope[at])
        assert (off <= (rel * (tail + m * phi) + 2.0 ** -22 * np.where(x >= 0, 1.0, 0.0) + 1e-44)[at]).all()


def test_gelu_in_bf16_is_rounded_once_in_its_tails():
    """lrbi.h: off by 2^-13 of itself before it is rounded, 2^-5 of a step at most; exp2 and its argument 2^-8 of one down to -10."""
    from scipy.special import erfcx
    b = _b()
    h = torch.linspace(-10, -1, 4096, device="cuda").to(BF16)[None]
    x = h.float().cpu().numpy().astype(np.float64)
    value = x * erfcx(-x / np.sqrt(2)) * np.exp(-x * x / 2) / 2
    a = b.lrbi_activation(h, "gelu").float().cpu().numpy().astype(np.float64)
    step = 2.0 ** (np.floor(np.log2(np.abs(value))) - 7)
    assert (np.abs(a - value) <= step * (0.5 + 2.0 ** -5 + 2.0 ** -8)).all()


def test_quantize_ranges_up_to_the_end_of_fp32():
    """A group's range is finite in fp32 up to its largest number; beyond that the scale is NaN."""
    import test_gpu_w4 as w4
    b = _b()
    top = float(w4.f32([0x7F7F])[0])                                  # the largest bf16
    W = np.zeros((16, 128), np.float32)
    for row, low in enumerate((0.0, -1e36, -1.2e36, -1.3e36, -2e36, -1e38)):
        W[row, 3], W[row, 5], W[row, 70] = top, low, 1.0
    bits = w4.bf16_bits(W)
    W = w4.f32(bits)
    q, scale, zero = w4.quantize(W, np.ones_like(W, bool), 64)
    with np.errstate(over="ignore"):
        over = np.isinf(W[:, :64].max(1) - W[:, :64].min(1))
    assert 0 < over[:6].sum() < 5
    scale[over, 0], zero[over, 0], q[over, :64] = 0x7FC0, 8, 8
    got = b.lrbi_w4_quantize((16, 128, 16, 128, 1), b.to_device_bf16(bits.astype(np.uint16)), 64)
    packed, meta = w4.lay_out(q, scale, zero, 64)
    assert (got.meta.cpu().numpy().view(np.uint32).reshape(meta.shape) == meta).all()
    assert (got.packed.cpu().numpy().view(np.uint32).reshape(packed.shape) == packed).all()


@pytest.mark.parametrize("rows", [3, 1500])              # a block has a row; a warp has one
@pytest.mark.parametrize("cols", [256, 20480])
def test_rstd_of_variances_that_are_zero_or_tiny(rows, cols):
    """1 / sqrt(var + eps) for eps = 0: infinite for equal values, and right where the variance is below fp32's normal range."""
    b = _b()
    rows = min(rows, 3 if cols > 16384 else rows)
    gamma = torch.ones(cols, device="cuda")
    x = torch.full((rows, cols), 0.75, device="cuda")
    y, mean, rstd = b.lrbi_layer_norm(x, gamma, eps=0.0)
    assert (mean == 0.75).all() and torch.isinf(rstd).all() and (rstd > 0).all() and torch.isnan(y).all()
    # pairs (v, -v), squares of two units of 2^-149 and (rounded) of four in turn: the mean is 0, the variance three units
    v = torch.tensor([1.0, -1.0, 1.41, -1.41], device="cuda") * 2.0 ** -74
    x = v.repeat(rows, cols // 4)
    _, mean, rstd = b.lrbi_layer_norm(x, gamma, eps=0.0)
    assert (mean == 0).all()
    want = (3 * 2.0 ** -149) ** -0.5
    assert ((rstd.double() / want - 1).abs() <= 2.0 ** -20).all()


def test_sizes_of_copies_and_weights_are_checked_by_the_calls():
    """A Checkpoint's or W4Weights' fields may have changed since it was made: calls look at the arrays that they are given."""
    b = _b()
    x = torch.randn((6, 300), device="cuda")
    gamma = torch.ones(300, device="cuda")
    _, mean, rstd = b.lrbi_layer_norm(x, gamma)

    def copies():
        yield {"cols": 305}                       # (301 has the same arrays)
        yield {"rows": 7}
        yield {"cols": 4096}
        yield {"rows": -1}
        yield {"cols": 1 << 40}
        good = b.lrbi_checkpoint_store(x)
        yield {"q": good.q[:5]}
        yield {"q": good.q.view(torch.uint8)}
        yield {"q": good.q.t()}
        yield {"q": good.q.cpu()}
        yield {"scale": good.scale[:, :2].contiguous()}
        yield {"scale": good.scale.double()}
        yield {"scale": good.scale.cpu()}

    before = None
    for change in copies():
        kept = b.lrbi_checkpoint_store(x)
        for name, v in change.items():
            setattr(kept, name, v)
        before = b.launch_count()
        with pytest.raises((ValueError, TypeError, OverflowError)):
            b.lrbi_checkpoint_load(kept)
        with pytest.raises((ValueError, TypeError, OverflowError)):
            b.lrbi_layer_norm_backward(torch.ones((kept.rows if 0 < kept.rows < 9 else 6, min(kept.cols, 5000)), device="cuda"), kept, gamma, mean, rstd)
        with pytest.raises((ValueError, TypeError, OverflowError)):
            b.lrbi_activation_backward(torch.ones((kept.rows if 0 < kept.rows < 9 else 6, min(kept.cols, 5000)), device="cuda"), kept, "relu")
        assert b.launch_count() == before, change

    W = b.lrbi_w4_quantize((20, 64, 20, 64, 1), torch.randn((20, 64), device="cuda").bfloat16(), 64)
    for name, v in (("rows", 33), ("cols", 65), ("group", 32), ("rows", 0), ("packed", W.packed[:-4]), ("meta", W.meta[:-4]), ("meta", W.meta.cpu()),
                    ("packed", W.packed.float())):
        changed = b.W4Weights(W.packed, W.meta, 20, 64, 64)
        setattr(changed, name, v)
        before = b.launch_count()
        with pytest.raises((ValueError, TypeError)):
            b.lrbi_w4_gemv(changed, torch.zeros((2, changed.cols), device="cuda").bfloat16())
        assert b.launch_count() == before, name


@pytest.mark.parametrize("dtype,stride", [(BF16, (1 << 30) + 8), (BF16, (1 << 30) + 5), (F32, (1 << 29) + 8), (F32, (1 << 28) + 1)])
@pytest.mark.parametrize("cols", [264, 9000])
def test_rows_more_than_two_gigabytes_apart(cols, dtype, stride):
    """The same bits as side by side."""
    b = _b()
    base = torch.empty(stride + cols, dtype=dtype, device="cuda")
    x = torch.as_strided(base, (2, cols), (stride, 1))
    own = torch.randn((2, cols), device="cuda").to(dtype)
    x.copy_(own)
    gamma = torch.ones(cols, device="cuda")
    got = []
    for t in (x, own):
        y, mean, rstd, kept = b.lrbi_layer_norm(t, gamma, checkpoint=True)
        a, _ = b.lrbi_activation(t, "gelu", checkpoint=True)
        got.append((y, mean, rstd, kept.q, a, b.lrbi_activation_backward(t, t, "silu"), *b.lrbi_layer_norm_backward(t, t, gamma, mean, rstd, dres=t),
                    b.lrbi_checkpoint_store(t).q))
    if stride % 8 == 0:                 # both are whole vectors: sums in the same order
        assert all(torch.equal(p, q) for p, q in zip(*got))
    else:
        assert all(torch.equal(got[0][i], got[1][i]) for i in (3, 4, 5, -1))
        assert all((p.float() - q.float()).abs().max() <= 2.0 ** -7 * q.float().abs().max() for p, q in zip(*got))
