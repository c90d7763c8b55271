"""Values of the serving calls where they are easily lost: tokens of a nonlinearity to all of fp32's bits, rows far from zero, tokens of
many rows one by one.

Tolerances count roundings, 2^-24 of a value each (half a step of fp32)."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_1905_05686_b200 import binding
    return binding


def act64(h, act):
    if act == "relu":
        return h.clamp(min=0)
    return h * torch.special.expit(h) if act == "silu" else h.clamp(min=0) - h.abs() * 0.5 * torch.erfc(h.abs() * 0.5 ** 0.5)


def act_bound(h, act):
    """How far off the library states a result in fp32 to be, of itself."""
    return {"relu": 0 * h, "gelu": 2.0 ** -20 * (1 + h * h / 8), "silu": 2.0 ** -20 * (1 + h.abs())}[act]


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_tokens_of_every_16_bit_value_in_32_bits(B, act):
    """Rows of one value: 127 times the scale is act(h), off by the bound of a result in fp32 and by one rounding (the scale's)."""
    h = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(BF16).view(-1, 1)
    h = h[torch.isfinite(h)].view(-1, 1)
    t = B.lrbi_i8_tokens(h, act=act)
    x = h.double()[:, 0]
    want = act64(x, act).abs()
    there = want >= 2.0 ** -100
    off = (127 * t.scale.double() - want).abs() / want.clamp(min=2.0 ** -100) - act_bound(x, act) - 2.0 ** -24
    assert off[there].max() <= 0, (off[there].max(), x[there][off[there].argmax()])


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("rows,cols,pad", [(3, 4096, 0), (64, 1157, 0), (1100, 4096, 8), (900, 2049, 0), (400, 16384, 0), (260, 20001, 0)])
def test_bytes_of_the_nonlinearity(B, act, rows, cols, pad):
    """A byte is the exact quotient rounded to a whole number: off by half, by the bound of act(h) and of the row's largest value, and by
    two roundings (127 / top and the product)."""
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    channel = torch.where(torch.rand(cols + pad, generator=g, device="cuda") < 0.01, 8.0, 1.0)
    x = (torch.randn((rows, cols + pad), generator=g, device="cuda") * channel).to(BF16)[:, :cols]
    t = B.lrbi_i8_tokens(x, act=act)
    h = x.double()
    want, bound = act64(h, act), act_bound(h, act)
    top, at = want.abs().max(1, keepdim=True)
    exact = want * (127 / top)
    slack = exact.abs() * (bound + bound.gather(1, at) + 2.0 ** -23)
    assert ((t.q[:, :cols].double() - exact).abs() <= 0.5 + slack).all()


def norm64(v, eps):
    mean = v.mean(1, keepdim=True)
    rstd = ((v - mean).square().mean(1, keepdim=True) + eps) ** -0.5
    return (v - mean) * rstd, mean[:, 0], rstd[:, 0]


@pytest.mark.parametrize("which", ["x", "f"])
@pytest.mark.parametrize("rows,cols", [(30, 1000), (7, 801), (900, 4096), (620, 4099), (300, 16384), (300, 20000), (300, 32760), (5, 32768)])
def test_rows_far_from_zero(B, rows, cols, which):
    """Means 1e5 times the spread, of the stream (the second norm) or of f (the first).

    A sum over a row is a chain of at most 31 additions for any one value: 16 in a thread (four spans, two values at a time), 1 for its
    pair, 5 in the warp, 9 over a row's warps.  The mean that is subtracted first is off by up to 31 roundings of 1e5, a fifth of the
    spread; what is left is summed anew, in magnitudes of the spread: a normalised value n is off by 31 roundings of the mean, 20 of the
    root and a few of its own, together below 2^-18 (|n| + 1).  The mean that is kept is off by its own rounding and by less than
    another."""
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    x, f = rand(rows, cols) + (1e5 if which == "x" else 0), rand(rows, cols) * 0.7 - (7e4 if which == "f" else 0)
    gamma, post, gate = 1 + 0.2 * rand(cols), 1 + 0.2 * rand(cols), 0.5 + 0.1 * rand(cols)
    beta, post_beta = 0.2 * rand(cols), 0.2 * rand(cols)
    how = dict(post_gamma=post, post_beta=post_beta, gate=gate, residual_scale=0.75, eps=1e-5)
    out, u, stats = B.lrbi_residual_norm(x, f, gamma, beta, **how)
    n, mean, rstd = norm64(f.double(), 1e-5)
    assert ((stats[2] - mean).abs() <= 2.0 ** -23 * mean.abs() + 2.0 ** -18).all() and ((stats[3] / rstd - 1).abs() <= 2.0 ** -18).all()
    z, size = n * post.double() + post_beta.double(), (n.abs() + 1) * post.abs() + post_beta.abs()
    want = 0.75 * x.double() + gate.double() * z
    assert ((out - want).abs() <= 2.0 ** -18 * gate.abs() * size + 2.0 ** -24 * (want.abs() + 0.75 * x.abs() + (gate * z).abs())).all()
    n, mean, rstd = norm64(out.double(), 1e-5)
    assert ((stats[0] - mean).abs() <= 2.0 ** -23 * mean.abs() + 2.0 ** -18).all() and ((stats[1] / rstd - 1).abs() <= 2.0 ** -18).all()
    want, size = n * gamma.double() + beta.double(), (n.abs() + 1) * gamma.abs() + beta.abs()
    assert ((u - want).abs() <= 2.0 ** -18 * size).all()
    again, t, _ = B.lrbi_residual_norm(x, f, gamma, beta, tokens=True, **how)
    step = t.scale.double()[:, None]
    assert torch.equal(again, out)
    assert ((t.q[:, :cols] * step - want).abs() <= step * (0.5 + 2.0 ** -16) + 2.0 ** -18 * size).all()


def test_rows_of_one_value(B):
    """A spread of nothing: n is 0 but for what the mean is off, and the root is that of eps."""
    for cols in (40, 1000, 4096, 12891):
        value = torch.tensor([1000.0, -3.3, 1e6, 1 / 3], device="cuda")[:, None]
        x = value.expand(4, cols).contiguous()
        gamma = torch.ones(cols, device="cuda")
        out, u, stats = B.lrbi_residual_norm(x, torch.zeros_like(x), gamma)
        assert torch.equal(out, x) and ((stats[0] - value[:, 0]).abs() <= 2.0 ** -23 * value[:, 0].abs()).all()
        # what is left of a value, some 31 roundings, is taken off to 2^-18 of itself
        assert (u.abs() <= 2.0 ** -18 * 31 * 2.0 ** -24 * value.abs() / 1e-5 ** 0.5).all() and ((stats[1] * 1e-5 ** 0.5 - 1).abs() <= 2.0 ** -18 + (31 * 2.0 ** -24 * value[:, 0]) ** 2 * 2.0 ** -18 / 1e-5).all()


# Rows with one span a warp and with four; whole vectors and not; in one block, with the vectors in shared memory or read for every row;
# shared by two, four and eight blocks.
TOKEN_ROWS = [(3, 520), (70, 801), (400, 1024), (650, 1030), (900, 4096), (640, 4104), (620, 4099), (500, 8192), (310, 8704), (330, 9216), (310, 12345), (310, 12896), (300, 16384),
              (160, 16381), (300, 20000), (299, 32760), (70, 32761), (3000, 512), (6000, 200), (2500, 777)]


@pytest.mark.parametrize("post,gate,beta", [(True, True, True), (True, True, False), (False, False, False), (True, False, True), (False, True, False)])
@pytest.mark.parametrize("rows,cols", TOKEN_ROWS)
def test_tokens_between_blocks(B, rows, cols, post, gate, beta):
    """u as 8-bit tokens, value by value: off by half a step and 2^-18 of the magnitudes that go into u (64 roundings: sums over a row of
    31 additions at most, the root's 20, a few of its own); in fp32 the bytes and scales of u itself."""
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    gamma, vec = 1 + 0.2 * rand(cols), 0.2 * rand(cols)
    how = dict(post_gamma=1 + vec if post else None, post_beta=vec if post and beta else None, gate=0.4 + vec if gate else None, residual_scale=0.8, eps=1e-5)
    for x, f in ((BF16, BF16), (F32, BF16), (F32, F32)):
        for kind in ("layer", "rms"):
            a, b = (rand(rows, cols) + 0.3).to(x), (0.7 * rand(rows, cols) - 0.3).to(f)
            out, t, stats = B.lrbi_residual_norm(a, b, gamma, vec if beta else None, kind=kind, tokens=True, **how)
            plain, u, _ = B.lrbi_residual_norm(a, b, gamma, vec if beta else None, kind=kind, **how)
            assert torch.equal(out, plain) and stats is None and not t.q[:, cols:].any() and (t.q.abs().amax(1) == 127).all()
            o = out.double()
            mean = o.mean(1, keepdim=True) if kind == "layer" else 0.0
            rstd = ((o - mean).square().mean(1, keepdim=True) + 1e-5) ** -0.5
            offset = vec.double() if beta else 0.0
            want = (o - mean) * rstd * gamma.double() + offset
            size = (o.abs() + o.abs().mean(1, keepdim=True)) * rstd * gamma.double().abs() + abs(offset)
            step, top = t.scale.double()[:, None], want.abs().amax(1)
            assert ((t.q[:, :cols] * step - want).abs() <= step * (0.5 + 2.0 ** -16) + size * 2.0 ** -18).all()
            assert ((127 * step[:, 0] - top).abs() <= 2.0 ** -18 * size.amax(1) + 2.0 ** -23 * top).all()
            if f == F32:
                same = B.lrbi_i8_tokens(u)
                assert torch.equal(t.q, same.q) and torch.equal(t.scale, same.scale)
