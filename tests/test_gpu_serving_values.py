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
