"""The pruned feed-forward block out of the library's calls, training and serving, against torch in 64 bits.

Tolerances.  Activations and gradients pass between calls in bf16: each rounding is 2^-9 of a value (1.1e-3 rms), and at most
eight of them lie one behind another; products average them.  2e-2 of the norm is several times their sum.  What 8 bits cost is
compared apart: the reference takes the 8-bit copies by their definition."""
import numpy as np
import pytest

import oracle
from paper_1905_05686_b200 import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TOL = 2e-2


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def kept64(x):
    """What the 8-bit copy of x stands for, by its definition in fp32 steps."""
    rows, cols = x.shape
    p = torch.nn.functional.pad(x.float(), (0, -cols % 128)).view(rows, -1, 128)
    top = p.abs().amax(2, keepdim=True)
    steps = torch.full_like(top, 127.0)
    return (torch.round(p * (steps / top)) * (top / steps)).view(rows, -1)[:, :cols].double()


def masked(layer):
    Ip, Iz = synth.make_factors(layer.layer)
    M = torch.from_numpy(oracle.decode_mask(Ip, Iz, layer.layer.rows, layer.layer.cols).astype(np.float64)).cuda()
    return layer.W.double() * M, M


def act64(h, act):
    if act == "relu":
        return h.clamp(min=0), (h > 0).double()
    if act == "silu":
        s = torch.sigmoid(h)
        return h * s, s * (1 + h * (1 - s))
    phi = torch.special.ndtr(h)
    return h * phi, phi + h * torch.exp(-h * h / 2) / np.sqrt(2 * np.pi)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("shape", [(512, 1024, 256, 200), (256, 512, 128, 1), (384, 640, 128, 72)], ids=lambda s: "x".join(map(str, s)))
def test_training_step(shape, act):
    from paper_1905_05686_b200 import binding as b
    from paper_1905_05686_b200 import ffn
    width, hidden, tile, tokens = shape
    block = ffn.synthetic_block(width, hidden, tile, act=act)
    g = torch.Generator(device="cuda").manual_seed(3)
    block.gamma += 0.2 * torch.randn(width, generator=g, device="cuda")
    block.beta += 0.2 * torch.randn(width, generator=g, device="cuda")
    block.up.W.mul_(4)
    block.up.refresh()
    x = torch.randn((tokens, width), generator=g, device="cuda").bfloat16()
    dout = torch.randn((tokens, width), generator=g, device="cuda").bfloat16()
    out, kept = block.forward(x)
    dx, grads = block.backward(dout, kept)
    assert kept.nbytes < 0.54 * 2 * tokens * (width + hidden) + 8 * tokens + 64 * tokens

    W1, M1 = masked(block.up)
    W2, M2 = masked(block.down)
    gamma, beta, x64, d64 = block.gamma.double(), block.beta.double(), x.double(), dout.double()
    mean = x64.mean(1, keepdim=True)
    rstd = ((x64 - mean).square().mean(1, keepdim=True) + block.eps).rsqrt()
    u = (x64 - mean) * rstd * gamma + beta
    h = u @ W1.t()
    a, _ = act64(h, act)
    want = x64 + a @ W2.t()
    assert off(out, want) <= TOL
    # the backward pass sees the copies: that of x by its definition, that of h as the library rounded h
    n = (kept64(x) - mean) * rstd
    h8 = b.lrbi_checkpoint_load(kept.h, torch.float32).double()
    a8, slope = act64(h8, act)
    dh = (d64 @ W2) * slope
    dy = dh @ W1
    gg = dy * gamma
    want = {"down": (d64.t() @ a8) * M2, "up": (dh.t() @ (n * gamma + beta)) * M1, "gamma": (dy * n).sum(0), "beta": dy.sum(0)}
    for name, w in want.items():
        assert off(grads[name], w) <= TOL, name
    assert not grads["up"][M1 == 0].any() and not grads["down"][M2 == 0].any()
    want = d64 + rstd * (gg - gg.mean(1, keepdim=True) - n * (gg * n).mean(1, keepdim=True))
    assert off(dx, want) <= TOL
    # what 8 bits cost: a step of top / 127 in 128 values, about 0.7 % of a normal value's deviation; relu's kink moves a little more
    exact = (d64.t() @ a) * M2
    assert off(grads["down"], exact) <= TOL + 2e-2
    assert b.device_status() == 0


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens", [1, 5, 16])
def test_tokens(group, tokens):
    from paper_1905_05686_b200 import binding as b
    from paper_1905_05686_b200 import ffn
    block = ffn.synthetic_block(512, 1280, 256)
    block.up.W.mul_(4)
    served = block.tokens(group)
    x = torch.randn((tokens, 512), generator=torch.Generator(device="cuda").manual_seed(tokens), device="cuda").bfloat16()
    got = served(x)
    eye = lambda n: torch.eye(n, device="cuda").bfloat16()
    W1 = b.lrbi_w4_gemv(served.up, eye(512), y_dtype=torch.float32).t().double()
    W2 = b.lrbi_w4_gemv(served.down, eye(1280), y_dtype=torch.float32).t().double()
    assert not W1[masked(block.up)[1] == 0].any() and not W2[masked(block.down)[1] == 0].any()
    x64 = x.double()
    u = torch.nn.functional.layer_norm(x64, (512,), block.gamma.double(), block.beta.double(), block.eps)
    want = act64(u @ W1.t(), "gelu")[0] @ W2.t()
    assert off(got.double() - x64, want) <= TOL + 2.0 ** -9 * float(got.double().norm() / want.norm())
    # a token's result does not depend on the tokens beside it
    assert torch.equal(served(x[:1].contiguous())[0], got[0])


def test_example_runs():
    from paper_1905_05686_b200 import ffn
    ffn.main()


def test_tokens_are_served_from_what_was_taken():
    """Training that goes on after tokens() does not reach the served block."""
    from paper_1905_05686_b200 import ffn
    block = ffn.synthetic_block(256, 512, 128)
    served = block.tokens(64)
    x = torch.randn((3, 256), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    before = served(x)
    out, kept = block.forward(x)
    _, grads = block.backward(torch.ones_like(out), kept)
    block.step(grads, 0.5)
    assert grads["gamma"].abs().max() > 0 and torch.equal(served(x), before)
