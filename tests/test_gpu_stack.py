"""Several pruned blocks in a row out of the library's calls, training and in 8 bits, against torch in 64 bits.

Tolerances.  Activations and gradients pass between calls in bf16: each rounding is 2^-9 of a value (1.1e-3 rms); behind one another
lie at most eight of them a block, and a block's share of the residual stream (a gate below 1) makes them smaller there.  2e-2 of the
norm a block is several times their sum.  An 8-bit value of 512 normal ones is off by up to half a step, top / 254, with top some
3.5 deviations: 0.8 % rms of the deviation; two of its kind (tokens, weights) in each of a block's two products: 1.6 %, and 3.2 %
where what an activation makes of it (0.8 % more of another scale) is counted twice."""
import numpy as np
import pytest

import oracle
from paper_1905_05686_b200 import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def masked(layer):
    Ip, Iz = synth.make_factors(layer.layer)
    M = torch.from_numpy(oracle.decode_mask(Ip, Iz, layer.layer.rows, layer.layer.cols).astype(np.float64)).cuda()
    return layer.W.double() * M, M


def act64(h, act):
    return {"relu": lambda: h.clamp(min=0), "silu": lambda: h * torch.sigmoid(h), "gelu": lambda: h * torch.special.ndtr(h)}[act]()


def make(width, hidden, depth, act="gelu", seed=3):
    from paper_1905_05686_b200 import ffn
    stack = ffn.synthetic_stack(width, hidden, depth, 128, act, residual_scale=0.9)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for i, (block, joint) in enumerate(zip(stack.blocks, stack.joints)):
        block.gamma += 0.2 * torch.randn(width, generator=g, device="cuda")
        block.beta += 0.2 * torch.randn(width, generator=g, device="cuda")
        block.up.W.mul_(4 + i)
        block.up.refresh()
        for v in joint.vectors().values():
            v += 0.1 * torch.randn(width, generator=g, device="cuda")
    return stack, g


def reference(stack, x, up, down, vectors):
    """The stack in 64 bits, on leaves."""
    eps = stack.blocks[0].eps
    norm = lambda v, w, b: torch.nn.functional.layer_norm(v, v.shape[1:], w, b, eps)
    for block, w1, w2, v in zip(stack.blocks, up, down, vectors):
        f = act64(norm(x, v["gamma"], v["beta"]) @ w1.t(), block.act) @ w2.t()
        x = stack.residual_scale * x + v["gate"] * norm(f, v["post_gamma"], v["post_beta"])
    return x


def leaves(stack, x):
    up, down = [masked(b.up)[0].requires_grad_() for b in stack.blocks], [masked(b.down)[0].requires_grad_() for b in stack.blocks]
    vectors = [{"gamma": b.gamma.double().requires_grad_(), "beta": b.beta.double().requires_grad_(),
                **{k: v.double().requires_grad_() for k, v in j.vectors().items()}} for b, j in zip(stack.blocks, stack.joints)]
    return x.double().requires_grad_(), up, down, vectors


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width,hidden,depth,act,tokens", [(256, 512, 1, "gelu", 72), (256, 640, 3, "silu", 200), (384, 512, 2, "gelu", 1)])
def test_training_step(width, hidden, depth, act, tokens, dtype):
    from paper_1905_05686_b200 import binding as b
    stack, g = make(width, hidden, depth, act)
    x = torch.randn((tokens, width), generator=g, device="cuda").to(dtype)
    dout = torch.randn((tokens, width), generator=g, device="cuda").to(dtype)
    out, kept = stack.forward(x)
    dx, grads = stack.backward(dout, kept)
    assert out.dtype == dx.dtype == dtype
    x64, up, down, vectors = leaves(stack, x)
    want = reference(stack, x64, up, down, vectors)
    want.backward(dout.double())
    tol = 2e-2 * depth
    assert off(out, want.detach()) <= tol and off(dx, x64.grad) <= tol
    for i, (block, got) in enumerate(zip(stack.blocks, grads)):
        assert set(got) == {"up", "down", "gamma", "beta", "post_gamma", "post_beta", "gate"}
        for name, leaf, layer in (("up", up[i], block.up), ("down", down[i], block.down)):
            M = masked(layer)[1]
            # the nonlinearity's input was kept in 8 bits: 2e-2 more, as for one block
            assert off(got[name], leaf.grad * M) <= tol + 2e-2, (i, name)
            assert not got[name][M == 0].any()
        for name, leaf in vectors[i].items():
            assert off(got[name], leaf.grad) <= tol + 2e-2, (i, name)
    assert b.device_status() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens", [1, 8, 33, 300])
def test_prompts(tokens, dtype):
    stack, g = make(512, 1024, 2)
    served = stack.prompts()
    x = torch.randn((tokens, 512), generator=g, device="cuda").to(dtype)
    got = served(x)
    assert got.dtype == dtype
    x64, up, down, vectors = leaves(stack, x)
    with torch.no_grad():
        want = reference(stack, x64, up, down, vectors)
        assert off(got, want) <= 2 * 3.2e-2 + 2e-2
        # closer, against the weights that the 8-bit ones stand for
        exact = lambda w: w.q[:, :w.cols].double() * w.scale.double()[:, None]
        for i, block in enumerate(served.blocks):
            for w, layer in ((block.up, stack.blocks[i].up), (block.down, stack.blocks[i].down)):
                assert not exact(w)[masked(layer)[1] == 0].any()
        want = reference(stack, x64, [exact(b.up) for b in served.blocks], [exact(b.down) for b in served.blocks], vectors)
        assert off(got, want) <= 2 * 2.4e-2 + 2e-2
    # a token's result does not depend on the tokens beside it, as long as the same kernel multiplies: sums are exact in all of them
    assert torch.equal(served(x[:1].contiguous())[0], got[0])


def test_one_block_in_8_bits():
    from paper_1905_05686_b200 import ffn
    block = ffn.synthetic_block(512, 1280, 256)
    block.up.W.mul_(4)
    served = block.prompts()
    x = torch.randn((50, 512), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    W1, W2 = masked(block.up)[0], masked(block.down)[0]
    u = torch.nn.functional.layer_norm(x.double(), (512,), block.gamma.double(), block.beta.double(), block.eps)
    want = act64(u @ W1.t(), "gelu") @ W2.t()
    got = served(x)
    assert off(got.double() - x.double(), want) <= 3.2e-2 + 2e-2 + 2.0 ** -9 * float(got.double().norm() / want.norm())
    before = served(x)
    block.step({"up": torch.ones_like(W1).float(), "down": torch.ones_like(W2).float(), "gamma": torch.ones(512, device="cuda"), "beta": torch.ones(512, device="cuda")}, 0.1)
    assert torch.equal(served(x), before)


def test_captured():
    """The stack in 8 bits captured into a graph while an eager pass is under way, and replayed on other inputs."""
    stack, g = make(256, 512, 2)
    served = stack.prompts()
    x = [torch.randn((40, 256), generator=g, device="cuda").bfloat16() for _ in range(3)]
    want = [served(v) for v in x]
    fixed = x[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = served(fixed)
    for v, w in zip(x, want):
        fixed.copy_(v)
        graph.replay()
        assert torch.equal(got, w) and torch.equal(served(v), w)


def test_wrong_stacks():
    from paper_1905_05686_b200 import ffn
    block = ffn.synthetic_block(256, 512, 128)
    with pytest.raises(ValueError):
        ffn.PrunedStack([block], [])
    with pytest.raises(ValueError):
        ffn.PrunedStack([], [])


def test_blocks_of_a_stack_are_alike():
    from paper_1905_05686_b200 import ffn
    joint = ffn.synthetic_stack(256, 512, 1, 128).joints[0]
    wide, other = ffn.synthetic_block(512, 512, 128), ffn.synthetic_block(256, 512, 128)
    other.eps = 1e-3
    for second in (wide, other):
        with pytest.raises(ValueError):
            ffn.PrunedStack([ffn.synthetic_block(256, 512, 128), second], [joint, joint])


def test_a_block_twice():
    """A stack that goes through the same block twice: the gradients of both uses, apart, are those of two equal blocks."""
    from paper_1905_05686_b200 import ffn
    one, two = ffn.synthetic_stack(256, 512, 1, 128), ffn.synthetic_stack(256, 512, 2, 128)
    shared = ffn.PrunedStack(one.blocks * 2, one.joints * 2)
    for block, joint in zip(two.blocks, two.joints):
        for a, b in ((block.up.W, one.blocks[0].up.W), (block.down.W, one.blocks[0].down.W)):
            a.copy_(b)
        block.up.refresh()
        block.down.refresh()
    x = torch.randn((70, 256), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    results = []
    for stack in (shared, two):
        out, kept = stack.forward(x)
        dx, grads = stack.backward(torch.ones_like(out), kept)
        results.append([out, dx, stack.prompts()(x)] + [g[name] for g in grads for name in sorted(g)])
    assert all(torch.equal(a, b) for a, b in zip(*results))
