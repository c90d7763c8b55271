"""A transformer's feed-forward block whose two layers are pruned by a low-rank binary index, out of the library's calls.

    out = x + act(norm(x) W1^T) W2^T,      W1, W2 seen through their index

``PrunedFFN`` retrains it: the forward pass keeps its input and the hidden layer's input in 8 bits (and two numbers a row),
the backward pass takes everything else from those copies.  ``TokenFFN`` serves it: both layers in 4 bits, pruned weights
exactly zero, a few tokens at a time.  ``PromptFFN`` serves it in 8 bits, any number of tokens at a time.

``PrunedStack`` retrains several blocks in a row, with a norm behind each, a gate and a residual scale between them,

    out = residual_scale x + gate norm(f),      f = act(norm(x) W1^T) W2^T,

what stands between two blocks being one call; ``PromptStack`` serves it in 8 bits.

    python -m paper_1905_05686_b200.ffn      retrains a small block for a few steps, runs tokens through its 4-bit and 8-bit forms,
                                             then does the same with a stack of blocks
"""
from __future__ import annotations

from dataclasses import dataclass

import torch

from . import binding as B
from .synth import Layer


@dataclass
class PrunedLayer:
    """Weights [rows, cols] bf16 of a layer and its packed index factors."""

    layer: Layer
    W: torch.Tensor
    ip: torch.Tensor
    iz: torch.Tensor
    Wt: torch.Tensor | None = None      # transposed, for the gradient of the layer's input

    def refresh(self):
        """To be called whenever W has changed: dx reads the transposed weights."""
        self.Wt = B.lrbi_transpose_bf16(self.W, self.Wt)

    def __call__(self, X):
        return B.lrbi_masked_gemm(self.layer, self.W, self.ip, self.iz, X)

    def dx(self, dY):
        return B.lrbi_masked_gemm_dx(self.layer, self.Wt, self.ip, self.iz, dY)

    def dw(self, dY, X):
        return B.lrbi_masked_gemm_dw(self.layer, dY, X, self.ip, self.iz, dtype=torch.float32)

    def quantize(self, group):
        return B.lrbi_w4_quantize(self.layer, self.W, group, self.ip, self.iz)

    def quantize8(self):
        return B.lrbi_i8_quantize(self.layer, self.W, self.ip, self.iz)


@dataclass
class Kept:
    """What a forward pass leaves for its backward pass."""

    x: B.Checkpoint
    mean: torch.Tensor
    rstd: torch.Tensor
    h: B.Checkpoint

    @property
    def nbytes(self):
        return self.x.nbytes + self.h.nbytes + 4 * (self.mean.numel() + self.rstd.numel())


class PrunedFFN:
    def __init__(self, up: PrunedLayer, down: PrunedLayer, gamma: torch.Tensor, beta: torch.Tensor, act: str = "gelu", eps: float = 1e-5):
        if up.layer.rows != down.layer.cols or up.layer.cols != down.layer.rows:
            raise ValueError("the second layer must take what the first one gives, and give what it takes")
        self.up, self.down, self.gamma, self.beta, self.act, self.eps = up, down, gamma, beta, act, eps
        up.refresh()
        down.refresh()

    def forward(self, x: torch.Tensor):
        """x [tokens, width] bf16 -> (out, what the backward pass needs)."""
        u, mean, rstd, kept_x = B.lrbi_layer_norm(x, self.gamma, self.beta, self.eps, checkpoint=True)
        a, kept_h = B.lrbi_activation(self.up(u), self.act, checkpoint=True)
        return x + self.down(a), Kept(kept_x, mean, rstd, kept_h)

    def backward(self, dout: torch.Tensor, kept: Kept):
        """Gradient of the input, and {"up", "down", "gamma", "beta"} in fp32."""
        dh, a = B.lrbi_activation_backward(self.down.dx(dout), kept.h, self.act, restore=True)
        grads = {"down": self.down.dw(dout, a)}
        dx, grads["gamma"], grads["beta"], u = B.lrbi_layer_norm_backward(self.up.dx(dh), kept.x, self.gamma, kept.mean, kept.rstd,
                                                                          beta=self.beta, dres=dout, restore=True)
        grads["up"] = self.up.dw(dh, u)
        return dx, grads

    def step(self, grads, rate: float):
        for layer, name in ((self.up, "up"), (self.down, "down")):
            layer.W.copy_(layer.W.float() - rate * grads[name])
            layer.refresh()
        self.gamma -= rate * grads["gamma"]
        self.beta -= rate * grads["beta"]

    def tokens(self, group: int = 128) -> "TokenFFN":
        """The block as it is now, in 4 bits; later steps do not change it."""
        return TokenFFN(self.up.quantize(group), self.down.quantize(group), self.gamma.clone(), self.beta.clone(), self.act, self.eps)


    def prompts(self) -> "PromptFFN":
        """The block as it is now, in 8 bits; later steps do not change it."""
        return PromptFFN(self.up.quantize8(), self.down.quantize8(), self.gamma.clone(), self.beta.clone(), self.act, self.eps)


class TokenFFN:
    """The block with 4-bit weights, for a few tokens at a time."""

    def __init__(self, up: B.W4Weights, down: B.W4Weights, gamma, beta, act, eps):
        self.up, self.down, self.gamma, self.beta, self.act, self.eps = up, down, gamma, beta, act, eps

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        u, _, _ = B.lrbi_layer_norm(x, self.gamma, self.beta, self.eps)
        return x + B.lrbi_w4_gemv(self.down, B.lrbi_activation(B.lrbi_w4_gemv(self.up, u), self.act))

    @property
    def nbytes(self):
        return self.up.nbytes + self.down.nbytes


class PromptFFN:
    """The block with 8-bit weights and tokens, for prompts."""

    def __init__(self, up: B.I8Weights, down: B.I8Weights, gamma, beta, act, eps):
        self.up, self.down, self.gamma, self.beta, self.act, self.eps = up, down, gamma, beta, act, eps

    def layers(self, u: B.I8Tokens) -> torch.Tensor:
        return B.lrbi_i8_gemm(self.down, B.lrbi_i8_tokens(B.lrbi_i8_gemm(self.up, u), act=self.act))

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        u, _, _ = B.lrbi_layer_norm(x, self.gamma, self.beta, self.eps)
        return x + self.layers(B.lrbi_i8_tokens(u))

    @property
    def nbytes(self):
        return self.up.nbytes + self.down.nbytes


@dataclass
class Joint:
    """What is learned behind a block: the norm of its result and the gate, a value for each channel of the residual stream."""

    post_gamma: torch.Tensor
    post_beta: torch.Tensor
    gate: torch.Tensor

    def vectors(self):
        return {"post_gamma": self.post_gamma, "post_beta": self.post_beta, "gate": self.gate}

    def clone(self):
        return Joint(*(v.clone() for v in self.vectors().values()))


@dataclass
class KeptBlock:
    """What a block of a stack leaves for the backward pass: the input of its first layer, that of its nonlinearity in 8 bits, what it
    gave, the residual stream behind it and two numbers a row for each norm."""

    u: torch.Tensor
    h: B.Checkpoint
    f: torch.Tensor
    out: torch.Tensor
    stats: torch.Tensor


class PrunedStack:
    """Blocks in a row; the gamma and beta of a block belong to the norm before it.  The residual stream is bf16 or fp32."""

    def __init__(self, blocks: list[PrunedFFN], joints: list[Joint], residual_scale: float = 1.0):
        if not blocks or len(blocks) != len(joints):
            raise ValueError("a stack has one joint for each of its blocks")
        if any(block.eps != blocks[0].eps or block.gamma.shape != blocks[0].gamma.shape for block in blocks):
            raise ValueError("the blocks of a stack have one width and one eps")
        self.blocks, self.joints, self.residual_scale = blocks, joints, residual_scale

    def _between(self, i):
        """(gamma, beta) of the norm behind joint i: the next block's, none behind the last."""
        return (self.blocks[i + 1].gamma, self.blocks[i + 1].beta) if i + 1 < len(self.blocks) else (None, None)

    def forward(self, x: torch.Tensor):
        """x [tokens, width] -> (out, what the backward pass needs)."""
        first = self.blocks[0]
        u, mean, rstd = B.lrbi_layer_norm(x, first.gamma, first.beta, first.eps, y_dtype=torch.bfloat16)
        kept = []
        out = x
        for i, (block, joint) in enumerate(zip(self.blocks, self.joints)):
            a, h = B.lrbi_activation(block.up(u), block.act, checkpoint=True)
            f = block.down(a)
            out, following, stats = B.lrbi_residual_norm(out, f, *self._between(i), **joint.vectors(), residual_scale=self.residual_scale, eps=block.eps)
            kept.append(KeptBlock(u, h, f, out, stats))
            u = following
        return out, (x, mean, rstd, kept)

    def backward(self, dout: torch.Tensor, kept):
        """Gradient of the input, and for each block {"up", "down", "gamma", "beta", "post_gamma", "post_beta", "gate"} in fp32."""
        x, mean, rstd, blocks = kept
        grads = [{} for _ in blocks]
        du = None
        for i in reversed(range(len(blocks))):
            block, k = self.blocks[i], blocks[i]
            dout, df, vectors = B.lrbi_residual_norm_backward(du, dout, k.out, k.f, *self._between(i), **self.joints[i].vectors(),
                                                              residual_scale=self.residual_scale, stats=k.stats)
            for name, g in vectors.items():
                grads[i + 1 if name in ("gamma", "beta") else i][name] = g
            dh, a = B.lrbi_activation_backward(block.down.dx(df), k.h, block.act, restore=True)
            grads[i]["down"], grads[i]["up"] = block.down.dw(df, a), block.up.dw(dh, k.u)
            du = block.up.dx(dh)
        first = self.blocks[0]
        dx, grads[0]["gamma"], grads[0]["beta"] = B.lrbi_layer_norm_backward(du, x, first.gamma, mean, rstd, dres=dout)
        return dx, grads

    def step(self, grads, rate: float):
        for block, joint, g in zip(self.blocks, self.joints, grads):
            block.step(g, rate)
            for name, v in joint.vectors().items():
                v -= rate * g[name]

    def prompts(self) -> "PromptStack":
        """The stack as it is now, in 8 bits; later steps do not change it."""
        return PromptStack([block.prompts() for block in self.blocks], [joint.clone() for joint in self.joints], self.residual_scale)


class PromptStack:
    """The stack with 8-bit weights and tokens: between two blocks the stream goes on in its own type, and the next block's tokens
    come in 8 bits out of the same call."""

    def __init__(self, blocks: list[PromptFFN], joints: list[Joint], residual_scale: float):
        self.blocks, self.joints, self.residual_scale = blocks, joints, residual_scale

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        first = self.blocks[0]
        u = B.lrbi_i8_tokens(B.lrbi_layer_norm(x, first.gamma, first.beta, first.eps, y_dtype=torch.bfloat16)[0])
        for i, (block, joint) in enumerate(zip(self.blocks, self.joints)):
            last = i + 1 == len(self.blocks)
            gamma, beta = (None, None) if last else (self.blocks[i + 1].gamma, self.blocks[i + 1].beta)
            x, u, _ = B.lrbi_residual_norm(x, block.layers(u), gamma, beta, **joint.vectors(), residual_scale=self.residual_scale, eps=block.eps, tokens=not last)
        return x

    @property
    def nbytes(self):
        return sum(block.nbytes for block in self.blocks)


def synthetic_block(width: int, hidden: int, tile: int = 256, rank: int = 32, density: float = 0.3, act: str = "gelu") -> PrunedFFN:
    """A block with seeded weights and index factors."""
    from . import synth

    layers = []
    for name, rows, cols in (("ffn_up", hidden, width), ("ffn_down", width, hidden)):
        layer = Layer(name, rows, cols, min(tile, rows), min(tile, cols), rank, density, 0.02)
        ip, iz = synth.make_factors(layer)
        layers.append(PrunedLayer(layer, B.to_device_bf16(synth.make_weights(layer)), B.to_device_words(synth.pack_ip(ip)), B.to_device_words(synth.pack_iz(iz))))
    return PrunedFFN(*layers, torch.ones(width, device="cuda"), torch.zeros(width, device="cuda"), act)


def synthetic_stack(width: int, hidden: int, depth: int, tile: int = 256, act: str = "gelu", residual_scale: float = 1.0) -> PrunedStack:
    """A stack of such blocks; joints that pass a fifth of a block's result on."""
    ones = torch.ones(width, device="cuda")
    joints = [Joint(ones.clone(), torch.zeros_like(ones), 0.2 * ones) for _ in range(depth)]
    return PrunedStack([synthetic_block(width, hidden, tile, act=act) for _ in range(depth)], joints, residual_scale)


def main():
    torch.manual_seed(0)
    width, hidden, tokens = 1024, 4096, 2048
    block, teacher = synthetic_block(width, hidden), synthetic_block(width, hidden)
    teacher.gamma += 0.3 * torch.randn(width, device="cuda")
    x = torch.randn((tokens, width), device="cuda").bfloat16()
    want = teacher.forward(x)[0]
    for i in range(5):
        out, kept = block.forward(x)
        off = out.float() - want.float()
        print("step %d: mean square error %.4f (%.1f KB kept a token, %.1f as bf16)" % (
            i, off.square().mean(), kept.nbytes / tokens / 1024, 2 * (2 * hidden + 2 * width) / 1024))
        _, grads = block.backward((off * (2 / tokens)).bfloat16(), kept)
        block.step(grads, 0.1)
    served = block.tokens()
    for batch in (1, 8):
        full, small = block.forward(x[:batch])[0].float() - x[:batch].float(), served(x[:batch]).float() - x[:batch].float()
        print("%d token(s) in 4 bits (%.1f MB of weights, %.1f as bf16): %.1f %% off" % (
            batch, served.nbytes / 2**20, 4 * width * hidden / 2**20, 100 * (full - small).norm() / full.norm()))
    prompt = block.prompts()
    full, small = block.forward(x)[0].float() - x.float(), prompt(x).float() - x.float()
    print("%d tokens in 8 bits (%.1f MB of weights): %.1f %% off" % (tokens, prompt.nbytes / 2**20, 100 * (full - small).norm() / full.norm()))
    stack = synthetic_stack(width, hidden, 3)
    want = stack.forward(x.float())[0] + 0.1 * torch.randn((tokens, width), device="cuda")
    for i in range(3):
        out, kept = stack.forward(x.float())
        off = out - want
        print("stack of %d, step %d: mean square error %.4f" % (len(stack.blocks), i, off.square().mean()))
        _, grads = stack.backward(off * (2 / tokens), kept)
        stack.step(grads, 0.1)
    full, small = stack.forward(x.float())[0], stack.prompts()(x.float())
    print("%d tokens through the stack in 8 bits: %.1f %% off" % (tokens, 100 * (full - small).norm() / full.norm()))


if __name__ == "__main__":
    main()
