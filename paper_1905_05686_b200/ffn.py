"""A transformer's feed-forward block whose two layers are pruned by a low-rank binary index, out of the library's calls.

    out = x + act(norm(x) W1^T) W2^T,      W1, W2 seen through their index

``PrunedFFN`` retrains it: the forward pass keeps its input and the hidden layer's input in 8 bits (and two numbers a row),
the backward pass takes everything else from those copies.  ``TokenFFN`` serves it: both layers in 4 bits, pruned weights
exactly zero, a few tokens at a time.

    python -m paper_1905_05686_b200.ffn      retrains a small block for a few steps, then runs tokens through its 4-bit form
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


def synthetic_block(width: int, hidden: int, tile: int = 256, rank: int = 32, density: float = 0.3, act: str = "gelu") -> PrunedFFN:
    """A block with seeded weights and index factors."""
    from . import synth

    layers = []
    for name, rows, cols in (("ffn_up", hidden, width), ("ffn_down", width, hidden)):
        layer = Layer(name, rows, cols, min(tile, rows), min(tile, cols), rank, density, 0.02)
        ip, iz = synth.make_factors(layer)
        layers.append(PrunedLayer(layer, B.to_device_bf16(synth.make_weights(layer)), B.to_device_words(synth.pack_ip(ip)), B.to_device_words(synth.pack_iz(iz))))
    return PrunedFFN(*layers, torch.ones(width, device="cuda"), torch.zeros(width, device="cuda"), act)


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


if __name__ == "__main__":
    main()
