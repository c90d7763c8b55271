"""The operators around the pruned layers of a transformer's feed-forward block, as cases to be measured.

  norm        layer norm, forward
  norm_back   layer norm, backward from the saved input: dx and the reduced gradients of gamma and beta
  norm_step   layer norm in a training step that keeps its input in 8 bits: forward, then backward from the 8-bit copy
              with the residual's gradient added, and the norm's output restored for the weight gradient of the next layer
  keep        an activation stored in 8 bits and loaded again
  act         the block's nonlinearity, forward
  act_step    the nonlinearity in a training step that keeps its input in 8 bits: forward, then backward from the copy
              with the nonlinearity's output restored for the weight gradient of the next layer
  gemv        products of a few rows of activations with 4-bit weights (a scale and a zero point for every group of columns)

`run` computes each in plain torch operations in 32 bits (own = False) or through the package's entry points (own = True).
"""
import math

import torch

own = False

EPS = 1e-5
KEEP = 128          # columns that share a scale in the 8-bit copies
TINY = 2.0 ** -118  # a group whose largest magnitude is below this is kept as zeros
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token through the norm in front of the 4096-column layers: latency
        {"name": "norm_token", "op": "norm", "rows": 1, "cols": 4096, "dtype": "bf16", "pad": 0},
        # the norm over the feed-forward layer's whole batch
        {"name": "norm_ffn", "op": "norm", "rows": 4096, "cols": 4096, "dtype": "bf16", "pad": 0},
        # its backward pass when the input was kept as it was
        {"name": "norm_back_ffn", "op": "norm_back", "rows": 4096, "cols": 4096, "dtype": "bf16", "pad": 0},
        # a small ragged batch in 32 bits: odd rows, a width that no vector load fits, a slice of a wider tensor
        {"name": "norm_back_ragged", "op": "norm_back", "rows": 1003, "cols": 801, "dtype": "f32", "pad": 6},
        # a training step over a long batch with the residual stream kept in 8 bits: the largest
        {"name": "norm_step_long", "op": "norm_step", "rows": 16384, "cols": 4096, "dtype": "bf16", "pad": 0},
        # the input of the 4096 x 9216 layer at batch 128, kept in 8 bits
        {"name": "keep_fc", "op": "keep", "rows": 128, "cols": 9216, "dtype": "bf16", "pad": 0},
        # the same for a ragged 32-bit activation
        {"name": "keep_ragged", "op": "keep", "rows": 12544, "cols": 1157, "dtype": "f32", "pad": 3},
        # the nonlinearity between the two feed-forward layers, training
        {"name": "act_step_ffn", "op": "act_step", "rows": 4096, "cols": 16384, "dtype": "bf16", "act": "gelu", "pad": 0},
        # the nonlinearity of the 500 x 800 layer at batch 32
        {"name": "act_small", "op": "act", "rows": 32, "cols": 500, "dtype": "bf16", "act": "relu", "pad": 0},
        # one token through the 500 x 800 layer: latency
        {"name": "gemv_small", "op": "gemv", "rows": 500, "cols": 800, "batch": 1, "group": 32, "out": "f32"},
        # one token through the 4096 x 9216 layer
        {"name": "gemv_fc", "op": "gemv", "rows": 4096, "cols": 9216, "batch": 1, "group": 128, "out": "bf16"},
        # eight sequences, a token each, through the 16384 x 4096 feed-forward layer
        {"name": "gemv_ffn_8", "op": "gemv", "rows": 16384, "cols": 4096, "batch": 8, "group": 64, "out": "bf16"},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5:
            n = (n + 7) // 8 * 8
        return max(lo, min(hi, n))

    op = rng.choice(("norm", "norm_back", "norm_step", "keep", "act", "act_step", "gemv", "gemv"))
    if op == "gemv":
        return {"op": op, "rows": size(64, 16384), "cols": size(64, 16384), "batch": rng.randint(1, 16), "group": rng.choice((32, 64, 128)),
                "out": rng.choice(("bf16", "bf16", "f32"))}
    dtype = rng.choice(("bf16", "bf16", "f32"))
    cols = size(64, 16384)
    rows = size(1, min(16384, (1 << (26 if dtype == "bf16" else 25)) // cols))
    # 32-bit results of a step depend on values kept in 8 bits and on sums over them: steps are in the type they run in
    case = {"op": op, "rows": rows, "cols": cols, "dtype": "bf16" if op.endswith("_step") else dtype, "pad": rng.choice((0, 0, 8, rng.randint(1, 64)))}
    if op.startswith("act"):
        case["act"] = rng.choice(("relu", "gelu", "silu"))
    return case


def padded(n, m):
    return (n + m - 1) // m * m


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows, cols = case["rows"], case["cols"]

    def normal(r, c, scale, dtype, pad=0):
        return (torch.randn((r, c + pad), generator=gen, device="cuda") * scale).to(dtype)[:, :c]

    s = {"op": case["op"]}
    if case["op"] == "gemv":
        # 4-bit values as a quantised layer holds them, most near the zero point, and their scales and zero points
        group = case["group"]
        wide, high = padded(cols, 64), padded(rows, 16)
        groups = -(-cols // group)
        zero = torch.randint(6, 10, (high, groups), generator=gen, device="cuda")
        q = torch.randn((high, wide), generator=gen, device="cuda") * 2.5
        each = zero.repeat_interleave(group, 1)
        each = torch.nn.functional.pad(each, (0, max(0, wide - each.shape[1])), value=8)[:, :wide]
        q = (q.round().to(torch.int64) + each).clamp_(0, 15)
        q = torch.where(torch.rand((high, wide), generator=gen, device="cuda") < 0.2, each, q)  # pruned weights stand at the zero point
        q[:, cols:] = each[:, cols:]
        scale = (0.004 + 0.004 * torch.rand((high, groups), generator=gen, device="cuda")).to(torch.bfloat16)
        s |= {"rows": rows, "cols": cols, "group": group, "out": DTYPES[case["out"]]}
        s["X"] = normal(case["batch"], cols, 1.0, torch.bfloat16).contiguous()
        s["rowwise"] = (q[:rows, 0::2] | q[:rows, 1::2] << 4).to(torch.uint8).contiguous()  # two neighbours a byte
        s["scale"], s["zero"] = scale[:rows].contiguous(), zero[:rows].to(torch.uint8).contiguous()
        # the weights as the library lays them out: words of 8 values in the order in which a warp takes 16 rows x 64 columns
        v = q.view(high // 16, 2, 8, wide // 64, 2, 4, 2, 2, 2)  # row tile, half, row, unit, step / 2, t, step % 2, pair, low/high
        v = v.permute(0, 3, 2, 5, 4, 6, 8, 7, 1).reshape(-1, 8)  # a word: low/high, pair, half
        word = torch.zeros(v.shape[0], dtype=torch.int64, device="cuda")
        for j in range(8):
            word |= v[:, j] << (4 * j)
        s["packed"] = (word - (word >> 31 << 32)).to(torch.int32)
        meta = (scale.view(torch.int16).to(torch.int64) & 0xFFFF) << 16 | zero
        meta = meta.view(high // 16, 16, groups).permute(0, 2, 1).reshape(-1)
        s["meta"] = (meta - (meta >> 31 << 32)).to(torch.int32)
        return s
    dtype, pad = DTYPES[case["dtype"]], case["pad"]
    if case["op"].startswith("norm"):
        # a residual stream: an offset, and a few channels far above the rest
        channel = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 12.0, 1.0)
        s["x"] = ((torch.randn((rows, cols + pad), generator=gen, device="cuda")[:, :cols] * channel) + 0.2).to(dtype)
        if pad:
            s["x"] = torch.nn.functional.pad(s["x"], (0, pad))[:, :cols]
        s["gamma"] = 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda")
        s["beta"] = 0.1 * torch.randn(cols, generator=gen, device="cuda")
        if case["op"] != "norm":
            s["dy"] = normal(rows, cols, 0.5, dtype, pad)
        if case["op"] == "norm_back":
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
        if case["op"] == "norm_step":
            s["dres"] = normal(rows, cols, 0.5, dtype, pad)
        return s
    s["h"] = normal(rows, cols, 1.5, dtype, pad)
    if case["op"].startswith("act"):
        s["act"] = case["act"]
    if case["op"] == "act_step":
        s["da"] = normal(rows, cols, 0.5, dtype, pad)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def plain_kept(x):
    """What the 8-bit copy of x stands for: a group of 128 columns shares scale = max|x| / 127, q = round(x * (127 / max|x|))."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.float(), (0, padded(cols, KEEP) - cols)).view(rows, -1, KEEP)
    top = x.abs().amax(2, keepdim=True)
    low, steps = top < TINY, torch.full_like(top, 127.0)  # a tensor: a number's quotient would be taken as a product
    q = torch.round(x * (steps / torch.where(low, 1.0, top)))
    return torch.where(low, 0.0, q * (top / steps)).view(rows, -1)[:, :cols]


def plain_act(h, act):
    if act == "relu":
        return h.clamp(min=0)
    if act == "silu":
        return h / (1 + torch.exp(-h))
    return 0.5 * h * (1 + torch.erf(h * math.sqrt(0.5)))


def plain_slope(h, act):
    if act == "relu":
        return (h > 0).float()
    if act == "silu":
        sig = 1 / (1 + torch.exp(-h))
        return sig * (1 + h * (1 - sig))
    return 0.5 * (1 + torch.erf(h * math.sqrt(0.5))) + h * torch.exp(-0.5 * h * h) * (1 / math.sqrt(2 * math.pi))


def plain_norm(x, gamma, beta):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
    return x * rstd * gamma + beta, mean, rstd


def plain_norm_back(dy, x, gamma, mean, rstd):
    dy = dy.float()
    n = (x.float() - mean) * rstd
    g = dy * gamma
    dx = rstd * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    return dx, (dy * n).sum(0), dy.sum(0), n


def plain(s):
    op = s["op"]
    if op == "norm":
        y, mean, rstd = plain_norm(s["x"], s["gamma"], s["beta"])
        return {"y": y.to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if op == "norm_back":
        dx, dgamma, dbeta, _ = plain_norm_back(s["dy"], s["x"], s["gamma"], s["mean"][:, None], s["rstd"][:, None])
        return {"dx": dx.to(s["x"].dtype), "dgamma": dgamma, "dbeta": dbeta}
    if op == "norm_step":
        dtype = s["x"].dtype
        y, mean, rstd = plain_norm(s["x"], s["gamma"], s["beta"])
        y = y.to(dtype)
        kept = plain_kept(s["x"])
        dx, dgamma, dbeta, n = plain_norm_back(s["dy"], kept, s["gamma"], mean, rstd)
        return {"y": y, "dx": (dx + s["dres"].float()).to(dtype), "dgamma": dgamma, "dbeta": dbeta, "restored": (n * s["gamma"] + s["beta"]).to(dtype)}
    if op == "keep":
        return {"loaded": plain_kept(s["h"]).to(s["h"].dtype)}
    if op == "act":
        return {"a": plain_act(s["h"].float(), s["act"]).to(s["h"].dtype)}
    if op == "act_step":
        dtype = s["h"].dtype
        a = plain_act(s["h"].float(), s["act"]).to(dtype)
        kept = plain_kept(s["h"])
        return {"a": a, "dh": (s["da"].float() * plain_slope(kept, s["act"])).to(dtype), "restored": plain_act(kept, s["act"]).to(dtype)}
    rows, cols, group = s["rows"], s["cols"], s["group"]
    q = torch.stack((s["rowwise"] & 15, s["rowwise"] >> 4), 2).view(rows, -1)[:, :cols].float()
    zero = s["zero"].float().repeat_interleave(group, 1)[:, :cols]
    w = (q - zero) * s["scale"].float().repeat_interleave(group, 1)[:, :cols]
    return {"Y": (s["X"].float() @ w.t()).to(s["out"])}


# ---------------------------------------------------------------------------------------------------------------------
# The package's entry points
# ---------------------------------------------------------------------------------------------------------------------
def ours(s):
    from paper_1905_05686_b200 import binding as b

    op = s["op"]
    if op == "norm":
        y, mean, rstd = b.lrbi_layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_back":
        dx, dgamma, dbeta = b.lrbi_layer_norm_backward(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"])
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if op == "norm_step":
        y, mean, rstd, kept = b.lrbi_layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS, checkpoint=True)
        dx, dgamma, dbeta, restored = b.lrbi_layer_norm_backward(s["dy"], kept, s["gamma"], mean, rstd, beta=s["beta"], dres=s["dres"], restore=True)
        return {"y": y, "dx": dx, "dgamma": dgamma, "dbeta": dbeta, "restored": restored}
    if op == "keep":
        return {"loaded": b.lrbi_checkpoint_load(b.lrbi_checkpoint_store(s["h"]), s["h"].dtype)}
    if op == "act":
        return {"a": b.lrbi_activation(s["h"], s["act"])}
    if op == "act_step":
        a, kept = b.lrbi_activation(s["h"], s["act"], checkpoint=True)
        dh, restored = b.lrbi_activation_backward(s["da"], kept, s["act"], restore=True)
        return {"a": a, "dh": dh, "restored": restored}
    if "weights" not in s:  # a view of tensors that are already laid out
        s["weights"] = b.W4Weights(s["packed"], s["meta"], s["rows"], s["cols"], s["group"])
    return {"Y": b.lrbi_w4_gemv(s["weights"], s["X"], y_dtype=s["out"])}


def run(state):
    return ours(state) if own else plain(state)


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    op, rows, cols = case["op"], case["rows"], case["cols"]
    if op == "gemv":
        batch, groups = case["batch"], -(-cols // case["group"])
        out = 4 if case["out"] == "f32" else 2
        return {"bytes": rows * (cols / 2 + 3 * groups) + batch * (2 * cols + out * rows), "flops": 2 * batch * rows * cols}
    n, e = rows * cols, 2 if case["dtype"] == "bf16" else 4
    kept = n + 4 * rows * -(-cols // KEEP)
    if op == "norm":
        return {"bytes": 2 * e * n + 8 * cols + 8 * rows, "flops": 8 * n}
    if op == "norm_back":
        return {"bytes": 3 * e * n + 12 * cols + 8 * rows, "flops": 14 * n}
    if op == "norm_step":  # forward: x, y, the copy; backward: dy, the copy, dres, dx, the restored y
        return {"bytes": 6 * e * n + 2 * kept + 24 * cols + 16 * rows, "flops": 28 * n}
    if op == "keep":
        return {"bytes": 2 * e * n + 2 * kept, "flops": 5 * n}
    if op == "act":
        return {"bytes": 2 * e * n, "flops": 10 * n}
    return {"bytes": 5 * e * n + 2 * kept, "flops": 40 * n}  # forward: h, a, the copy; backward: da, the copy, dh, the restored a


def exact_kept(x):
    """The 8-bit copy by its definition: the scale and the quotient that is rounded are 32-bit numbers, what they stand for is not rounded."""
    rows, cols = x.shape
    out = torch.zeros((rows, padded(cols, KEEP)), dtype=torch.float64, device=x.device)
    out[:, :cols] = x.double()
    parts = out.unflatten(1, (-1, KEEP))
    top = parts.abs().max(dim=2, keepdim=True).values
    steps = torch.tensor(127.0, dtype=torch.float64, device=x.device).expand_as(top)
    q = (parts * (steps / top).float().double()).float().double().round()
    out = torch.where(top < TINY, torch.zeros_like(q), q * (top / steps).float().double())
    return out.flatten(1)[:, :cols]


def exact_act(h, act):
    """(value, slope) in 64 bits."""
    if act == "relu":
        return torch.where(h > 0, h, 0.0), torch.where(h > 0, 1.0, 0.0).double()
    if act == "silu":
        t = torch.special.expit(h)
        return h * t, t + h * t * torch.special.expit(-h)
    t = torch.special.ndtr(h)
    return h * t, t + h * torch.exp(-h.square() / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "gemv":
        group, cols = s["group"], s["cols"]
        y = torch.zeros((s["X"].shape[0], s["rows"]), dtype=torch.float64, device="cuda")
        both = torch.empty((s["rows"], padded(cols, 64)), dtype=torch.float64, device="cuda")
        both[:, 0::2], both[:, 1::2] = (s["rowwise"] % 16).double(), (s["rowwise"] // 16).double()
        x = s["X"].double()
        for g in range(s["scale"].shape[1]):
            at = slice(g * group, min(cols, (g + 1) * group))
            part = x[:, at] @ both[:, at].t() - x[:, at].sum(1, keepdim=True) * s["zero"][:, g].double()
            y += part * s["scale"][:, g].double()
        return {"Y": y}
    if op.startswith("norm"):
        x, gamma, beta = s["x"].double(), s["gamma"].double(), s["beta"].double()
        if op == "norm_back":
            mean, rstd = s["mean"].double()[:, None], s["rstd"].double()[:, None]
        else:
            var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
            rstd = (var + EPS) ** -0.5
            y = torch.addcmul(beta, (x - mean) * rstd, gamma)
            if op == "norm":
                return {"y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]}
            x = exact_kept(s["x"])
        n, dy = (x - mean) * rstd, s["dy"].double()
        dbeta, dgamma = dy.sum(0), torch.einsum("rc,rc->c", dy, n)
        along = torch.einsum("rc,rc,c->r", dy, n, gamma)[:, None] / x.shape[1]
        flat = (dy @ gamma)[:, None] / x.shape[1]
        dx = (dy * gamma - flat - n * along) * rstd
        if op == "norm_back":
            return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
        return {"y": y, "dx": dx + s["dres"].double(), "dgamma": dgamma, "dbeta": dbeta, "restored": n * gamma + beta}
    if op == "keep":
        return {"loaded": exact_kept(s["h"])}
    a, _ = exact_act(s["h"].double(), s["act"])
    if op == "act":
        return {"a": a}
    restored, slope = exact_act(exact_kept(s["h"]), s["act"])
    return {"a": a, "dh": s["da"].double() * slope, "restored": restored}
