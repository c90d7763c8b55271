"""What stands between and inside the pruned blocks when prompts are served and several blocks are trained, as cases to be measured.

  linear      a layer on a batch of tokens in 8-bit integers: tokens quantised with a scale each (after the nonlinearity where the
              case has one), product with 8-bit weights that have a scale for each channel
  mlp         both layers of a feed-forward block that way, the nonlinearity between them
  join        between two blocks: out = residual_scale * x + gate * norm(f), u = norm(out), with x the residual stream and f the
              block's result
  join_back   its backward pass
  join_step   both, as in a training step
  seam        join with u as 8-bit tokens, then the next block's first layer on them

`run` computes each in plain torch operations in 32 bits (own = False) or through the package's entry points (own = True).
"""
import math

import torch

own = False

EPS = 1e-5
TINY = 2.0 ** -118  # a row whose largest magnitude is below this is kept as zeros
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token through the 4096 x 9216 layer
        {"name": "token_fc", "op": "linear", "batch": 1, "rows": 4096, "cols": 9216, "act": "", "in": "bf16", "out": "bf16", "pad": 0},
        # the same layer at batch 128
        {"name": "batch_fc", "op": "linear", "batch": 128, "rows": 4096, "cols": 9216, "act": "", "in": "bf16", "out": "bf16", "pad": 0},
        # a long prompt through the feed-forward block's first layer: the largest
        {"name": "prompt_ffn", "op": "linear", "batch": 4096, "rows": 16384, "cols": 4096, "act": "", "in": "bf16", "out": "bf16", "pad": 0},
        # a shorter one through its second layer, the nonlinearity applied as the tokens are quantised
        {"name": "prompt_down", "op": "linear", "batch": 1000, "rows": 4096, "cols": 16384, "act": "gelu", "in": "bf16", "out": "bf16", "pad": 0},
        # odd sizes in 32 bits: tokens sliced out of a wider tensor, a layer of no whole vector
        {"name": "linear_ragged", "op": "linear", "batch": 333, "rows": 500, "cols": 801, "act": "", "in": "f32", "out": "f32", "pad": 3},
        # eight sequences, a token each, through the whole feed-forward block
        {"name": "mlp_8", "op": "mlp", "batch": 8, "rows": 16384, "cols": 4096, "act": "gelu", "in": "bf16", "out": "bf16", "pad": 0},
        # one token between two blocks: latency
        {"name": "join_token", "op": "join", "rows": 1, "cols": 4096, "kind": "rms", "x": "bf16", "f": "bf16", "post": True, "gate": True, "beta": False, "pad": 0},
        # a batch between two blocks
        {"name": "join_ffn", "op": "join", "rows": 4096, "cols": 4096, "kind": "layer", "x": "bf16", "f": "bf16", "post": True, "gate": True, "beta": True, "pad": 0},
        # its backward pass
        {"name": "join_back_ffn", "op": "join_back", "rows": 4096, "cols": 4096, "kind": "layer", "x": "bf16", "f": "bf16", "post": True, "gate": True, "beta": True, "pad": 0},
        # the backward pass of a small ragged batch in 32 bits, rows sliced out of wider ones
        {"name": "join_back_ragged", "op": "join_back", "rows": 1003, "cols": 801, "kind": "rms", "x": "f32", "f": "f32", "post": True, "gate": True, "beta": False, "pad": 6},
        # a long training batch whose residual stream is kept in 32 bits
        {"name": "join_step_long", "op": "join_step", "rows": 16384, "cols": 4096, "kind": "rms", "x": "f32", "f": "bf16", "post": True, "gate": True, "beta": False, "pad": 0},
        # a prompt from one block into the next block's first layer
        {"name": "seam_prompt", "op": "seam", "rows": 2048, "cols": 4096, "next": 16384, "kind": "layer", "x": "bf16", "f": "bf16", "post": True, "gate": True, "beta": True, "pad": 0},
    ]


def draw(rng):
    def size(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5:
            n = (n + 15) // 16 * 16
        return max(lo, min(hi, n))

    op = rng.choice(("linear", "linear", "linear", "mlp", "join", "join_back", "join_step", "seam"))
    pad = rng.choice((0, 0, 8, rng.randint(1, 64)))
    if op in ("linear", "mlp"):
        rows, cols = size(64, 16384), size(64, 16384)
        batch = size(1, min(4096, (1 << (37 if op == "mlp" else 38)) // (rows * cols)))
        if op == "mlp":
            return {"op": op, "batch": batch, "rows": rows, "cols": cols, "act": rng.choice(("relu", "gelu", "silu")), "in": "bf16", "out": "bf16", "pad": pad}
        # 32-bit results of tokens that went through a nonlinearity hang on which way its values round to 8 bits
        act = rng.choice(("", "", "relu", "gelu", "silu"))
        return {"op": op, "batch": batch, "rows": rows, "cols": cols, "act": act, "in": rng.choice(("bf16", "bf16", "f32")),
                "out": "bf16" if act else rng.choice(("bf16", "bf16", "f32")), "pad": pad}
    x, f = rng.choice((("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")))
    if op == "seam":
        x, f = "bf16", "bf16"
    if op == "join_step":
        x = "f32"  # in 16 bits, gradients in 32 bits would hang on which way values of the stream round
    cols = size(64, 16384)
    rows = size(1, min(16384, (1 << (26 if f == "bf16" else 25)) // cols))
    case = {"op": op, "rows": rows, "cols": cols, "kind": rng.choice(("layer", "rms")), "x": x, "f": f, "post": rng.random() < 0.75,
            "gate": rng.random() < 0.75, "beta": rng.random() < 0.5, "pad": pad}
    if op == "seam":
        case["rows"] = min(rows, 4096)
        case["next"] = size(64, max(64, min(16384, (1 << 37) // (case["rows"] * cols))))
    return case


def padded(n, m):
    return (n + m - 1) // m * m


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    pad = case["pad"]

    def normal(r, c, scale, dtype, pad=0, offset=0.0):
        return (torch.randn((r, c + pad), generator=gen, device="cuda") * scale + offset).to(dtype)[:, :c]

    def weights(rows, cols):
        # 8-bit weights as a quantised layer holds them: most small, a part of them pruned, and a scale for each channel
        q = (torch.randn((rows, padded(cols, 16)), generator=gen, device="cuda") * 34).round_().clamp_(-127, 127)
        q[torch.rand(q.shape, generator=gen, device="cuda") < 0.3] = 0
        q[:, cols:] = 0
        return q.to(torch.int8), 0.0005 + 0.0005 * torch.rand(rows, generator=gen, device="cuda")

    op = case["op"]
    s = dict(case)
    if op in ("linear", "mlp"):
        rows, cols = case["rows"], case["cols"]
        # activations: a few channels far above the rest, each token at a scale of its own
        channel = torch.where(torch.rand(cols + pad, generator=gen, device="cuda") < 0.01, 8.0, 1.0)
        level = torch.exp(0.5 * torch.randn((case["batch"], 1), generator=gen, device="cuda"))
        s["X"] = (torch.randn((case["batch"], cols + pad), generator=gen, device="cuda") * channel * level).to(DTYPES[case["in"]])[:, :cols]
        s["q"], s["scale"] = weights(rows, cols)
        if op == "mlp":
            s["q2"], s["scale2"] = weights(cols, rows)
        return s
    rows, cols = case["rows"], case["cols"]
    x, f = DTYPES[case["x"]], DTYPES[case["f"]]
    # a residual stream: an offset, and a few channels far above the rest
    channel = torch.where(torch.rand(cols + pad, generator=gen, device="cuda") < 0.01, 12.0, 1.0)
    s["X"] = (torch.randn((rows, cols + pad), generator=gen, device="cuda") * channel + 0.2).to(x)[:, :cols]
    s["F"] = normal(rows, cols, 0.7, f, pad, 0.1)
    s["scale"] = 0.9

    def vector(offset, spread, there=True):
        v = offset + spread * torch.randn(cols, generator=gen, device="cuda")
        return v if there else None

    s["gamma"], s["post_gamma"], s["gain"] = vector(1, 0.1), vector(1, 0.1, case["post"]), vector(0.3, 0.1, case["gate"])
    s["offset"], s["post_offset"] = vector(0, 0.1, case["beta"]), vector(0, 0.1, case["beta"] and case["post"])
    if op in ("join_back", "join_step"):
        s["du"] = normal(rows, cols, 0.5, f, pad)
        s["dout"] = normal(rows, cols, 0.5, x, pad)
    if op == "join_back":
        s["X"] = (s["scale"] * s["X"].float() + (s["F"].float() if s["gain"] is None else s["F"].float() * s["gain"])).to(x)  # a stream that a forward pass left
        s["stats"] = torch.stack((*plain_stats(s["X"].float(), case["kind"]), *plain_stats(s["F"].float(), case["kind"])))
    if op == "seam":
        s["q"], s["channel"] = weights(case["next"], cols)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def plain_act(h, act):
    if act == "relu":
        return h.clamp(min=0)
    if act == "silu":
        return h / (1 + torch.exp(-h))
    if act == "gelu":
        return 0.5 * h * (1 + torch.erf(h * math.sqrt(0.5)))
    return h


def plain_tokens(x):
    """Whole numbers -127 .. 127 and a scale for each row: scale = max|x| / 127, q = round(x * (127 / max|x|))."""
    top = x.abs().amax(1, keepdim=True)
    low, steps = top < TINY, torch.full_like(top, 127.0)  # a tensor: a number's quotient would be taken as a product
    q = torch.round(x * (steps / torch.where(low, 1.0, top)))
    return torch.where(low, 0.0, q), torch.where(low, 0.0, top / steps)


def plain_product(q, scale, w, channel):
    return (q @ w[:, :q.shape[1]].float().t()) * scale * channel


def plain_stats(x, kind):
    if kind == "rms":
        return torch.zeros_like(x[:, 0]), torch.rsqrt(x.square().mean(1) + EPS)
    mean = x.mean(1)
    return mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS)


def plain_join(s):
    """(out as it is stored, u in 32 bits, statistics)."""
    z, f_mean, f_rstd = s["F"].float(), None, None
    if s["post_gamma"] is not None:
        f_mean, f_rstd = plain_stats(z, s["kind"])
        z = (z - f_mean[:, None]) * f_rstd[:, None] * s["post_gamma"]
        if s["post_offset"] is not None:
            z = z + s["post_offset"]
    if s["gain"] is not None:
        z = z * s["gain"]
    out = (s["scale"] * s["X"].float() + z).to(s["X"].dtype)
    mean, rstd = plain_stats(out.float(), s["kind"])
    u = (out.float() - mean[:, None]) * rstd[:, None] * s["gamma"]
    if s["offset"] is not None:
        u = u + s["offset"]
    return out, u, (mean, rstd, f_mean, f_rstd)


def plain_norm_back(g, n, rstd, kind):
    """Through n = (x - mean) * rstd."""
    g = g - n * (g * n).mean(1, keepdim=True) - (0 if kind == "rms" else g.mean(1, keepdim=True))
    return g * rstd


def plain_join_back(s, out, stats):
    mean, rstd, f_mean, f_rstd = (v if v is None else v[:, None] for v in stats)
    du = s["du"].float()
    n = (out.float() - mean) * rstd
    ds = s["dout"].float() + plain_norm_back(du * s["gamma"], n, rstd, s["kind"])
    result = {"dx": (s["scale"] * ds).to(out.dtype), "dgamma": (du * n).sum(0)}
    if s["offset"] is not None:
        result["dbeta"] = du.sum(0)
    z = nf = s["F"].float()
    if s["post_gamma"] is not None:
        nf = (nf - f_mean) * f_rstd
        z = nf * s["post_gamma"]
        if s["post_offset"] is not None:
            z = z + s["post_offset"]
    if s["gain"] is not None:
        result["dgate"] = (ds * z).sum(0)
        ds = ds * s["gain"]
    if s["post_gamma"] is not None:
        result["dpost_gamma"] = (ds * nf).sum(0)
        if s["post_offset"] is not None:
            result["dpost_beta"] = ds.sum(0)
        ds = plain_norm_back(ds * s["post_gamma"], nf, f_rstd, s["kind"])
    result["df"] = ds.to(s["F"].dtype)
    return result


def plain(s):
    op = s["op"]
    if op == "linear":
        return {"Y": plain_product(*plain_tokens(plain_act(s["X"].float(), s["act"])), s["q"], s["scale"]).to(DTYPES[s["out"]])}
    if op == "mlp":
        h = plain_product(*plain_tokens(s["X"].float()), s["q"], s["scale"]).to(torch.bfloat16)
        return {"Y": plain_product(*plain_tokens(plain_act(h.float(), s["act"])), s["q2"], s["scale2"]).to(DTYPES[s["out"]])}
    if op == "join_back":
        return plain_join_back(s, s["X"], s["stats"])
    out, u, stats = plain_join(s)
    if op == "seam":
        return {"out": out, "Y": plain_product(*plain_tokens(u), s["q"], s["channel"]).to(torch.bfloat16)}
    result = {"out": out, "u": u.to(s["F"].dtype)}
    if op == "join_step":
        result |= plain_join_back(s, out, stats)
    return result


# ---------------------------------------------------------------------------------------------------------------------
# The package's entry points
# ---------------------------------------------------------------------------------------------------------------------
def ours_join(b, s, tokens=False):
    return b.lrbi_residual_norm(s["X"], s["F"], s["gamma"], s["offset"], post_gamma=s["post_gamma"], post_beta=s["post_offset"], gate=s["gain"],
                                residual_scale=s["scale"], eps=EPS, kind=s["kind"], tokens=tokens)


def ours_join_back(b, s, out, stats):
    dx, df, grads = b.lrbi_residual_norm_backward(s["du"], s["dout"], out, s["F"], s["gamma"], s["offset"], post_gamma=s["post_gamma"],
                                                  post_beta=s["post_offset"], gate=s["gain"], residual_scale=s["scale"], stats=stats, kind=s["kind"])
    return {"dx": dx, "df": df} | {"d" + name: g for name, g in grads.items()}


def ours(s):
    from paper_1905_05686_b200 import binding as b

    op = s["op"]
    if op in ("linear", "mlp", "seam") and "weights" not in s:  # a view of tensors that are already laid out
        s["weights"] = b.I8Weights(s["q"], s["channel" if op == "seam" else "scale"], s["q"].shape[0], s["cols"])
        if op == "mlp":
            s["weights2"] = b.I8Weights(s["q2"], s["scale2"], s["cols"], s["rows"])
    if op == "linear":
        return {"Y": b.lrbi_i8_gemm(s["weights"], b.lrbi_i8_tokens(s["X"], act=s["act"] or None), y_dtype=DTYPES[s["out"]])}
    if op == "mlp":
        h = b.lrbi_i8_gemm(s["weights"], b.lrbi_i8_tokens(s["X"]))
        return {"Y": b.lrbi_i8_gemm(s["weights2"], b.lrbi_i8_tokens(h, act=s["act"]), y_dtype=DTYPES[s["out"]])}
    if op == "join_back":
        return ours_join_back(b, s, s["X"], s["stats"])
    if op == "seam":
        out, tokens, _ = ours_join(b, s, tokens=True)
        return {"out": out, "Y": b.lrbi_i8_gemm(s["weights"], tokens)}
    out, u, stats = ours_join(b, s)
    result = {"out": out, "u": u}
    if op == "join_step":
        result |= ours_join_back(b, s, out, stats)
    return result


def run(state):
    return ours(state) if own else plain(state)


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without, and its results in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    op, rows, cols = case["op"], case["rows"], case["cols"]
    size = {"bf16": 2, "f32": 4}
    if op in ("linear", "mlp"):
        batch = case["batch"]
        if op == "linear":
            return {"bytes": size[case["in"]] * batch * cols + rows * cols + 4 * rows + size[case["out"]] * batch * rows, "flops": 2 * batch * rows * cols}
        return {"bytes": batch * (size[case["in"]] * cols + size[case["out"]] * cols) + 2 * rows * cols + 4 * (rows + cols), "flops": 4 * batch * rows * cols}
    n, x, f = rows * cols, size[case["x"]], size[case["f"]]
    vectors = 1 + (2 if case["post"] and case["beta"] else 1 if case["post"] else 0) + case["gate"] + case["beta"]
    if op == "seam":
        return {"bytes": n * (2 * x + f) + case["next"] * (cols + 4) + 2 * rows * case["next"] + 4 * cols * vectors, "flops": 2 * n * case["next"]}
    forward = {"bytes": n * (2 * x + 2 * f) + 4 * cols * vectors, "flops": 20 * n}
    back = {"bytes": n * (3 * x + 3 * f) + 8 * cols * vectors, "flops": 36 * n}  # in: du, f, dout, out; out: dx, df
    return {"bytes": 0, "flops": 0} | {k: (op != "join_back") * forward[k] + (op != "join") * back[k] for k in forward}


def exact_act(h, act):
    if act == "relu":
        return torch.where(h > 0, h, 0.0)
    if act == "silu":
        return h * torch.special.expit(h)
    if act == "gelu":
        return h * torch.special.ndtr(h)
    return h


def exact_tokens(v):
    """By the definition: scale and the quotient that is rounded are 32-bit numbers, what they stand for is not rounded."""
    v = v.float().double()
    top = torch.linalg.vector_norm(v, ord=math.inf, dim=1)[:, None]
    steps = torch.tensor(127.0, dtype=torch.float64, device=v.device)
    there = top >= TINY
    q = (v * (steps / top).float().double()).float().double().round()
    return torch.where(there, q * (top / steps).float().double(), torch.zeros_like(v))


def exact_norm(x, kind):
    """(normalised, 1 / its root)."""
    if kind == "layer":
        x = x - torch.mean(x, dim=1, keepdim=True)
    rstd = (torch.einsum("rc,rc->r", x, x)[:, None] / x.shape[1] + EPS) ** -0.5
    return x * rstd, rstd


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]

    def layer(v, q, scale):
        return torch.einsum("bi,oi->bo", exact_tokens(v), q[:, :v.shape[1]].double() * scale.double()[:, None])

    if op == "linear":
        return {"Y": layer(exact_act(s["X"].double(), s["act"]), s["q"], s["scale"])}
    if op == "mlp":
        h = layer(s["X"].double(), s["q"], s["scale"]).to(torch.bfloat16)  # the hidden layer is kept in 16 bits
        return {"Y": layer(exact_act(h.double(), s["act"]), s["q2"], s["scale2"])}
    kind = s["kind"]
    one = torch.ones(s["cols"], dtype=torch.float64, device="cuda")
    gamma, offset = s["gamma"].double(), 0 * one if s["offset"] is None else s["offset"].double()
    gain = one if s["gain"] is None else s["gain"].double()
    x, f = s["X"].double(), s["F"].double()
    if s["post_gamma"] is None:
        nf, post, shift = f, one, 0 * one
    else:
        if op == "join_back":
            nf, f_rstd = (f - s["stats"][2].double()[:, None]) * s["stats"][3].double()[:, None], s["stats"][3].double()[:, None]
        else:
            nf, f_rstd = exact_norm(f, kind)
        post, shift = s["post_gamma"].double(), 0 * one if s["post_offset"] is None else s["post_offset"].double()
    result = {}
    if op == "join_back":
        rstd = s["stats"][1].double()[:, None]
        n = (x - s["stats"][0].double()[:, None]) * rstd
    else:
        out = x * s["scale"] + torch.addcmul(shift, nf, post) * gain
        n, rstd = exact_norm(out.to(s["X"].dtype).double(), kind)  # the stream as it is stored is what is normalised
        u = torch.addcmul(offset, n, gamma)
        if op == "seam":
            return {"out": out, "Y": layer(u, s["q"], s["channel"])}
        result = {"out": out, "u": u}
        if op == "join":
            return result

    def back(g, n, rstd):
        along = torch.einsum("rc,rc->r", g, n)[:, None] / g.shape[1]
        flat = torch.mean(g, dim=1, keepdim=True) if kind == "layer" else 0.0
        return rstd * (g - flat - along * n)

    du = s["du"].double()
    ds = s["dout"].double() + back(du * gamma, n, rstd)
    first, second = torch.einsum("rc,rc->c", ds, nf), ds.sum(0)
    result |= {"dx": s["scale"] * ds, "dgamma": torch.einsum("rc,rc->c", du, n)}
    if s["offset"] is not None:
        result["dbeta"] = du.sum(0)
    if s["gain"] is not None:
        result["dgate"] = post * first + shift * second
    if s["post_gamma"] is not None:
        result["dpost_gamma"] = gain * first
        if s["post_offset"] is not None:
            result["dpost_beta"] = gain * second
    result["df"] = ds * gain if s["post_gamma"] is None else back(ds * gain * post, nf, f_rstd)
    return result
