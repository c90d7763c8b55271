"""The norms, the gate and the residual scale between two blocks against the formulas in 64 bits, forward and backward.

Tolerances, with e = 2^-24 (half a step of fp32): a sum over a row takes at most 3 + 2 + 5 + 2 + 5 additions for any one value (a
chunk, its pairs, the warp, the entries of a lane, the warp), so it is off by 17 e of the sum of magnitudes; a mean or a root by
some 20 e, and a result, behind fewer than ten more roundings and two sums, by less than 64 e = 2^-18 of the magnitudes that
went into it.  The backward pass's second mean is put together out of seven sums, each of magnitudes that are counted: twice as
much.  Sums over rows: a thread adds rows / 148 values or fewer after another, the blocks' sums 148 / 16 + 16: at most
rows / 148 + 42 additions, 2^-16 for the rows tested here.  Outputs are rounded once: eps / 2 of the value."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def B():
    from paper_1905_05686_b200 import binding
    return binding


def near(got, want, size, bits):
    """got is want within 2^-bits of size, and half a step of its type."""
    half = torch.finfo(got.dtype).eps / 2
    got = got.double()
    assert got.shape == want.shape and bool(got.isfinite().all())
    off = (got - want).abs() - (size * 2.0 ** -bits) * (1 + half) - half * want.abs()
    assert off.max() <= 1e-30, (off.max(), off.argmax())


class Case:
    def __init__(self, rows, cols, x=BF16, f=BF16, kind="layer", post=True, gate=True, beta=True, pre=True, pad=0, params=F32, seed=0, offset=0.3):
        g = torch.Generator(device="cuda").manual_seed(seed + 7 * rows + cols)
        rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")
        wide = cols + pad
        self.kind, self.scale, self.eps = kind, 0.8, 1e-5
        self.x = (rand(rows, wide) * torch.where(rand(wide) > 2, 9.0, 1.0) + offset).to(x)[:, :cols]
        self.f = (rand(rows, wide) * 0.7 - offset).to(f)[:, :cols]
        self.du = (rand(rows, wide) * 0.5).to(f)[:, :cols]
        self.dout = (rand(rows, wide) * 0.5).to(x)[:, :cols]
        vec = lambda at, there: (at + 0.2 * rand(cols)).to(params) if there else None
        self.gamma, self.post_gamma, self.gate = vec(1, pre), vec(1, post), vec(0.4, gate)
        self.beta, self.post_beta = vec(0, beta and pre), vec(0, beta and post)

    def vectors(self):
        return dict(post_gamma=self.post_gamma, post_beta=self.post_beta, gate=self.gate, residual_scale=self.scale, kind=self.kind)

    def forward(self, B, **more):
        return B.lrbi_residual_norm(self.x, self.f, self.gamma, self.beta, eps=self.eps, **self.vectors(), **more)

    def backward(self, B, out, stats, dout=True, **more):
        return B.lrbi_residual_norm_backward(self.du if self.gamma is not None else None, self.dout if dout else None, out, self.f, self.gamma, self.beta, stats=stats,
                                             **self.vectors(), **more)

    def wide(self, name):
        """A vector in 64 bits, and what stands for one that is not there."""
        v = getattr(self, name)
        return v.double() if v is not None else (0.0 if name.endswith("beta") else 1.0)


def norm64(v, kind, eps):
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    rstd = ((v - mean).square().mean(1, keepdim=True) + eps) ** -0.5
    return (v - mean) * rstd, mean, rstd, (v.abs() + v.abs().mean(1, keepdim=True)) * rstd       # last: magnitudes


def check_forward(c, out, u, stats):
    f, x = c.f.double(), c.x.double()
    if c.post_gamma is not None:
        n, mean, rstd, size = norm64(f, c.kind, c.eps)
        near(stats[2], mean[:, 0], f.abs().mean(1), 18)
        near(stats[3], rstd[:, 0], rstd[:, 0], 18)
    else:
        n, size = f, f.abs()
        assert not stats[2].any() and (stats[3] == 1).all()
    z = n * c.wide("post_gamma") + c.wide("post_beta")
    sizes = size * abs(c.wide("post_gamma")) + abs(c.wide("post_beta"))
    near(out, c.scale * x + c.wide("gate") * z, c.scale * x.abs() + abs(c.wide("gate")) * sizes, 18)
    if c.gamma is None:
        assert u is None
        return
    n, mean, rstd, size = norm64(out.double(), c.kind, c.eps)
    near(stats[0], mean[:, 0], out.double().abs().mean(1), 18)
    near(stats[1], rstd[:, 0], rstd[:, 0], 18)
    if u is not None:
        near(u, n * c.wide("gamma") + c.wide("beta"), size * abs(c.wide("gamma")) + abs(c.wide("beta")), 18)


def back64(g, sizes, n, size, rstd, kind):
    """Gradient through n = (v - mean) rstd, and its magnitudes."""
    flat, flats = (g.mean(1, keepdim=True), sizes.mean(1, keepdim=True)) if kind == "layer" else (0.0, 0.0)
    return (rstd * (g - flat - n * (g * n).mean(1, keepdim=True)), rstd * (sizes + flats + size * (sizes * size).mean(1, keepdim=True)))


def check_backward(c, out, stats, dout, dx, df, grads):
    ds = c.dout.double() if dout else torch.zeros_like(c.f.double())
    sizes = ds.abs()
    want, bound = {}, {}
    st = None if stats is None else stats.double()
    if c.gamma is not None:
        mean, rstd = st[0][:, None], st[1][:, None]
        o, du = out.double(), c.du.double()
        n, size = (o - mean) * rstd, (o.abs() + mean.abs()) * rstd
        part, parts = back64(du * c.wide("gamma"), (du * c.wide("gamma")).abs(), n, size, rstd, c.kind)
        ds, sizes = ds + part, sizes + parts
        want["gamma"], bound["gamma"] = (du * n).sum(0), (du.abs() * size).sum(0)
        want["beta"], bound["beta"] = du.sum(0), du.abs().sum(0)
    f = c.f.double()
    if c.post_gamma is not None:
        mean, rstd = st[2][:, None], st[3][:, None]
        nf, nsize = (f - mean) * rstd, (f.abs() + mean.abs()) * rstd
    else:
        nf, nsize = f, f.abs()
    pg, pb, gate = c.wide("post_gamma"), c.wide("post_beta"), c.wide("gate")
    a, s = (ds * nf).sum(0), ds.sum(0)
    asize, ssize = (sizes * nsize).sum(0), sizes.sum(0)
    want["gate"], bound["gate"] = pg * a + pb * s, abs(pg) * asize + abs(pb) * ssize
    want["post_gamma"], bound["post_gamma"] = gate * a, abs(gate) * asize
    want["post_beta"], bound["post_beta"] = gate * s, abs(gate) * ssize
    near(dx, c.scale * ds, c.scale * sizes, 18)
    w = gate * pg
    if c.post_gamma is not None:
        ref, size = back64(ds * w, sizes * abs(w), nf, nsize, rstd, c.kind)
    else:
        ref, size = ds * w, sizes * abs(w)
    near(df, ref, size, 17)
    assert set(grads) == {k for k in ("gamma", "beta", "post_gamma", "post_beta", "gate") if getattr(c, k) is not None}
    for k, got in grads.items():
        assert got.dtype == F32
        near(got, want[k] + torch.zeros_like(bound[k]), bound[k], 16)


SIZES = [(1, 1), (1, 4096), (3, 7), (5, 33), (64, 64), (1003, 801), (37, 256), (300, 257), (200, 1000), (129, 1032), (64, 4096), (50, 4097), (33, 4104), (20, 8192),
         (9, 9216), (7, 12345), (6, 16384), (3, 20000), (5, 32768), (2, 32761), (4099, 64)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_sizes(B, rows, cols, kind):
    for x, f in ((BF16, BF16), (F32, BF16), (F32, F32)):
        c = Case(rows, cols, x, f, kind)
        out, u, stats = c.forward(B)
        assert out.dtype == x and u.dtype == f and stats.shape == (4, rows)
        check_forward(c, out, u, stats)
        check_backward(c, out, stats, True, *c.backward(B, out, stats))


# More rows: a warp has four spans (forward) or two (backward) of a row, all of them there or not; rows in one block whose vectors stay
# in memory; rows shared by two, four and eight blocks.
MANY = [(400, 1024), (650, 1030), (900, 4096), (640, 4104), (620, 4099), (500, 8192), (330, 9216), (310, 12345), (300, 16384), (300, 20000), (299, 32760), (3000, 512),
        (6000, 200), (2500, 777)]


@pytest.mark.parametrize("kind,beta", [("layer", True), ("rms", False), ("layer", False), ("rms", True)])
@pytest.mark.parametrize("rows,cols", MANY)
def test_many_rows(B, rows, cols, kind, beta):
    for x, f in ((BF16, BF16), (F32, BF16), (F32, F32)):
        c = Case(rows, cols, x, f, kind, beta=beta)
        out, u, stats = c.forward(B)
        check_forward(c, out, u, stats)
        check_backward(c, out, stats, True, *c.backward(B, out, stats))
    out, t, _ = c.forward(B, tokens=True)
    assert (t.q[:, :cols].abs().amax(1) == 127).all() and not t.q[:, cols:].any()


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("beta", [False, True])
@pytest.mark.parametrize("pre", [False, True])
def test_parts(B, post, gate, beta, pre):
    for rows, cols, pad, params in ((40, 500, 0, BF16), (40, 512, 8, F32), (40, 777, 5, BF16), (2600, 1024, 0, F32), (600, 16000, 0, BF16)):
        for x, f, kind in ((BF16, BF16, "layer"), (F32, F32, "rms")):
            c = Case(rows, cols, x, f, kind, post, gate, beta, pre, pad, params)
            out, u, stats = c.forward(B)
            check_forward(c, out, u, stats)
            for dout in (True, False) if pre else (True,):
                check_backward(c, out, stats, dout, *c.backward(B, out, stats, dout))


@pytest.mark.parametrize("post,gate,beta,pre", [(False, False, False, True), (True, False, False, True), (True, True, False, True), (False, False, True, True),
                                               (True, False, True, False), (False, True, False, False), (True, True, True, True), (True, True, True, False)])
@pytest.mark.parametrize("rows,cols,x", [(310, 8704, F32), (150, 8701, F32), (310, 12896, BF16), (305, 12891, BF16), (160, 16381, F32)])
def test_vectors_that_leave_room(B, rows, cols, x, post, gate, beta, pre):
    """Long rows in one block beside few vectors, without them, or shared by blocks."""
    c = Case(rows, cols, x, BF16, "rms", post, gate, beta, pre)
    out, u, stats = c.forward(B)
    check_forward(c, out, u, stats)
    if pre:
        again, t, _ = c.forward(B, tokens=True)
        assert torch.equal(again, out) and (t.q[:, :cols].abs().amax(1) == 127).all() and not t.q[:, cols:].any()


def test_values_far_from_zero(B):
    """A mean a thousand times the spread: squares are summed about it."""
    c = Case(30, 1000, F32, F32, offset=1000.0)
    out, u, stats = c.forward(B)
    check_forward(c, out, u, stats)
    n, _, rstd, _ = norm64(c.f.double(), "layer", c.eps)
    assert ((stats[3].double() - rstd[:, 0]) / rstd[:, 0]).abs().max() < 2.0 ** -18


@pytest.mark.parametrize("rows,cols,kind", [(1, 4096, "rms"), (70, 800, "layer"), (9, 801, "rms"), (12, 9216, "layer"), (3, 16400, "layer")])
def test_tokens(B, rows, cols, kind):
    """u as 8-bit tokens: the values that u has, in steps of their row's scale."""
    c = Case(rows, cols, BF16, BF16, kind, pad=3)
    out, t, stats = c.forward(B, tokens=True)
    same, _, _ = c.forward(B)
    assert stats is None and torch.equal(out, same) and isinstance(t, B.I8Rows) and t.shape == (rows, cols)
    n, _, _, size = norm64(out.double(), kind, c.eps)
    u, size = n * c.wide("gamma") + c.wide("beta"), size * abs(c.wide("gamma")) + abs(c.wide("beta"))
    assert not t.q[:, cols:].any() and (t.q.abs().amax(1) == 127).all()
    assert ((t.q[:, :cols].double() * t.scale.double()[:, None] - u).abs() <= t.scale.double()[:, None] * (0.5 + 2.0 ** -16) + size * 2.0 ** -18).all()
    w = B.lrbi_i8_tokens(torch.randn((100, cols), device="cuda"))
    y = B.lrbi_i8_gemm(w, t, y_dtype=F32)
    want = (t.q[:, :cols].double() * t.scale.double()[:, None]) @ (w.q[:, :cols].double() * w.scale.double()[:, None]).t()
    assert (y.double() - want).abs().max() <= 2.0 ** -22 * want.abs().max()


def test_odd_rows(B):
    """A row that holds a NaN or an infinity concerns itself alone; no rows are no work, and gradients of zero."""
    c = Case(6, 40, F32, F32)
    c.f[1, 3], c.x[2, 5], c.x[3, 0] = float("nan"), float("inf"), float("nan")
    out, u, stats = c.forward(B)
    assert u[1].isnan().all() and u[2].isnan().any() and u[3].isnan().all() and u[[0, 4, 5]].isfinite().all()
    _, t, _ = c.forward(B, tokens=True)
    assert t.scale[[1, 2, 3]].isnan().all() and not t.q[[1, 2, 3]].any() and t.scale[[0, 4, 5]].isfinite().all()
    dx, df, _ = c.backward(B, out, stats)
    assert dx[[0, 4, 5]].isfinite().all() and df[[0, 4, 5]].isfinite().all() and dx[[1, 2, 3]].isnan().any(1).all()
    none = Case(0, 40)
    out, u, stats = none.forward(B)
    assert out.shape == u.shape == (0, 40) and stats.shape == (4, 0)
    dx, df, grads = none.backward(B, out, stats)
    assert dx.shape == df.shape == (0, 40) and len(grads) == 5 and not any(g.any() for g in grads.values())
    zero = Case(3, 40)
    zero.f.zero_()
    zero.x.zero_()
    zero.gate.zero_()
    out, u, stats = zero.forward(B)
    assert not out.any() and torch.equal(u, zero.beta.to(BF16).expand(3, 40))
    check_backward(zero, out, stats, True, *zero.backward(B, out, stats))


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_gradients_against_differences(B, kind):
    """Along a random direction of each input, the formula's central difference (64 bits, steps of 1e-5) is the gradient's product
    with the direction: off by the fp32 gradient's own 1e-5 or so of the product of norms, and 1e-9 of truncation."""
    c = Case(7, 90, F32, F32, kind)
    out, u, stats = c.forward(B)
    dx, df, grads = c.backward(B, out, stats)
    grads |= {"x": dx, "f": df}

    def loss(name, step):
        v = {k: getattr(c, k).double() for k in ("x", "f", "gamma", "beta", "post_gamma", "post_beta", "gate")}
        v[name] = v[name] + step
        z = norm64(v["f"], kind, c.eps)[0] * v["post_gamma"] + v["post_beta"]
        o = c.scale * v["x"] + v["gate"] * z
        w = norm64(o, kind, c.eps)[0] * v["gamma"] + v["beta"]
        return (o * c.dout.double()).sum() + (w * c.du.double()).sum()

    for name, got in grads.items():
        d = torch.randn(got.shape, device="cuda", dtype=torch.float64)
        want = (loss(name, 1e-5 * d) - loss(name, -1e-5 * d)) / 2e-5
        assert abs((got.double() * d).sum() - want) <= 1e-5 * got.double().norm() * d.norm(), name


@pytest.mark.parametrize("rows,cols", [(500, 800), (11, 9000)])
def test_repeatable_on_streams_and_in_graphs(B, rows, cols):
    """The same bits every time: eagerly, on another stream, and replayed from a graph on inputs that changed meanwhile."""
    c = Case(rows, cols, pad=8)

    def both(**more):
        out, u, stats = c.forward(B, **more)
        dx, df, grads = c.backward(B, out, stats, **more)
        return [out, u, stats, dx, df, *grads.values()]

    want = both()
    assert all(torch.equal(a, b) for a, b in zip(want, both()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    x = c.x.clone()
    for k in range(3):
        c.x.copy_(x if k != 1 else -x)
        graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_surroundings(B):
    """Through the C entry: strided outputs, and nothing beyond them is written."""
    rows, cols = 21, 300
    for pad in (0, 5, 8):
        c = Case(rows, cols, pad=3)
        out, u, stats = c.forward(B)
        room = [torch.full((rows + 1, cols + pad), 7.0, device="cuda", dtype=BF16) for _ in range(2)]
        how = B.Residual(rows, cols, 0, 0, 0, 1, c.scale, c.eps, *[v.data_ptr() for v in (c.gamma, c.beta, c.post_gamma, c.post_beta, c.gate)])
        s = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        rc = B.lib().lrbi_residual_norm(ctypes.byref(how), c.x.data_ptr(), c.x.stride(0), c.f.data_ptr(), c.f.stride(0), room[0].data_ptr(), cols + pad,
                                        room[1].data_ptr(), cols + pad, None, None, None, s)
        assert rc == B.OK
        for r, want in zip(room, (out, u)):
            assert torch.equal(r[:rows, :cols], want) and (r[:rows, cols:] == 7).all() and (r[rows] == 7).all()
