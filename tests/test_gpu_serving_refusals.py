"""What the Python calls of the 8-bit products and between two blocks refuse, on tensors of the GPU, and streams other than the current one."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
SLEEP = 60_000_000      # cycles: some 30 ms


@pytest.fixture(scope="module")
def b():
    from paper_1905_05686_b200 import binding
    return binding


def test_i8(b):
    x = torch.zeros((4, 64), device="cuda")
    w = b.lrbi_i8_tokens(x)
    for bad in (x.half(), x[0], x.cpu(), x.to_sparse()):
        with pytest.raises(TypeError):
            b.lrbi_i8_tokens(bad)
    for bad in (x.t(), x[:, ::2], torch.zeros((2, (1 << 17) + 1), device="cuda"), torch.zeros((3, 0), device="cuda")):
        with pytest.raises(ValueError):
            b.lrbi_i8_tokens(bad)
    with pytest.raises(ValueError):
        b.lrbi_i8_tokens(x, act="tanh")
    with pytest.raises(ValueError):
        b.lrbi_i8_gemm(w, b.lrbi_i8_tokens(x[:, :48].contiguous()))
    with pytest.raises(TypeError):
        b.lrbi_i8_gemm(w, x)
    with pytest.raises(TypeError):
        b.lrbi_i8_gemm(w, w, y_dtype=torch.float16)
    for q, scale, rows, cols in ((w.q[:, :32], w.scale, 4, 32), (w.q, w.scale[:3], 4, 64), (w.q, w.scale, 4, 65), (w.q, w.scale, 3, 64), (w.q, w.scale, 4, 0)):
        with pytest.raises((ValueError, TypeError)):
            b.I8Weights(q, scale, rows, cols)
    with pytest.raises(TypeError):
        b.I8Weights(w.q.int(), w.scale, 4, 64)
    # rows that do not start on a 16-byte boundary
    room = torch.zeros(4 * 64 + 8, dtype=torch.int8, device="cuda")
    off = b.I8Weights(room[8:].view(4, 64), w.scale, 4, 64)
    for pair in ((off, w), (w, off)):
        with pytest.raises(b.LrbiError):
            b.lrbi_i8_gemm(*pair)
    with pytest.raises(ValueError):
        b.lrbi_i8_quantize((4, 64, 4, 64, 1), torch.zeros((4, 65), device="cuda", dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        b.lrbi_i8_quantize((4, 64, 4, 64, 1), x)
    with pytest.raises(ValueError):
        b.lrbi_i8_quantize((4, 64, 4, 64, 1), x.bfloat16(), ip=torch.zeros(4, dtype=torch.int32, device="cuda"))


def test_between(b):
    x, f = torch.zeros((4, 64), device="cuda"), torch.zeros((4, 64), device="cuda").bfloat16()
    v, half = torch.ones(64, device="cuda"), torch.ones(64, device="cuda").bfloat16()
    out, u, stats = b.lrbi_residual_norm(x, f, v)
    both = dict(post_gamma=v, gate=v)
    for kind, args, more in ((TypeError, (x.half(), f, v), {}), (TypeError, (f, x, v), {}), (ValueError, (x, f[:3], v), {}), (ValueError, (x, f, v[:5]), {}),
                             (ValueError, (x, f, v, half), {}), (ValueError, (x, f, None, v), {}), (ValueError, (x, f, v), dict(post_beta=v)),
                             (ValueError, (x, f, None), dict(tokens=True)), (ValueError, (x, f, v), dict(kind="group")), (TypeError, (x, f, v.cpu()), {}),
                             (ValueError, (x.t(), f.t(), v), {}), (b.LrbiError, (x, f, v), dict(eps=-1.0))):
        with pytest.raises(kind):
            b.lrbi_residual_norm(*args, **more)
    wide = torch.zeros((1, 32769), device="cuda")
    with pytest.raises(ValueError):
        b.lrbi_residual_norm(wide, wide, None)
    back = b.lrbi_residual_norm_backward
    for kind, args, more in ((TypeError, (u, x, out, f, v), {}), (TypeError, (u, x, out, f, v), dict(stats=stats[:3])), (ValueError, (u, x, None, f, v), dict(stats=stats)),
                             (ValueError, (x, x, out, f, v), dict(stats=stats)), (ValueError, (u, f, out, f, v), dict(stats=stats)), (ValueError, (u, x, out, f, None), {}),
                             (ValueError, (None, None, None, f, None), dict(gate=v)), (TypeError, (None, x, out, f, v), dict(stats=stats)),
                             (ValueError, (u, x[:, :32], out, f, v), dict(stats=stats)), (TypeError, (u, x, out, f, v), dict(stats=stats.double(), **both))):
        with pytest.raises(kind):
            back(*args, **more)


def calls(b, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").bfloat16()
    x, f, du, W, gamma = normal(700, 1000), normal(700, 1000), normal(700, 1000), normal(512, 1000), torch.ones(1000, device="cuda")
    tokens, weights = b.lrbi_i8_tokens(x), b.lrbi_i8_tokens(W)
    out, _, stats = b.lrbi_residual_norm(x, f, gamma, post_gamma=gamma, gate=gamma)
    return {
        "tokens": lambda s: b.lrbi_i8_tokens(x, act="silu", stream=s),
        "quantize": lambda s: b.lrbi_i8_quantize((512, 1000, 512, 1000, 1), W, stream=s),
        "product": lambda s: b.lrbi_i8_gemm(weights, tokens, stream=s),
        "between": lambda s: b.lrbi_residual_norm(x, f, gamma, post_gamma=gamma, gate=gamma, stream=s),
        "between_tokens": lambda s: b.lrbi_residual_norm(x, f, gamma, post_gamma=gamma, gate=gamma, tokens=True, stream=s),
        "between_backward": lambda s: b.lrbi_residual_norm_backward(du, x, out, f, gamma, post_gamma=gamma, gate=gamma, stats=stats, stream=s),
    }


def tensors(out):
    if isinstance(out, torch.Tensor):
        return [out]
    if isinstance(out, dict):
        out = list(out.values())
    if isinstance(out, (tuple, list)):
        return [t for o in out for t in tensors(o)]
    return [] if out is None else [out.q, out.scale]


@pytest.mark.parametrize("name", ["tokens", "quantize", "product", "between", "between_tokens", "between_backward"])
def test_results_that_the_current_stream_still_reads(b, name):
    """Results are freed while the current stream has yet to read them, and the call is made again on the other stream."""
    call, other = calls(b, 1)[name], calls(b, 2)[name]
    want = tensors(call(None))
    side = torch.cuda.Stream()
    room = [call(side) for _ in range(6)]
    del room
    torch.cuda.synchronize()
    got = tensors(call(side))
    side.synchronize()
    torch.cuda._sleep(SLEEP)
    copies = [t.clone() for t in got]
    del got
    again = [other(side) for _ in range(3)]
    side.synchronize()
    assert not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert all(torch.equal(c, t) for c, t in zip(copies, want))
    assert all(torch.equal(p, q) for a in again for p, q in zip(tensors(a), tensors(other(None))))


def test_two_at_once(b):
    """Two streams at work on calls of their own, with clusters and pairs among them."""
    w, many, few = (b.lrbi_i8_tokens(torch.randn((n, 2048), device="cuda")) for n in (2000, 1500, 40))
    f = torch.randn((300, 16400), device="cuda")
    v = torch.ones(16400, device="cuda")
    one, two = lambda s=None: [b.lrbi_i8_gemm(w, many, stream=s), b.lrbi_i8_gemm(w, few, stream=s)], lambda s=None: list(b.lrbi_residual_norm(f, f, v, post_gamma=v, stream=s))
    want = one(), two()
    sides = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for side, call, k in zip(sides, (one, two), (0, 1)):
            got[k].append(call(side))
    torch.cuda.synchronize()
    assert b.device_status() == 0
    for k in (0, 1):
        assert all(torch.equal(p, q) for g in got[k] for p, q in zip(g, want[k]))
