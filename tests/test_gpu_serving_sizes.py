"""8-bit products and what stands between two blocks on arrays of more than 2^31 values: the last rows are those of a small call."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROWS, COLS, TAIL = 66000, 32768, 40      # 2.16e9 values, 4.3 GB in bf16


@pytest.fixture(scope="module")
def b():
    from paper_1905_05686_b200 import binding
    yield binding
    torch.cuda.empty_cache()


def noise(rows, cols, seed):
    """bf16 rows, most of them alike: a block of 500 noisy rows over and over, and a tail of its own."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    part = torch.randn((500, cols), generator=g, device="cuda").bfloat16()
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, 500):
        x[r:r + 500] = part[:min(500, rows - r)]
    x[-TAIL:] = torch.randn((TAIL, cols), generator=g, device="cuda").bfloat16()
    return x


def test_products(b):
    x = noise(ROWS, COLS, 1)
    tokens = b.lrbi_i8_tokens(x)
    few = b.lrbi_i8_tokens(x[-TAIL:])
    assert torch.equal(tokens.q[-TAIL:], few.q) and torch.equal(tokens.scale[-TAIL:], few.scale)
    weights = b.lrbi_i8_tokens(x[:300])
    del x
    y, want = b.lrbi_i8_gemm(weights, tokens), b.lrbi_i8_gemm(weights, few)           # tokens that pass 2^31 bytes
    assert torch.equal(y[-TAIL:], want)
    wide = b.lrbi_i8_gemm(tokens, few)                                                 # weights that do
    assert torch.equal(wide[:, :300], b.lrbi_i8_gemm(b.I8Weights(tokens.q[:300], tokens.scale[:300], 300, COLS), few))
    assert torch.equal(wide[:, -TAIL:], b.lrbi_i8_gemm(few, few))
    del tokens, y, wide
    narrow = noise(ROWS, 64, 2)
    tokens = b.lrbi_i8_tokens(narrow)
    last = b.I8Tokens(tokens.q[-TAIL:].contiguous(), tokens.scale[-TAIL:].contiguous(), TAIL, 64)
    weights = b.lrbi_i8_tokens(narrow[:COLS + 8])
    y = b.lrbi_i8_gemm(weights, tokens)                                                # an output that does
    assert torch.equal(y[-TAIL:], b.lrbi_i8_gemm(weights, last)) and b.device_status() == 0


def test_between(b):
    x, f = noise(ROWS, COLS, 3), noise(ROWS, COLS, 4)
    v = [1 + 0.1 * torch.randn(COLS, device="cuda") for _ in range(3)]
    how = dict(post_gamma=v[1], gate=v[2])
    out, u, stats = b.lrbi_residual_norm(x, f, v[0], **how)
    few = b.lrbi_residual_norm(x[-TAIL:], f[-TAIL:], v[0], **how)
    assert torch.equal(out[-TAIL:], few[0]) and torch.equal(u[-TAIL:], few[1]) and torch.equal(stats[:, -TAIL:], few[2])
    del u
    dx, df, grads = b.lrbi_residual_norm_backward(f, x, out, f, v[0], stats=stats, **how)
    small = b.lrbi_residual_norm_backward(f[-TAIL:], x[-TAIL:], few[0], f[-TAIL:], v[0], stats=few[2], **how)
    assert torch.equal(dx[-TAIL:], small[0]) and torch.equal(df[-TAIL:], small[1])
    # 131 equal blocks of 500 rows, and the rest
    block = b.lrbi_residual_norm_backward(f[:500], x[:500], out[:500], f[:500], v[0], stats=stats[:, :500].contiguous(), **how)[2]
    rest = b.lrbi_residual_norm_backward(f[65500:], x[65500:], out[65500:], f[65500:], v[0], stats=stats[:, 65500:].contiguous(), **how)[2]
    for name, g in grads.items():
        # 66000 values a column: chains of 8250 sums on a group of blocks, 2^-24 each of what has been added up to there
        want = 131 * block[name].double() + rest[name].double()
        assert (g.double() - want).norm() <= 1e-4 * want.norm(), name
