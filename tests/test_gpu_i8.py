"""8-bit rows and their products against the definition: the bytes, the scales and the products bit for bit (the sums are whole
numbers, and every other step is one fp32 operation that torch makes too)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -118


@pytest.fixture(scope="module")
def B():
    from paper_1905_05686_b200 import binding
    return binding


def rows8(v):
    """(q, scale) of fp32 rows by the definition."""
    v = v.float()
    steps = torch.full((v.shape[0], 1), 127.0, device=v.device)
    top = v.abs().amax(1, keepdim=True)
    bad = ~torch.isfinite(v).all(1, keepdim=True)
    low = bad | (top < TINY)
    top = torch.where(low, torch.ones_like(top), top)
    q = torch.where(low, torch.zeros_like(v), torch.round(v * (steps / top)))
    scale = torch.where(bad, torch.full_like(top, float("nan")), torch.where(low, torch.zeros_like(top), top / steps))
    return q.to(torch.int8), scale[:, 0]


def product(w, x, dtype):
    """By the definition, from I8Rows."""
    total = x.q[:, :x.cols].double() @ w.q[:, :w.cols].double().t()        # whole numbers below 2^31: exact
    return ((total.float() * x.scale[:, None]) * w.scale[None, :]).to(dtype)


def same(a, b):
    return a.dtype == b.dtype and a.shape == b.shape and bool(((a == b) | (a.isnan() & b.isnan())).all())


def activations(rows, cols, dtype, pad=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * rows + cols + seed)
    wide = torch.randn((rows, cols + pad), generator=g, device="cuda") * torch.exp(torch.randn((rows, 1), generator=g, device="cuda"))
    return wide.to(dtype)[:, :cols]


def random_rows8(B, rows, cols, seed=0, most=127):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-most, most + 1, (rows, (cols + 15) // 16 * 16), generator=g, device="cuda").to(torch.int8)
    q[:, cols:] = 0
    return B.I8Rows(q, torch.rand(rows, generator=g, device="cuda") + 0.5, rows, cols)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 0), (1, 4096, 0), (5, 801, 3), (33, 256, 8), (130, 257, 0), (17, 4104, 0), (9, 9216, 0),
                                           (4, 16384, 1), (3, 20000, 0), (2, 40003, 0), (2, 131072, 0), (1000, 64, 0), (1000, 4096, 0), (900, 4097, 0),
                                           (600, 16384, 8), (250, 20001, 3), (3000, 1000, 0)])
def test_tokens_are_the_definition(B, rows, cols, pad, dtype):
    x = activations(rows, cols, dtype, pad)
    t = B.lrbi_i8_tokens(x)
    q, scale = rows8(x)
    assert t.shape == (rows, cols) and t.q.shape == (rows, (cols + 15) // 16 * 16)
    assert torch.equal(t.q[:, :cols], q) and torch.equal(t.scale, scale)
    assert not t.q[:, cols:].any()


@pytest.mark.parametrize("cols", [24, 33])
def test_tokens_of_odd_rows(B, cols):
    x = activations(8, cols, torch.float32)
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 0] = float("inf")
    x[4] = 2.0 ** -120
    x[5] = 0
    x[5, cols - 1] = -(2.0 ** -117)
    x[6] *= 2.0 ** 120
    t = B.lrbi_i8_tokens(x)
    q, scale = rows8(x)
    assert torch.equal(t.q[:, :cols], q) and same(t.scale, scale)
    w = random_rows8(B, 5, cols)
    y = B.lrbi_i8_gemm(w, t, y_dtype=torch.float32)
    assert y[[2, 3]].isnan().all() and not y[[1, 4]].any() and same(y, product(w, t, torch.float32))


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("rows,cols,dtype", [(5, 800, torch.bfloat16), (7, 1157, torch.float32), (3, 16384, torch.bfloat16), (2, 20001, torch.bfloat16),
                                             (1100, 4096, torch.bfloat16), (700, 5000, torch.float32), (300, 18000, torch.bfloat16)])
def test_tokens_of_the_nonlinearity(B, act, rows, cols, dtype):
    x = activations(rows, cols, dtype, pad=2)
    t = B.lrbi_i8_tokens(x, act=act)
    h = x.double()
    want = {"relu": h.clamp(min=0), "gelu": h * torch.special.ndtr(h), "silu": h * torch.special.expit(h)}[act]
    # an 8-bit value is off by half a step, and by as much as its fp32 value is: 2^-20 (1 + h^2 / 8), and 2^-13 from 16 bits
    off = 2.0 ** -13 * want.abs() + 2.0 ** -20 * (1 + h * h) * want.abs() + 2.0 ** -100
    assert ((t.q[:, :cols].double() * t.scale.double()[:, None] - want).abs() <= t.scale.double()[:, None] * (0.5 + 2.0 ** -12) + off).all()
    assert (t.scale.double() * 127 - want.abs().amax(1)).abs().max() <= 2.0 ** -12 * want.abs().max()
    assert (t.q[:, :cols].abs().amax(1) == 127).all()


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_nonlinearity_of_every_16_bit_value(B, act):
    """Rows of one value: 127 times the scale is the value's magnitude.  Off by 2^-20 (1 + h^2 / 8) and 2^-13 of it, and by three
    roundings of 2^-24; rows below 2^-118 are zeros.  No finite result comes of an infinity or a NaN, but relu's of -inf."""
    x = torch.arange(65536, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(-1, 1)
    t = B.lrbi_i8_tokens(x, act=act)
    h, got = x.double()[:, 0], 127 * t.scale.double()
    want = {"relu": h.clamp(min=0), "gelu": -h.abs() * 0.5 * torch.erfc(h.abs() * 0.5 ** 0.5) + h.clamp(min=0), "silu": h * torch.special.expit(h)}[act].abs()
    finite = torch.isfinite(h)
    near = finite & (want >= 2.0 ** -100)
    assert ((got - want).abs() <= want * (2.0 ** -13 + 2.0 ** -20 * (1 + h * h / 8) + 2.0 ** -22))[near].all()
    assert (got <= 2.0 ** -99)[finite & ~near].all()
    assert (t.q[:, 0].double() == torch.where(t.scale > 0, torch.where(h < 0, -127., 127.), 0.))[finite].all()
    lost = torch.isnan(h) | (torch.isinf(h) & (h > 0 if act == "relu" else True))
    assert torch.isnan(t.scale[lost]).all() and not t.q[lost].any()
    # the same among many columns, in rows that are and are not whole vectors
    for cols in (2048, 2049):
        y = torch.zeros((64, cols), dtype=torch.bfloat16, device="cuda")
        values = x[finite & (h.abs() < 60)][:, 0]
        y[:, :1024] = values[torch.randint(0, values.numel(), (64, 1024), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")]
        big = B.lrbi_i8_tokens(y.repeat(200, 1), act=act)
        one = B.lrbi_i8_tokens(y, act=act)
        assert same(big.q, one.q.repeat(200, 1)) and same(big.scale, one.scale.repeat(200))


SHAPES = [(1, 1, 1), (16, 64, 1), (500, 800, 1), (500, 801, 3), (33, 17, 9), (4096, 9216, 1), (4096, 9216, 8), (1000, 4096, 16), (129, 1000, 17), (500, 801, 333),
          (256, 2304, 40), (640, 320, 64), (100, 129, 100), (4096, 512, 128), (300, 3000, 129), (2000, 1024, 200), (1024, 640, 256), (130, 16, 257),
          (4097, 384, 300), (1000, 257, 1000), (257, 4096, 511), (3000, 144, 2000), (8192, 1040, 1500), (16384, 128, 520), (64, 16384, 700), (12, 131072, 5),
          (24, 100000, 70)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,batch", SHAPES)
def test_products_are_exact(B, rows, cols, batch, dtype):
    w, x = random_rows8(B, rows, cols, 1), random_rows8(B, batch, cols, 2)
    y = B.lrbi_i8_gemm(w, x, y_dtype=dtype)
    assert same(y, product(w, x, dtype))
    assert B.device_status() == 0


@pytest.mark.parametrize("batch", [1, 2, 8, 15, 31, 32, 33, 48, 63, 65, 96, 127, 160, 192, 255, 384, 512, 640, 1024])
def test_every_size_of_batch(B, batch):
    w, x = random_rows8(B, 777, 1300, 3), random_rows8(B, batch, 1300, 4)
    assert same(B.lrbi_i8_gemm(w, x), product(w, x, torch.bfloat16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,batch", [(4490, 65, 1028), (4491, 65, 1028), (3180, 281, 1325), (3181, 281, 1325), (3140, 679, 987), (3141, 679, 987),
                                             (3974, 598, 780), (3975, 598, 780), (3976, 598, 780), (4098, 577, 808), (4100, 577, 808)])
def test_sizes_between_rounds_of_tiles(B, rows, cols, batch, dtype):
    """Many tokens, the outputs cut into 128 to 256 channels for the last round's sake."""
    w, x = random_rows8(B, rows, cols, 9), random_rows8(B, batch, cols, 10)
    assert same(B.lrbi_i8_gemm(w, x, y_dtype=dtype), product(w, x, dtype))
    assert B.device_status() == 0


@pytest.mark.parametrize("batch", [3, 40, 300, 600])
def test_largest_sums(B, batch):
    """131072 columns of 127 * 127 on top of one another stay in 32 bits."""
    w, x = random_rows8(B, 20, 131072, 5), random_rows8(B, batch, 131072, 6)
    w.q.fill_(127)
    w.q[7:].fill_(-127)
    x.q.fill_(127)
    y = B.lrbi_i8_gemm(w, x, y_dtype=torch.float32)
    assert same(y, product(w, x, torch.float32)) and y[0, 0] != 0


@pytest.mark.parametrize("batch", [1, 20, 600])
def test_no_rows_and_surroundings(B, batch):
    """Nothing beyond the output is written, and no tokens are no work."""
    w = random_rows8(B, 301, 200, 7)
    assert B.lrbi_i8_gemm(w, B.lrbi_i8_tokens(torch.empty((0, 200), device="cuda"))).shape == (0, 301)
    x = random_rows8(B, batch, 200, 8)
    room = torch.full((batch * 301 + 64,), 7.0, device="cuda", dtype=torch.bfloat16)
    import ctypes
    for first in (0, 1, 8):       # also off a 16-byte boundary
        room.fill_(7.0)
        rc = B.lib().lrbi_i8_gemm(w.q.data_ptr(), w.scale.data_ptr(), 301, 200, x.q.data_ptr(), x.scale.data_ptr(), batch,
                                  room.data_ptr() + 2 * first, B.Y_BF16, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == B.OK
        assert same(room[first:first + batch * 301].view(batch, 301), product(w, x, torch.bfloat16))
        assert (room[:first] == 7).all() and (room[first + batch * 301:] == 7).all()


@pytest.mark.parametrize("rows,cols,tile,rank", [(500, 800, (500, 800), 16), (300, 1000, (128, 96), 40), (64, 130, (7, 33), 3)])
def test_weights_are_the_definition(B, rows, cols, tile, rank):
    from paper_1905_05686_b200 import synth

    layer = synth.Layer("i8", rows, cols, *tile, rank, 0.3, 0.05)
    ip, iz = synth.make_factors(layer)
    ip, iz = B.to_device_words(synth.pack_ip(ip)), B.to_device_words(synth.pack_iz(iz))
    W = B.to_device_bf16(synth.make_weights(layer))
    bits = B.lrbi_decode_mask(layer, ip, iz).cpu().numpy().view(np.uint32)
    mask = torch.from_numpy(((bits[:, :, None] >> np.arange(32, dtype=np.uint32)) & 1).reshape(rows, -1)[:, :cols].astype(bool)).cuda()
    for m, args in ((torch.ones_like(mask), ()), (mask, (ip, iz))):
        V = W.clone()
        V[~m] = float("nan")                       # what pruned places hold is not looked at
        if bool(m[3].any()):
            V[3] = torch.where(m[3], float("inf"), float("nan"))
        q = B.lrbi_i8_quantize(layer, V, *args)
        want, scale = rows8(torch.where(m, V.float(), 0.0))
        assert torch.equal(q.q[:, :cols], want) and same(q.scale, scale) and not q.q[:, cols:].any()


def test_streams_and_graphs(B):
    """Calls on another stream, and a captured sequence that is replayed on new inputs."""
    w = random_rows8(B, 1000, 520, 9)
    for batch in (1, 100, 700):
        x = activations(batch, 520, torch.bfloat16)
        want = B.lrbi_i8_gemm(w, B.lrbi_i8_tokens(x, act="gelu"))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        y = B.lrbi_i8_gemm(w, B.lrbi_i8_tokens(x, act="gelu", stream=side), stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert same(y, want)
        fixed = torch.zeros_like(x)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = B.lrbi_i8_gemm(w, B.lrbi_i8_tokens(fixed, act="gelu"))
        for k in range(3):
            fixed.copy_(x if k != 1 else -x)
            graph.replay()
        assert same(y, want)


def test_weights_written_just_before(B):
    """Weights and tokens that the calls right before a product wrote."""
    a, b = activations(2000, 1024, torch.bfloat16, seed=1), activations(24, 1024, torch.bfloat16, seed=2)
    for batch in (1, 24):
        for _ in range(20):
            x = B.lrbi_i8_tokens(b[:batch])
            w = B.lrbi_i8_tokens(a)
            y = B.lrbi_i8_gemm(w, x)
            del w
        w = B.lrbi_i8_tokens(a)
        assert same(y, product(w, x, torch.bfloat16))
