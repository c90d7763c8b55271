"""The forms of the 8-bit product: which one a size takes, that no size takes one that is not tested here, and each of them bit for
bit.

A form is a kernel with what distinguishes its code and its waits: warp-level products by tokens of a tile, threads and steps under
way; tiles in tensor memory by tokens (up to), CTAs that share the columns and CTAs an SM; pairs by channels of a tile.  Sizes are
among the smallest that take the form, with rows of Y that are and are not whole vectors."""
import ctypes
import math
import random

import pytest
import torch

BF16, F32 = torch.bfloat16, torch.float32
TILES = (16, 32, 64, 128, 192, 256)

FORMS = {
    ("few", 8, 256, 2): [(2384, 144, 1, BF16), (2379, 130, 1, BF16), (2380, 999, 7, F32)],
    ("few", 8, 256, 4): [(2384, 1040, 1, BF16), (2377, 1032, 1, BF16), (4097, 4100, 8, F32)],
    ("few", 8, 512, 4): [(144, 144, 1, F32), (131, 130, 1, F32), (500, 5003, 8, BF16)],
    ("few", 16, 512, 4): [(144, 144, 9, BF16), (133, 130, 9, BF16), (600, 801, 16, F32)],
    ("long", 128): [(4624, 400, 781, BF16), (4721, 401, 780, BF16)],
    ("long", 160): [(9488, 272, 258, BF16), (9505, 257, 274, BF16)],
    ("long", 192): [(39456, 144, 17, F32), (38033, 132, 17, F32)],
    ("long", 224): [(45936, 144, 9, F32), (45887, 137, 9, F32)],
    ("long", 256): [(50400, 144, 9, BF16), (51603, 130, 9, F32)],
    ("split", 16, 1, 1): [(144, 144, 17, F32), (131, 130, 17, F32)],
    ("split", 16, 1, 2): [(18960, 144, 9, F32), (19061, 133, 9, F32)],
    ("split", 16, 2, 1): [(144, 1184, 131, F32), (135, 1170, 131, BF16)],
    ("split", 16, 4, 1): [(144, 784, 17, F32), (131, 771, 19, BF16)],
    ("split", 16, 4, 2): [(4272, 19744, 9, BF16), (4225, 20672, 9, BF16)],
    ("split", 16, 8, 1): [(144, 2576, 18, F32), (131, 2680, 17, F32)],
    ("split", 16, 8, 2): [(1936, 28720, 10, F32), (1929, 27758, 11, BF16)],
    ("split", 32, 1, 1): [(144, 144, 307, BF16), (133, 132, 306, BF16)],
    ("split", 32, 1, 2): [(19184, 144, 17, F32), (19535, 133, 17, BF16)],
    ("split", 32, 2, 1): [(144, 1184, 243, BF16), (137, 1193, 242, F32)],
    ("split", 32, 2, 2): [(9504, 67392, 19, F32), (9477, 57303, 18, F32)],
    ("split", 32, 4, 1): [(144, 1168, 116, F32), (131, 1163, 116, F32)],
    ("split", 32, 4, 2): [(4288, 22592, 23, BF16), (4245, 20484, 18, BF16)],
    ("split", 32, 8, 1): [(144, 2592, 49, F32), (133, 2589, 52, BF16)],
    ("split", 32, 8, 2): [(1936, 34800, 18, BF16), (1923, 33673, 19, F32)],
    ("split", 64, 1, 1): [(2336, 144, 33, F32), (2339, 132, 33, F32)],
    ("split", 64, 1, 2): [(19968, 144, 33, BF16), (18969, 142, 33, F32)],
    ("split", 64, 2, 1): [(144, 1680, 938, BF16), (137, 1690, 946, F32)],
    ("split", 64, 2, 2): [(9504, 74960, 35, BF16), (9477, 74108, 34, BF16)],
    ("split", 64, 4, 1): [(944, 1296, 33, BF16), (903, 1295, 34, BF16)],
    ("split", 64, 4, 2): [(4272, 25216, 34, BF16), (4253, 24948, 33, F32)],
    ("split", 64, 8, 1): [(528, 2592, 35, BF16), (523, 2573, 33, F32)],
    ("split", 64, 8, 2): [(1984, 39520, 33, F32), (1943, 38555, 33, F32)],
    ("split", 128, 1, 1): [(3520, 144, 66, BF16), (3457, 132, 65, F32)],
    ("split", 128, 1, 2): [(19200, 144, 65, F32), (18951, 131, 65, F32)],
    ("split", 128, 2, 1): [(2816, 1744, 65, F32), (2753, 1733, 69, F32)],
    ("split", 128, 2, 2): [(9520, 113184, 74, BF16), (9491, 103554, 71, F32)],
    ("split", 128, 4, 1): [(1296, 1808, 66, F32), (1283, 1918, 65, F32)],
    ("split", 128, 4, 2): [(2112, 30352, 255, BF16), (2131, 29320, 242, BF16)],
    ("split", 128, 8, 1): [(656, 3680, 68, BF16), (653, 3756, 66, BF16)],
    ("split", 128, 8, 2): [(144, 29728, 966, BF16), (131, 32918, 928, BF16)],
    ("split", 192, 1, 1): [(5664, 144, 135, F32), (5817, 134, 129, BF16)],
    ("split", 192, 2, 1): [(3648, 2784, 130, F32), (3567, 2810, 129, F32)],
    ("split", 192, 4, 1): [(1568, 3376, 129, BF16), (1565, 3368, 130, BF16)],
    ("split", 256, 1, 1): [(9584, 144, 197, BF16), (9699, 130, 200, F32)],
    ("split", 256, 2, 1): [(7232, 4144, 201, BF16), (6855, 4324, 199, BF16)],
    ("split", 256, 4, 1): [(2112, 6928, 199, F32), (2127, 7100, 194, BF16)],
}
# Pairs that go through several tiles, so that both accumulators are used again: tiles of each width, tokens and channels running
# fastest, rows of Y that are and are not whole vectors.
ROUNDS = [(6240, 1950, 760, BF16, 128), (1131, 1929, 3932, F32, 128), (2071, 5357, 4146, F32, 160), (2080, 3091, 4333, F32, 160),
          (3871, 3747, 1044, BF16, 160), (2848, 3961, 4683, BF16, 192), (3857, 4426, 3499, F32, 192), (3424, 2708, 2906, BF16, 192), (4781, 2295, 4931, BF16, 224),
          (16565, 2304, 1572, F32, 224), (6688, 2629, 3398, BF16, 224), (8645, 2123, 3269, F32, 256), (11456, 1201, 4359, F32, 256), (4943, 1869, 4998, BF16, 256)]


@pytest.fixture(scope="module")
def B():
    from paper_1905_05686_b200 import build
    build.build()
    from paper_1905_05686_b200 import binding
    return binding


def form(B, plan):
    if plan.kernel == B.I8_FEW:
        return "few", plan.tokens, plan.threads, plan.stages
    if plan.kernel == B.I8_LONG:
        return "long", plan.channels
    return "split", min(n for n in TILES if n >= plan.tokens), plan.split, plan.per_sm


def test_sizes_take_the_forms_named_here(B):
    for want, sizes in FORMS.items():
        for rows, cols, batch, dtype in sizes:
            assert form(B, B.i8_gemm_plan(rows, cols, batch, dtype)) == want, (rows, cols, batch)
    for rows, cols, batch, dtype, channels in ROUNDS:
        plan = B.i8_gemm_plan(rows, cols, batch, dtype)
        assert form(B, plan) == ("long", channels) and math.ceil(batch / 256) * math.ceil(rows / channels) > 74, (rows, cols, batch)


def test_no_size_takes_another_form(B):
    """Sizes over the whole range, spread over their logarithms."""
    rng = random.Random(1905)

    def size(hi):
        n = int(math.exp(rng.uniform(0, math.log(hi + 1))))
        return max(1, min(hi, (n + 15) // 16 * 16 if rng.random() < 0.5 else n))

    for _ in range(40000):
        rows, cols, batch, dtype = size(1 << rng.choice((14, 20))), size(1 << rng.choice((14, 17))), size(1 << rng.choice((8, 12, 18))), rng.choice((BF16, F32))
        plan = B.i8_gemm_plan(rows, cols, batch, dtype)
        assert form(B, plan) in FORMS, (rows, cols, batch, dtype, form(B, plan))
        # what the kernels are built for
        assert 2 <= plan.stages <= 8 and plan.split in (1, 2, 4, 8) and plan.split <= math.ceil(cols / 128)
        if plan.kernel == B.I8_SPLIT:
            assert plan.tokens % 16 == 0 and 16 <= plan.tokens <= 256 and plan.channels == 128 and (plan.per_sm == 1 or plan.tokens <= 128)
            assert plan.stages * (16384 + 128 * plan.tokens) >= 512 * plan.tokens       # the sums take the stages' place
        if plan.kernel == B.I8_LONG:
            assert plan.channels % 32 == 0 and 128 <= plan.channels <= 256 and plan.tokens == 256


def test_plan_arguments(B):
    L, plan = B.lib(), B.I8Plan()
    for args in ((0, 64, 4, 0), (64, 0, 4, 0), (64, (1 << 17) + 1, 4, 0), (64, 64, 0, 0), (64, 64, -1, 0), (64, 64, 4, 2)):
        assert L.lrbi_i8_gemm_plan(*args, ctypes.byref(plan)) == B.ERR_INVALID_ARG, args
    assert L.lrbi_i8_gemm_plan(64, 64, 4, 0, None) == B.ERR_INVALID_ARG
    for args in ((2 ** 31 - 4095, 64, 4, 0), (64, 64, 2 ** 31 - 4095, 0)):
        assert L.lrbi_i8_gemm_plan(*args, ctypes.byref(plan)) == B.ERR_UNSUPPORTED
    assert L.lrbi_i8_gemm_plan(2 ** 31 - 4096, 1 << 17, 2 ** 31 - 4096, 1, ctypes.byref(plan)) == B.OK and plan.kernel == B.I8_LONG
    with pytest.raises(TypeError):
        B.i8_gemm_plan(64, 64, 4, torch.float16)
    with pytest.raises(B.LrbiError):
        B.i8_gemm_plan(64, 64, 0)


def check(B, rows, cols, batch, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + cols + batch)

    def rows8(n):
        q = torch.randint(-127, 128, (n, (cols + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)
        q[:, cols:] = 0
        return B.I8Rows(q, torch.rand(n, generator=g, device="cuda") + 0.5, n, cols)

    w, x = rows8(rows), rows8(batch)
    y = B.lrbi_i8_gemm(w, x, y_dtype=dtype)
    for r in range(0, rows, 1 << 13):                   # whole numbers below 2^31: exact in 64 bits, and rounded as the definition says
        total = x.q[:, :cols].double() @ w.q[r:r + (1 << 13), :cols].double().t()
        want = ((total.float() * x.scale[:, None]) * w.scale[None, r:r + (1 << 13)]).to(dtype)
        assert torch.equal(y[:, r:r + (1 << 13)], want)
    assert B.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("at", sorted(FORMS, key=str), ids=lambda at: "-".join(map(str, at)))
def test_products_of_every_form(B, at):
    for size in FORMS[at]:
        assert form(B, B.i8_gemm_plan(*size)) == at
        check(B, *size)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,batch,dtype,channels", ROUNDS)
def test_pairs_through_several_tiles(B, rows, cols, batch, dtype, channels):
    check(B, rows, cols, batch, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols,batch", [(4096, 9216, 128), (4096, 4096, 64), (4096, 4096, 200), (4096, 4096, 512), (2518, 8772, 729), (249, 1249, 324), (6606, 12584, 124), (4192, 13222, 269),
                                             (1634, 9632, 291), (3996, 6624, 248), (154, 14703, 469), (1922, 49592, 41)])
def test_products_of_common_sizes(B, rows, cols, batch):
    for dtype in (BF16, F32):
        check(B, rows, cols, batch, dtype)
