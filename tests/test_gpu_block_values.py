"""Values at the edges of the block's operators' range, where a formula meets infinities, zeros and the ends of a type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def _b():
    from paper_1905_05686_b200 import binding
    return binding


@pytest.mark.parametrize("rows,cols,pad", [(5, 512, 0), (3, 16, 8), (7, 301, 0), (4, 256, 3)], ids=lambda v: str(v))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_activation_of_infinities(act, dtype, rows, cols, pad):
    """The formula's own result: +inf for +inf; 0 for relu of -inf, NaN (infinity times zero) for gelu and silu of it."""
    b = _b()
    h = torch.randn((rows, cols + pad), device="cuda").to(dtype)[:, :cols]
    plain = b.lrbi_activation(h.contiguous(), act)
    at = {(0, 0): INF, (1, 7): -INF, (rows - 1, cols - 1): INF, (rows - 1, cols - 2): NAN, (2, 3): -INF, (0, cols // 2): INF}
    for place, v in at.items():
        h[place] = v
    want = {INF: INF, -INF: 0.0 if act == "relu" else NAN}
    a, kept = b.lrbi_activation(h, act, checkpoint=True)
    _, again = b.lrbi_activation_backward(torch.ones_like(h), h, act, restore=True)
    rest = torch.ones((rows, cols), dtype=torch.bool)
    for got in (a, b.lrbi_activation(h, act), again):
        got = got.float().cpu()
        for place, v in at.items():
            w = want.get(v, NAN)
            assert got[place] == w or (np.isnan(w) and torch.isnan(got[place])), (place, v)
            rest[place] = False
        assert torch.equal(got[rest], plain.float().cpu()[rest])
    stands = b.lrbi_checkpoint_load(kept, F32)
    assert all(torch.isnan(stands[place]) for place in at)          # a group with either restores as NaN
