"""The same checks as test_gpu_block.py and test_gpu_w4.py at sizes that take the other kernels: many rows of whole vectors (a
warp, or several, has a row), layers of more 4-bit tiles than the GPU has warps to share them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import test_gpu_block as block
import test_gpu_w4 as w4

BF16, F32 = torch.bfloat16, torch.float32

# Rows times warps of a row are 1480 or more (1184 with one warp).  Chunks a lane has of a row: 1, 2, 4, 8, 8 in two warps, 7 in
# three (the last one's part not whole), 16 in three and in four.
NORM_SHAPES = [(1200, 256, 0), (1500, 264, 0), (1300, 1024, 8), (1201, 2048, 0), (900, 4096, 0), (1000, 5000, 0), (600, 12288, 0), (401, 16384, 16)]


@pytest.mark.parametrize("shape", NORM_SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype,y_dtype", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=["bf16", "bf16-f32", "f32"])
def test_layer_norm_of_many_rows(shape, dtype, y_dtype):
    block.test_layer_norm(shape, dtype, y_dtype, F32)


@pytest.mark.parametrize("shape", NORM_SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_layer_norm_backward_of_many_rows(shape, dtype):
    block.test_layer_norm_backward(shape, dtype, dtype, F32)


# 296 tiles of 16 rows or more: a warp takes two (297 and 1025: the last by itself); 9473 rows or more, by how evenly they fall on
# the SMs: four, two or one of a block's eight warps share the tiles.
W4_SHAPES = [(4737, 200, 32, 3), (5000, 1000, 128, 16), (4736, 2056, 64, 1), (9500, 264, 64, 8), (16384, 320, 64, 8), (16390, 333, 32, 16),
             (16384, 4096, 128, 2), (32768, 136, 128, 5), (65500, 72, 32, 9), (65536, 129, 64, 17), (4721, 8200, 128, 8)]


@pytest.mark.parametrize("shape", W4_SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gemv_of_many_rows(shape):
    w4.test_gemv(shape)


@pytest.mark.parametrize("shape", [(16384, 264, 128, 256, 16, 128), (9500, 75, 64, 32, 8, 32)], ids=lambda s: "x".join(map(str, s)))
def test_quantize_many_rows(shape):
    w4.test_quantize(shape, True)
