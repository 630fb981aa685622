"""Many short rows, several of them in a workgroup: the statements of test_gpu_rows at their sizes."""
import pytest

import test_gpu_rows
from test_gpu_rows import KINDS, q  # noqa: F401

pytestmark = pytest.mark.gpu

# n, rows, block
SHAPES = [(1, 300, 0), (2, 257, 0), (3, 1029, 0), (4, 258, 0), (15, 259, 0), (16, 261, 0), (60, 300, 0), (63, 271, 0), (64, 272, 0),
          (65, 273, 0), (100, 1000, 0), (127, 257, 0), (128, 2049, 0), (129, 258, 0), (200, 259, 0), (255, 260, 0), (256, 1023, 0),
          (257, 261, 0), (260, 262, 0), (500, 263, 0), (511, 257, 0), (512, 1021, 0), (513, 257, 0),
          (16, 257, 16), (32, 1030, 32), (48, 258, 16), (64, 259, 64), (64, 300, 32), (80, 261, 16), (96, 262, 32), (128, 263, 128),
          (128, 2050, 64), (112, 265, 16), (144, 257, 16), (192, 259, 64), (256, 1021, 256), (256, 261, 128), (240, 263, 16),
          (256, 265, 64), (272, 257, 16), (512, 300, 512)]


@pytest.mark.parametrize("n,rows,block", SHAPES)
@pytest.mark.parametrize("dtype,gated,pad,lead", [("f16", False, 0, 0), ("bf16", True, 3, 1), ("f32", False, 8, 2)])
def test_quantize_short_rows(q, n, rows, block, dtype, gated, pad, lead):
    test_gpu_rows.test_quantize_rows(q, n, rows, block, pad, lead, dtype, gated)


@pytest.mark.parametrize("n,rows,block", SHAPES)
@pytest.mark.parametrize("kind", KINDS, ids=[k[0] for k in KINDS])
@pytest.mark.parametrize("y_type,h_type,x_type,pad", [("f16", "f16", "f16", 0), ("bf16", "f32", "i8", 1), ("f32", "f32", "bf16", 4)])
def test_norm_of_short_rows(q, n, rows, block, kind, y_type, h_type, x_type, pad):
    test_gpu_rows.test_norm_residual(q, n, rows, block, pad, kind, y_type, h_type, x_type)


def test_one_bad_row_leaves_its_neighbours(q):
    import torch
    for n, block in ((64, 0), (100, 0), (256, 0), (64, 64), (128, 128), (256, 256)):
        x = torch.randn(600, n, device="cuda", generator=torch.Generator("cuda").manual_seed(n)).half()
        signs = torch.ones(n, dtype=torch.int8, device="cuda") if block else None
        good, scale = torch.empty(600, n, dtype=torch.int8, device="cuda"), torch.empty(600, device="cuda")
        q.qtip_quantize_rows_i8(x, None, q.F16, 600, n, n, signs, block, good, n, scale)
        bad = x.clone()
        bad[7, 3], bad[8, n - 1], bad[597] = float("nan"), float("inf"), 0
        out, scale2 = torch.empty_like(good), torch.empty_like(scale)
        q.qtip_quantize_rows_i8(bad, None, q.F16, 600, n, n, signs, block, out, n, scale2)
        torch.cuda.synchronize()
        keep = torch.ones(600, dtype=torch.bool, device="cuda")
        keep[[7, 8, 597]] = False
        assert torch.equal(out[keep], good[keep]) and torch.equal(scale2[keep], scale[keep])
        assert bool(torch.isnan(scale2[[7, 8]]).all()) and float(scale2[597]) == 0 and int(out[[7, 8, 597]].abs().max()) == 0
