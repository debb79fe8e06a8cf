"""GPU: the values that the tests of the products give codes and scales are those of the library's own dequantization (BF16: a value without alpha is
exact, times alpha in fp32 it rounds once, to BF16 once more)."""
import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import linear as L

from .test_gpu_weight_product import values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block2d", [False, True])
@pytest.mark.parametrize("N, K", [(64, 96), (544, 288)])
def test_values_are_the_librarys(N, K, block2d):
    w = torch.randn((N, K), generator=torch.Generator().manual_seed(5)).cuda()
    q = L.quantize_weight(w, block2d=block2d)
    for codes, scales, layout in ((q["codes_row"], q["scales_row"], B.BLOCK2D if block2d else B.ROWWISE),
                                  (q["codes_col"], q["scales_col"], B.BLOCK2D | B.COLWISE if block2d else B.COLWISE)):
        mine = (q["alpha"].double() * values(codes, scales, block2d)).float().bfloat16()
        got = B.nvfp4_46_dequantize(codes, scales, q["alpha"], N, K, layout)
        assert torch.equal(got, mine.T if layout & B.COLWISE else mine)
