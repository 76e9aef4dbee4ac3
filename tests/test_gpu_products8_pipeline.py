"""The large tiles' loop at work: products of four and five steps of k, so that every stage is refilled, read and
refilled again, which what has one or two steps never does.  Two sizes for each tile that the choice knows, rows of results
that are whole sectors and others, k that ends in the first and in the second half of a step."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import test_gpu_products8 as T
from paper_2206_01299_amd import binding as B

# columns of the tile, of the narrower ones behind it (0: none), then m, n, k
LOOPS = [(64, 0, 65, 5471, 432), (64, 0, 74, 5664, 624), (128, 0, 2328, 6445, 432), (128, 0, 6459, 2368, 624),
         (256, 0, 2067, 6348, 432), (256, 0, 6615, 2096, 624), (256, 64, 4247, 4742, 432), (256, 64, 5372, 6672, 624),
         (256, 96, 5645, 3609, 432), (256, 96, 4440, 4864, 624), (256, 128, 3351, 6664, 432), (256, 128, 3133, 7040, 624),
         (256, 160, 1165, 6550, 432), (256, 160, 2186, 3600, 624), (256, 192, 1313, 6748, 432), (256, 192, 1814, 5136, 624),
         (256, 224, 1580, 7096, 432), (256, 224, 1835, 6176, 624)]
GATED_LOOPS = [(64, 0, 33, 4166, 432), (64, 0, 34, 4112, 624), (128, 0, 1039, 6572, 432), (128, 0, 1318, 5424, 624),
               (256, 0, 771, 6161, 432), (256, 0, 801, 6592, 624), (256, 64, 4244, 2378, 432), (256, 64, 4506, 3664, 624),
               (256, 128, 1571, 6919, 432), (256, 128, 2349, 4416, 624), (256, 192, 520, 6634, 432), (256, 192, 522, 6752, 624)]


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.fail("these tests need an MI355X")
    B.lib()


@pytest.mark.parametrize("dtype", T.DTYPES)
@pytest.mark.parametrize("tile,narrow,m,n,k", LOOPS)
def test_products_of_several_steps(dtype, tile, narrow, m, n, k):
    """Plain, added to in place, of a message, and through an activation."""
    T.test_products_by_every_kernel(dtype, m, n, k)


@pytest.mark.parametrize("dtype", T.DTYPES)
@pytest.mark.parametrize("tile,narrow,m,f,k", GATED_LOOPS)
def test_gated_blocks_of_several_steps(dtype, tile, narrow, m, f, k):
    T.test_gated_blocks_by_every_kernel(dtype, m, f, k)
