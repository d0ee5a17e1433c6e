"""The feed-forward block's workspace sizes (include/layer.h): no GPU is needed."""
import pytest
import torch

from paper_2607_20548_gb300 import build
from paper_2607_20548_gb300 import soap as S


@pytest.fixture(scope="module")
def lib():
    build.build()
    return S.load_library()


@pytest.mark.parametrize("rows,hidden,width,groups", [(70000, 2048, 8192, 1), (200000, 2048, 768, 1), (200000, 1024, 1024, 4)])
def test_long_sums_take_their_parts_alone(lib, rows, hidden, width, groups):
    """Beside dg, du and h: of the weights' gradients a block of 256 x 256 sums for each run of 65536 rows, which groups of
    their own at most double, and blocks for 76 pairs in each of three phases."""
    size = lib.layer_ffn_workspace_bytes(rows, hidden, width, groups, S.DTYPES[torch.bfloat16], 1, 1)
    kept, block, tiles = 3 * rows * width * 2, 256 * 256 * 4, 3 * (hidden // 256) * (width // 256)
    runs = -(-rows // 65536)
    assert size >= kept + tiles * runs * block
    assert size <= kept + tiles * (runs + (min(groups, runs) if groups > 1 else 0)) * block + 3 * 76 * block + (8 << 20)
