"""What the stand-alone operators' binding and planning do on the host: no GPU is needed."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2607_20548_gb300 import build, layers
from paper_2607_20548_gb300 import soap as S


@pytest.mark.parametrize("batch", [1, 30, 5000, 65535])
@pytest.mark.parametrize("rows,cols,dtype,planes", [(130, 200, 1, 1), (200, 140, 0, 2), (2000, 136, 1, 1)])
def test_workspace_is_what_the_kernels_use(batch, rows, cols, dtype, planes):
    """X twice, S and B in fp16 with rows of whole 16-byte units, and for all matrices together no more than
    1216 partial sums, or one each, a scale and a counter; seven pieces rounded up to 256 bytes."""
    build.build()
    got = S.load_library().muon_orthogonalize_workspace_bytes(batch, rows, cols, dtype)
    up8 = lambda n: (n + 7) // 8 * 8  # noqa: E731
    r = min(rows, cols)
    need = 2 * planes * batch * (2 * rows * up8(cols) + 2 * r * up8(r))
    assert need <= got <= need + 12 * max(1216, batch) + 8 * batch + 12 + 7 * 256


def test_imports_on_a_torch_without_cuda():
    """A CPU-only torch has none of torch._C's CUDA functions: the package (its oracle-side and planning parts
    are of use there) imports all the same, and the operators refuse what is no CUDA tensor."""
    code = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, name)
import paper_2607_20548_gb300 as lib
from paper_2607_20548_gb300 import layerwise, workloads
try:
    lib.layer_norm_forward(torch.zeros(2, 8))
except TypeError:
    print("refused")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "refused", r.stderr


@pytest.mark.parametrize("make,copies", [
    (lambda t: t, False),
    (lambda t: t[..., :5], False),              # a slice of every row
    (lambda t: t[..., 2:7], False),
    (lambda t: t[:1, 1:2, :, :5], False),       # dimensions of one
    (lambda t: t[1:, :, :, 3:], False),
    (lambda t: t[0], False),
    (lambda t: t[0, 0, :, 1:], False),
    (lambda t: t[:, :, 0, :5], False),          # a longer step between rows
    (lambda t: t[:, :, ::2], False),
    (lambda t: t[..., 0:1], False),
    (lambda t: t[0, 0, 0, 1:4], False),
    (lambda t: t[..., ::2], True),              # elements apart
    (lambda t: t[:, 1:, :, :5], True),          # two steps between rows
    (lambda t: t[:, 1:2, :, :5], True),
    (lambda t: t[:, :, :1, :5].expand(2, 3, 4, 5), True),
    (lambda t: t.transpose(0, 1)[..., :5], True),
    (lambda t: t.mT, True),
    (lambda t: t[0, 0, 0, ::3], True),
])
def test_rows_are_copied_only_where_no_leading_dimension_describes_them(make, copies):
    t = make(torch.arange(2 * 3 * 4 * 9, dtype=torch.float32).view(2, 3, 4, 9))
    got, rows, ld = layers._rows(t)
    width = t.shape[-1]
    assert (got.data_ptr() != t.data_ptr()) == copies
    assert rows == t.numel() // width and ld >= width
    assert torch.equal(torch.as_strided(got, (rows, width), (ld, 1), got.storage_offset()), t.reshape(rows, width))
