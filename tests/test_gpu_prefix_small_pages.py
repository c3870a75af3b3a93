"""Shared prefixes over pages of fewer than eight tokens, which the fp32-arithmetic kernels read, in every type."""
import pytest
import torch

from prompt_util import verify
from test_gpu_prefix import _grouped

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d,page,ks", [(8, 2, 64, 4, [4, 0]), (7, 1, 128, 1, [0, 2]), (16, 4, 128, 2, [15])])
@pytest.mark.parametrize("dtype,kind", [(torch.bfloat16, "rows"), (torch.bfloat16, "e4m3"), (torch.float32, "rows"), (torch.float32, "e4m3")])
def test_groups(hq, hkv, d, page, ks, dtype, kind):
    b, groups = _grouped([5, 1, 9], [700, 300, 129], [1, 90, 128, 17], ks, hq, hkv, d, page, dtype=dtype, kind=kind, seed=hq)
    out, lse, status = verify(b, groups)
    assert status == 0
    b.check(out, lse)
