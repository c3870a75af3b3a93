"""Scales that are not finite in 8-bit pools: rows that see such a token are not finite, the others are as without it."""
import math

import pytest
import torch

from prompt_util import Batch, prompt, verify

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_scale_that_is_not_finite(which, bad, dtype):
    """Keys and values of one sign: a NaN that were taken for an infinity would drop the token from the softmax, or be an infinity."""
    lens, m = [300, 200], [300, 40]
    b = Batch(lens, m, 8, 2, 128, 16, dtype=dtype, kind="e4m3", sb=8, seed=3)
    ones = torch.full((), 0x38, dtype=torch.uint8)                        # 1.0
    b.q = -b.q.abs() if not math.isinf(bad) else b.q
    for x in (b.k, b.v):
        x[:] = torch.where(x != 0x7F, ones if which == "k" else x & 0x7F, x)
    hit = [(0, 100), (1, 184)]                                            # first token of the block of eight
    ref = {r: b.exact(r) for r in range(2)}
    for r, t in hit:
        getattr(b, which + "_scales")[b.table[r, t // 16], :, t % 16 // 8] = bad
    out, lse, status = prompt(b)
    assert status == 0
    for r, t in hit:
        t = t // 8 * 8
        n = max(0, t - (lens[r] - m[r]))
        o, l, to, tl = ref[r]
        rows = slice(b.starts[r], b.starts[r + 1])
        assert bool(((out[rows][:n].double() - o[:n]).abs() <= to[:n]).all()) and bool(((lse[rows][:n].double() - l[:n]).abs() <= tl[:n]).all())
        seen = out[rows][n:].float()
        if math.isnan(bad):
            assert bool(torch.isnan(seen).all())
        elif which == "v":
            assert not bool(torch.isfinite(seen).any())
    if math.isnan(bad):
        # as the attention of verify steps has it, alone and behind a shared prefix
        one = Batch([300] * 3, [4] * 3, 8, 2, 128, 16, dtype=dtype, kind="e4m3", sb=8, seed=4, shared=[(0, 3, 256)])
        one.q = -one.q.abs()
        for x in (one.k, one.v):
            x[:] = torch.where(x != 0x7F, ones if which == "k" else x & 0x7F, x)
        getattr(one, which + "_scales")[one.table[0, 3], :, 1] = bad
        for groups in (None, ([0, 3], [256])):
            out, _, status = verify(one, groups)
            assert status == 0 and bool(torch.isnan(out.float()).all()), groups
