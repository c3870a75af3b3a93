"""Prompt attention where q_indptr holds wrong bounds: the requests they belong to are flagged and left alone, the others are right."""
import pytest
import torch

import paper_2609_34370_b200 as spx
from prompt_util import DEV, Batch

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _run(b, starts, lens):
    """b's requests with these bounds and lengths; rows that no valid request has keep what they held."""
    (q, k, v, strides, table, n, _, *rest), scales = b.device()
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    out, lse = torch.full_like(q, 3.25), torch.full(q.shape[:2], -7.0, device=DEV)
    _, _, ws = spx.prompt_attention(q, k, v, strides, table, ints(lens), ints(starts), *rest, out=out, lse=lse, **scales)
    assert int(ws.status.item()) == spx.DEV_BAD_LEN
    return out, lse


@pytest.mark.parametrize("dtype,kind", [(BF16, "rows"), (BF16, "e4m3"), (F32, "rows")])
@pytest.mark.parametrize("starts,lens", [([0, 1000, 18, 27], [1200, 30, 40]), ([0, 2147483647, 18, 27], [1200, 30, 40]), ([0, -2000000000, 18, 27], [30, 30, 40]),
                                         ([-5, 18, 18, 27], [30, 0, 40])])
def test_the_request_behind_a_wrong_bound(starts, lens, dtype, kind):
    b = Batch([30, 18, 40], [9, 9, 9], 8, 2, 64, 16, dtype=dtype, kind=kind, seed=1)
    out, lse = _run(b, starts, lens)
    b.check(out, lse, requests=[2])
    assert bool((out[:18] == 3.25).all()) and bool((lse[:18] == -7.0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_several_requests_claim(dtype):
    """More row blocks than the rows could make.  The requests are alike, so that the rows come out the same whoever writes them."""
    b = Batch([900], [700], 8, 2, 64, 16, dtype=dtype, seed=2)
    many = Batch.__new__(Batch)
    many.__dict__.update(b.__dict__)
    many.table = b.table.repeat(9, 1)
    out, lse = _run(many, [0, 700] * 5, [900] * 9)
    b.check(out, lse)
