"""Requests that the append skips: K, V and query rows, with and without a rotation."""
import numpy as np
import pytest
import torch

import paper_2609_34370_b200 as spx
from prompt_util import DEV, Batch, turned

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("base", [0.0, 10000.0])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_skipped_request_leaves_k_v_and_query_rows(dtype, base):
    """A bad page among a prompt's new positions, and fewer tokens than rows: nothing of the request is written, all of the others is."""
    lens, m = [400, 300, 90, 33], [400, 300, 50, 6]
    b = Batch(lens, m, 4, 2, 64, 16, dtype=dtype, seed=6, poison=0.5)
    b.table[1, 15] = -1
    g = torch.Generator().manual_seed(6)
    new_k, new_v = (torch.randn(b.starts[-1], 2, 64, generator=g).to(dtype) for _ in range(2))
    (q, k, v, strides, table, n, starts, _, page, pages), _ = b.device()
    n[2] = 49
    status = spx.kv_append(new_k.to(DEV), new_v.to(DEV), k, v, strides, table, n, starts, page, pages, rope_base=base, q_rows=q)
    assert int(status.item()) == (spx.DEV_BAD_PAGE | spx.DEV_BAD_LEN)
    want_k, want_v, want_q = b.k.clone(), b.v.clone(), b.q.clone()
    got_k, got_q = k.cpu(), q.cpu()
    unit = {BF16: 2.0 ** -8 + 2.0 ** -24, F32: 2.0 ** -24}[dtype]
    for r in (0, 3):
        t = torch.arange(lens[r] - m[r], lens[r])
        rows = slice(b.starts[r], b.starts[r + 1])
        where = (b.table[r].long()[t // 16], t % 16)
        want_v.transpose(1, 2)[where] = new_v[rows]
        want_k.transpose(1, 2)[where] = new_k[rows] if base == 0 else got_k.transpose(1, 2)[where]
        if base:
            for got, x in ((got_k.transpose(1, 2)[where], new_k[rows]), (got_q[rows], b.q[rows])):
                w = turned(x.double().numpy(), t[None].numpy().astype(np.float64), base, [32], False)
                pair = np.sqrt((w ** 2).reshape(*w.shape[:-1], 2, -1).sum(-2))
                assert (np.abs(got.double().numpy() - w) <= unit * np.abs(w) + 2.0 ** -38 * np.concatenate((pair, pair), -1)).all()
            want_q[rows] = got_q[rows]
    assert torch.equal(got_k, want_k) and torch.equal(v.cpu(), want_v) and torch.equal(got_q, want_q)
