"""Appends of tens of thousands of rows: blocks of several steps."""
import numpy as np
import pytest
import torch

import paper_2609_34370_b200 as spx
from prompt_util import turned

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


def _pool(lens, page, d, dtype, seed):
    need = [-(-n // page) for n in lens]
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(sum(need), generator=g).to(torch.int32).split(need)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    for r, ids in enumerate(order):
        table[r, :len(ids)] = ids
    return table, torch.full((sum(need), 1, page, d), 0.5, dtype=dtype, device=DEV), g


@pytest.mark.parametrize("lens,m,page,d,dtype,base", [
    ([40000], [40000], 1, 64, BF16, 0.0), ([40000], [40000], 1, 64, BF16, 10000.0), ([33000, 20, 70001, 9], [33000, 6, 70000, 9], 8, 64, F32, 10000.0),
    ([16384 + 3], [16384 + 3], 16, 128, BF16, 10000.0), ([17000, 1000], [17000, 1000], 16, 512, BF16, 10000.0), ([131072], [131072], 16, 64, BF16, 0.0),
    ([30 + i % 7 for i in range(1100)] + [50000], [1 + i % 30 for i in range(1100)] + [49999], 16, 64, BF16, 10000.0)])
def test_rows_of_long_prompts(lens, m, page, d, dtype, base):
    table, k, g = _pool(lens, page, d, dtype, 1)
    v = k.clone()
    starts = [0] + np.cumsum(m).tolist()
    new = [torch.randn(starts[-1], 1, d, generator=g).to(dtype) for _ in range(2)]
    q = torch.randn(starts[-1], 2, d, generator=g).to(dtype)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    qd = q.to(DEV)
    status = spx.kv_append(new[0].to(DEV), new[1].to(DEV), k, v, k.stride()[:3], table.to(DEV), ints(lens), ints(starts), page, k.shape[0], rope_base=base,
                           q_rows=qd)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    t = torch.cat([torch.arange(n - c, n) for n, c in zip(lens, m)])
    r = torch.cat([torch.full((c,), i) for i, c in enumerate(m)])
    where = (table[r, t // page].long(), 0, t % page)
    want_v = torch.full(v.shape, 0.5, dtype=dtype)
    want_v[where] = new[1][:, 0]
    assert torch.equal(v.cpu(), want_v)
    got = k.cpu()
    want_k = torch.full(v.shape, 0.5, dtype=dtype)
    want_k[where] = got[where] if base else new[0][:, 0]
    assert torch.equal(got, want_k)               # no other slot
    if not base:
        return
    unit = {BF16: 2.0 ** -8 + 2.0 ** -24, F32: 2.0 ** -24}[dtype]
    for have, x in ((got[where][:, None], new[0]), (qd.cpu(), q)):
        w = turned(x.double().numpy(), t[None].numpy().astype(np.float64), base, [d // 2], False)
        pair = np.sqrt((w ** 2).reshape(*w.shape[:-1], 2, -1).sum(-2))
        # an angle below 2^17 is off by 2^-35
        assert (np.abs(have.double().numpy() - w) <= unit * np.abs(w) + 2.0 ** -34 * np.concatenate((pair, pair), -1)).all()


@pytest.mark.parametrize("base", [0.0, 10000.0])
def test_a_bad_page_at_the_end_of_a_long_prompt(base):
    """The first of its 40,000 rows stay out too, and its query rows; the requests beside it enter."""
    lens = m = [100, 40000, 30]
    table, k, g = _pool(lens, 4, 64, BF16, 2)
    table[1, 9999] = k.shape[0]
    v = k.clone()
    new = torch.randn(40130, 1, 64, generator=g).bfloat16()
    q = new.clone().to(DEV)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    status = spx.kv_append(new.to(DEV), new.to(DEV), k, v, k.stride()[:3], table.to(DEV), ints(lens), ints([0, 100, 40100, 40130]), 4, k.shape[0],
                           rope_base=base, q_rows=q)
    assert int(status.item()) == spx.DEV_BAD_PAGE
    want = torch.full(v.shape, 0.5, dtype=BF16)
    for r, a, n in ((0, 0, 100), (2, 40100, 30)):
        t = torch.arange(n)
        want[table[r].long()[t // 4], 0, t % 4] = new[a:a + n, 0]
    assert torch.equal(v.cpu(), want) and torch.equal(q[100:40100].cpu(), new[100:40100])
    assert bool((k.cpu() == 0.5).all(-1).sum() == (want == 0.5).all(-1).sum())
