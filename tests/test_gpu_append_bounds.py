"""The append where q_indptr holds wrong bounds: the requests they belong to are skipped and flagged, the others enter the cache whole, and
nothing else is written."""
import numpy as np
import pytest
import torch

import paper_2609_34370_b200 as spx
from prompt_util import DEV, turned

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
PAGE, HKV, HQ, D = 16, 2, 4, 64


def _run(starts, total, lens, dtype, base, query):
    """Requests of their own pages, in pools, tables and rows with guards on both sides; what is in the cache and the rows afterwards."""
    n = len(lens)
    g = torch.Generator().manual_seed(len(starts))
    valid = [0 <= a <= b <= total and b > a and length >= b - a for a, b, length in zip(starts, starts[1:], lens)]
    need = [max(1, -(-length // PAGE)) for length in lens]
    width = max(need)
    pages = sum(need)
    table = torch.full((n + 2, width), -7, dtype=torch.int32)
    order, at = torch.randperm(pages, generator=g).to(torch.int32), 0
    for r in range(n):
        table[1 + r, :need[r]] = order[at:at + need[r]]
        at += need[r]
    pools = [torch.full((pages + 8, HKV, PAGE, D), 0.5, dtype=dtype) for _ in range(2)]
    rows = [torch.randn(total + 64, HKV, D, generator=g).to(dtype) for _ in range(2)]
    q = torch.randn(total + 64, HQ, D, generator=g).to(dtype)
    on = [x.to(DEV) for x in pools + rows + [q]]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    k, v = (x[4:4 + pages] for x in on[:2])
    new = [x[32:32 + total] for x in on[2:4]]
    qd = on[4][32:32 + total]
    status = spx.kv_append(new[0], new[1], k, v, k.stride()[:3], table.to(DEV)[1:1 + n], ints(lens), ints(starts), PAGE, pages, rope_base=base,
                           q_rows=qd if query else None)
    torch.cuda.synchronize()
    got = [x.cpu() for x in on]
    want_v, want_k, want_q = pools[1].clone(), pools[0].clone(), q.clone()
    unit = {BF16: 2.0 ** -8 + 2.0 ** -24, F32: 2.0 ** -24}[dtype]

    def take(have, x, t, into, where):
        """The rotated rows that are there, after a look at them."""
        if base:
            w = turned(x.double().numpy(), t[None].numpy().astype(np.float64), base, [D // 2], False)
            pair = np.sqrt((w ** 2).reshape(*w.shape[:-1], 2, -1).sum(-2))
            assert (np.abs(have.double().numpy() - w) <= unit * np.abs(w) + 2.0 ** -38 * np.concatenate((pair, pair), -1)).all()
        into[where] = have if base else x

    for r in range(n):
        if not valid[r]:
            continue
        a, b = starts[r], starts[r + 1]
        t = torch.arange(lens[r] - (b - a), lens[r])
        where = (4 + table[1 + r].long()[t // PAGE], slice(None), t % PAGE)
        want_v[where] = rows[1][32 + a:32 + b]
        take(got[0][where], rows[0][32 + a:32 + b], t, want_k, where)
        if query and base:
            take(got[4][32 + a:32 + b], q[32 + a:32 + b], t, want_q, slice(32 + a, 32 + b))
    assert torch.equal(got[0], want_k) and torch.equal(got[1], want_v) and torch.equal(got[4], want_q)
    assert torch.equal(got[2], rows[0]) and torch.equal(got[3], rows[1])
    assert int(status.item()) == (0 if all(valid) else spx.DEV_BAD_LEN)


@pytest.mark.parametrize("base", [0.0, 10000.0])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("starts,total,lens,query", [
    ([0, 1000, 18, 27], 27, [1200, 30, 40], True),                 # a bound past the rows, and the request behind it runs backwards
    ([-5, 3, 10], 10, [9, 30], True),
    ([0, 8, -2000000000, 8, 20], 20, [8, 8, 40, 31], True),
    ([0, 2147483647, 8, 20], 20, [8, 40, 31], True),
    ([0, 80, 0, 16], 80, [90, 5, 16], False),                      # rows that two requests claim enter the pages of both
    ([0, 80, 16, 64, 64, 80], 80, [80, 5, 300, 3, 16], False),
    ([40, 0, 40, 0, 40], 40, [7, 40, 7, 60], False),
    ([5, 14], 14, [9], True),                                      # rows before the first request's
])
def test_wrong_bounds(starts, total, lens, query, dtype, base):
    _run(starts, total, lens, dtype, base, query)


@pytest.mark.parametrize("base", [0.0, 10000.0])
def test_wrong_bounds_in_the_middle_of_a_batch(base):
    """200 requests of 1 to 20 rows; some of their bounds point past the rows, behind them, or far ahead."""
    m = [1 + (5 * i) % 20 for i in range(200)]
    starts = [0] + np.cumsum(m).tolist()
    total = starts[-1]
    for at, x in ((30, 100000), (70, -4), (110, 2), (150, total), (199, total + 1)):
        starts[at] = x
    lens = [max(1, min(b - a, total)) + i % 33 for i, (a, b) in enumerate(zip(starts, starts[1:]))]
    _run(starts, total, lens, BF16, base, False)


@pytest.mark.parametrize("base", [0.0, 10000.0])
@pytest.mark.parametrize("n", [256, 257, 700, 1024, 1025, 1400])
def test_steps_of_many_requests_do_not_hang_on_each_others_bounds(n, base):
    """Up to 16 rows a request, as a verify step brings them: the requests whose own bounds hold enter the cache, whatever the others' are."""
    m = [1 + (5 * i) % 16 for i in range(n)]
    starts = [0] + np.cumsum(m).tolist()
    total = starts[-1]
    for at, x in ((30, 100000), (70, -4), (110, total), (111, 3), (150, 0), (n - 1, total + 1)):
        starts[at] = x
    lens = [max(1, b - a) + i % 33 if b - a <= 16 else 2 for i, (a, b) in enumerate(zip(starts, starts[1:]))]
    _run(starts, total, lens, BF16, base, False)


@pytest.mark.parametrize("base", [0.0, 10000.0])
@pytest.mark.parametrize("n,d_rows", [(3, 1), (255, 9), (300, 17), (300, 16), (1030, 33), (1030, 16)])
def test_prompts_among_steps(n, d_rows, base):
    """Ascending bounds: every row of prompts of many lengths enters, among requests of d_rows rows."""
    m = [1 + (7 * i) % d_rows for i in range(n)]
    for i, k in enumerate((8, 9, 16, 17, 24, 25, 31, 128, 129, 500)):
        m[(i * 101) % n] = k
    starts = [0] + np.cumsum(m).tolist()
    _run(starts, starts[-1], [k + i % 50 for i, k in enumerate(m)], F32, base, True)
