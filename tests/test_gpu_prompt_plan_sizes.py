"""Plans of more requests, row blocks and tokens than one pass of the planner takes, against the definition in 64 bits."""
import pytest
import torch

import paper_2609_34370_b200 as spx
from prompt_util import DEV, Batch, prompt, verify

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_requests_than_threads_of_the_planner(dtype):
    """2500 requests in three passes, some without rows, some prompts, one with a bad length in the last pass."""
    n = 2500
    lens = [1 + (7 * i) % 40 for i in range(n)]
    m = [0 if i % 11 == 3 else min(x, 1 + i % 5) for i, x in enumerate(lens)]
    for r, x in ((5, 300), (1023, 150), (1024, 200), (2040, 129)):
        lens[r] = m[r] = x
    b = Batch(lens, m, 4, 1, 64, 16, dtype=dtype, seed=1, poison=0.5)
    (q, k, v, strides, table, n_d, starts, hkv, page, pages), _ = b.device()
    n_d[2400] = -1
    assert m[2400] > 0
    out, lse, ws = spx.prompt_attention(q, k, v, strides, table, n_d, starts, hkv, page, pages)
    assert int(ws.status.item()) == spx.DEV_BAD_LEN
    b.check(out, lse, requests=list(range(0, 2400, 61)) + [5, 1022, 1023, 1024, 1025, 2040, 2047, 2048, 2049, 2399, 2401, 2499])
    bad = slice(b.starts[2400], b.starts[2401])
    assert bool((out[bad] == 0).all()) and bool(torch.isnan(lse[bad]).all())
    good = torch.ones(b.starts[-1], dtype=torch.bool)
    good[bad] = False
    assert bool(torch.isfinite(lse[good]).all())


@pytest.mark.parametrize("dtype,m", [(F32, 20000), (BF16, 40000)])
def test_more_row_blocks_than_threads_of_the_planner(dtype, m):
    """One prompt of more than 1024 row blocks (fp32: 64 packed rows each, 16 bits: 256), eight heads of a group, behind another request."""
    lens = [40, m]
    b = Batch(lens, [40, m], 8, 1, 64, 128, dtype=dtype, seed=2, poison=0.5)
    out, lse, status = prompt(b)
    assert status == 0 and bool(torch.isfinite(out).all())
    rows = torch.tensor([0, 1, 63, 127, 128, 1000, m // 2, m // 2 + 1, m - 129, m - 2, m - 1])
    _check_rows(b, out, lse, 1, rows)


def _check_rows(b, out, lse, r, rows):
    """Some rows of a long prompt: each as the one new row of a request of its own length."""
    for j in rows.tolist():
        one = Batch.__new__(Batch)
        one.__dict__.update(b.__dict__)
        seen = b.lens[r] - b.m[r] + j + 1
        one.lens, one.m, one.starts, one.table, one.q = [seen], [1], [0, 1], b.table[r:r + 1], b.q[b.starts[r] + j:b.starts[r] + j + 1]
        one.check(out[b.starts[r] + j:b.starts[r] + j + 1], lse[b.starts[r] + j:b.starts[r] + j + 1])


@pytest.mark.parametrize("dtype,kind", [(BF16, "rows"), (BF16, "e4m3"), (F32, "rows")])
def test_more_tokens_than_the_sort_tells_apart(dtype, kind):
    """140,000 cached tokens: 1094 tiles, past the last length that the planner sorts by, beside ordinary requests."""
    b = Batch([140000, 50, 131072 + 5], [70, 50, 1], 4, 1, 64, 128, dtype=dtype, kind=kind, seed=3)
    out, lse, status = prompt(b)
    assert status == 0
    b.check(out, lse, requests=[1, 2])
    _check_rows(b, out, lse, 0, torch.tensor([0, 1, 31, 63, 64, 69]))


def _groups(n, size, page, own):
    """n groups of `size` requests behind 128 or 256 tokens, and a request of its own behind every tenth group."""
    lens, m, shared, bounds, prefixes = [], [], [], [0], []
    for i in range(n):
        p = 128 * (1 + i % 2)
        shared.append((len(lens), len(lens) + size, p))
        for j in range(size):
            m.append(1 + (i + j) % 3)
            lens.append(p + m[-1] + (own * (i + 3 * j)) % 50)
        bounds.append(len(lens))
        prefixes.append(p)
        if i % 10 == 9:
            m.append(2), lens.append(20)
            bounds.append(len(lens))
            prefixes.append(1000)
    return lens, m, shared, bounds, prefixes


@pytest.mark.parametrize("dtype,kind,n,size", [(BF16, "rows", 550, 2), (BF16, "e4m3", 550, 2), (F32, "rows", 550, 2), (BF16, "rows", 1100, 2), (BF16, "rows", 3, 700)])
def test_groups_of_more_than_a_thousand_requests(dtype, kind, n, size):
    lens, m, shared, bounds, prefixes = _groups(n, size, 16, 7)
    assert len(lens) > 1024
    b = Batch(lens, m, 4, 1, 64, 16, dtype=dtype, kind=kind, shared=shared, seed=n, poison=0.5)
    out, lse, status = verify(b, (bounds, prefixes))
    assert status == 0 and bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    b.check(out, lse, requests=sorted(set(range(0, len(lens), 37)) | {1022, 1023, 1024, 1025, len(lens) - 2, len(lens) - 1}))


def test_a_thousand_grouped_requests_with_bad_data():
    """The requests' own errors are found behind the first thousand too."""
    lens, m, shared, bounds, prefixes = _groups(550, 2, 16, 7)
    b = Batch(lens, m, 4, 1, 64, 16, shared=shared, seed=9, poison=0.5)
    r0 = bounds[540]
    r1 = bounds[545]
    assert r0 > 1024 and bounds[541] == r0 + 2 and bounds[546] == r1 + 2
    b.table[r0 + 1, 0] = b.table[0, 0]                     # another page than its group's
    (args, _) = b.device()
    args[5][r1] = prefixes[545] + m[r1] - 1                # a prefix that holds a new position
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    out, lse, ws = spx.verify_attention(*args, max_q_len=3, group_indptr=ints(bounds), prefix_lens=ints(prefixes))
    assert int(ws.status.item()) == (spx.DEV_BAD_PAGE | spx.DEV_BAD_LEN)
    for r in (r0 + 1, r1):
        rows = slice(b.starts[r], b.starts[r + 1])
        assert bool((out[rows] == 0).all()) and bool(torch.isnan(lse[rows]).all())
    b.check(out, lse, requests=[0, r0 - 1, r0, r0 + 2, r1 - 1, r1 + 1, r1 + 2])
