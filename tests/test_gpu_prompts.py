"""Attention for prompts against the definition in 64 bits: types, pools, heads, pages, lengths, masks, errors, streams."""
import math

import pytest
import torch

import paper_2609_34370_b200 as spx
from prompt_util import Batch, prompt

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# new rows behind cached ones: none, single tokens, the edges of tiles and of row blocks, odd ones
RAGGED = [(1, 0), (0, 5), (97, 0), (128, 0), (129, 3), (31, 128), (64, 64), (1, 300), (0, 0), (33, 1000), (257, 127), (2, 126)]


def _ragged(part):
    m = [a for a, _ in part]
    return [a + h for a, h in part], m


@pytest.mark.parametrize("layout", ["HND", "NHD"])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 64, 16), (32, 8, 128, 16), (14, 2, 128, 8), (6, 6, 64, 128), (4, 4, 128, 32), (24, 1, 128, 64), (12, 4, 64, 8),
                                           (128, 1, 128, 16), (100, 2, 64, 16), (66, 1, 128, 32)])
def test_ragged_bf16(hq, hkv, d, page, layout):
    lens, m = _ragged(RAGGED)
    b = Batch(lens, m, hq, hkv, d, page, layout=layout, seed=hq + page)
    out, lse, status = prompt(b)
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("layout", ["HND", "NHD"])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 64, 16), (7, 1, 128, 4), (4, 4, 128, 1), (30, 2, 64, 2)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ragged_fp32_arithmetic(hq, hkv, d, page, layout, dtype):
    lens, m = _ragged(RAGGED)
    b = Batch(lens, m, hq, hkv, d, page, dtype=dtype, layout=layout, seed=hq + page)
    out, lse, status = prompt(b)
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("hq,hkv,d,page,sb,layout", [(8, 2, 64, 16, 16, "HND"), (32, 8, 128, 16, 4, "NHD"), (14, 2, 128, 8, 8, "NHD"), (6, 6, 64, 128, 32, "HND"),
                                                     (4, 4, 128, 32, 1, "HND"), (5, 1, 128, 4, 2, "HND")])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ragged_8_bit(hq, hkv, d, page, sb, layout, dtype):
    lens, m = _ragged(RAGGED)
    b = Batch(lens, m, hq, hkv, d, page, dtype=dtype, kind="e4m3", sb=sb, layout=layout, seed=hq + page)
    out, lse, status = prompt(b)
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("scale_kind", ["powers", "mixed"])
@pytest.mark.parametrize("hq,hkv,d,page,sb", [(8, 2, 128, 16, 16), (7, 1, 64, 32, 1), (4, 2, 128, 128, 128)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scales_of_8_bit_pools(hq, hkv, d, page, sb, dtype, scale_kind):
    lens, m = _ragged(RAGGED)
    b = Batch(lens, m, hq, hkv, d, page, dtype=dtype, kind="e4m3", sb=sb, seed=hq + page, scale_kind=scale_kind)
    out, lse, status = prompt(b)
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("dtype,kind", [(BF16, "rows"), (F32, "rows"), (BF16, "e4m3")])
@pytest.mark.parametrize("m,hist", [(3, 9000), (40, 6000), (500, 5000), (1, 12345)])
def test_few_rows_behind_a_long_history(m, hist, dtype, kind):
    b = Batch([m + hist], [m], 8, 2, 128, 16, dtype=dtype, kind=kind, seed=m)
    out, lse, status = prompt(b)
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("kind", ["rows", "e4m3"])
def test_long_prompts(kind):
    b = Batch([3001, 2000, 700], [3001, 1500, 700], 8, 2, 128, 32, kind=kind, seed=5)
    out, lse, status = prompt(b)
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("n", [1, 17, 148, 149, 600])
def test_many_requests_of_few_rows(n):
    lens = [1 + (37 * i) % 300 for i in range(n)]
    m = [min(x, 1 + (11 * i) % 9) for i, x in enumerate(lens)]
    b = Batch(lens, m, 8, 2, 64, 16, seed=n)
    out, lse, status = prompt(b)
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("dtype,kind,page", [(BF16, "rows", 16), (F32, "rows", 16), (BF16, "e4m3", 16), (BF16, "rows", 4)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_nothing_behind_a_row_reaches_it(dtype, kind, page, bad):
    """Tokens near the end hold NaN and infinities in K and V: the rows before them are as without, those that see them are not finite."""
    if kind == "e4m3" and not math.isnan(bad):
        pytest.skip("the 8-bit format has no infinities")
    lens, m = [300, 150, 64], [300, 100, 3]
    b = Batch(lens, m, 8, 2, 128, page, dtype=dtype, kind=kind, seed=9)
    hit = [(0, 40, "v", 5), (0, 200, "v", 127), (0, 250, "k", 3), (1, 120, "v", 64), (2, 63, "k", 0), (2, 62, "v", 1)]
    ref = {r: b.exact(r) for r in range(3)}
    for r, t, which, col in hit:
        getattr(b, which)[b.table[r, t // page], :, t % page, col] = 0x7F if kind == "e4m3" else bad
    out, lse, status = prompt(b)
    assert status == 0
    for r in range(3):
        o, l, to, tl = ref[r]
        rows = slice(b.starts[r], b.starts[r + 1])
        clean = min([t for rr, t, _, _ in hit if rr == r])
        n = clean - (lens[r] - m[r])                       # rows before the first of them
        n = max(n, 0)
        assert bool(((out[rows][:n].double() - o[:n]).abs() <= to[:n]).all()) and bool(((lse[rows][:n].double() - l[:n]).abs() <= tl[:n]).all())
        # a poisoned V element reaches its column of the rows that see it, and no other before a poisoned K
        k_at = min([t for rr, t, w, _ in hit if rr == r and w == "k"], default=lens[r])
        for rr, t, which, col in hit:
            if rr == r and which == "v":
                j = t - (lens[r] - m[r])
                seen = out[rows][j:max(j, k_at - (lens[r] - m[r])), :, col].float()
                assert not bool(torch.isfinite(seen).any())
        cols = [c for rr, _, w, c in hit if rr == r and w == "v"]
        last = max(0, k_at - (lens[r] - m[r]))
        keep = [c for c in range(128) if c not in cols]
        assert bool(((out[rows][:last].double() - o[:last]).abs() <= to[:last])[..., keep].all())
        assert bool(((lse[rows][:last].double() - l[:last]).abs() <= tl[:last]).all())


def test_masked_scores_of_the_lowest_value():
    """Keys that give the lowest finite and minus infinite scores inside the visible range: those tokens weigh nothing."""
    b = Batch([200], [200], 4, 1, 64, 16, dtype=F32, seed=2)
    b.q[:] = 0
    b.q[:, :, 0] = 1.0
    b.k[b.table[0, :13].long()] = 0
    for t, x in ((0, 0.0), (7, -math.inf), (8, -3e38), (100, -math.inf)):
        b.k[b.table[0, t // 16], :, t % 16, 0] = x
    out, lse, status = prompt(b)
    n = torch.arange(1, 201, dtype=torch.float64, device="cuda")
    n -= (n > 7).double() + (n > 8).double() + (n > 100).double()
    assert status == 0 and bool(((lse.double() - torch.log(n)[:, None]).abs() < 1e-5).all()) and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
def test_large_scores_and_a_scale(dtype, d):
    """Scores of some thousands, rising and falling along the axis: the running maximum moves by more than an exponent's range."""
    b = Batch([700, 400], [700, 130], 8, 2, d, 16, dtype=dtype, seed=4, spread=30.0)
    out, lse, status = prompt(b, sm_scale=1.0)
    assert status == 0 and bool(torch.isfinite(out).all())
    b.check(out, lse, scale=1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_behind_the_last_request_and_no_lse(dtype):
    b = Batch([50, 20], [50, 7], 8, 2, 64, 16, dtype=dtype, tail_rows=9)
    args, _ = b.device()
    out = torch.full_like(args[0], 3.25)
    lse = torch.full(args[0].shape[:2], -7.0, device="cuda")
    got, l, ws = spx.prompt_attention(*args, out=out, lse=lse)
    none = spx.prompt_attention(*args, want_lse=False)
    assert int(ws.status.item()) == 0 and got is out and l is lse and none[1] is None
    b.check(out[:57], lse[:57])
    assert bool((out[57:] == 3.25).all()) and bool((lse[57:] == -7.0).all()) and torch.equal(none[0][:57], out[:57])


@pytest.mark.parametrize("dtype,kind", [(BF16, "rows"), (F32, "rows"), (BF16, "e4m3")])
def test_bad_data_voids_its_request_alone(dtype, kind):
    lens, m = [90, 300, 40, 200, 30], [90, 120, 40, 8, 30]
    b = Batch(lens, m, 8, 2, 64, 16, dtype=dtype, kind=kind, seed=1)
    b.table[1, 3] = b.num_pages
    b.table[3, 1] = -5
    (q, k, v, strides, table, n, starts, *rest), scales = b.device()
    n[2] = 39                            # fewer tokens than rows
    out, lse, ws = spx.prompt_attention(q, k, v, strides, table, n, starts, *rest, **scales)
    assert int(ws.status.item()) == (spx.DEV_BAD_PAGE | spx.DEV_BAD_LEN)
    b.check(out, lse, requests=[0, 4])
    for r in (1, 2, 3):
        rows = slice(b.starts[r], b.starts[r + 1])
        assert bool((out[rows] == 0).all()) and bool(torch.isnan(lse[rows]).all())


def test_too_many_pages_and_wrong_bounds():
    b = Batch([90, 60, 40], [9, 9, 9], 4, 2, 64, 16)
    (q, k, v, strides, table, n, starts, *rest), _ = b.device()
    n[0] = 16 * table.shape[1] + 1
    out, lse, ws = spx.prompt_attention(q, k, v, strides, table, n, starts, *rest)
    assert int(ws.status.item()) == spx.DEV_BAD_LEN and bool(torch.isnan(lse[:9]).all())
    b.check(out, lse, requests=[1, 2])
    starts[3] = 1000                      # the last request's rows end outside the tensor: it is left alone
    n[0] = 90
    ws.status.zero_()
    out.fill_(2.0)
    out, lse, ws = spx.prompt_attention(q, k, v, strides, table, n, starts, *rest, out=out, ws=ws)
    assert int(ws.status.item()) == spx.DEV_BAD_LEN and bool((out[18:] == 2.0).all())
    b.check(out, lse, requests=[0, 1])


def test_no_requests_and_no_rows():
    b = Batch([5], [5], 4, 2, 64, 16)
    (q, k, v, strides, table, n, starts, *rest), _ = b.device()
    out, lse, ws = spx.prompt_attention(q[:0], k, v, strides, table[:0], n[:0], starts[:1], *rest)
    assert out.shape[0] == 0 and int(ws.status.item()) == 0
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    out, lse, ws = spx.prompt_attention(q[:0], k, v, strides, table, n, zero, *rest)
    assert out.shape[0] == 0 and int(ws.status.item()) == 0


@pytest.mark.parametrize("m,hist", [(500, 4000), (300, 0)])
def test_the_same_bits_from_call_to_call_on_any_stream_and_replayed(m, hist):
    b = Batch([m + hist, 77], [m, 77], 8, 2, 128, 16, seed=8)
    args, _ = b.device()
    first, lse, ws = spx.prompt_attention(*args)
    torch.cuda.synchronize()
    b.check(first, lse)
    again = torch.empty_like(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _, lse2, ws2 = spx.prompt_attention(*args, out=again)
    side.synchronize()
    assert torch.equal(first, again) and torch.equal(lse, lse2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spx.prompt_attention(*args, out=again, lse=lse2, ws=ws)
    for _ in range(3):
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, again) and torch.equal(lse, lse2)
    # two calls at once, a workspace each
    outs = [torch.empty_like(first) for _ in range(2)]
    wss = [ws, ws2]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s, o, w in zip(streams, outs, wss):
            with torch.cuda.stream(s):
                spx.prompt_attention(*args, out=o, ws=w)
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)


@pytest.mark.parametrize("dtype,kind", [(BF16, "rows"), (F32, "rows"), (BF16, "e4m3")])
def test_agrees_with_verify_attention_on_a_step(dtype, kind):
    b = Batch([400, 90, 16], [5, 1, 16], 8, 2, 128, 16, dtype=dtype, kind=kind, seed=3)
    args, scales = b.device()
    out, lse, _ = spx.prompt_attention(*args, **scales)
    ref, ref_lse, _ = spx.verify_attention(*args, **scales)
    torch.cuda.synchronize()
    b.check(out, lse)
    b.check(ref, ref_lse) if dtype == F32 or kind == "rows" else None
    assert float((lse - ref_lse).abs().max()) < 2e-5
