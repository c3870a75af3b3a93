"""Verify attention over a paged cache of 8-bit floats and the append that fills it, against plain 64-bit
references; the cache's codes and scales bit for bit."""
import math

import numpy as np
import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding
from parity_util import Guarded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


def _starts(m):
    return torch.tensor([0, *np.cumsum(m).tolist()], dtype=torch.int32, device=DEV)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _attend(c, q, lens, m, **kw):
    k, v, strides, table, ks, vs = c.on(DEV)
    kw.setdefault("max_q_len", max(m, default=0))
    out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, _ints(lens), _starts(m), c.hkv, c.page, c.num_pages,
                                        k_scales=ks, v_scales=vs, **kw)
    torch.cuda.synchronize()
    return out, lse, int(ws.status.item())


def _check(c, q, lens, m, out, lse, sm_scale=0.0):
    ref, ref_lse, spread, reach = R.attention(c, q, lens, m, sm_scale)
    tol, tol_lse = R.attention_bounds(ref, spread, reach, max(lens), q.shape[2], q.dtype)
    err = np.abs(out.cpu().double().numpy() - ref)
    assert (err <= tol).all(), (err - tol).max()
    err = np.abs(lse.cpu().double().numpy() - ref_lse)
    assert (err <= tol_lse).all(), (err - tol_lse).max()


CASES = [
    # hq, hkv, d, page, sb, layout, lens, m
    (8, 2, 64, 16, 16, "HND", [40, 1, 128, 129, 5], [5, 1, 5, 2, 5]),
    (8, 2, 64, 16, 4, "NHD", [127, 255, 256, 257], [1, 3, 5, 4]),
    (32, 8, 128, 16, 16, "HND", [300, 17, 512, 64], [6, 6, 6, 6]),
    (32, 8, 128, 32, 32, "NHD", [700, 33], [9, 9]),
    (64, 8, 128, 16, 8, "NHD", [129, 1000, 4], [4, 4, 4]),
    (32, 8, 128, 128, 128, "HND", [500, 128, 129], [1, 2, 16]),
    (28, 4, 128, 64, 16, "HND", [333, 90], [5, 2]),
    (8, 1, 128, 8, 1, "HND", [200, 31], [16, 3]),
    (16, 16, 64, 8, 8, "NHD", [150, 77], [1, 16]),
    (12, 4, 128, 4, 2, "HND", [100, 9], [4, 1]),
    (4, 4, 64, 1, 1, "NHD", [30, 7], [2, 7]),
    (16, 2, 64, 2, 2, "HND", [66], [3]),
    (8, 8, 128, 16, 16, "HND", [3000], [1]),
    (128, 1, 128, 32, 16, "HND", [400], [1]),
    (8, 1, 64, 64, 64, "NHD", [900, 130], [16, 9]),
]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("case", CASES)
def test_attention_matches_the_reference(case, dtype):
    hq, hkv, d, page, sb, layout, lens, m = case
    c = R.Cache(lens, hkv, d, page, sb, layout, seed=sum(lens))
    c.poison(lens)
    q = torch.randn(sum(m), hq, d, generator=torch.Generator().manual_seed(3)).to(dtype)
    out, lse, status = _attend(c, q, lens, m)
    assert status == 0
    _check(c, q, lens, m, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
def test_many_ragged_requests(dtype):
    g = np.random.RandomState(11)
    m = g.choice([1, 3, 5, 7], 70).tolist()
    lens = [max(int(n), k) for n, k in zip(np.exp(g.uniform(0, 6.2, 70)), m)]
    c = R.Cache(lens, 2, 64, 16, 8, seed=5)
    c.poison(lens)
    q = torch.randn(sum(m), 8, 64, generator=torch.Generator().manual_seed(4)).to(dtype)
    out, lse, status = _attend(c, q, lens, m, max_q_len=0)
    assert status == 0
    _check(c, q, lens, m, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("size", [1e-25, 1.0, 1e25])
def test_query_magnitudes_and_outlier_columns(dtype, size):
    """Rows of any magnitude, one column far above the others, rows of zeros; a scale that undoes the magnitude."""
    lens, m = [150, 40], [4, 4]
    c = R.Cache(lens, 2, 128, 16, 16, seed=6)
    q = torch.randn(8, 8, 128, generator=torch.Generator().manual_seed(5)) * size
    q[:, :, 7] *= 30
    q[2, 3] = 0
    q[1, 1, 5:] *= 2.0 ** -12
    q = q.to(dtype)
    sm = 0.09 / size
    out, lse, status = _attend(c, q, lens, m, sm_scale=sm)
    assert status == 0
    _check(c, q, lens, m, out, lse, sm_scale=float(np.float32(sm)))


@pytest.mark.parametrize("dtype", [BF, F])
def test_peaked_and_flat_rows(dtype):
    """Scores far apart (one token takes all, at either end of a long row) and all equal."""
    lens, m = [2000, 2000, 900], [2, 2, 2]
    c = R.Cache(lens, 2, 64, 16, 16, seed=7, spread=0.2)
    q = torch.randn(6, 8, 64, generator=torch.Generator().manual_seed(8))
    q[:4] *= 12
    q[4:] = 0
    q = q.to(dtype)
    out, lse, status = _attend(c, q, lens, m)
    assert status == 0
    _check(c, q, lens, m, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("hq,hkv,d,m", [(8, 2, 64, 3), (32, 8, 128, 6), (36, 1, 128, 1), (64, 8, 128, 9), (8, 1, 64, 16)])
def test_scores_that_grow_from_tile_to_tile(hq, hkv, d, m, dtype):
    """Maxima that rise by a few, by a hundred and by a million times, at any place of the sequence: the first token of a later tile,
    the last token, one tile after another, for some rows only, beside V scales that rise with them."""
    lens = [700, 1290, 520, 128, 385]
    c = R.Cache(lens, hkv, d, 16, 16, seed=31, spread=0.1)
    q = torch.randn(m * len(lens), hq, d, generator=torch.Generator().manual_seed(9)) * 0.1
    def lift(r, t, size, lanes=slice(None)):
        # key t of request r along the mean of some of its queries: a score near `size`
        page, slot = int(c.table[r, t // 16]), t % 16
        for h in range(hkv):
            rows = q[m * r:m * r + m, h * (hq // hkv):(h + 1) * (hq // hkv)].reshape(-1, d)[lanes]
            mean = rows.mean(0)
            k = mean / mean.norm() ** 2 * size * math.sqrt(d)
            s = float(k.abs().max()) / 400
            block = torch.from_numpy(R.decode(c.k[page, h])) * float(c.k_scales[page, h, 0])
            s = max(s, float(block.abs().max()) / 440)
            block[slot] = k.double()
            c.k[page, h] = torch.from_numpy(R.encode((block / s).numpy()))
            c.k_scales[page, h, 0] = s
    for i, t in enumerate((130, 270, 390, 513, 699)):
        lift(0, t, 6.0 * (i + 1))
    for t, size in ((200, 3.0), (1024, 20.0), (1289, 45.0)):
        lift(1, t, size)
    lift(2, 260, 15.0, slice(0, 2))
    lift(2, 511, 30.0, slice(2, None))
    lift(4, 384, 25.0)
    c.v_scales[c.table[1, 70:].clamp(min=0).long()] *= 2.0 ** 9
    q = q.to(dtype)
    out, lse, status = _attend(c, q, lens, [m] * len(lens))
    assert status == 0
    _check(c, q, lens, [m] * len(lens), out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
def test_value_scales_of_very_different_size(dtype):
    lens, m = [260, 513], [3, 2]
    c = R.Cache(lens, 2, 128, 16, 16, seed=9, spread=0.3)
    c.v_scales *= 2.0 ** torch.randint(-30, 30, c.v_scales.shape, generator=torch.Generator().manual_seed(1))
    c.v_scales[:, 1] = 0
    q = torch.randn(5, 8, 128, generator=torch.Generator().manual_seed(10)).to(dtype)
    out, lse, status = _attend(c, q, lens, m)
    assert status == 0
    _check(c, q, lens, m, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("length", [200, 131, 128])
def test_nan_in_a_position_reaches_only_the_queries_that_see_it(dtype, length):
    """A NaN in one column of V at new position 2 of 5: queries 0 and 1 do not see it; a NaN in K likewise."""
    lens, m = [length, 64], [5, 5]
    c = R.Cache(lens, 2, 64, 16, 16, seed=12)
    q = torch.randn(10, 8, 64, generator=torch.Generator().manual_seed(2)).to(dtype)
    clean, clean_lse, _ = _attend(c, q, lens, m)
    t = length - 3
    page, slot = int(c.table[0, t // 16]), t % 16
    c.v[page, 1, slot, 9] = 0xFF
    out, lse, status = _attend(c, q, lens, m)
    assert status == 0
    want = clean.clone()
    want[2:5, 4:, 9] = math.nan
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(out[~torch.isnan(want)], want[~torch.isnan(want)]) and torch.equal(lse, clean_lse)
    c.k[page, 0, slot, 3] = 0x7F
    out, lse, status = _attend(c, q, lens, m)
    want[2:5, :4] = math.nan
    assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.isnan(lse[2:5, :4]).all()
    assert torch.equal(out[~torch.isnan(want)], want[~torch.isnan(want)])


def test_queries_that_are_not_finite_stay_in_their_row():
    lens, m = [140, 30], [4, 4]
    c = R.Cache(lens, 2, 128, 16, 16, seed=13)
    q = torch.randn(8, 8, 128, generator=torch.Generator().manual_seed(2)).to(BF)
    clean, clean_lse, _ = _attend(c, q, lens, m)
    q[1, 2, 100], q[6, 5, 0] = math.inf, math.nan
    out, lse, status = _attend(c, q, lens, m)
    assert status == 0
    hit = torch.zeros(8, 8, dtype=torch.bool, device=DEV)
    hit[1, 2] = hit[6, 5] = True
    assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])


def test_bad_pages_and_lengths_give_sentinels_and_leave_the_others():
    lens, m = [300, 200, 100, 50], [4, 4, 4, 4]
    c = R.Cache(lens, 8, 128, 16, 16, seed=14)
    q = torch.randn(16, 32, 128, generator=torch.Generator().manual_seed(2)).to(BF)
    clean, clean_lse, _ = _attend(c, q, lens, m)
    c.table[1, 3] = c.num_pages
    out, lse, status = _attend(c, q, [300, 200, 2, 50], m)
    assert status == (spx.DEV_BAD_PAGE | spx.DEV_BAD_LEN)
    for a, b in ((4, 8), (8, 12)):
        assert (out[a:b] == 0).all() and torch.isnan(lse[a:b]).all()
    for a, b in ((0, 4), (12, 16)):
        assert torch.equal(out[a:b], clean[a:b]) and torch.equal(lse[a:b], clean_lse[a:b])


def test_attention_without_lse_and_with_empty_batches():
    c = R.Cache([20], 2, 64, 16, 16)
    q = torch.randn(2, 8, 64).to(BF)
    out, lse, status = _attend(c, q, [20], [2], want_lse=False)
    assert lse is None and status == 0
    ref, *_ = R.attention(c, q, [20], [2])
    assert np.abs(out.cpu().double().numpy() - ref).max() < 0.05
    k, v, strides, table, ks, vs = c.on(DEV)
    none, _, _ = spx.verify_attention(q[:0].to(DEV), k, v, strides, table[:0], _ints([]), _ints([0]), 2, 16, c.num_pages, k_scales=ks, v_scales=vs)
    assert none.shape[0] == 0


# ------------------------------------------------------------------------------------------------
# append
# ------------------------------------------------------------------------------------------------
def _append(c, nk, nv, lens, m, q=None, q_out=None, base=0.0, state=None):
    k, v, strides, table, ks, vs = state or c.on(DEV)
    status = spx.kv_append(nk.to(DEV), nv.to(DEV), k, v, strides, table, _ints(lens), _starts(m), c.page, c.num_pages, rope_base=base,
                           q_rows=q, q_out=q_out, k_scales=ks, v_scales=vs)
    torch.cuda.synchronize()
    return k, v, ks, vs, int(status.item())


def _same(c, k, v, ks, vs):
    for got, want in ((k, c.k), (v, c.v)):
        assert torch.equal(got.view(torch.uint8).cpu(), want)
    assert torch.equal(ks.cpu(), c.k_scales) and torch.equal(vs.cpu(), c.v_scales)


def _rows(total, hkv, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(total, hkv, d, generator=g) * s).to(dtype) for s in (1.0, 3.0)]


APPENDS = [
    # hkv, d, page, sb, layout, lens, m
    (2, 64, 16, 16, "HND", [40, 1, 16, 17, 300], [5, 1, 16, 1, 7]),
    (8, 128, 16, 16, "NHD", [6, 100, 37], [6, 6, 6]),
    (2, 128, 16, 4, "HND", [33, 5], [3, 5]),
    (2, 128, 8, 1, "NHD", [9, 20], [2, 1]),
    (4, 64, 128, 128, "HND", [500, 127, 129, 128], [200, 127, 2, 1]),
    (2, 128, 128, 128, "NHD", [300, 129], [299, 1]),
    (1, 128, 64, 64, "HND", [70, 64, 1000], [1, 64, 936]),
    (2, 64, 32, 2, "HND", [65], [64]),
    (3, 128, 1, 1, "HND", [5], [5]),
    (2, 128, 32, 32, "HND", [31, 32, 33, 700], [31, 1, 2, 600]),
    (2, 64, 4, 4, "NHD", [13, 4], [6, 4]),
    (1, 64, 64, 32, "HND", [97], [40]),
]


@pytest.mark.parametrize("base", [0.0, 10000.0])
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("case", APPENDS)
def test_append_is_bit_exact(case, dtype, base):
    hkv, d, page, sb, layout, lens, m = case
    c = R.Cache(lens, hkv, d, page, sb, layout, seed=1)
    c.k_scales, c.v_scales = [torch.exp2(torch.log2(s).round()) for s in (c.k_scales, c.v_scales)]
    nk, nv = _rows(sum(m), hkv, d, dtype, 2)
    state = c.on(DEV)
    *got, status = _append(c, nk, nv, lens, m, base=base, state=state)
    assert status == 0
    R.append(c, nk, nv, lens, m, base)
    _same(c, *got)
    # the same rows again: nothing changes
    *got, status = _append(c, nk, nv, lens, m, base=base, state=state)
    _same(c, *got)


def test_append_under_scales_that_are_no_powers_of_two():
    """Older tokens under another quantiser's scales: values to 32 bits, then rounded anew."""
    lens, m = [40, 21], [3, 2]
    c = R.Cache(lens, 2, 64, 16, 16, seed=3)
    c.k_scales, c.v_scales = [(s * 0 + 0.25).float() for s in (c.k_scales, c.v_scales)]
    c.v_scales[:] = 0.375          # 1.5 * 2^-2: code * scale is exact in 32 bits
    nk, nv = _rows(5, 2, 64, BF, 4)
    *got, status = _append(c, nk, nv, lens, m)
    assert status == 0
    R.append(c, nk, nv, lens, m)
    _same(c, *got)


@pytest.mark.parametrize("dtype", [BF, F])
def test_append_of_extreme_values(dtype):
    """Zeros, subnormals, the largest finite values, infinities and NaN; a later row that makes the scale grow by far."""
    lens, m = [20, 20, 20, 20, 20], [4, 4, 4, 4, 4]
    c = R.Cache(lens, 1, 64, 16, 16, seed=3)
    c.k_scales[:], c.v_scales[:] = 2.0 ** -9, 2.0 ** -9
    nk, nv = _rows(20, 1, 64, F, 4)
    nk[0:4], nv[0:4] = 0.0, -0.0
    nk[4:8] *= 1e-39
    nv[4:8] *= 1e-37
    nk[8:12], nv[8:12] = 3.38e38, -1e30
    nk[13, 0, 3], nk[13, 0, 40], nv[14, 0, 5] = math.inf, math.nan, -math.inf
    nk[16:20] *= 1e5
    nk, nv = nk.to(dtype), nv.to(dtype)
    *got, status = _append(c, nk, nv, lens, m)
    assert status == 0
    R.append(c, nk, nv, lens, m)
    # the sign of a stored NaN is not told
    for a, b in ((got[0], c.k), (got[1], c.v)):
        a = a.view(torch.uint8).cpu()
        assert torch.equal(torch.where((a & 0x7F) == 0x7F, 0x7F, a), torch.where((b & 0x7F) == 0x7F, 0x7F, b))
    assert torch.equal(got[2].cpu(), c.k_scales) and torch.equal(got[3].cpu(), c.v_scales)


def test_rejected_tokens_leave_the_scale_they_found():
    """Large rows appended, rejected and overwritten by small ones: the scales are what they would be without them, and so
    are the codes but for what the larger scale pushed out.  Under a scale s a multiple of s / 2^9 below s / 2^6 is what
    is left of a smaller value (off by s / 2^10 at most), larger ones keep their three bits."""
    c, plain = (R.Cache([30], 2, 128, 16, 16, seed=8) for _ in range(2))
    for x in (c, plain):
        x.k_scales[:], x.v_scales[:] = 2.0 ** -7, 2.0 ** -7
    state = c.on(DEV)
    big, small = _rows(6, 2, 128, BF, 1), _rows(3, 2, 128, BF, 2)
    _append(c, big[0] * 8, big[1] * 8, [28], [6], state=state)     # 22 tokens + 6
    page, n = int(plain.table[0, 1]), 26 - 16
    largest = state[4][page].amax().item()
    *got, status = _append(c, small[0], small[1], [26], [3], state=state)   # 23 kept
    assert status == 0
    R.append(plain, big[0][:1] * 8, big[1][:1] * 8, [23], [1])
    R.append(plain, small[0], small[1], [26], [3])
    assert torch.equal(got[2].cpu(), plain.k_scales) and torch.equal(got[3].cpu(), plain.v_scales)
    scale = plain.k_scales[page].double().numpy()[:, :, None]
    a, b = (R.decode(x.view(torch.uint8).cpu()[page, :, :n]) * scale for x in (got[0], plain.k))
    assert (np.abs(a - b) <= largest / 2 ** 10 + (np.abs(b) < largest / 2 ** 6) * largest / 2 ** 10).all()
    assert (a == b)[np.abs(b) >= largest / 2 ** 6].all() and largest > scale.max()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("hq,hkv,d,page,sb", [(8, 2, 64, 16, 16), (32, 8, 128, 16, 16), (5, 1, 128, 128, 128), (12, 4, 64, 64, 64)])
def test_queries_are_rotated(hq, hkv, d, page, sb, dtype):
    lens, m = [3, 1000, 40], [3, 150, 1]
    c = R.Cache(lens, hkv, d, page, sb, seed=1)
    nk, nv = _rows(sum(m), hkv, d, dtype, 2)
    q = torch.randn(sum(m), hq, d, generator=torch.Generator().manual_seed(1)).to(dtype)
    want = np.concatenate([R.rotate(q[i:i + 1].double().numpy()[0], n - k + j, 500000.0)[None]
                           for i, (n, k, j) in enumerate((n, k, j) for n, k in zip(lens, m) for j in range(k))])
    held, out = q.to(DEV), Guarded(tuple(q.shape), dtype, DEV, "q_out")
    *_, status = _append(c, nk, nv, lens, m, q=held, q_out=out.view, base=500000.0)
    out.check()
    assert status == 0 and torch.equal(held.cpu(), q)
    # float64 -> binary32 -> the type: at most half a step of each
    tol = (torch.finfo(dtype).eps / 2 + 2.0 ** -24) * np.abs(want) + 1e-30 + 1e-13
    assert (np.abs(out.view.cpu().double().numpy() - want) <= tol).all()
    *_, status = _append(c, nk, nv, lens, m, q=held, base=500000.0)
    assert torch.equal(held, out.view)


def test_sixteen_bit_pools_take_q_out_too():
    lens, m = [40, 7], [4, 4]
    c = R.Cache(lens, 2, 64, 16, 16)
    _, _, strides, table, _, _ = c.on(DEV)
    pool = torch.zeros(c.num_pages, 2, 16, 64, dtype=BF, device=DEV)
    pool2 = torch.zeros_like(pool)
    nk, nv = (x.to(DEV) for x in _rows(8, 2, 64, BF, 3))
    q = torch.randn(8, 8, 64, device=DEV).to(BF)
    kept, out = q.clone(), torch.empty_like(q)
    spx.kv_append(nk, nv, pool, pool2, strides, table, _ints(lens), _starts(m), 16, c.num_pages, rope_base=10000.0, q_rows=q, q_out=out)
    assert torch.equal(q, kept)
    spx.kv_append(nk, nv, pool, pool2, strides, table, _ints(lens), _starts(m), 16, c.num_pages, rope_base=10000.0, q_rows=q)
    torch.cuda.synchronize()
    assert torch.equal(q, out) and not torch.equal(q, kept)


def test_append_skips_bad_requests_whole():
    lens, m = [300, 50, 2, 40], [290, 3, 4, 2]
    c = R.Cache(lens, 2, 64, 16, 16, seed=4)
    c.k_scales[:], c.v_scales[:] = 0.25, 0.25
    c.table[0, 18] = -1                    # the last of request 0's pages; its first ones are fine
    nk, nv = _rows(sum(m), 2, 64, BF, 5)
    *got, status = _append(c, nk, nv, lens, m)
    assert status == (spx.DEV_BAD_PAGE | spx.DEV_BAD_LEN)
    R.append(c, nk, nv, lens, m, skip=(0, 2))
    _same(c, *got)


def test_append_many_requests():
    g = np.random.RandomState(3)
    m = g.randint(1, 12, 700).tolist()
    lens = [k + int(g.randint(0, 40)) for k in m]
    c = R.Cache(lens, 1, 64, 16, 8, seed=6)
    c.k_scales[:], c.v_scales[:] = 0.5, 0.5
    nk, nv = _rows(sum(m), 1, 64, BF, 7)
    *got, status = _append(c, nk, nv, lens, m, base=10000.0)
    assert status == 0
    R.append(c, nk, nv, lens, m, 10000.0)
    _same(c, *got)


# ------------------------------------------------------------------------------------------------
# together
# ------------------------------------------------------------------------------------------------
def test_prompt_then_steps_then_rollback():
    """A prompt enters the cache, then two verify steps with a rollback between them: append, attend, LM head, sample, log-probabilities."""
    hq, hkv, d, page, vocab, B = 8, 2, 128, 16, 1000, 3
    prompt, k = [60, 33, 128], 3
    c = R.Cache([n + 3 * k for n in prompt], hkv, d, page, 16, seed=20)
    k_cache, v_cache, strides, table, ks, vs = c.on(DEV)
    state = (k_cache, v_cache, strides, table, ks, vs)
    g = torch.Generator().manual_seed(7)
    weight = (torch.randn(vocab, hq * d, generator=g) * 0.05).to(BF).to(DEV)
    nk, nv = _rows(sum(prompt), hkv, d, BF, 30)
    _append(c, nk, nv, prompt, prompt, base=10000.0, state=state)
    R.append(c, nk, nv, prompt, prompt, 10000.0)
    lens, ws, ws2 = [n + k + 1 for n in prompt], None, None
    for step in range(2):
        m = [k + 1] * B
        nk, nv = _rows(sum(m), hkv, d, BF, 40 + step)
        q = torch.randn(sum(m), hq, d, generator=g).to(BF).to(DEV)
        *got, status = _append(c, nk, nv, lens, m, q=q, base=10000.0, state=state)
        assert status == 0
        R.append(c, nk, nv, lens, m, 10000.0)
        _same(c, *got)
        out, lse, ws = spx.verify_attention(q, k_cache, v_cache, strides, table, _ints(lens), _starts(m), hkv, page, c.num_pages,
                                            max_q_len=k + 1, ws=ws, k_scales=ks, v_scales=vs)
        _check(c, q.cpu(), lens, m, out, lse)
        logits, stats, _ = spx.lm_head(out.view(sum(m), -1), weight)
        draft = logits.view(B, k + 1, -1)[:, :k].reshape(B * k, -1).contiguous()
        ids = draft[:, :vocab].float().argmax(1).int()
        acc, tok, _, ws2 = spx.rejection_sample(logits, draft, ids, _starts(m), torch.rand(B * k, generator=g).to(DEV),
                                                torch.rand(B, generator=g).to(DEV), vocab=vocab, target_tile_stats=stats, ws=ws2)
        lp, ent, top, top_lp, _ = spx.token_logprobs(logits, tok, top_n=4, vocab=vocab)
        torch.cuda.synchronize()
        assert int(ws.status.item()) == 0 and int(ws2.status.item()) == 0
        for i, t in enumerate(tok.tolist()):
            if t < 0:
                assert math.isnan(lp[i]) and top[i].tolist() == [-1] * 4
                continue
            want = R.logprobs(logits[i, :vocab].float().cpu().numpy(), t, 4)
            assert abs(lp[i].item() - want[0]) < 1e-5 and top[i].tolist() == want[2]
        new, _ = spx.kv_rollback(_ints(lens), _starts(m), acc)
        lens = [n + k + 1 for n in new.tolist()]
        assert max(lens) <= max(prompt) + 3 * k + k


def test_verify_step_and_captured_graph():
    """The whole step over an 8-bit cache, eager and as a replayed graph on another stream, gives the halves' results."""
    import spx_workloads as W
    spec = W.scaled(W.CONFIGS[1], batch=6, ctx_div=8, vocab=4000)
    b = W.generate(spec).to(DEV)
    lens, m = b.seq_lens_host, [k + 1 for k in b.k_host]
    c = R.Cache(lens, spec.num_kv_heads, spec.head_dim, 16, 16, seed=2)
    k, v, strides, table, ks, vs = c.on(DEV)
    out = torch.empty_like(b.q)
    lse = torch.empty(b.q.shape[:2], dtype=F, device=DEV)
    acc, tok = torch.empty(6, dtype=torch.int32, device=DEV), torch.empty(b.total_q, dtype=torch.int32, device=DEV)
    a = binding.make_attn_args(b.q, k, v, strides, table, b.seq_lens, b.q_indptr, spec.num_kv_heads, 16, c.num_pages, out, lse,
                               max_q_len=max(m), k_scales=ks, v_scales=vs)
    s = binding.make_sample_args(b.target_logits, b.draft_logits, b.draft_ids, b.q_indptr, b.u_accept, b.u_sample, acc, tok)
    ws = spx.Workspace.allocate(spx.workspace_size(a, s), DEV)
    spx.verify_step(a, s, ws, DEV)
    torch.cuda.synchronize()
    _check(c, b.q.cpu(), lens, m, out, lse)
    ref_acc, ref_tok, _, _ = spx.rejection_sample(b.target_logits, b.draft_logits, b.draft_ids, b.q_indptr, b.u_accept, b.u_sample)
    assert torch.equal(acc, ref_acc) and torch.equal(tok, ref_tok)
    want, want_lse = out.clone(), lse.clone()
    nk, nv = (x.to(DEV) for x in _rows(b.total_q, spec.num_kv_heads, spec.head_dim, BF, 3))
    q_in = b.q.clone()
    lp = torch.empty(b.total_q, dtype=F, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    lws = spx.token_logprobs(b.target_logits, tok, top_n=3, logprobs=lp)[4]
    torch.cuda.synchronize()
    want_lp = lp.clone()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        spx.kv_append(nk, nv, k, v, strides, table, b.seq_lens, b.q_indptr, 16, c.num_pages, status=status, rope_base=10000.0,
                      q_rows=q_in, q_out=b.q, k_scales=ks, v_scales=vs)
        spx.verify_step(a, s, ws, DEV)
        spx.token_logprobs(b.target_logits, tok, top_n=3, logprobs=lp, ws=lws)
    graph.replay()
    torch.cuda.synchronize()
    R.append(c, nk.cpu(), nv.cpu(), lens, m, 10000.0)
    _same(c, k, v, ks, vs)
    _check(c, b.q.cpu(), lens, m, out, lse)
    first, first_lse = out.clone(), lse.clone()
    for t in (out, lse, acc, tok, lp):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first) and torch.equal(lse, first_lse) and torch.equal(tok, ref_tok) and torch.equal(acc, ref_acc)
    assert not torch.equal(first, want)
    assert torch.equal(torch.isnan(lp), torch.isnan(want_lp)) and torch.equal(lp[~torch.isnan(lp)], want_lp[~torch.isnan(lp)])


def test_host_step_copies_the_scales():
    import spx_workloads as W
    spec = W.scaled(W.CONFIGS[0], batch=3, vocab=512)
    b = W.generate(spec)
    lens, m = b.seq_lens_host, [k + 1 for k in b.k_host]
    c = R.Cache(lens, spec.num_kv_heads, spec.head_dim, spec.page_size, 4, seed=2)
    s0 = c.k.stride()
    pin = lambda t: t.contiguous().pin_memory()  # noqa: E731
    q, k, v, table, ks, vs = (pin(t) for t in (b.q, c.k, c.v, c.table, c.k_scales, c.v_scales))
    out, lse = pin(torch.zeros_like(q)), pin(torch.zeros(q.shape[:2]))
    acc, tok = pin(torch.zeros(3, dtype=torch.int32)), pin(torch.zeros(b.total_q, dtype=torch.int32))
    a = binding.make_attn_args(q, k, v, (s0[0], s0[1], s0[2]), table, pin(b.seq_lens), pin(b.q_indptr), spec.num_kv_heads, spec.page_size,
                               c.num_pages, out, lse, k_scales=ks, v_scales=vs)
    keep = [pin(t) for t in (b.target_logits, b.draft_logits, b.draft_ids, b.q_indptr, b.u_accept, b.u_sample, b.seq_lens)]
    a.seq_lens, a.q_indptr = keep[6].data_ptr(), keep[3].data_ptr()
    s = binding.make_sample_args(*keep[:6], acc, tok)
    arena = torch.empty(spx.host_step_arena_size(a, s, k.numel()), dtype=torch.uint8, device=DEV)
    status = pin(torch.zeros(1, dtype=torch.int32))
    spx.verify_step_host(a, s, k.numel(), arena, status, torch.device(DEV))
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    _check(c, b.q, lens, m, out, lse)


def test_cache_offsets_past_32_bits():
    """A page whose byte offset passes 2^31 in both the pool and (through the stride) the tensor map."""
    page, hkv, d = 16, 2, 64
    stride_page = 1 << 24
    pages = 160
    need = (pages - 1) * stride_page + hkv * page * d
    k = torch.zeros(need, dtype=torch.uint8, device=DEV)
    v = torch.zeros(need, dtype=torch.uint8, device=DEV)
    strides = (stride_page, page * d, d)
    small = R.Cache([40], hkv, d, page, 16, seed=1)
    table = torch.tensor([[158, 3, 157]], dtype=torch.int32, device=DEV)
    ks = torch.full((pages, hkv, 1), 0.25, device=DEV)
    vs = torch.full((pages, hkv, 1), 0.25, device=DEV)
    for i, p in enumerate(table[0].tolist()):
        n = int(small.table[0, i])
        for pool, codes in ((k, small.k), (v, small.v)):
            pool[p * stride_page:p * stride_page + hkv * page * d] = codes[n].reshape(-1).to(DEV)
    small.k_scales[:], small.v_scales[:] = 0.25, 0.25
    nk, nv = _rows(4, hkv, d, BF, 3)
    status = spx.kv_append(nk.to(DEV), nv.to(DEV), k, v, strides, table, _ints([40]), _starts([4]), page, pages, k_scales=ks, v_scales=vs)
    R.append(small, nk, nv, [40], [4])
    for dtype in (BF, F):
        q = torch.randn(4, 8, d, generator=torch.Generator().manual_seed(3)).to(dtype)
        out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, _ints([40]), _starts([4]), hkv, page, pages, k_scales=ks, v_scales=vs)
        torch.cuda.synchronize()
        assert int(ws.status.item()) == 0 and int(status.item()) == 0
        _check(small, q, [40], [4], out, lse)
