"""How many bits the attention over 8-bit pools keeps of its weights, at the bounds that its kernels state; the same results from call
to call; and the fp32 kernels' rows of requests with a bad page id."""
import math

import numpy as np
import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx
from test_piece_arithmetic import weight_error

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _attend(c, q, lens, m, times=1, **kw):
    k, v, strides, table, ks, vs = c.on(DEV)
    got = []
    ws = None
    for _ in range(times):
        out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, _ints(lens), _ints([0, *np.cumsum(m).tolist()]), c.hkv, c.page, c.num_pages,
                                            k_scales=ks, v_scales=vs, max_q_len=max(m), ws=ws, **kw)
        got.append((out, lse))
    torch.cuda.synchronize()
    return got, int(ws.status.item())


SHAPES = [(8, 2, 128, 16, 3), (32, 8, 128, 16, 6), (8, 2, 64, 16, 4), (36, 4, 128, 32, 5), (16, 2, 64, 8, 6), (64, 4, 128, 16, 6), (128, 8, 64, 16, 5)]


@pytest.mark.parametrize("hq,hkv,d,page,m", SHAPES)
def test_weights_keep_nine_bits(hq, hkv, d, page, m):
    """bf16 queries.  A weight times its V scale is off by 2^-9 + 2^-11 at most (its pieces and their rounding to binary16), and in the mean
    square by what test_piece_arithmetic counts.  That is the numerator only: the sum below it adds the weights before their rounding.
    fp32 terms as in attention_bounds, the reference's and the score's error in numerator and sum.  Beside it the output's own rounding.
    The root mean square over all outputs tells a lost bit that the largest error does not: the weights' errors are independent, so their
    squares add up, p^2 v^2 each, with the output's own rounding; a bit less would make the weights' part four times as large, the bound
    leaves it twice."""
    lens = [300, 1000, 129]
    c = R.Cache(lens, hkv, d, page, page, seed=hq, spread=0.3)
    c.poison(lens)
    n = m * len(lens)
    q = torch.randn(n, hq, d, generator=torch.Generator().manual_seed(d)).to(BF)
    (got, *_), status = _attend(c, q, lens, [m] * 3)
    assert status == 0
    ref, ref_lse, spread, reach = R.attention(c, q, lens, [m] * 3)
    u = 2.0 ** -24
    # reach holds the queries' least step for the bound of (d + 4) 4u below; spread what lies below the weights' range for the 2^-7 that
    # attention_bounds charges: it is scaled up here to keep its value
    weight = 2 * (d + 4) * 4 * u * reach + 2.0 ** -20 + 4 * max(lens) * u
    plain, squares = np.zeros_like(ref), np.zeros_like(ref)
    q0 = 0
    g = hq // hkv
    for r, k_ in zip(range(3), [m] * 3):
        keys, values = c.values("k", r, lens[r]), c.values("v", r, lens[r])
        for j in range(k_):
            seen = lens[r] - k_ + j + 1
            s = np.einsum("hgd,thd->hgt", q[q0 + j].double().numpy().reshape(hkv, g, d), keys[:seen]) / math.sqrt(d)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            plain[q0 + j] = np.einsum("hgt,thd->hgd", p, np.abs(values[:seen])).reshape(hq, d)
            squares[q0 + j] = np.einsum("hgt,thd->hgd", p ** 2, values[:seen] ** 2).reshape(hq, d)
        q0 += k_
    below = (spread - plain) * 2.0 ** -7
    tol = torch.finfo(BF).eps / 2 * np.abs(ref) + (2.0 ** -9 + 2.0 ** -11 + 2 * weight[..., None]) * plain + below
    err = got[0].cpu().double().numpy() - ref
    assert (np.abs(err) <= tol).all(), (np.abs(err) / tol).max()
    rounding = torch.from_numpy(ref).to(BF).double().numpy() - ref
    part = weight_error()[1] ** 2 * squares.mean()
    assert (err ** 2).mean() <= (rounding ** 2).mean() + 2 * part, ((err ** 2).mean() - (rounding ** 2).mean()) / part


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("hq,hkv,d,page,m", SHAPES)
def test_the_same_bits_from_call_to_call(hq, hkv, d, page, m, dtype):
    lens = [2000, 700, 90, 1300]
    c = R.Cache(lens, hkv, d, page, page, seed=hq + 1)
    q = torch.randn(m * 4, hq, d, generator=torch.Generator().manual_seed(d)).to(dtype)
    got, status = _attend(c, q, lens, [m] * 4, times=10)
    assert status == 0
    assert all(torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1]) for out, lse in got)


@pytest.mark.parametrize("dtype,page", [(F, 16), (BF, 4), (F, 1)])
@pytest.mark.parametrize("e4m3", [True, False])
def test_a_bad_page_gives_the_requests_sentinel_rows(e4m3, dtype, page):
    """The kernels in fp32 arithmetic: a page id out of range anywhere in a request, which may be cut into several chunks or be one."""
    lens, m = [4000, 200, 90, 3], [3, 2, 4, 3]
    c = R.Cache(lens, 2, 64, page, page, seed=5)
    q = torch.randn(sum(m), 8, 64, generator=torch.Generator().manual_seed(2)).to(dtype)
    starts = [0, *np.cumsum(m).tolist()]
    k, v, strides, table, ks, vs = c.on(DEV)
    kw = dict(k_scales=ks, v_scales=vs)
    if not e4m3:
        k, v = ((x.float() * s.repeat_interleave(page, 2)[..., None]).to(dtype) for x, s in ((k, ks), (v, vs)))
        kw = {}
    args = (_ints(lens), _ints(starts), 2, page, c.num_pages)
    clean, clean_lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, *args, max_q_len=4, **kw)
    assert int(ws.status.item()) == 0
    for r, at, bad in ((0, 3, -1), (0, 3999 // page, c.num_pages), (1, 199 // page, -5), (2, 0, 1 << 30), (3, 2 // page, -1)):
        broken = table.clone()
        broken[r, at] = bad
        out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, broken, *args, max_q_len=4, **kw)
        torch.cuda.synchronize()
        assert int(ws.status.item()) == spx.DEV_BAD_PAGE
        rows = torch.zeros(sum(m), dtype=torch.bool, device=DEV)
        rows[starts[r]:starts[r + 1]] = True
        assert (out[rows] == 0).all() and torch.isnan(lse[rows]).all()
        assert torch.equal(out[~rows], clean[~rows]) and torch.equal(lse[~rows], clean_lse[~rows])
