"""The append on positions of several axes, and prompts entering 16- and 32-bit pools, against 64-bit references."""
import numpy as np
import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx
from prompt_util import DEV, Batch, prompt, turned

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
HALF_STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def _positions(axes, rows, seed, top=4000):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, top, (axes, rows), generator=g, dtype=torch.int32)


def _append(b, new_k, new_v, q, positions, sections, interleaved, base, q_out=None, rows=None):
    (_, k, v, strides, table, n, starts, _, page, pages), scales = b.device()
    status = spx.kv_append(new_k.to(DEV), new_v.to(DEV), k, v, strides, table, n, starts, page, pages, rope_base=base, q_rows=q, q_out=q_out,
                           positions=None if positions is None else positions.to(DEV), rope_sections=sections, rope_interleaved=interleaved, **scales)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return k, v, scales


def _check_rows(got, want, dtype):
    """One rounding to fp32, one to the type, and an angle off by 2^-53 of itself (positions below 2^13: 2^-39 of the row)."""
    size = np.abs(want) + 1e-30
    pair = np.sqrt((want ** 2).reshape(*want.shape[:-1], 2, -1).sum(-2))
    tol = (HALF_STEP[dtype] + (2.0 ** -24 if dtype == BF16 else 0)) * size + 2.0 ** -38 * np.concatenate((pair, pair), -1)
    bad = ~(np.abs(got.double().cpu().numpy() - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist())


@pytest.mark.parametrize("layout", ["HND", "NHD"])
@pytest.mark.parametrize("d,sections,interleaved", [(128, [16, 24, 24], False), (128, [24, 20, 20], True), (64, [8, 12, 12], False), (64, [32], False), (64, [0, 32], False),
                                                    (128, [60, 1, 1, 2], True), (64, [31, 1], True)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_the_pools_type(d, sections, interleaved, dtype, layout):
    lens, m = [700, 40, 16, 90, 1], [700, 33, 1, 17, 1]
    b = Batch(lens, m, 6, 2, d, 16, dtype=dtype, layout=layout, seed=d, poison=1.5)
    g = torch.Generator().manual_seed(1)
    rows = b.starts[-1]
    new_k, new_v = (torch.randn(rows, 2, d, generator=g).to(dtype) for _ in range(2))
    pos = _positions(len(sections), rows, 3)
    q = b.q.to(DEV)
    before = [b.k.clone(), b.v.clone()]
    k, v, _ = _append(b, new_k, new_v, q, pos, sections, interleaved, 10000.0)
    want_q = turned(b.q.double().numpy(), pos.numpy().astype(np.float64), 10000.0, sections, interleaved)
    want_k = turned(new_k.double().numpy(), pos.numpy().astype(np.float64), 10000.0, sections, interleaved)
    _check_rows(q, want_q, dtype)
    k, v = k.cpu(), v.cpu()
    for r in range(len(lens)):
        t = torch.arange(lens[r] - m[r], lens[r])
        pages = b.table[r].long()[t // 16]
        rows = slice(b.starts[r], b.starts[r + 1])
        _check_rows(k.transpose(1, 2)[pages, t % 16], want_k[rows], dtype)
        assert torch.equal(v.transpose(1, 2)[pages, t % 16], new_v[rows])
        before[0].transpose(1, 2)[pages, t % 16] = k.transpose(1, 2)[pages, t % 16]
        before[1].transpose(1, 2)[pages, t % 16] = new_v[rows]
    assert torch.equal(before[0], k) and torch.equal(before[1], v)      # and no other slot


@pytest.mark.parametrize("sections,interleaved", [([16, 24, 24], False), ([24, 20, 20], True)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_8_bit_pools(sections, interleaved, dtype):
    """The stored values are those of the 64-bit rotation, quantised: half a step of the format under the block's scale."""
    lens, m = [300, 37, 16], [300, 30, 1]
    b = Batch(lens, m, 4, 2, 128, 16, dtype=dtype, kind="e4m3", sb=8, seed=5)
    g = torch.Generator().manual_seed(2)
    rows = b.starts[-1]
    new_k, new_v = (torch.randn(rows, 2, 128, generator=g).to(dtype) for _ in range(2))
    pos = _positions(3, rows, 4)
    q, out = b.q.to(DEV), torch.empty_like(b.q, device=DEV)
    k, v, scales = _append(b, new_k, new_v, q, pos, sections, interleaved, 500000.0, q_out=out)
    assert torch.equal(q.cpu(), b.q)
    turn = lambda x: turned(x.double().numpy(), pos.numpy().astype(np.float64), 500000.0, sections, interleaved)  # noqa: E731
    want = turn(b.q)
    pair = np.sqrt((want ** 2).reshape(*want.shape[:-1], 2, -1).sum(-2))
    tol = HALF_STEP[dtype] * np.abs(want) + 3 * 2.0 ** -23 * np.concatenate((pair, pair), -1)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    for which, codes, new in (("k", k, torch.from_numpy(turn(new_k))), ("v", v, new_v.double())):
        values = torch.from_numpy(R.decode(codes))
        sc = scales[which + "_scales"].cpu().double()
        for r in range(len(lens)):
            for t in range(lens[r] - m[r], lens[r]):
                page, slot = int(b.table[r, t // 16]), t % 16
                s = sc[page, :, slot // 8][:, None]
                w = new[b.starts[r] + t - (lens[r] - m[r])]
                assert bool(((values[page, :, slot] * s - w).abs() <= w.abs() / 16 + s * 2.0 ** -10 + w.abs() * 2.0 ** -20).all())


@pytest.mark.parametrize("kind", ["rows", "e4m3"])
def test_one_axis_of_the_places_is_the_plain_rotation(kind):
    lens, m = [90, 40, 16], [16, 7, 1]
    b = Batch(lens, m, 6, 2, 128, 16, dtype=BF16, kind=kind, seed=7)
    g = torch.Generator().manual_seed(3)
    rows = b.starts[-1]
    new_k, new_v = (torch.randn(rows, 2, 128, generator=g).to(BF16) for _ in range(2))
    pos = torch.cat([torch.arange(n - k, n) for n, k in zip(lens, m)]).to(torch.int32)
    q1, q2 = b.q.to(DEV), b.q.to(DEV)
    k1, v1, s1 = _append(b, new_k, new_v, q1, None, None, False, 10000.0)
    k2, v2, s2 = _append(b, new_k, new_v, q2, pos[None].repeat(3, 1), [16, 24, 24], False, 10000.0)
    raw = lambda x: x.view(torch.uint8) if kind == "e4m3" else x.view(torch.int16)  # noqa: E731
    if kind == "rows":
        assert torch.equal(raw(k1), raw(k2)) and torch.equal(raw(v1), raw(v2)) and torch.equal(q1, q2)
    else:   # (angles by turning on from token to token there, by a sine each here: last bits of 64)
        assert (raw(k1) != raw(k2)).sum() <= 1 and torch.equal(raw(v1), raw(v2)) and float((q1 - q2).abs().max()) <= 2.0 ** -6


def test_negative_and_far_positions():
    b = Batch([5], [5], 2, 1, 64, 16, dtype=F32)
    g = torch.Generator().manual_seed(4)
    new = torch.randn(5, 1, 64, generator=g)
    pos = torch.tensor([[-3, 0, 2 ** 31 - 1, -2 ** 31, 70000], [1, -1, 5, 7, -70000]], dtype=torch.int32)
    q = b.q.to(DEV)
    _append(b, new, new, q, pos, [20, 12], False, 10000.0)
    want = turned(b.q.double().numpy(), pos.numpy().astype(np.float64), 10000.0, [20, 12], False)
    # an angle of 2^31 is off by 2^-22 in 64 bits
    assert (np.abs(q.double().cpu().numpy() - want) <= 2.0 ** -24 * np.abs(want) + 4 * 2.0 ** -20).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 96, 128, 256, 512])
def test_prompts_enter_pools_of_their_type(dtype, d):
    """Any head size, plain copies, a batch of prompts and single tokens; rows behind the last request stay out."""
    lens, m = [513, 17, 300, 16], [513, 1, 40, 16]
    b = Batch(lens, m, 2, 2, d, 32, dtype=dtype, seed=d, poison=0.25)
    g = torch.Generator().manual_seed(5)
    rows = b.starts[-1]
    new_k, new_v = (torch.randn(rows + 21, 2, d, generator=g).to(dtype) for _ in range(2))
    k, v, _ = _append(b, new_k, new_v, None, None, None, False, 0.0)
    for cache, was, new in ((k.cpu(), b.k, new_k), (v.cpu(), b.v, new_v)):
        want = was.clone()
        for r in range(len(lens)):
            t = torch.arange(lens[r] - m[r], lens[r])
            want.transpose(1, 2)[b.table[r].long()[t // 32], t % 32] = new[b.starts[r]:b.starts[r + 1]]
        assert torch.equal(cache, want)


def test_a_prompt_with_a_bad_page_or_length_is_skipped_as_a_whole():
    lens, m = [400, 300, 90], [400, 300, 50]
    b = Batch(lens, m, 2, 2, 64, 16, dtype=BF16, seed=6, poison=0.5)
    b.table[1, 15] = -1
    g = torch.Generator().manual_seed(6)
    rows = b.starts[-1]
    new = torch.randn(rows, 2, 64, generator=g).bfloat16()
    (_, k, v, strides, table, n, starts, _, page, pages), _ = b.device()
    n[2] = 49
    status = spx.kv_append(new.to(DEV), new.to(DEV), k, v, strides, table, n, starts, page, pages)
    assert int(status.item()) == (spx.DEV_BAD_PAGE | spx.DEV_BAD_LEN)
    want = b.k.clone()
    t = torch.arange(400)
    want.transpose(1, 2)[b.table[0].long()[t // 16], t % 16] = new[:400]
    assert torch.equal(k.cpu(), want)


@pytest.mark.parametrize("kind,dtype", [("rows", BF16), ("rows", F32), ("e4m3", BF16)])
def test_prompts_with_images_enter_and_attend(kind, dtype):
    """The run a server makes: prompts enter the cache on three axes, attend, then a step behind them does."""
    lens, m = [200, 333], [200, 333]
    b = Batch(lens, m, 8, 2, 128, 16, dtype=dtype, kind=kind, seed=12)
    g = torch.Generator().manual_seed(7)
    rows = b.starts[-1]
    new_k, new_v = (torch.randn(rows, 2, 128, generator=g).to(dtype) for _ in range(2))
    pos = _positions(3, rows, 9, 500)
    (q, k, v, strides, table, n, starts, hkv, page, pages), scales = b.device()
    status = spx.kv_append(new_k.to(DEV), new_v.to(DEV), k, v, strides, table, n, starts, page, pages, rope_base=1e6, q_rows=q, positions=pos.to(DEV),
                           rope_sections=[16, 24, 24], **scales)
    out, lse, ws = spx.prompt_attention(q, k, v, strides, table, n, starts, hkv, page, pages, **scales)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and int(ws.status.item()) == 0
    b.q = q.cpu()
    raw = (lambda x: x.view(torch.uint8)) if kind == "e4m3" else (lambda x: x)
    b.k, b.v = raw(k).cpu(), raw(v).cpu()
    if scales:
        b.k_scales, b.v_scales = scales["k_scales"].cpu(), scales["v_scales"].cpu()
    b.check(out, lse)


@pytest.mark.parametrize("rope", [False, True])
def test_a_batch_of_many_requests(rope):
    """More requests than a block looks at in one go, one of them invalid, prompts among single tokens."""
    n = 700
    m = [1 + (i % 3) for i in range(n)]
    m[300], m[650] = 100, 37
    lens = [x + i % 20 for i, x in enumerate(m)]
    b = Batch(lens, m, 2, 1, 64, 16, dtype=F32, seed=13, poison=0.5)
    g = torch.Generator().manual_seed(8)
    new_k, new_v = (torch.randn(b.starts[-1], 1, 64, generator=g) for _ in range(2))
    (_, k, v, strides, table, lens_d, starts, _, page, pages), _ = b.device()
    lens_d[5] = 0
    status = spx.kv_append(new_k.to(DEV), new_v.to(DEV), k, v, strides, table, lens_d, starts, page, pages, rope_base=10000.0 if rope else 0.0)
    assert int(status.item()) == spx.DEV_BAD_LEN
    t = torch.cat([torch.arange(a - c, a) for a, c in zip(lens, m)])
    want_k = turned(new_k.double().numpy(), t[None].numpy().astype(np.float64), 10000.0, [32], False) if rope else new_k.double().numpy()
    want = b.v.clone()
    got_k = []
    for r in range(n):
        at = torch.arange(lens[r] - m[r], lens[r])
        where = (b.table[r].long()[at // 16], at % 16)
        if r != 5:
            want.transpose(1, 2)[where] = new_v[b.starts[r]:b.starts[r + 1]]
            got_k.append(k.cpu().transpose(1, 2)[where] if r % 50 == 0 or m[r] > 3 else None)
        else:
            got_k.append(None)
    assert torch.equal(v.cpu(), want)
    for r, x in enumerate(got_k):
        if x is not None:
            _check_rows(x, want_k[b.starts[r]:b.starts[r + 1]], F32)
