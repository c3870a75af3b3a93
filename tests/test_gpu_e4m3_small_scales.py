"""Attention over 8-bit pools whose V scales are zero or tiny while the scores rise from tile to tile, against the plain
64-bit reference: a row's weights and its sum are kept under one reference, and the sum has to stay in range where the
weights times the scales do not tell that it leaves it."""
import math

import numpy as np
import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
TILE = 128


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _rising_cache(lens, hkv, d, steps, seed):
    """Every key of tile i of request r is the same direction, its score (for a query along it) steps[r][i] nats above tile 0's."""
    c = R.Cache(lens, hkv, d, 16, 16, seed=seed, spread=0.2)
    g = torch.Generator().manual_seed(seed)
    signs = torch.where(torch.rand(hkv, d, generator=g) < 0.5, -1.0, 1.0)
    ones = torch.from_numpy(R.encode((signs * 256.0).double().numpy()))            # code +-256
    for r, n in enumerate(lens):
        for t0 in range(0, n, 16):
            page = int(c.table[r, t0 // 16])
            c.k[page] = ones[:, None].expand(-1, 16, -1)
            # <q, k> sm_scale = 256 ks d / sqrt(d) for q = signs; a little different from block to block
            c.k_scales[page] = (steps[r][t0 // TILE] + 0.25 * math.sin(t0)) / (256 * math.sqrt(d))
    return c, signs


def _queries(signs, m, hq, hkv, d, seed):
    g = torch.Generator().manual_seed(seed)
    q = signs.repeat_interleave(hq // hkv, 0)[None].repeat(m, 1, 1)
    return q * (0.5 + 0.5 * torch.rand(m, hq, 1, generator=g))                      # from half of the steps to all of them


def _check(c, q, lens, m):
    k, v, strides, table, ks, vs = c.on(DEV)
    starts = _ints([0, *np.cumsum(m).tolist()])
    out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, _ints(lens), starts, c.hkv, c.page, c.num_pages, k_scales=ks, v_scales=vs,
                                        max_q_len=max(m))
    torch.cuda.synchronize()
    assert int(ws.status.item()) == 0
    ref, ref_lse, spread, reach = R.attention(c, q, lens, m)
    if q.dtype == BF:
        # What lies below the range kept for a row: half a least step of a weight times its scale is 2^-27 of the reference, the
        # largest p_t max(scale_t, 2^-90) (smaller scales count as 2^-90 in it); a token adds that times its code, at most 448.
        # Divided by the 2^-7 at least that the bound multiplies spread with.
        q0 = 0
        g = q.shape[1] // c.hkv
        for r, (n, k_) in enumerate(zip(lens, m)):
            keys, sc = c.values("k", r, n), np.maximum(c.token_scales("v", r, n), 2.0 ** -90)
            live = np.abs(R.decode(getattr(c, "v")[c.table[r, : -(-n // c.page)].long()]).transpose(0, 2, 1, 3).reshape(-1, c.hkv, c.d)[:n])
            live = np.where(c.token_scales("v", r, n)[..., None] > 0, live, 0.0)
            for j in range(k_):
                seen = n - k_ + j + 1
                x = q[q0 + j].double().numpy().reshape(c.hkv, g, c.d)
                s = np.einsum("hgd,thd->hgt", x, keys[:seen]) / math.sqrt(c.d)
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                top = (p * sc[:seen].T[:, None]).max(-1)
                spread[q0 + j] += (2.0 ** -20 * top[..., None] * live[:seen].sum(0)[:, None]).reshape(-1, c.d)
            q0 += k_
    tol, tol_lse = R.attention_bounds(ref, spread, reach, max(lens), q.shape[2], q.dtype)
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    # A weight e^(s - m) below the smallest normal number may vanish (z >= 1 and |v| times it at most, summed over the tokens),
    # and so may a result that is below it itself.
    tiny = np.full_like(ref, 2.0 ** -126)
    q0 = 0
    for r, (n, k_) in enumerate(zip(lens, m)):
        all_v = np.abs(c.values("v", r, n)).sum(0)
        tiny[q0:q0 + k_] += 2.0 ** -126 * np.repeat(all_v, q.shape[1] // c.hkv, 0)
        q0 += k_
    assert (np.abs(out - ref) <= tol + tiny).all(), (np.abs(out - ref) - tol).max()
    assert (np.abs(lse - ref_lse) <= tol_lse).all(), (np.abs(lse - ref_lse) - tol_lse).max()


# packed rows: up to 32, 64 and 128 a request (the three accumulator layouts), and head_dim 64
SHAPES = [(8, 2, 128, 3), (8, 2, 64, 4), (36, 4, 128, 5), (16, 2, 64, 6), (64, 4, 128, 6), (128, 8, 64, 5)]
PATTERNS = ["all zero", "first tile zero", "first two tiles zero", "zero from the second tile on", "zero but for the last tile", "tiny", "mixed"]


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("hq,hkv,d,m", SHAPES)
@pytest.mark.parametrize("pattern", PATTERNS)
def test_rising_scores_under_zero_and_tiny_value_scales(pattern, hq, hkv, d, m, dtype):
    lens = [770, 515, 640, 128 + m]
    steps = [[0, 25, 50, 75, 100, 125, 150], [0, 0, 90, 95, 190], [0, 100, 3, 200, 10], [0, 120]]
    c, signs = _rising_cache(lens, hkv, d, steps, seed=3)
    g = torch.Generator().manual_seed(5)
    for r, n in enumerate(lens):
        tiles = -(-n // TILE)
        for t0 in range(0, n, 16):
            page, i = int(c.table[r, t0 // 16]), t0 // TILE
            if pattern == "all zero":
                s = 0.0
            elif pattern == "first tile zero":
                s = 0.0 if i < 1 else None
            elif pattern == "first two tiles zero":
                s = 0.0 if i < 2 else None
            elif pattern == "zero from the second tile on":
                s = 0.0 if i >= 1 else None
            elif pattern == "zero but for the last tile":
                s = 0.0 if i < tiles - 1 else None
            elif pattern == "tiny":
                s = [2.0 ** -100, 2.0 ** -116, 2.0 ** -95, 2.0 ** -110][i % 4]
            else:
                s = [0.0, 2.0 ** -105, 2.0 ** -60, 1.0, 2.0 ** 40][int(torch.randint(0, 5, (1,), generator=g))]
            if s is not None:
                c.v_scales[page] = s
    q = _queries(signs, m * len(lens), hq, hkv, d, 6).to(dtype)
    _check(c, q, lens, [m] * len(lens))


@pytest.mark.parametrize("hq,hkv,d,m", SHAPES)
def test_a_chunk_of_zero_scales_among_others(hq, hkv, d, m):
    """One long request cut over many CTAs: chunks with nothing but zero scales merge with ordinary ones."""
    n = 6000
    tiles = -(-n // TILE)
    steps = [[5.0 * i for i in range(tiles)]]
    c, signs = _rising_cache([n], hkv, d, steps, seed=7)
    for t0 in range(0, n, 16):
        if (t0 // TILE) % 11 < 6:
            c.v_scales[int(c.table[0, t0 // 16])] = 0.0
    q = _queries(signs, m, hq, hkv, d, 8).to(BF)
    _check(c, q, [n], [m])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("large", [30, 60, 90])
@pytest.mark.parametrize("hq,hkv,d,m", SHAPES)
def test_zero_and_large_value_scales_in_one_row(hq, hkv, d, m, large, dtype):
    """Scales of zero beside scales of 2^30 to 2^90: what has weight and what has size lie in different tiles (every other one, the first or the
    last ones), or in different chunks of a long request; the row's sum is that of the weights."""
    lens = [770, 515, 900, 700, 7000]
    c, signs = _rising_cache(lens, hkv, d, [[0] * 64, [6, 0, 6, 0, 6], [0] * 64, [4, 3, 2, 1, 0, 0], [0] * 64], seed=9)
    for r, n in enumerate(lens):
        tiles = -(-n // TILE)
        for t0 in range(0, n, 16):
            page, i = int(c.table[r, t0 // 16]), t0 // TILE
            zero = (i % 2 == 0, i % 2 == 1, i < tiles // 2, i >= tiles // 2, i % 9 < 5)[r]
            c.v_scales[page] = 0.0 if zero else c.v_scales[page] * 2.0 ** large
    q = _queries(signs, m * len(lens), hq, hkv, d, 10).to(dtype)
    _check(c, q, lens, [m] * len(lens))
