"""Invariants of the attention work plan over 8-bit pools, read back from the workspace after a call: the rules of the
tensor-core kernel (an entry costs 14/8 of a tile) and of the fp32 kernel (cuts down to a tile), and the one that cuts few
requests with long contexts over the SMs too."""
import types

import numpy as np
import pytest
import torch

import paper_2609_34370_b200 as spx
import spx_workloads as W
import test_gpu_plan as plan
from paper_2609_34370_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
TILE = 128
COST = 8   # of a tile on the planner's axis


def _plan_of(lens, m, hq, hkv, d, page, dtype):
    g = torch.Generator(DEV).manual_seed(sum(lens) % 1000)
    pages = 64   # the plan goes by lengths alone: all requests share a small pool
    codes = torch.randint(0, 0x70, (2, pages, hkv, page, d), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.full((pages, hkv, 1), 2.0 ** -6, device=DEV)
    table = torch.randint(0, pages, (len(lens), -(-max(lens) // page)), generator=g, device=DEV, dtype=torch.int32)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    starts = np.concatenate([[0], np.cumsum(m)]).tolist()
    q = torch.randn(starts[-1], hq, d, generator=g, device=DEV).to(dtype)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    n, qi = ints(lens), ints(starts)
    strides = (hkv * page * d, page * d, d)
    a = binding.make_attn_args(q, codes[0], codes[1], strides, table, n, qi, hkv, page, pages, out, lse, max_q_len=max(m), k_scales=scales,
                               v_scales=scales)
    lay = spx.plan_layout(a)
    ws = spx.Workspace.allocate(spx.workspace_size(a, None), DEV)
    spx.verify_attention(q, codes[0], codes[1], strides, table, n, qi, hkv, page, pages, out=out, lse=lse, max_q_len=max(m), k_scales=scales,
                         v_scales=scales, ws=ws)
    torch.cuda.synchronize()
    raw = ws.buf.cpu().numpy()
    n_work, n_cta, n_slots, total_tiles, _, overflow = (int(v) for v in raw[lay["header"]:lay["header"] + 24].view(np.int32))
    pairs = len(lens) * hkv
    part = lambda key, count: raw[lay[key]:lay[key] + 4 * count].view(np.int32)  # noqa: E731
    P = dict(n_work=n_work, n_cta=n_cta, n_slots=n_slots, total_tiles=total_tiles, overflow=overflow, cta_off=part("cta_off", n_cta + 1),
             work=part("work", 8 * n_work).reshape(-1, 8), nch=part("pair_nchunks", pairs), base=part("pair_part_base", pairs), lay=lay,
             seq_lens=np.array(lens), status=int(ws.status.item()))
    invalid = {r for r, (n_, k) in enumerate(zip(lens, m)) if n_ < k}
    assert (P["status"] != 0) == bool(invalid)
    batch = types.SimpleNamespace(batch=len(lens), q_indptr=starts, spec=types.SimpleNamespace(num_kv_heads=hkv))
    plan._check_plan(batch, P, invalid=invalid)
    return P


def _loads(P, entry_cost):
    """Ranges' lengths on the planner's axis: tiles, and an entry's cost where a pair begins."""
    tiles = [-(-int(n) // TILE) for n in P["seq_lens"]]
    loads = []
    for c in range(P["n_cta"]):
        load = 0
        for req, begin, end, *_ in P["work"][P["cta_off"][c]:P["cta_off"][c + 1]]:
            load += COST * (end - begin) + (entry_cost + 2 * (tiles[req] <= 2) if begin == 0 else 0)
        loads.append(load)
    return loads


def _lens(spec):
    """Lengths and new positions as the named workload draws them (its tensors are not needed)."""
    rng = np.random.default_rng(spec.index)
    batch = min(spec.batch, 160)
    m = [k + 1 for k in (rng.choice(spec.k[1], batch).tolist() if spec.k[0] == "choice" else [spec.k[1]] * batch)]
    if spec.ctx[0] == "uniform":
        lens = rng.integers(spec.ctx[1], spec.ctx[2] + 1, batch)
    else:
        _, median, sigma, lo, hi = spec.ctx
        lens = np.clip(median * np.exp(sigma * rng.standard_normal(batch)), lo, hi).astype(int)
    return [max(int(n), k) for n, k in zip(lens, m)], m


@pytest.mark.parametrize("index", [1, 2, 4])
def test_named_workloads_are_cut_into_ranges_of_equal_cost(index):
    spec = W.CONFIGS[index]
    lens, m = _lens(spec)
    P = _plan_of(lens, m, spec.num_q_heads, spec.num_kv_heads, spec.head_dim, spec.page_size, BF)
    loads = _loads(P, 14)
    mean = sum(loads) / len(loads)
    # a cut lies at a multiple of the mean, moved back by less than an entry's cost (16), the two tiles that are not split off
    # and a part of a tile (39 in all), or forward by less than two tiles
    assert P["n_cta"] == 148 and max(abs(x - mean) for x in loads) <= 39 + 16 + 1


@pytest.mark.parametrize("dtype,lens,hkv,ranges", [
    # one request of 32 tiles and 8 heads: 256 tiles, ranges of four (tensor cores) or two (fp32) tiles at least
    (BF, [4096], 8, 64), (F, [4096], 8, 128), (BF, [8000, 8000], 1, 31), (F, [8000, 8000], 1, 63), (BF, [1200], 1, 2),
    # pairs no longer than two ranges' least lengths stay whole, one CTA each
    (BF, [1024], 8, 148), (F, [500], 8, 148), (BF, [100] * 20, 2, 148),
    # an axis long enough for every SM
    (BF, [9000], 16, 148), (F, [4500], 16, 148)])
def test_few_requests_with_long_contexts_are_cut_too(dtype, lens, hkv, ranges):
    P = _plan_of(lens, [1] * len(lens), hkv, hkv, 128, 16, dtype)
    assert P["n_cta"] == ranges
    tiles = [-(-n // TILE) for n in lens]
    least = 2 if dtype == BF else 1
    longest = max(e[2] - e[1] for e in P["work"])
    if ranges < 148 or sum(tiles) * hkv >= 2 * least * 148:
        # every pair that is longer than a range is cut, no piece is shorter than the least, none much longer than its share
        assert (P["nch"] > 1).all()
        assert min(e[2] - e[1] for e in P["work"]) >= least
        share = sum(_loads(P, 14 if dtype == BF else 3)) / P["n_cta"] / COST
        assert longest <= share + 2 * least + 4
    else:
        assert (P["nch"] == 1).all() and P["n_work"] == len(lens) * hkv


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("seed", range(5))
def test_invariants_on_random_batches(seed, dtype):
    rng = np.random.default_rng(seed)
    batch = int(rng.choice([1, 2, 7, 40, 300, 1500]))
    hi = int(rng.choice([40, 700, 5000])) if batch >= 300 else int(rng.choice([40, 700, 5000, 30000]))
    hkv = int(rng.choice([1, 2, 4]))
    m = rng.choice([1, 2, 4, 6], batch).tolist()
    lens = [max(int(x), k) for x, k in zip(rng.integers(1, hi, batch), m)]
    if seed % 2:
        for r in rng.choice(batch, size=min(batch, 3), replace=False):
            lens[int(r)] = 0
    _plan_of(lens, m, 2 * hkv, hkv, 64, 16, dtype)
