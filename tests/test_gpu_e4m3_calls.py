"""Calls over the 8-bit cache that a program makes beside the plain one: on other streams, two at once, captured and
replayed under other lengths, with rows behind the last request, with the same page twice; and by keyword."""
import numpy as np
import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _starts(m):
    return _ints([0, *np.cumsum(m).tolist()])


def _check(c, q, lens, m, out, lse):
    ref, ref_lse, spread, reach = R.attention(c, q, lens, m)
    tol, tol_lse = R.attention_bounds(ref, spread, reach, max(lens), q.shape[2], q.dtype)
    assert (np.abs(out.cpu().double().numpy() - ref) <= tol).all()
    assert (np.abs(lse.cpu().double().numpy() - ref_lse) <= tol_lse).all()


def _queries(m, hq, d, dtype, seed):
    return torch.randn(sum(m), hq, d, generator=torch.Generator().manual_seed(seed)).to(dtype)


SHAPES = [(32, 8, 128, 16, BF), (64, 8, 128, 16, BF), (64, 4, 128, 32, BF), (8, 2, 64, 8, BF), (8, 2, 64, 16, F)]


@pytest.mark.parametrize("hq,hkv,d,page,dtype", SHAPES)
def test_two_calls_at_once(hq, hkv, d, page, dtype):
    """Two streams, each with its own workspace and outputs, over one cache; many calls in flight, the same results bit for bit."""
    lens, m = [900, 33, 2000, 140], [5, 1, 6, 6]
    c = R.Cache(lens, hkv, d, page, page, seed=1)
    k, v, strides, table, ks, vs = c.on(DEV)
    streams = [torch.cuda.Stream() for _ in range(2)]
    qs = [_queries(m, hq, d, dtype, 2 + i).to(DEV) for i in range(2)]
    args = (k, v, strides, table, _ints(lens), _starts(m), hkv, page, c.num_pages)
    outs, lses, wss = [[], []], [[], []], [None, None]
    torch.cuda.synchronize()
    for _ in range(12):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                out, lse, wss[i] = spx.verify_attention(qs[i], *args, k_scales=ks, v_scales=vs, ws=wss[i], max_q_len=6)
                outs[i].append(out)
                lses[i].append(lse)
    torch.cuda.synchronize()
    for i in range(2):
        assert int(wss[i].status.item()) == 0
        _check(c, qs[i].cpu(), lens, m, outs[i][0], lses[i][0])
        assert all(torch.equal(o, outs[i][0]) for o in outs[i]) and all(torch.equal(x, lses[i][0]) for x in lses[i])


def test_a_side_stream_needs_no_other():
    """Append, attention and log-probabilities in order on one stream that is not the default one, behind work that keeps it busy."""
    lens, m = [40, 300], [6, 4]
    c = R.Cache(lens, 8, 128, 16, 16, seed=3)
    c.k_scales, c.v_scales = [torch.exp2(torch.log2(s).round()) for s in (c.k_scales, c.v_scales)]
    k, v, strides, table, ks, vs = c.on(DEV)
    g = torch.Generator().manual_seed(4)
    nk, nv = (torch.randn(10, 8, 128, generator=g).to(BF) for _ in range(2))
    q = _queries(m, 32, 128, BF, 5)
    logits = torch.randn(10, 1000, generator=g).to(BF)
    dev = [t.to(DEV) for t in (nk, nv, q, logits)]
    n, starts, ids = _ints(lens), _starts(m), _ints(list(range(10)))
    busy = torch.zeros(1 << 26, device=DEV)
    staged = [torch.empty_like(t) for t in dev]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for _ in range(8):
            busy.add_(1)
        for a, b in zip(staged, dev):
            a.copy_(b)
        status = spx.kv_append(staged[0], staged[1], k, v, strides, table, n, starts, 16, c.num_pages, k_scales=ks, v_scales=vs)
        out, lse, ws = spx.verify_attention(staged[2], k, v, strides, table, n, starts, 8, 16, c.num_pages, k_scales=ks, v_scales=vs)
        lp, ent, top, top_lp, lws = spx.token_logprobs(staged[3], ids, top_n=2)
    stream.synchronize()
    assert int(status.item()) == 0 and int(ws.status.item()) == 0 and int(lws.status.item()) == 0
    R.append(c, nk, nv, lens, m)
    assert torch.equal(k.view(torch.uint8).cpu(), c.k) and torch.equal(vs.cpu(), c.v_scales)
    _check(c, q, lens, m, out, lse)
    for i in range(10):
        want = R.logprobs(logits[i].float().numpy(), i, 2)
        assert abs(lp[i].item() - want[0]) < 1e-4 and top[i].tolist() == want[2]


@pytest.mark.parametrize("hq,hkv,d,page,dtype", SHAPES)
def test_a_captured_call_follows_its_lengths_and_pages(hq, hkv, d, page, dtype):
    """One graph, replayed under other lengths, other pages and other queries in the same tensors."""
    m = [3, 3, 3]
    c = R.Cache([1500, 1500, 1500], hkv, d, page, page, seed=6)
    k, v, strides, table, ks, vs = c.on(DEV)
    q, n = torch.empty(9, hq, d, dtype=dtype, device=DEV), _ints([1500] * 3)
    q.zero_()
    starts = _starts(m)
    out, lse, ws = spx.verify_attention(q, k, v, strides, table, n, starts, hkv, page, c.num_pages, k_scales=ks, v_scales=vs, max_q_len=3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spx.verify_attention(q, k, v, strides, table, n, starts, hkv, page, c.num_pages, out=out, lse=lse, k_scales=ks, v_scales=vs, max_q_len=3, ws=ws)
    for seed, lens in enumerate(([3, 4, 5], [1500, 3, 129], [700, 1400, 1500])):
        x = _queries(m, hq, d, dtype, seed)
        q.copy_(x)
        n.copy_(_ints(lens))
        c.table[:] = c.table.flip(0) if torch.is_tensor(c.table) else c.table[::-1].copy()
        table.copy_(torch.as_tensor(np.ascontiguousarray(c.table)))
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        assert int(ws.status.item()) == 0
        _check(c, x, lens, m, out, lse)


@pytest.mark.parametrize("hq,hkv,d,page,dtype", SHAPES)
def test_rows_behind_the_last_request_stay(hq, hkv, d, page, dtype):
    """A batch padded with rows that belong to no request: neither written nor, whatever they hold, of any effect."""
    lens, m, pad = [200, 9], [4, 2], 5
    c = R.Cache(lens, hkv, d, page, page, seed=8)
    c.k_scales, c.v_scales = [torch.exp2(torch.log2(s).round()) for s in (c.k_scales, c.v_scales)]
    k, v, strides, table, ks, vs = c.on(DEV)
    total = sum(m) + pad
    q = _queries([total], hq, d, dtype, 9)
    g = torch.Generator().manual_seed(10)
    nk, nv = (torch.randn(total, hkv, d, generator=g).to(dtype) for _ in range(2))
    for t in (q, nk, nv):
        t[sum(m):] = float("nan")
    q_out = torch.full((total, hq, d), 7.0, dtype=dtype, device=DEV)
    status = spx.kv_append(nk.to(DEV), nv.to(DEV), k, v, strides, table, _ints(lens), _starts(m), page, c.num_pages, rope_base=10000.0,
                           q_rows=q.to(DEV), q_out=q_out, k_scales=ks, v_scales=vs)
    R.append(c, nk, nv, lens, m, 10000.0)
    assert int(status.item()) == 0 and torch.equal(k.view(torch.uint8).cpu(), c.k) and torch.equal(ks.cpu(), c.k_scales)
    assert (q_out[sum(m):] == 7).all() and not torch.isnan(q_out[:sum(m)]).any()
    out = torch.full((total, hq, d), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((total, hq), 7.0, device=DEV)
    _, _, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, _ints(lens), _starts(m), hkv, page, c.num_pages, out=out, lse=lse,
                                    k_scales=ks, v_scales=vs, max_q_len=4)
    assert int(ws.status.item()) == 0
    assert (out[sum(m):] == 7).all() and (lse[sum(m):] == 7).all()
    _check(c, q[:sum(m)], lens, m, out[:sum(m)], lse[:sum(m)])


@pytest.mark.parametrize("hq,hkv,d,page,dtype", SHAPES)
def test_the_same_page_twice(hq, hkv, d, page, dtype):
    """A page that stands twice in a request's table, and in two requests' tables (a shared prefix), is read twice."""
    lens, m = [400, 400], [2, 5]
    c = R.Cache(lens, hkv, d, page, page, seed=11)
    c.table[0, 1] = c.table[0, 0]
    c.table[1, :4] = c.table[0, :4]
    k, v, strides, table, ks, vs = c.on(DEV)
    q = _queries(m, hq, d, dtype, 12)
    out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, _ints(lens), _starts(m), hkv, page, c.num_pages, k_scales=ks, v_scales=vs,
                                    max_q_len=5)
    assert int(ws.status.item()) == 0
    _check(c, q, lens, m, out, lse)


def test_keywords_and_byte_pools():
    """Every argument by keyword, the pools as plain bytes."""
    lens, m = [50, 20], [3, 2]
    c = R.Cache(lens, 2, 64, 16, 8, seed=13)
    c.k_scales, c.v_scales = [torch.exp2(torch.log2(s).round()) for s in (c.k_scales, c.v_scales)]
    k, v, strides, table, ks, vs = c.on(DEV)
    k, v = k.view(torch.uint8), v.view(torch.uint8)
    g = torch.Generator().manual_seed(14)
    nk, nv = (torch.randn(5, 2, 64, generator=g).to(BF) for _ in range(2))
    status = spx.kv_append(new_k=nk.to(DEV), new_v=nv.to(DEV), k_cache=k, v_cache=v, kv_strides=strides, block_table=table, seq_lens=_ints(lens),
                           q_indptr=_starts(m), page_size=16, num_pages=c.num_pages, k_scales=ks, v_scales=vs)
    R.append(c, nk, nv, lens, m)
    assert int(status.item()) == 0 and torch.equal(k.cpu(), c.k) and torch.equal(v.cpu(), c.v)
    q = _queries(m, 8, 64, BF, 15)
    out, lse, _ = spx.verify_attention(q=q.to(DEV), k_cache=k, v_cache=v, kv_strides=strides, block_table=table, seq_lens=_ints(lens),
                                       q_indptr=_starts(m), num_kv_heads=2, page_size=16, num_pages=c.num_pages, k_scales=ks, v_scales=vs)
    _check(c, q, lens, m, out, lse)
    x = torch.randn(2, 64, generator=g)
    lp, *_ = spx.token_logprobs(logits=x.to(DEV), token_ids=_ints([3, 4]))
    assert abs(lp[1].item() - R.logprobs(x[1].numpy(), 4, 1)[0]) < 1e-4
