"""Calls over 8-bit pools that the interface allows and an ordinary program seldom makes: pools that are views with odd strides and
offsets, positions far out, the whole step in every variant, thousands of requests; log-probabilities of very many rows."""
import math

import numpy as np
import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding

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


def _strided(codes, order, pad, offset):
    """The pool in a byte buffer that begins `offset` bytes in, its dimensions in `order` (outer to inner), each stride padded by `pad`."""
    shape = codes.shape
    strides, step = [0, 0, 0, 1], shape[3] + pad
    for dim in reversed(order):
        strides[dim] = step
        step = step * shape[dim] + pad
    buf = torch.full((offset + step + 256,), 0x7F, dtype=torch.uint8, device=DEV)
    pool = buf[offset:].as_strided(shape, strides)
    pool.copy_(codes.to(DEV))
    return buf, pool, tuple(strides[:3])


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("order,pad,offset", [((0, 1, 2), 16, 16), ((0, 2, 1), 48, 80), ((1, 0, 2), 0, 16), ((1, 2, 0), 32, 0), ((2, 0, 1), 16, 48)])
def test_pools_that_are_views(order, pad, offset, d, dtype):
    """Pages, heads and slots in any order, strides and base addresses that are multiples of 16 bytes and no more; what lies between stays."""
    lens, m = [300, 40, 129], [5, 2, 4]
    c = R.Cache(lens, 2, d, 16, 8, seed=9)
    c.k_scales, c.v_scales = [torch.exp2(torch.log2(s).round()) for s in (c.k_scales, c.v_scales)]
    _, _, _, table, ks, vs = c.on(DEV)
    (kb, k, strides), (vb, v, _) = _strided(c.k, order, pad, offset), _strided(c.v, order, pad, offset)
    between = [torch.ones_like(b, dtype=torch.bool) for b in (kb, vb)]
    for mask, b in zip(between, (kb, vb)):
        mask[offset:].as_strided(k.shape, k.stride()).fill_(False)
    g = torch.Generator().manual_seed(1)
    nk, nv = (torch.randn(sum(m), 2, d, generator=g).to(dtype) for _ in range(2))
    q = torch.randn(sum(m), 8, d, generator=g).to(dtype)
    status = spx.kv_append(nk.to(DEV), nv.to(DEV), k, v, strides, table, _ints(lens), _starts(m), 16, c.num_pages, rope_base=10000.0, k_scales=ks, v_scales=vs)
    R.append(c, nk, nv, lens, m, 10000.0)
    out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, _ints(lens), _starts(m), 2, 16, c.num_pages, k_scales=ks, v_scales=vs, max_q_len=5)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and int(ws.status.item()) == 0
    assert torch.equal(k.cpu(), c.k) and torch.equal(v.cpu(), c.v) and torch.equal(ks.cpu(), c.k_scales) and torch.equal(vs.cpu(), c.v_scales)
    assert (kb[between[0]] == 0x7F).all() and (vb[between[1]] == 0x7F).all()
    _check(c, q, lens, m, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
def test_keys_and_values_in_one_tensor(dtype):
    """[pages, 2, heads, slots, d]: both pools are views of it with the page stride of both."""
    lens, m = [200, 77], [3, 6]
    c = R.Cache(lens, 2, 128, 16, 16, seed=3)
    both = torch.stack((c.k, c.v), 1).to(DEV)
    _, _, _, table, ks, vs = c.on(DEV)
    k, v = both[:, 0], both[:, 1]
    q = torch.randn(9, 8, 128, generator=torch.Generator().manual_seed(2)).to(dtype)
    out, lse, ws = spx.verify_attention(q.to(DEV), k, v, k.stride()[:3], table, _ints(lens), _starts(m), 2, 16, c.num_pages, k_scales=ks, v_scales=vs)
    torch.cuda.synchronize()
    assert int(ws.status.item()) == 0
    _check(c, q, lens, m, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("position", [131071, 1 << 20, 16000000])
def test_positions_far_out(position, dtype):
    """New rows at positions whose angles are large: only the pages of the new positions are looked at."""
    hkv, hq, d, page, m = 2, 4, 128, 16, 20
    n = position + m
    c = R.Cache([64], hkv, d, page, page, seed=1)
    c.k_scales[:], c.v_scales[:] = 0.25, 0.25
    real = c.table.clone()
    c.table = torch.full((1, -(-n // page)), -1, dtype=torch.int32)
    first = position // page
    c.table[0, first:first + 3] = real[0, :3][: c.table.shape[1] - first]
    k, v, strides, table, ks, vs = c.on(DEV)
    g = torch.Generator().manual_seed(4)
    nk, nv = (torch.randn(m, hkv, d, generator=g).to(dtype) for _ in range(2))
    q = torch.randn(m, hq, d, generator=g).to(dtype)
    out = torch.empty(q.shape, dtype=dtype, device=DEV)
    status = spx.kv_append(nk.to(DEV), nv.to(DEV), k, v, strides, table, _ints([n]), _starts([m]), page, c.num_pages, rope_base=10000.0,
                           q_rows=q.to(DEV), q_out=out, k_scales=ks, v_scales=vs)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    want = np.stack([R.rotate(q[j].double().numpy(), position + j, 10000.0) for j in range(m)])
    # the angle t f in 64 bits, f of four roundings: t f 2^-51, and a few steps of 2^-52 from the turns between neighbours, each times
    # the pair's elements; then the rounding to binary32 (two of its steps for 16-bit rows) and to the type
    angle = (position + m) * 2.0 ** -51 + 2.0 ** -49
    size = np.abs(q.double().numpy())
    size = size + np.concatenate((size[..., d // 2:], size[..., :d // 2]), -1)
    tol = (torch.finfo(dtype).eps / 2 + (2.0 ** -24 if dtype == F else 2.0 ** -22)) * np.abs(want) + (angle + 2.0 ** -44 + (2.0 ** -22 if dtype == BF else 0)) * size
    assert (np.abs(out.cpu().double().numpy() - want) <= tol).all()
    R.append(c, nk, nv, [n], [m], 10000.0)
    got = k.view(torch.uint8).cpu()
    # a code may be its neighbour where the value lies within that error of a border
    same = got == c.k
    assert same.double().mean() > 0.9999 and ((got.int() - c.k.int()).abs() <= 1).all()
    assert torch.equal(v.view(torch.uint8).cpu(), c.v) and torch.equal(ks.cpu(), c.k_scales) and torch.equal(vs.cpu(), c.v_scales)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("variant", ["plain", "temperature", "top-k", "top-p"])
def test_the_whole_step_in_every_variant(variant, dtype):
    """spx_verify_step over 8-bit pools gives what the two halves give, bit for bit, and again when it is repeated."""
    import spx_workloads as W
    spec = W.scaled(W.CONFIGS[1], batch=5, ctx_div=8, vocab=5000)
    b = W.generate(spec).to(DEV)
    lens, m = b.seq_lens_host, [k + 1 for k in b.k_host]
    hq, hkv, d = spec.num_q_heads, spec.num_kv_heads, spec.head_dim
    c = R.Cache(lens, hkv, d, 16, 16, seed=2)
    k, v, strides, table, ks, vs = c.on(DEV)
    q = b.q.to(dtype)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=F, device=DEV)
    acc, tok = torch.empty(5, dtype=torch.int32, device=DEV), torch.empty(b.total_q, dtype=torch.int32, device=DEV)
    extra = {"plain": {}, "temperature": dict(temperature=torch.tensor([0.7, 1.0, 0.0, 1.3, 0.9], device=DEV)),
             "top-k": dict(top_k=_ints([50, 1, 5000, 7, 300])), "top-p": dict(top_p=torch.tensor([0.9, 0.5, 1.0, 0.2, 0.99], device=DEV))}[variant]
    a = binding.make_attn_args(q, k, v, strides, table, b.seq_lens, b.q_indptr, hkv, 16, c.num_pages, out, lse, max_q_len=max(m), k_scales=ks, v_scales=vs)
    s = binding.make_sample_args(b.target_logits, b.draft_logits, b.draft_ids, b.q_indptr, b.u_accept, b.u_sample, acc, tok, **extra)
    ws = spx.Workspace.allocate(spx.workspace_size(a, s), DEV)
    want, want_lse, _ = spx.verify_attention(q, k, v, strides, table, b.seq_lens, b.q_indptr, hkv, 16, c.num_pages, max_q_len=max(m), k_scales=ks, v_scales=vs)
    want_acc, want_tok, _, _ = spx.rejection_sample(b.target_logits, b.draft_logits, b.draft_ids, b.q_indptr, b.u_accept, b.u_sample, **extra)
    for _ in range(3):
        for t in (out, lse, acc, tok):
            t.fill_(3)
        spx.verify_step(a, s, ws, DEV)
        torch.cuda.synchronize()
        assert int(ws.status.item()) == 0
        assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.equal(acc, want_acc) and torch.equal(tok, want_tok)
    _check(c, q.cpu(), lens, m, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
def test_thousands_of_short_requests(dtype):
    """More requests than the planner keeps in shared memory, of one token up to two tiles."""
    g = np.random.RandomState(2)
    m = g.choice([1, 2, 5], 2500).tolist()
    lens = [max(int(n), k) for n, k in zip(np.exp(g.uniform(0, 4, 2500)), m)]
    lens[7], lens[2400] = 150, 256
    c = R.Cache(lens, 1, 64, 16, 16, seed=5, tables_from=1)
    q = torch.randn(sum(m), 4, 64, generator=torch.Generator().manual_seed(4)).to(dtype)
    k, v, strides, table, ks, vs = c.on(DEV)
    out, lse, ws = spx.verify_attention(q.to(DEV), k, v, strides, table, _ints(lens), _starts(m), 1, 16, c.num_pages, k_scales=ks, v_scales=vs, max_q_len=5)
    torch.cuda.synchronize()
    assert int(ws.status.item()) == 0
    _check(c, q, lens, m, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
def test_very_many_rows_of_few_logits(dtype):
    """More rows than a grid's other dimensions could hold."""
    rows, vocab, top = 200001, 24, 5
    g = torch.Generator(DEV).manual_seed(1)
    logits = (3 * torch.randn(rows, vocab, generator=g, device=DEV)).to(dtype)
    tokens = torch.randint(-1, vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    lp, ent, ids, top_lp, ws = spx.token_logprobs(logits, tokens, top_n=top)
    torch.cuda.synchronize()
    assert int(ws.status.item()) == 0
    ref = torch.log_softmax(logits.double(), -1)
    none = tokens < 0
    assert torch.equal(torch.isnan(lp), none) and torch.equal(torch.isnan(ent), none) and (ids[none] == -1).all() and torch.isnan(top_lp[none]).all()
    want = ref.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0]
    assert ((lp.double() - want).abs()[~none] <= 2.0 ** -15 + 2.0 ** -24 * want.abs()[~none]).all()
    entropy = -(ref.exp() * ref).sum(1)
    assert ((ent.double() - entropy).abs()[~none] <= 2.0 ** -15 * (1 + 2 * entropy[~none] + 2 * 24)).all()
    order = torch.sort(logits.float(), dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(ids[~none].long(), order[~none])
    assert ((top_lp.double() - ref.gather(1, order)).abs()[~none] <= 2.0 ** -15 + 2.0 ** -24 * 40).all()


def test_logits_that_are_a_slice_of_a_wider_tensor():
    g = torch.Generator(DEV).manual_seed(2)
    wide = torch.randn(6, 4096 + 64, generator=g, device=DEV).to(BF)
    for lo, vocab in ((8, 4000), (64, 4096), (16, 1)):
        x = wide[1:5, lo:lo + vocab]
        lp, ent, ids, top, ws = spx.token_logprobs(x, _ints([0, vocab - 1, -1, vocab // 2]), top_n=2, vocab=vocab)
        whole = spx.token_logprobs(x.contiguous() if vocab % 8 == 0 else torch.nn.functional.pad(x, (0, 7)), _ints([0, vocab - 1, -1, vocab // 2]), top_n=2, vocab=vocab)
        torch.cuda.synchronize()
        assert int(ws.status.item()) == 0
        for a, b in zip((lp, ent, ids, top), whole):
            assert torch.equal(torch.nan_to_num(a.float(), nan=7.0), torch.nan_to_num(b.float(), nan=7.0))
        assert math.isnan(lp[2].item())
