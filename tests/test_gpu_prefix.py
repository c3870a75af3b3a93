"""Verify attention behind shared prefixes against the definition in 64 bits, and the whole step with it."""
import pytest
import torch

import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding
from prompt_util import DEV, Batch, verify

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _grouped(sizes, prefixes, own, ks, hq, hkv, d, page, **kw):
    """Groups of sizes[i] requests behind prefixes[i] tokens; own and ks are gone through in turn."""
    lens, m, shared, at = [], [], [], 0
    for n, p in zip(sizes, prefixes):
        if n:
            shared.append((at, at + n, p))
        for _ in range(n):
            m.append(ks[len(m) % len(ks)] + 1)
            lens.append(p + max(m[-1], own[len(lens) % len(own)]))
        at += n
    groups = [0]
    for n in sizes:
        groups.append(groups[-1] + n)
    return Batch(lens, m, hq, hkv, d, page, shared=shared, **kw), (groups, list(prefixes))


@pytest.mark.parametrize("layout", ["HND", "NHD"])
@pytest.mark.parametrize("hq,hkv,d,page,ks", [(8, 2, 64, 16, [4]), (32, 8, 128, 16, [5, 0]), (28, 4, 128, 8, [0, 2, 4]), (64, 8, 128, 32, [3]), (16, 16, 64, 128, [0]),
                                              (32, 2, 128, 16, [5, 7, 1]), (8, 1, 64, 64, [15])])
@pytest.mark.parametrize("dtype,kind", [(BF16, "rows"), (BF16, "e4m3"), (F32, "rows"), (F32, "e4m3")])
def test_groups(hq, hkv, d, page, ks, dtype, kind, layout):
    b, groups = _grouped([5, 0, 1, 9], [700, 50, 300, 129], [1, 90, 128, 300, 17], ks, hq, hkv, d, page, dtype=dtype, kind=kind, layout=layout, seed=hq)
    out, lse, status = verify(b, groups)
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("prefix", [0, 1, 127, 128, 255, 256, 3000])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_lengths_of_the_prefix(prefix, dtype):
    b, groups = _grouped([7], [prefix], [3, 40], [2], 8, 2, 128, 16, dtype=dtype, seed=prefix)
    out, lse, status = verify(b, groups)
    assert status == 0
    b.check(out, lse)


def test_one_prefix_of_many_requests_and_many_groups():
    b, groups = _grouped([150], [1000], [30], [1], 8, 2, 64, 16, seed=1)
    out, lse, status = verify(b, groups)
    assert status == 0
    b.check(out, lse)
    b, groups = _grouped([2] * 70, [128 + 13 * i for i in range(70)], [20, 200], [0, 3], 8, 2, 64, 16, seed=2)
    out, lse, status = verify(b, groups)
    assert status == 0
    b.check(out, lse)


def test_long_prefix_is_cut():
    b, groups = _grouped([3], [20000], [10], [0, 1], 8, 1, 128, 16, seed=3)
    out, lse, status = verify(b, groups)
    assert status == 0
    b.check(out, lse)


def test_groups_that_leave_requests_out():
    b, _ = _grouped([4, 4, 4], [256, 400, 300], [33], [2], 8, 2, 128, 16, seed=4)
    out, lse, status = verify(b, ([4, 8], [400]))
    assert status == 0
    b.check(out, lse)
    out, lse, status = verify(b, ([12, 12, 0], [400, 400]))      # empty, and one that runs backwards: nothing is shared
    assert status == 0
    b.check(out, lse)
    out, lse, status = verify(b, ([0, 4, 8, 12], [-5, 0, 99]))
    assert status == 0
    b.check(out, lse)


@pytest.mark.parametrize("dtype,kind", [(BF16, "rows"), (F32, "rows"), (BF16, "e4m3")])
def test_bad_data(dtype, kind):
    b, groups = _grouped([4, 3, 3], [512, 300, 600], [50, 60], [2], 8, 2, 128, 16, dtype=dtype, kind=kind, seed=6)
    b.table[2, 5] = b.table[0, 0]                # another page inside the shared tiles: request 2 alone is void
    b.table[4:7, 2] = b.num_pages + 3            # a bad page of group 1's prefix: the whole group
    b.table[8, 600 // 16 + 1] = -7               # a bad page of request 8's own
    (args, scales) = b.device()
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    out, lse, ws = spx.verify_attention(*args, **scales, max_q_len=3, group_indptr=ints(groups[0]), prefix_lens=ints(groups[1]))
    assert int(ws.status.item()) == spx.DEV_BAD_PAGE
    b.check(out, lse, requests=[0, 1, 3, 7, 9])
    for r in (2, 4, 5, 6, 8):
        rows = slice(b.starts[r], b.starts[r + 1])
        assert bool((out[rows] == 0).all()) and bool(torch.isnan(lse[rows]).all())


def test_a_prefix_that_holds_new_positions():
    b, groups = _grouped([3], [400], [10], [2], 8, 2, 64, 16, seed=7)
    (q, k, v, strides, table, n, *rest), _ = b.device()
    n[1] = 386                                    # 383 tokens behind the three new ones: below the 384 that are read once
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    out, lse, ws = spx.verify_attention(q, k, v, strides, table, n, *rest, max_q_len=3, group_indptr=ints([0, 3]), prefix_lens=ints([400]))
    assert int(ws.status.item()) == spx.DEV_BAD_LEN and bool(torch.isnan(lse[3:6]).all()) and bool((out[3:6] == 0).all())
    b.check(out, lse, requests=[0, 2])


@pytest.mark.parametrize("dtype,kind", [(BF16, "rows"), (F32, "rows"), (BF16, "e4m3")])
def test_replayed_and_the_same_bits(dtype, kind):
    b, (gi, pl) = _grouped([12, 20], [900, 300], [100, 40], [4, 1], 32, 8, 128, 16, dtype=dtype, kind=kind, seed=8)
    args, scales = b.device()
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    kw = dict(max_q_len=5, group_indptr=ints(gi), prefix_lens=ints(pl), **scales)
    first, lse, ws = spx.verify_attention(*args, **kw)
    torch.cuda.synchronize()
    assert int(ws.status.item()) == 0
    b.check(first, lse)
    again, lse2 = torch.empty_like(first), torch.empty_like(lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spx.verify_attention(*args, out=again, lse=lse2, ws=ws, **kw)
    for _ in range(3):
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("filtered", [False, True])
def test_the_whole_step(filtered):
    b, (gi, pl) = _grouped([6, 3], [640, 200], [90, 30], [3, 0], 32, 8, 128, 16, seed=9)
    (q, k, v, strides, table, n, starts, hkv, page, pages), _ = b.device()
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    g = torch.Generator().manual_seed(1)
    tq, nb, vocab = b.starts[-1], len(b.lens), 4096
    target = (3 * torch.randn(tq, vocab, generator=g)).bfloat16().to(DEV)
    draft = (3 * torch.randn(tq - nb, vocab, generator=g)).bfloat16().to(DEV)
    ids = torch.randint(0, vocab, (tq - nb,), generator=g, dtype=torch.int32).to(DEV)
    ua, us = torch.rand(tq - nb, generator=g).to(DEV), torch.rand(nb, generator=g).to(DEV)
    extra = dict(top_k=ints([20] * nb), temperature=torch.full((nb,), 0.8, device=DEV)) if filtered else {}
    acc, tok, _, _ = spx.rejection_sample(target, draft, ids, starts, ua, us, **extra)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    acc2, tok2 = torch.empty_like(acc), torch.empty_like(tok)
    groups = (ints(gi), ints(pl))
    a = spx.make_attn_args(q, k, v, strides, table, n, starts, hkv, page, pages, out, lse, max_q_len=4, group_indptr=groups[0], prefix_lens=groups[1])
    s = spx.make_sample_args(target, draft, ids, starts, ua, us, acc2, tok2, **extra)
    ws = spx.Workspace.allocate(spx.workspace_size(a, s), DEV)
    for _ in range(3):
        spx.verify_step(a, s, ws, torch.device(DEV, 0))
    torch.cuda.synchronize()
    assert int(ws.status.item()) == 0 and torch.equal(acc, acc2) and torch.equal(tok, tok2)
    b.check(out, lse)


def test_the_step_from_host_buffers():
    b, (gi, pl) = _grouped([4], [300], [50], [2], 8, 2, 64, 16, dtype=F32, seed=10)
    g = torch.Generator().manual_seed(2)
    tq, nb, vocab = b.starts[-1], len(b.lens), 512
    pin = lambda x: x.contiguous().pin_memory()  # noqa: E731
    ints = lambda x: pin(torch.tensor(x, dtype=torch.int32))  # noqa: E731
    q, k, v, table, n, starts = pin(b.q), pin(b.k), pin(b.v), pin(b.table), ints(b.lens), ints(b.starts)
    target, draft = pin(torch.randn(tq, vocab, generator=g)), pin(torch.randn(tq - nb, vocab, generator=g))
    ids, ua, us = ints([5] * (tq - nb)), pin(torch.rand(tq - nb, generator=g)), pin(torch.rand(nb, generator=g))
    out, lse, acc, tok = pin(torch.empty_like(q)), pin(torch.empty(q.shape[:2])), ints([0] * nb), ints([0] * tq)
    gi, pl, status = ints(gi), ints(pl), ints([7])
    a = spx.make_attn_args(q, k, v, k.stride()[:3], table, n, starts, 2, 16, b.num_pages, out, lse, max_q_len=3, group_indptr=gi, prefix_lens=pl)
    s = spx.make_sample_args(target, draft, ids, starts, ua, us, acc, tok)
    arena = torch.empty(binding.host_step_arena_size(a, s, k.numel()), dtype=torch.uint8, device=DEV)
    spx.verify_step_host(a, s, k.numel(), arena, status, torch.device(DEV, 0))
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    b.check(out.to(DEV), lse.to(DEV))
