"""Several host threads, each with its own stream, workspace and outputs, make calls whose kernels need different amounts of
shared memory: every call is launched, and its results are those it has alone."""
import threading

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


def _in_threads(calls, times, monkeypatch):
    """Makes every call once through the binding on a stream of its own, then repeats its library call, and nothing else, in a thread of its
    own; returns the statuses that are not OK."""
    lib, made = spx.load_library(), []

    class Recorder:
        def __getattr__(self, name):
            def call(*args):
                made.append((getattr(lib, name), args))
                return made[-1][0](*args)
            return call

    loops = []
    with monkeypatch.context() as patch:
        patch.setattr(binding, "load_library", Recorder)
        for call in calls:
            with torch.cuda.stream(torch.cuda.Stream()):
                call()
            loops.append(made[-1])
    torch.cuda.synchronize()
    bad, go = [], threading.Barrier(len(loops))

    def body(fn, args):
        go.wait()
        bad.extend(s for s in (fn(*args) for _ in range(times)) if s != binding.OK)

    threads = [threading.Thread(target=body, args=x) for x in loops]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return bad


@pytest.mark.parametrize("e4m3", [True, False])
def test_fp32_attention_with_few_and_with_many_packed_rows(e4m3, monkeypatch):
    """The same kernel for 4 and for 64 packed rows of 32-bit pools, for 20 and for 32 of 8-bit ones."""
    hkv, d, page = 2, 128, 16
    calls, outs, wants = [], [], []
    for hq, m in ([(8, 5), (16, 4)] if e4m3 else [(2, 4), (16, 8)]) * 2:
        lens = [100, 40]
        c = R.Cache(lens, hkv, d, page, page, seed=hq)
        k, v, strides, table, ks, vs = c.on(DEV)
        kw = dict(k_scales=ks, v_scales=vs)
        if not e4m3:
            k, v = ((x.float() * s.repeat_interleave(page, 2)[..., None]).contiguous() for x, s in ((k, ks), (v, vs)))
            kw = {}
        q = torch.randn(2 * m, hq, d, generator=torch.Generator().manual_seed(hq)).to(DEV)
        args = (q, k, v, strides, table, _ints(lens), _ints([0, m, 2 * m]), hkv, page, c.num_pages)
        want, _, ws = spx.verify_attention(*args, max_q_len=m, **kw)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
        calls.append(lambda args=args, kw=dict(kw, out=out, lse=lse, max_q_len=m, ws=ws): spx.verify_attention(*args, **kw))
        outs.append(out)
        wants.append(want.clone())
    torch.cuda.synchronize()
    assert _in_threads(calls, 3000, monkeypatch) == []
    for out, want in zip(outs, wants):
        assert torch.equal(out, want)


def test_appends_with_small_and_with_large_scale_blocks(monkeypatch):
    """head_dim 128 with the angles of 64 and of 128 tokens in shared memory."""
    hkv, d, page = 2, 128, 128
    calls, states = [], []
    for sb in (64, 128, 32, 128):
        lens, m = [300, 40], [7, 3]
        c = R.Cache(lens, hkv, d, page, sb, seed=sb)
        c.k_scales[:], c.v_scales[:] = 0.25, 0.25
        k, v, strides, table, ks, vs = c.on(DEV)
        g = torch.Generator().manual_seed(sb)
        nk, nv = (torch.randn(10, hkv, d, generator=g).to(BF) for _ in range(2))
        R.append(c, nk, nv, lens, m, 10000.0)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        args = (nk.to(DEV), nv.to(DEV), k, v, strides, table, _ints(lens), _ints([0, *np.cumsum(m).tolist()]), page, c.num_pages)
        calls.append(lambda args=args, kw=dict(rope_base=10000.0, k_scales=ks, v_scales=vs, status=status): spx.kv_append(*args, **kw))
        states.append((c, k, v, ks, vs, status))
    torch.cuda.synchronize()
    assert _in_threads(calls, 3000, monkeypatch) == []
    for c, k, v, ks, vs, status in states:
        assert int(status.item()) == 0
        assert torch.equal(k.view(torch.uint8).cpu(), c.k) and torch.equal(v.view(torch.uint8).cpu(), c.v)
        assert torch.equal(ks.cpu(), c.k_scales) and torch.equal(vs.cpu(), c.v_scales)
