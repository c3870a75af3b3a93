"""Query rows beside the append: buffers longer than the batch, rows that a call without a rotation ignores, in place and out of place."""
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


class _Call:
    """One append of m new rows each over a pool of 8-bit floats or of the rows' type."""

    def __init__(self, e4m3, dtype, hq=8, hkv=2, d=64, lens=(40, 7), m=(4, 3)):
        self.c = R.Cache(list(lens), hkv, d, 16, 16)
        k, v, strides, table, ks, vs = self.c.on(DEV)
        self.kw = dict(k_scales=ks, v_scales=vs)
        if not e4m3:
            k, v, self.kw = torch.zeros(k.shape, dtype=dtype, device=DEV), torch.zeros(v.shape, dtype=dtype, device=DEV), {}
        g = torch.Generator().manual_seed(3)
        self.total = sum(m)
        nk, nv = (torch.randn(self.total, hkv, d, generator=g).to(dtype).to(DEV) for _ in range(2))
        self.q = torch.randn(self.total + 5, hq, d, generator=g).to(dtype).to(DEV)
        self.args = (nk, nv, k, v, strides, table, _ints(lens), _ints([0, *np.cumsum(m).tolist()]), 16, self.c.num_pages)
        self.k = k

    def run(self, **kw):
        status = spx.kv_append(*self.args, **self.kw, **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == 0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("e4m3", [True, False])
def test_a_buffer_longer_than_the_batch(e4m3, dtype):
    """Rows kept for a larger batch: those of this one are rotated, the others left as they are; with and without q_out."""
    call = _Call(e4m3, dtype)
    n = call.total
    want = call.q[:n].clone()
    call.run(rope_base=10000.0, q_rows=want)                       # in place, rows as many as new ones
    assert not torch.equal(want, call.q[:n])
    held = call.q.clone()
    call.run(rope_base=10000.0, q_rows=held)
    assert torch.equal(held[:n], want) and torch.equal(held[n:], call.q[n:])
    for rows, out_rows in ((n, n + 2), (n + 5, n), (n + 5, n + 3)):
        src, out = call.q[:rows].clone(), torch.full((out_rows, *call.q.shape[1:]), 7.0, dtype=dtype, device=DEV)
        call.run(rope_base=10000.0, q_rows=src, q_out=out)
        assert torch.equal(out[:n], want) and (out[n:] == 7).all() and torch.equal(src, call.q[:rows])


@pytest.mark.parametrize("e4m3", [True, False])
def test_without_a_rotation_the_rows_are_ignored(e4m3):
    call = _Call(e4m3, BF)
    for q in (call.q, call.q[:2], call.q.view(-1, 64), call.q[:, :, :32].contiguous()):
        before = q.clone()
        call.run(q_rows=q)
        assert torch.equal(q, before)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("e4m3", [True, False])
def test_in_place_beside_and_behind_one_another(e4m3, dtype):
    """Many rows of many heads (each place read and written by one lane only), and two halves of one buffer."""
    call = _Call(e4m3, dtype, hq=32, hkv=4, d=128, lens=(300, 200, 17), m=(16, 12, 16))
    n = call.total
    want = torch.empty_like(call.q[:n])
    call.run(rope_base=500000.0, q_rows=call.q[:n], q_out=want)
    for _ in range(20):
        held = call.q[:n].clone()
        call.run(rope_base=500000.0, q_rows=held)
        assert torch.equal(held, want)
    both = torch.empty(2 * n, *call.q.shape[1:], dtype=dtype, device=DEV)
    for a, b in ((slice(0, n), slice(n, 2 * n)), (slice(n, 2 * n), slice(0, n))):
        both[a].copy_(call.q[:n])
        call.run(rope_base=500000.0, q_rows=both[a], q_out=both[b])
        assert torch.equal(both[b], want) and torch.equal(both[a], call.q[:n])


@pytest.mark.parametrize("e4m3", [True, False])
def test_shapes_that_do_not_fit_are_refused(e4m3):
    call = _Call(e4m3, BF)
    q, n = call.q, call.total
    for rows, out in ((q[:n - 1], None), (q.view(-1, 64), None), (q[:, :, :32].contiguous(), None), (q, q[:n - 1].clone()), (q, q[:, :4].contiguous()),
                      (q, q.float()), (None, q), (q[:, ::2], None), (q[:n + 2], q[1:n + 3])):
        with pytest.raises(spx.SpxError):
            spx.kv_append(*call.args, **call.kw, rope_base=10000.0, q_rows=rows, q_out=out)
    with pytest.raises(spx.SpxError):
        spx.kv_append(*call.args, **call.kw, q_rows=q, q_out=q.clone())    # no rotation: nothing would be written
    with pytest.raises(spx.SpxError):
        spx.kv_append(*call.args, **call.kw, rope_base=10000.0, q_rows=q.cpu())
