"""Log-probabilities of given tokens, entropies and top alternatives against a plain 64-bit reference."""
import math

import numpy as np
import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32
U = 2.0 ** -24


def _check(logits, tokens, top_n, vocab, got):
    """Bounds: e^(x - m) in fp32 is off by |x - m| * 2u (the difference's and the conversion to powers of two's rounding) + 2^-21 (the
    approximate power of two); with terms below e^-90 of the sum not counting, |x - m| <= 90.  Sums of at most 2^14 fp32 terms before they
    are merged in 64 bits, in pairs of a lane's few hundred: 2^10 u.  Together c = 2^-15 on every sum of exponentials without the largest
    logit's own one, so log_z = log1p(rest) is off by c * rest / (1 + rest), and the expectation by 2 c * E|x - m|.  Results are rounded to fp32."""
    lp, ent, ids, top = (t.cpu().numpy() for t in got)
    c = 2.0 ** -15
    for i, t in enumerate(tokens):
        if t < 0 or t >= vocab:
            assert math.isnan(lp[i]) and math.isnan(ent[i]) and (ids[i] == -1).all() and np.isnan(top[i]).all(), i
            continue
        x = logits[i, :vocab].float().cpu().numpy()
        w_lp, w_ent, w_ids, w_top = R.logprobs(x, t, top_n)
        assert ids[i].tolist() == w_ids, (i, ids[i].tolist(), w_ids)
        if math.isnan(w_ent):
            assert math.isnan(lp[i]) and math.isnan(ent[i]) and np.isnan(top[i]).all()
            continue
        x = x.astype(np.float64)
        rest_part = -math.expm1(w_top[0]) if top_n else 1.0     # rest / (1 + rest)
        mean = float((np.exp(x - x.max()) * np.where(np.isinf(x), 0, x.max() - x)[...]).sum() / np.exp(x - x.max()).sum())
        # an exponential below the smallest normal fp32 number may vanish, the product with its x - m with it
        tol = c * rest_part + vocab * 2.0 ** -119
        assert lp[i] == w_lp or abs(lp[i] - w_lp) <= tol + U * abs(w_lp), (i, lp[i], w_lp)
        assert abs(ent[i] - w_ent) <= tol + 2 * c * mean + U * w_ent, (i, ent[i], w_ent)
        for a, b in zip(top[i], w_top):
            assert (math.isnan(b) and math.isnan(a)) or a == b or abs(a - b) <= tol + U * abs(b), (i, a, b)


def _run(logits, tokens, top_n, vocab=None, **kw):
    *got, ws = spx.token_logprobs(logits.to(DEV), torch.tensor(tokens, dtype=torch.int32, device=DEV), top_n=top_n, vocab=vocab, **kw)
    torch.cuda.synchronize()
    return got, int(ws.status.item())


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab,rows,top_n", [(1, 3, 1), (2, 2, 2), (7, 5, 7), (8, 4, 3), (500, 9, 32), (1024, 20, 5), (2049, 3, 20), (4095, 6, 1),
                                             (16384, 2, 10), (16385, 3, 32), (32000, 40, 10), (128256, 4, 20), (150001, 2, 32), (1000003, 1, 5)])
def test_matches_the_reference(vocab, rows, top_n, dtype):
    g = torch.Generator().manual_seed(vocab)
    stride = -(-vocab // 8) * 8 + 8
    logits = torch.full((rows, stride), 1e4)
    logits[:, :vocab] = 3 * torch.randn(rows, vocab, generator=g)
    logits = logits.to(dtype)
    tokens = torch.randint(0, vocab, (rows,), generator=g).tolist()
    tokens[0] = vocab - 1
    got, status = _run(logits, tokens, top_n, vocab)
    assert status == 0
    _check(logits, tokens, top_n, vocab, got)


@pytest.mark.parametrize("dtype", [BF, F])
def test_many_rows(dtype):
    g = torch.Generator().manual_seed(1)
    logits = (2 * torch.randn(700, 1000, generator=g)).to(dtype)
    tokens = torch.randint(-1, 1000, (700,), generator=g).tolist()
    got, status = _run(logits, tokens, 6)
    assert status == 0
    _check(logits, tokens, 6, 1000, got)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab", [3000, 40000])
def test_ties_go_to_the_lowest_id(vocab, dtype):
    """Rows of a few distinct values (hundreds of ties at the top), all equal, -0 beside +0, the ties at the very end."""
    g = torch.Generator().manual_seed(2)
    logits = torch.randint(0, 4, (6, vocab), generator=g).float()
    logits[1] = 1.5
    logits[2] = torch.where(torch.arange(vocab) % 3 == 0, -0.0, 0.0)
    logits[3] = -5.0
    logits[3, -20:] = 2.0
    logits[4] = torch.arange(vocab, 0, -1) // 7
    logits[5] = torch.arange(vocab) // 5
    logits = logits.to(dtype)
    got, status = _run(logits, [5, 0, vocab - 1, vocab - 1, 3, 9], 32)
    assert status == 0
    _check(logits, [5, 0, vocab - 1, vocab - 1, 3, 9], 32, vocab, got)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab", [304, 20000])
def test_masked_and_extreme_rows(vocab, dtype):
    """-inf masks (all but few, all), the type's lowest value as a mask, +inf, NaN, huge and tiny spreads, near-certain rows."""
    g = torch.Generator().manual_seed(3)
    low = torch.finfo(dtype).min
    x = torch.randn(12, vocab, generator=g).to(dtype).float()
    x[0, torch.arange(vocab) % 50 != 7] = -math.inf
    x[1] = -math.inf
    x[2, 10:] = low
    x[3] = low
    x[4, 99] = math.inf
    x[5, 123] = math.nan
    x[5, 7] = math.inf
    x[6] *= 1e4
    x[7] *= 1e-6
    x[8, 200] = 40.0
    x[9, 0] = 16.0
    x[10] = -math.inf
    x[10, vocab - 1] = 3.0
    x[11, 5] = torch.finfo(dtype).max
    logits = x.to(dtype)
    tokens = [7, 3, 4, 250, 99, 123, 0, 1, 200, 0, vocab - 1, 5]
    got, status = _run(logits, tokens, 8)
    assert status == 0
    _check(logits, tokens, 8, vocab, got)
    tokens = [8, 3, 11, 0, 98, 0, 17, 2, 4, 250, 0, 6]
    got, status = _run(logits, tokens, 8)
    _check(logits, tokens, 8, vocab, got)


@pytest.mark.parametrize("dtype", [BF, F])
def test_near_certain_rows_keep_relative_accuracy(dtype):
    """A top logit so far above the rest that 1 + rest rounds to 1 in fp32: log-probability -rest, not 0."""
    vocab = 9000
    logits = torch.zeros(4, vocab)
    for i, gap in enumerate((18.0, 22.0, 30.0, 12.0)):
        logits[i, 4567] = gap
    logits = logits.to(dtype)
    (lp, ent, ids, top), status = _run(logits, [4567] * 4, 2)
    for i in range(4):
        want = R.logprobs(logits[i].float().numpy(), 4567, 2)
        assert abs(lp[i].item() / want[0] - 1) < 2.0 ** -14 and abs(ent[i].item() / want[1] - 1) < 2.0 ** -13
        assert ids[i].tolist() == want[2]


@pytest.mark.parametrize("dtype", [BF, F])
def test_bad_tokens_are_flagged_and_unused_rows_are_not_read(dtype):
    g = torch.Generator().manual_seed(4)
    logits = torch.randn(6, 800, generator=g).to(dtype)
    logits[2] = math.nan
    tokens = [3, -1, -1, 800, -2, 799]
    got, status = _run(logits, tokens, 3)
    assert status == spx.DEV_BAD_TOKEN
    _check(logits, tokens, 3, 800, got)
    got, status = _run(logits, [3, -1, -1, -1, -1, 799], 3)
    assert status == 0


def test_optional_outputs():
    logits = torch.randn(5, 640, generator=torch.Generator().manual_seed(5)).to(BF).to(DEV)
    tok = torch.tensor([1, 2, 3, 4, 5], dtype=torch.int32, device=DEV)
    lp, ent, ids, top, ws = spx.token_logprobs(logits, tok, top_n=4)
    a = spx.token_logprobs(logits, tok, want_entropy=False, ws=ws)
    assert a[1] is None and a[2] is None and a[3] is None and torch.equal(a[0], lp)
    b = spx.token_logprobs(logits, None, top_n=4, ws=ws)
    assert b[0] is None and torch.equal(b[1], ent) and torch.equal(b[2], ids) and torch.equal(b[3], top)
    c = spx.token_logprobs(logits, None, ws=ws)
    assert torch.equal(c[1], ent)
    d = spx.token_logprobs(logits[:0], tok[:0], top_n=4, ws=ws)
    assert d[0].shape == (0,) and d[2].shape == (0, 4)
    one = spx.token_logprobs(logits[3:4], tok[3:4], top_n=4, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(one[2], ids[3:4]) and torch.equal(one[0], lp[3:4])


def test_same_results_from_call_to_call_and_in_a_graph():
    logits = (3 * torch.randn(40, 33000, generator=torch.Generator().manual_seed(6))).to(BF).to(DEV)
    tok = torch.arange(40, dtype=torch.int32, device=DEV)
    *a, ws = spx.token_logprobs(logits, tok, top_n=20)
    a = [t.clone() for t in a]
    outs = [torch.empty_like(t) for t in a]
    kw = dict(top_n=20, logprobs=outs[0], entropy=outs[1], top_ids=outs[2], top_logprobs=outs[3], ws=ws)
    ws.buf.fill_(255)
    spx.token_logprobs(logits, tok, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spx.token_logprobs(logits, tok, **kw)
    for _ in range(2):
        for t in outs:
            t.zero_()
        ws.buf.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, outs))


def test_rows_past_32_bit_offsets():
    vocab, stride = 1000, 1 << 24
    rows = 140
    logits = torch.zeros(rows * stride - stride + vocab, dtype=BF, device=DEV)
    view = logits.as_strided((rows, vocab), (stride, 1))
    fill = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(8)).to(BF)
    view.copy_(fill.to(DEV))
    tokens = [i * 7 for i in range(rows)]
    *got, ws = spx.token_logprobs(view, torch.tensor(tokens, dtype=torch.int32, device=DEV), top_n=3)
    torch.cuda.synchronize()
    _check(fill, tokens, 3, vocab, got)
