"""Rows of finite logits further apart than the largest float: their differences overflow, their log-probabilities, entropies and
order are those of the definition all the same."""
import math

import pytest
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("vocab", [40, 4096, 20000, 128256])
def test_a_forced_token_over_a_mask_of_the_lowest_value(vocab, dtype):
    """One or a few tokens at the type's largest value, all others at its lowest, in one sub-segment of the row and across them."""
    lo, hi = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = torch.full((5, vocab), lo)
    x[0, 0] = hi
    x[1, vocab - 1] = hi
    x[2, [1, vocab // 2]] = hi                       # two of them: ln 2
    x[3, vocab // 3] = hi
    x[3, : vocab // 4] = 0.0                         # and a stretch between the two
    x[4] = hi
    x[4, 3:] = lo
    logits = x.to(dtype)
    tokens = [0, vocab - 1, 1, vocab // 3, 2]
    want_lp = [0.0, 0.0, -math.log(2), 0.0, -math.log(3)]
    lp, ent, ids, top, ws = spx.token_logprobs(logits.to(DEV), torch.tensor(tokens, dtype=torch.int32, device=DEV), top_n=4)
    torch.cuda.synchronize()
    assert int(ws.status.item()) == 0
    for i, t in enumerate(tokens):
        w_lp, w_ent, w_ids, w_top = R.logprobs(logits[i].float().numpy(), t, 4)
        assert math.isclose(w_lp, want_lp[i], abs_tol=1e-12) and math.isclose(w_ent, -want_lp[i], abs_tol=1e-12)
        assert ids[i].tolist() == w_ids
        # log z and the entropy are ln 1, ln 2 or ln 3 of whole sums: half a step of fp32, and of the approximate power of two 2^-21
        assert abs(lp[i].item() - w_lp) <= 2.0 ** -20, (i, lp[i].item())
        assert abs(ent[i].item() - w_ent) <= 2.0 ** -20, (i, ent[i].item())
        for a, b in zip(top[i].tolist(), w_top):
            # differences below the lowest float are rounded to -inf
            assert abs(a - b) <= 2.0 ** -20 if b > -100 else (a == -math.inf or abs(a / b - 1) <= 2.0 ** -23), (i, a, b)
            if b < -2.0 ** 128:
                assert a == -math.inf
