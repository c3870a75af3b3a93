"""Plain 64-bit references of attention for prompts, behind shared prefixes, and of rotations on several axes.

Tolerances count roundings.  With u = half a step of the rows' type (bf16 2^-8, fp32 2^-24, relative) and A = sum_t p_t |v_t|:
  * an output is rounded once (u |out|) and, for 16-bit rows, each weight is rounded once before it meets V (u A);
  * a score is a sum of D fp32 products: off by (D + 3) 2^-24 scale sum_d |q_d k_d| at most (products of 16-bit elements are
    exact, so half of that); e^x turns that into a relative error of the weights, once in the numerator and once in the sum;
    2^-22 of a weight are ex2's, and n 2^-24 of a sum of n weights its own;
  * the log-sum-exp is off by the scores' error, the sum's, and one rounding of itself to fp32 with two for the logarithm.
"""
import math

import numpy as np
import torch

import e4m3_util as R
import paper_2609_34370_b200 as spx

DEV = "cuda"


class Batch:
    """Requests of lens[r] cached tokens, m[r] of them new, over pools of `kind` ("rows": the rows' type, "e4m3").  Pages are
    dealt out at random from a pool that is larger than needed; every slot that no request owns is `poison`."""

    def __init__(self, lens, m, hq, hkv, d, page, dtype=torch.bfloat16, kind="rows", layout="HND", sb=None, seed=0, poison=math.nan,
                 shared=None, spread=1.0, tail_rows=0, scale_kind="any"):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.m, self.hq, self.hkv, self.d, self.page, self.dtype, self.kind = lens, m, hq, hkv, d, page, dtype, kind
        self.sb = sb or page
        shared = shared or []                  # (first request, one past the last, tokens)
        need = [-(-n // page) for n in lens]
        total = sum(need) + 3
        order = torch.randperm(total, generator=g).tolist()
        self.table = torch.full((len(lens), max(need + [1]) + 1), -1, dtype=torch.int32)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        for a, b, n in shared:
            self.table[a:b, : n // page] = self.table[a, : n // page].clone()
        self.num_pages = total
        self.k, self.v = (spread * torch.randn(total, hkv, page, d, generator=g) for _ in range(2))
        self.k_scales = self.v_scales = None
        if kind == "e4m3":
            for w in "kv":
                x = getattr(self, w).double().clamp(-5.5, 5.5).numpy() * 80
                codes = torch.from_numpy(R.encode(x))
                scales = (torch.exp(0.7 * torch.randn(total, hkv, page // self.sb, generator=g)) / 80).float()
                if scale_kind == "powers":           # as the append writes them
                    scales = torch.exp2(torch.round(torch.log2(scales)))
                elif scale_kind == "mixed":          # powers of two, others, zeros
                    pick = torch.randint(0, 3, scales.shape, generator=g)
                    scales = torch.where(pick == 0, scales, torch.where(pick == 1, torch.exp2(torch.round(torch.log2(scales))), torch.zeros(())))
                setattr(self, w, codes)
                setattr(self, w + "_scales", scales)
        else:
            self.k, self.v = self.k.to(dtype), self.v.to(dtype)
        owned = torch.zeros(total, page, dtype=torch.bool)
        for r, n in enumerate(lens):
            for t in range(n):
                owned[self.table[r, t // page], t % page] = True
        for x in (self.k, self.v):
            x.transpose(1, 2)[~owned] = 0x7F if kind == "e4m3" else poison
        self.layout = layout
        self.starts = [0]
        for x in m:
            self.starts.append(self.starts[-1] + x)
        self.q = torch.randn(self.starts[-1] + tail_rows, hq, d, generator=g).to(dtype)

    def device(self):
        move = (lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)) if self.layout == "NHD" else (lambda x: x)
        k, v = (move(x).to(DEV) if self.layout == "HND" else move(x.to(DEV)) for x in (self.k, self.v))
        if self.kind == "e4m3":
            k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        scales = {} if self.k_scales is None else dict(k_scales=self.k_scales.to(DEV), v_scales=self.v_scales.to(DEV))
        return (self.q.to(DEV), k, v, tuple(k.stride()[:3]), self.table.to(DEV), ints(self.lens), ints(self.starts), self.hkv, self.page,
                self.num_pages), scales

    def tokens(self, which, r):
        n = self.lens[r]
        pages = self.table[r, : -(-n // self.page)].long()
        x = getattr(self, which)[pages]
        if self.kind == "e4m3":
            x = torch.from_numpy(R.decode(x)) * getattr(self, which + "_scales")[pages].double().repeat_interleave(self.sb, 2)[..., None]
        return x.double().transpose(0, 1).reshape(self.hkv, -1, self.d)[:, :n]

    def exact(self, r, scale=None):
        """out, lse and their tolerances of request r, [m, hq, d] and [m, hq]."""
        n, m, G = self.lens[r], self.m[r], self.hq // self.hkv
        scale = scale or 1 / math.sqrt(self.d)
        k, v = self.tokens("k", r).to(DEV), self.tokens("v", r).to(DEV)
        q = self.q[self.starts[r]:self.starts[r + 1]].double().to(DEV).view(m, self.hkv, G, self.d)
        x = scale * torch.einsum("jhgd,htd->jhgt", q, k)
        size = scale * torch.einsum("jhgd,htd->jhgt", q.abs(), k.abs())
        hidden = torch.arange(n, device=DEV)[None] > (n - m + torch.arange(m, device=DEV))[:, None]
        x = x.masked_fill(hidden[:, None, None], -math.inf)
        size = size.masked_fill(hidden[:, None, None], 0.0)
        lse = torch.logsumexp(x, -1)
        p = torch.exp(x - lse[..., None])
        v = torch.where(torch.isfinite(v), v, 0.0) if not torch.isfinite(v).all() else v
        out, mass = torch.einsum("jhgt,htd->jhgd", p, v), torch.einsum("jhgt,htd->jhgd", p, v.abs())
        u = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[self.dtype]
        score = (self.d + 3) * 2.0 ** -24 * size.amax(-1)          # of any weight's exponent
        sums = 2.0 ** -22 + n * 2.0 ** -24
        weight = u if self.dtype == torch.bfloat16 else 0.0
        tol = u * out.abs() + (weight + 2 * score[..., None] + 2 * sums) * mass * 1.01 + 1e-30
        tol_lse = score + sums + 3 * 2.0 ** -24 * (lse.abs() + 1)
        shape = (m, self.hq)
        return out.reshape(*shape, self.d), lse.reshape(shape), tol.reshape(*shape, self.d), tol_lse.reshape(shape)

    def check(self, out, lse, requests=None, scale=None):
        for r in range(len(self.lens)) if requests is None else requests:
            if self.m[r] == 0:
                continue
            o, l, to, tl = self.exact(r, scale)
            rows = slice(self.starts[r], self.starts[r + 1])
            bad = ~((out[rows].double() - o).abs() <= to)
            assert not bool(bad.any()), (r, self.lens[r], self.m[r], int(bad.sum()), float(((out[rows].double() - o).abs() / to).nan_to_num(1e9).max()),
                                         bad.nonzero()[:4].tolist())
            if lse is not None:
                bad = ~((lse[rows].double() - l).abs() <= tl)
                assert not bool(bad.any()), (r, "lse", float(((lse[rows].double() - l).abs() / tl).nan_to_num(1e9).max()), bad.nonzero()[:4].tolist())


def prompt(b, **kw):
    args, scales = b.device()
    out, lse, ws = spx.prompt_attention(*args, **scales, **kw)
    torch.cuda.synchronize()
    return out, lse, int(ws.status.item())


def verify(b, groups=None, **kw):
    args, scales = b.device()
    if groups is not None:
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        kw |= dict(group_indptr=ints(groups[0]), prefix_lens=ints(groups[1]))
    kw.setdefault("max_q_len", max(b.m))
    out, lse, ws = spx.verify_attention(*args, **scales, **kw)
    torch.cuda.synchronize()
    return out, lse, int(ws.status.item())


def axis_of(i, sections, interleaved):
    if interleaved:
        a = i % len(sections)
        return a if i < len(sections) * sections[a] else 0
    return next(a for a in range(len(sections)) if i < sum(sections[: a + 1]))


def turned(x, positions, base, sections, interleaved):
    """x [rows, heads, d] in 64 bits (numpy), turned to positions [axes, rows]."""
    half = x.shape[-1] // 2
    angle = np.stack([positions[axis_of(i, sections, interleaved)] * base ** (-2.0 * i / (2 * half)) for i in range(half)], -1)[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate((lo * np.cos(angle) - hi * np.sin(angle), hi * np.cos(angle) + lo * np.sin(angle)), -1)
