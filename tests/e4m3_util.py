"""Plain 64-bit references of the 8-bit cache and of token log-probabilities (CPU, numpy and torch).

The format's 127 non-negative values are tabulated from its definition and rounding is a search in the
table, so no conversion of torch's or of the library's is relied on.
"""
import math

import numpy as np
import torch


def _values():
    v = [m / 8 * 2.0 ** -6 for m in range(8)]
    for e in range(1, 16):
        v += [(1 + m / 8) * 2.0 ** (e - 7) for m in range(8)]
    return np.array(v[:-1])   # the last pattern is NaN


VALUES = _values()
DECODE = np.concatenate((VALUES, [np.nan], -VALUES, [np.nan]))


def decode(codes: torch.Tensor) -> np.ndarray:
    return DECODE[codes.detach().cpu().contiguous().view(torch.uint8).numpy()]


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest value, ties to the even pattern; not finite: NaN."""
    a = np.abs(x)
    fine = np.isfinite(a)
    assert (a[fine] <= 448).all()
    hi = np.clip(np.searchsorted(VALUES, np.where(fine, a, 0.0)), 1, len(VALUES) - 1)
    lo = hi - 1
    d_lo, d_hi = a - VALUES[lo], VALUES[hi] - a
    pick = np.where((d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0)), hi, lo)
    return np.where(fine, pick | (np.signbit(x).astype(np.int64) << 7), 0x7F).astype(np.uint8)


def scale_of(amax: float) -> float:
    if amax == 0:
        return 1.0
    e = -126
    while 448 * 2.0 ** e < amax:
        e += 1
    return 2.0 ** e


def rotate(x: np.ndarray, t: int, base: float) -> np.ndarray:
    """x [heads, d] in 64 bits, turned to position t."""
    half = x.shape[-1] // 2
    a = t * base ** (-np.arange(half) / half)
    lo, hi = x[:, :half], x[:, half:]
    return np.concatenate((lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)), -1)


class Cache:
    """Pools [pages, heads, slots, d] of codes (either layout in memory), scales, a table with gaps; on the CPU."""

    def __init__(self, lens, hkv, d, page, sb, layout="HND", seed=0, spread=1.0, tables_from=2):
        g = torch.Generator().manual_seed(seed)
        self.hkv, self.d, self.page, self.sb, self.layout = hkv, d, page, sb, layout
        need = [-(-max(n, 1) // page) for n in lens]
        self.num_pages = sum(need) * tables_from + 1
        order = torch.randperm(self.num_pages, generator=g).tolist()
        self.table = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        shape = (self.num_pages, hkv, page, d)
        self.k, self.v, self.k_scales, self.v_scales = None, None, None, None
        for which in "kv":
            codes = torch.randint(0, 127, shape, generator=g, dtype=torch.int32).to(torch.uint8)
            codes |= (torch.randint(0, 2, shape, generator=g, dtype=torch.int32) << 7).to(torch.uint8)
            # normal values: the code of a normal draw
            x = torch.randn(shape, generator=g).double().clamp(-5.5, 5.5).numpy() * 80
            codes = torch.from_numpy(encode(x))
            scales = torch.exp(spread * torch.randn(self.num_pages, hkv, page // sb, generator=g)) / 80
            setattr(self, which, codes)
            setattr(self, which + "_scales", scales.float())

    def poison(self, lens):
        """NaN codes in every slot past a request's length and in unused pages, NaN scales in wholly unused blocks."""
        live = torch.zeros(self.num_pages, self.page, dtype=torch.bool)
        for r, n in enumerate(lens):
            for t in range(n):
                live[self.table[r, t // self.page], t % self.page] = True
        dead = ~live[:, None, :, None].expand(-1, self.hkv, -1, self.d)
        block_dead = ~live.view(self.num_pages, -1, self.sb).any(-1)[:, None].expand(-1, self.hkv, -1)
        for which in "kv":
            getattr(self, which)[dead] = 0x7F
            getattr(self, which + "_scales")[block_dead] = math.nan

    def on(self, device):
        """(k_cache, v_cache, strides, table, k_scales, v_scales) as device tensors; strides (page, head, token)."""
        out = []
        for codes in (self.k, self.v):
            x = codes.to(device)
            if self.layout == "NHD":
                x = x.transpose(1, 2).contiguous().transpose(1, 2)
            out.append(x.view(torch.float8_e4m3fn))
        s = out[0].stride()
        return (*out, (s[0], s[1], s[2]), self.table.to(device), self.k_scales.clone().to(device), self.v_scales.clone().to(device))

    def token_scales(self, which, r, n):
        """The scales of the first n tokens of request r: [n, hkv] in 64 bits."""
        pages = self.table[r, : -(-n // self.page)].long()
        return np.repeat(getattr(self, which + "_scales")[pages].double().numpy(), self.sb, axis=2).transpose(0, 2, 1).reshape(-1, self.hkv)[:n]

    def values(self, which, r, n):
        """The first n tokens of request r: [n, hkv, d] in 64 bits."""
        codes, scales = getattr(self, which), getattr(self, which + "_scales")
        pages = self.table[r, : -(-n // self.page)].long()
        x = decode(codes[pages]) * np.repeat(scales[pages].double().numpy(), self.sb, axis=2)[..., None]
        return x.transpose(0, 2, 1, 3).reshape(-1, self.hkv, self.d)[:n]


def attention(c: Cache, q: torch.Tensor, lens, m, sm_scale=0.0):
    """(out, lse, spread, reach) in 64 bits; spread = sum_t p_t |v_t| and reach = max_t sum_d |q_d k_td| sm_scale, for
    the bounds on rounding errors.

    For 16-bit types spread also holds what lies below the range the kernel keeps for a row.  A weight times its
    token's V scale is held in binary16 pieces with a least step of 2^-16 under a reference that puts the largest of
    the row at 2^10 at least: half a step, 2^-17, is 2^-27 of the largest, and a token's value is its code times that.  Divided by the
    2^-7 that attention_bounds multiplies spread with for these types it is added here: 2^-20 max_t(p_t scale_t)
    sum_t |code_t|.  reach likewise holds the queries' least step: an element is the sum of an e4m3 and an e5m2 value under a scale that
    puts the row's largest at 2^7 at least; below 2^-6 the first is off by 2^-10 at most and the second takes
    three bits of that, so an element is off by 2^-13, 2^-20 of the largest: 2^-20 max|q| max_t sum_d |k_td| sm_scale, divided by the
    (d + 4) 2^-22 that scores are bounded with.
    """
    hq, d = q.shape[1], q.shape[2]
    g = hq // c.hkv
    scale = sm_scale or 1 / math.sqrt(d)
    outs, lses, spreads, reaches = [], [], [], []
    q0 = 0
    for r, (n, k) in enumerate(zip(lens, m)):
        keys, values = c.values("k", r, n), c.values("v", r, n)
        x = q[q0:q0 + k].double().numpy().reshape(k, c.hkv, g, d)
        for j in range(k):
            seen = n - k + j + 1
            kk, vv = keys[:seen], values[:seen]
            s = np.einsum("ghd,tgd->ght", x[j], kk) * scale
            top = s.max(-1, keepdims=True)
            e = np.exp(s - top)
            z = e.sum(-1, keepdims=True)
            p = e / z
            outs.append(np.einsum("ght,tgd->ghd", p, vv).reshape(hq, d))
            below = 0.0
            if q.dtype == torch.bfloat16:
                sc = c.token_scales("v", r, seen)
                codes = np.abs(vv) / np.where(sc > 0, sc, 1.0)[..., None]
                below = (2.0 ** -20 * (p * sc.T[:, None]).max(-1)[..., None] * codes.sum(0)[:, None]).reshape(hq, d)
            lses.append((top + np.log(z)).reshape(hq))
            spreads.append(np.einsum("ght,tgd->ghd", p, np.abs(vv)).reshape(hq, d) + below)
            reach = np.einsum("ghd,tgd->ght", np.abs(x[j]), np.abs(kk)).max(-1) * scale
            if q.dtype == torch.bfloat16:
                reach = reach + 2.0 ** -20 / ((d + 4) * 2.0 ** -22) * np.abs(x[j]).max(-1) * np.abs(kk).sum(-1).max(0)[:, None] * scale
            reaches.append(reach.reshape(hq))
        q0 += k
    return tuple(np.stack(v) if v else np.zeros((0,)) for v in (outs, lses, spreads, reaches))


def attention_bounds(out, spread, reach, n_max, d, dtype):
    """Bounds of |out - exact| and |lse - exact|, with u = 2^-24 the rounding of one fp32 operation (tensor cores may drop
    two more bits of a partial sum: 4u).
      a score: d products added, the K scale and the two factors of the exponent: (d + 4) * 4u * reach;
      a weight: twice that (its own score and the reference's) + 2^-20 for the approximate power of two;
      a sum of n weights or products: n * u relative at most, in whatever order (pairs of partial sums included);
      weights are rounded to 8 significant bits before the value product for 16-bit types: 2^-8;
      the output's own rounding: eps / 2.
    """
    u = 2.0 ** -24
    score = (d + 4) * 4 * u * reach
    weight = 2 * score + 2.0 ** -20 + 4 * n_max * u
    if dtype == torch.bfloat16:
        weight = weight + 2.0 ** -8
    # a normalised sum: the numerator's and the denominator's relative errors add
    return torch.finfo(dtype).eps / 2 * np.abs(out) + (weight[..., None] + weight[..., None]) * spread, 2 * score + 2.0 ** -20 + 4 * n_max * u + 2 * u * (1 + reach)


def append(c: Cache, new_k, new_v, lens, m, base=0.0, skip=()):
    """Appends in place (CPU, block by block)."""
    q0 = 0
    for r, (n, k) in enumerate(zip(lens, m)):
        if r not in skip:
            rows = {"k": new_k[q0:q0 + k].double().numpy().copy(), "v": new_v[q0:q0 + k].double().numpy()}
            if base:
                rows["k"] = np.stack([rotate(rows["k"][j], n - k + j, base) for j in range(k)]).astype(np.float32).astype(np.float64)
            for which in "kv":
                codes, scales = getattr(c, which), getattr(c, which + "_scales")
                for b in range((n - k) // c.sb, (n - 1) // c.sb + 1):
                    t0, t1 = b * c.sb, min(n, (b + 1) * c.sb)
                    page, slot = int(c.table[r, t0 // c.page]), t0 % c.page
                    old = decode(codes[page, :, slot:slot + t1 - t0]) * scales[page, :, slot // c.sb].double().numpy()[:, None, None]
                    y = old.transpose(1, 0, 2).copy()                       # [tokens, hkv, d]
                    a = max(t0, n - k)
                    y[a - t0:] = rows[which][a - (n - k):t1 - (n - k)]
                    for h in range(c.hkv):
                        mag = np.abs(y[:, h])
                        scale = scale_of(float(mag[np.isfinite(mag)].max(initial=0.0)))
                        codes[page, h, slot:slot + t1 - t0] = torch.from_numpy(encode(y[:, h] / scale))
                        scales[page, h, slot // c.sb] = scale
        q0 += k


def logprobs(x: np.ndarray, token, top_n):
    """(logprob, entropy, ids, their log-probabilities) of one row in 64 bits."""
    x = x.astype(np.float64)
    v = len(x)
    # NaN above +inf, equal values by the lowest id
    nan = np.isnan(x)
    order = np.lexsort((np.arange(v), -np.where(nan, 0.0, x), ~nan))[:top_n].tolist()
    ids = order + [-1] * (top_n - len(order))
    if nan.any() or (x == np.inf).any() or (x == -np.inf).all():
        return math.nan, math.nan, ids, [math.nan] * top_n
    top = x.max()
    first = int(np.argmax(x))
    rest = np.exp(np.delete(x, first) - top)
    log_z = math.log1p(math.fsum(rest.tolist()))
    lp = x - top - log_z
    p = np.exp(lp)
    ent = -math.fsum((p[p > 0] * lp[p > 0]).tolist())
    return lp[token], ent, ids, [lp[i] if i >= 0 else math.nan for i in ids]
