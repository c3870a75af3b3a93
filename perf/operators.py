"""Cases and plain forms of three serving operators around the verify step:

  attn     verify attention over a paged cache held in e4m3, with one float32 scale per block of
           tokens and kv head;
  append   new K/V rows rotated to their positions, quantised and stored in that cache (the query rows
           rotated beside them);
  logprob  log-probabilities of given tokens, the entropy of their rows and the top alternatives.

`run` computes them with elementary torch operations in 32 bits (64 for the rotation's angles), or,
with `own`, by the calls a program makes of paper_2609_34370_b200.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------
# cases
# ------------------------------------------------------------------------------------------------
def _attn(name, batch, hq, hkv, d, page, sb, dist, lo, hi, ks, dtype="bf16", layout="HND"):
    return {"name": name, "op": "attn", "batch": batch, "hq": hq, "hkv": hkv, "d": d, "page": page, "sb": sb, "dist": dist,
            "lo": lo, "hi": hi, "ks": ks, "dtype": dtype, "layout": layout}


def _append(name, batch, mlo, mhi, hist, hq, hkv, d, page, sb, rope=500000.0, dtype="bf16", layout="HND"):
    return {"name": name, "op": "append", "batch": batch, "mlo": mlo, "mhi": mhi, "hist": hist, "hq": hq, "hkv": hkv, "d": d,
            "page": page, "sb": sb, "rope": rope, "dtype": dtype, "layout": layout}


def _logprob(name, rows, vocab, top, skip=0, dtype="bf16"):
    return {"name": name, "op": "logprob", "rows": rows, "vocab": vocab, "top": top, "skip": skip, "dtype": dtype}


def listed():
    return [
        # the fp32 configuration: four short requests, five positions each, exact arithmetic
        _attn("attn-tiny-f32", 4, 8, 2, 64, 16, 16, "uniform", 32, 256, "4", dtype="f32"),
        # plain decode (no drafts) of a few requests: one query position each, latency counts
        _attn("attn-decode", 8, 32, 8, 128, 16, 16, "uniform", 100, 2000, "0"),
        # the Llama-3-8B layer shape's verify step
        _attn("attn-8b", 64, 32, 8, 128, 16, 16, "uniform", 512, 4096, "5"),
        # the Llama-3-70B layer shape: mixed lengths, eight query heads per kv head, pool in token order
        _attn("attn-70b", 128, 64, 8, 128, 16, 16, "lognormal", 16, 8192, "3", layout="NHD"),
        # long contexts, nine positions each: the largest case
        _attn("attn-long", 16, 32, 8, 128, 32, 32, "const", 32768, 32768, "8"),
        # one new token for each of four requests, fp32 rows, blocks of half a page
        _append("append-one-f32", 4, 1, 1, 256, 8, 2, 64, 16, 8, rope=10000.0, dtype="f32"),
        # a verify step's new positions on the Llama-3-8B layer shape
        _append("append-step", 64, 6, 6, 4096, 32, 8, 128, 16, 16),
        # prompts of a few thousand tokens entering the cache
        _append("append-prompt", 6, 1000, 8191, 0, 32, 8, 128, 32, 32),
        # the fp32 configuration's rows on a small vocabulary
        _logprob("logprob-tiny-f32", 20, 1024, 5, dtype="f32"),
        # one request's bonus token: a single row, latency counts
        _logprob("logprob-one-row", 1, 128256, 5),
        # the rows of a 16-request verify step on a 32000-token vocabulary, unused slots behind the accepted ones
        _logprob("logprob-32k", 144, 32000, 10, skip=1),
        # the Llama-3-8B shape's verify step with twenty alternatives for every row
        _logprob("logprob-8b", 384, 128256, 20),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "append", "logprob"])
    hq, hkv, d = rng.choice([(32, 8, 128), (64, 8, 128), (8, 2, 64), (16, 16, 64), (28, 4, 128), (12, 4, 128), (8, 1, 64)])
    page = rng.choice([8, 16, 32, 64, 128])
    sb = rng.choice([s for s in (1, 4, 8, 16, 32, 64, 128) if s <= page])
    layout = rng.choice(["HND", "NHD"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "attn":
        batch = _log_int(rng, 1, 200)
        # padded lengths, heads and columns together stay below the largest listed case
        top = min(32768, (16 * 32768 * 8 * 128) // (batch * hkv * d))
        if dtype == "f32":
            top = min(top, 4096)
        hi = _log_int(rng, 17, top)
        lo = rng.randint(16, hi)
        most = min(15, 128 // (hq // hkv) - 1)
        ks = rng.choice([str(rng.randint(0, most)), "0", ",".join(str(k) for k in (0, 2, 4, 6) if k <= most)])
        c = _attn("", batch, hq, hkv, d, page, sb, "uniform", lo, hi, ks, dtype, layout)
    elif op == "append":
        batch = _log_int(rng, 1, 256)
        mhi = _log_int(rng, 1, max(2, 48000 // batch)) if rng.random() < 0.4 else rng.randint(1, 16)
        mhi = min(mhi, 8191)
        mlo = rng.randint(1, mhi)
        hist = _log_int(rng, 1, 4096) if batch * hkv * d <= 65536 else rng.randint(0, 200)
        c = _append("", batch, mlo, mhi, hist, hq, hkv, d, page, sb, rng.choice([10000.0, 500000.0]), dtype, layout)
    else:
        vocab = _log_int(rng, 500, 150000)
        rows = _log_int(rng, 1, min(1500, 384 * 128256 // vocab))
        if dtype == "f32":
            rows = (rows + 1) // 2
        c = _logprob("", rows, vocab, rng.randint(1, 20), rng.randint(0, 1), dtype)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------
# what a program has in hand
# ------------------------------------------------------------------------------------------------
def _fixed(case):
    """Lengths go by the case alone, so that work() can count them."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lens(case):
    """(cached tokens with the new ones, new positions) of every request."""
    rng, n = _fixed(case), case["batch"]
    if case["op"] == "append":
        m = [rng.randint(case["mlo"], case["mhi"]) for _ in range(n)]
        return [x + rng.randint(0, case["hist"]) for x in m], m
    ks = [int(k) for k in case["ks"].split(",")]
    m = [rng.choice(ks) + 1 for _ in range(n)]
    if case["dist"] == "lognormal":
        lens = [min(case["hi"], max(case["lo"], round(1024 * math.exp(rng.gauss(0.0, 1.0))))) for _ in range(n)]
    else:
        lens = [rng.randint(case["lo"], case["hi"]) for _ in range(n)]
    return [max(a, b) for a, b in zip(lens, m)], m


def _skips(case):
    """Rows without a token (slots behind the accepted ones)."""
    rng = _fixed(case)
    return [bool(case["skip"]) and rng.random() < 0.4 for _ in range(case["rows"])]


def _scale_of(amax):
    """2^e with the smallest e for which amax <= 448 * 2^e; 1 for an amax of zero."""
    f, x = torch.frexp(amax)
    e = torch.where(f > 0.875, x - 8, x - 9).clamp(-126, 120)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def _pool(case, num_pages, gen):
    """A pool [pages, heads, slots, d] of e4m3 codes (as bytes) and its scales, with channels of unequal size."""
    hkv, d, page, sb = case["hkv"], case["d"], case["page"], case["sb"]
    x = torch.randn(num_pages, hkv, page // sb, sb, d, generator=gen, device=DEV)
    x *= torch.exp(0.5 * torch.randn(hkv, 1, 1, d, generator=gen, device=DEV))
    scale = _scale_of(x.abs().amax((3, 4)))
    x = x.div_(scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(num_pages, hkv, page, d)
    if case["layout"] == "NHD":
        x = x.transpose(1, 2).contiguous().transpose(1, 2)
    return x.view(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    rng = random.Random(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    if case["op"] == "logprob":
        rows, vocab = case["rows"], case["vocab"]
        stride = -(-vocab // 8) * 8
        logits = torch.full((rows, stride), 1e4, dtype=TYPES[case["dtype"]], device=DEV)
        logits[:, :vocab] = 3.0 * torch.randn(rows, vocab, generator=gen, device=DEV)
        # tokens as sampling would give them: mostly likely ones (the largest of logits plus Gumbel noise)
        tokens = torch.empty(rows, dtype=torch.int32, device=DEV)
        for at in range(0, rows, 64):
            u = torch.rand(min(64, rows - at), vocab, generator=gen, device=DEV).clamp_(1e-20, 1 - 1e-7)
            tokens[at:at + 64] = (logits[at:at + 64, :vocab].float() - torch.log(-torch.log(u))).argmax(1)
        tokens[torch.tensor(_skips(case), device=DEV)] = -1
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
        return {"case": case, "logits": logits, "tokens": tokens, "ws": None, "logprobs": new(rows), "entropy": new(rows),
                "top_ids": new(rows, case["top"], dtype=torch.int32), "top_logprobs": new(rows, case["top"])}
    lens, m = _lens(case)
    page, hkv, hq, d = case["page"], case["hkv"], case["hq"], case["d"]
    need = [-(-n // page) for n in lens]
    num_pages = sum(need)
    order = list(range(num_pages))
    rng.shuffle(order)
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [-1] * (max(need) - n))
        at += n
    starts = [0]
    for x in m:
        starts.append(starts[-1] + x)
    total, kind = starts[-1], TYPES[case["dtype"]]
    k_cache, k_scales = _pool(case, num_pages, gen)
    v_cache, v_scales = _pool(case, num_pages, gen)
    s = {"case": case, "k_cache": k_cache, "v_cache": v_cache, "k_scales": k_scales, "v_scales": v_scales, "num_pages": num_pages,
         "strides": (k_cache.stride(0), k_cache.stride(1), k_cache.stride(2)), "table": ints(table), "lens": ints(lens), "starts": ints(starts),
         "most": max(m), "rows_r": ints([r for r, x in enumerate(m) for _ in range(x)]), "rows_j": ints([j for x in m for j in range(x)]),
         "q": torch.randn(total, hq, d, generator=gen, device=DEV).to(kind), "out": torch.empty(total, hq, d, dtype=kind, device=DEV)}
    if case["op"] == "attn":
        s |= {"ws": None, "lse": torch.empty(total, hq, dtype=torch.float32, device=DEV)}
    else:
        s |= {"status": torch.zeros(1, dtype=torch.int32, device=DEV), "new_k": torch.randn(total, hkv, d, generator=gen, device=DEV).to(kind),
              "new_v": torch.randn(total, hkv, d, generator=gen, device=DEV).to(kind)}
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2609_34370_b200 as spx
        return {"attn": _own_attn, "append": _own_append, "logprob": _own_logprob}[op](spx, state)
    return {"attn": _plain_attn, "append": _plain_append, "logprob": _plain_logprob}[op](state)


def _own_attn(spx, s):
    c = s["case"]
    out, lse, s["ws"] = spx.verify_attention(
        s["q"], s["k_cache"], s["v_cache"], s["strides"], s["table"], s["lens"], s["starts"], c["hkv"], c["page"], s["num_pages"],
        out=s["out"], lse=s["lse"], max_q_len=s["most"], ws=s["ws"], k_scales=s["k_scales"], v_scales=s["v_scales"])
    return {"out": out, "lse": lse}


def _own_append(spx, s):
    c = s["case"]
    spx.kv_append(s["new_k"], s["new_v"], s["k_cache"], s["v_cache"], s["strides"], s["table"], s["lens"], s["starts"], c["page"],
                  s["num_pages"], status=s["status"], rope_base=c["rope"], q_rows=s["q"], q_out=s["out"], k_scales=s["k_scales"],
                  v_scales=s["v_scales"])
    return _appended(s)


def _own_logprob(spx, s):
    c = s["case"]
    logprobs, entropy, top_ids, top_logprobs, s["ws"] = spx.token_logprobs(
        s["logits"], s["tokens"], top_n=c["top"], vocab=c["vocab"], logprobs=s["logprobs"], entropy=s["entropy"], top_ids=s["top_ids"],
        top_logprobs=s["top_logprobs"], ws=s["ws"])
    return {"logprobs": logprobs, "entropy": entropy, "top_ids": top_ids, "top_logprobs": top_logprobs}


def _appended(s):
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "k_scales": s["k_scales"], "v_scales": s["v_scales"], "q": s["out"]}


def _gathered(s, cache, scales):
    """Dequantised K or V of every request, [batch, hkv, tokens, d], padded to the longest block-table row."""
    c, table = s["case"], s["table"].long().clamp(min=0)
    x = cache.view(torch.uint8)[table].view(torch.float8_e4m3fn).float()          # [batch, pages, hkv, slots, d]
    x = x * scales[table].repeat_interleave(c["sb"], dim=3)[..., None]
    return x.transpose(1, 2).reshape(table.shape[0], c["hkv"], -1, c["d"])


def _plain_attn(s):
    c = s["case"]
    hkv, d, most = c["hkv"], c["d"], s["most"]
    group, batch = c["hq"] // hkv, c["batch"]
    k, v = _gathered(s, s["k_cache"], s["k_scales"]), _gathered(s, s["v_cache"], s["v_scales"])
    lens, starts = s["lens"].long(), s["starts"].long()
    t = torch.arange(k.shape[2], device=DEV)
    j = torch.arange(most, device=DEV)
    m = starts[1:] - starts[:-1]
    at = (starts[:-1, None] + j).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().view(batch, most, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(batch, hkv, most * group, d)
    x = torch.matmul(q, k.transpose(2, 3)).view(batch, hkv, most, group, -1) * (1.0 / math.sqrt(d))
    seen = t <= ((lens - m)[:, None] + j).clamp(max=lens[:, None] - 1)[..., None]  # [batch, most, tokens]
    x = torch.where(seen[:, None, :, None], x, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    v = torch.where((t < lens[:, None])[:, None, :, None], v, 0.0)
    o = torch.matmul(p.view(batch, hkv, most * group, -1), v).view(batch, hkv, most, group, d) / total
    rows = (s["rows_r"].long(), s["rows_j"].long())
    o = o.permute(0, 2, 1, 3, 4).reshape(batch, most, c["hq"], d)[rows]
    lse = (top + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(batch, most, c["hq"])[rows]
    return {"out": o.to(s["q"].dtype), "lse": lse}


def _rotated(x, t, base):
    """x [rows, heads, d] rotated to positions t [rows], rounded once to 32 bits."""
    d = x.shape[-1]
    f = torch.pow(base, -2.0 * torch.arange(d // 2, device=DEV, dtype=torch.float64) / d)
    a = (t.double()[:, None] * f)[:, None]
    lo, hi = x[..., : d // 2].double(), x[..., d // 2:].double()
    return torch.cat((lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()), -1).float()


def _plain_append(s):
    c = s["case"]
    page, sb, hkv, d, batch = c["page"], c["sb"], c["hkv"], c["d"], c["batch"]
    lens, starts, r, j = s["lens"].long(), s["starts"].long(), s["rows_r"].long(), s["rows_j"].long()
    m = starts[1:] - starts[:-1]
    t_row = (lens - m)[r] + j
    s["out"].copy_(_rotated(s["q"], t_row, c["rope"]))
    # the scale blocks that hold new tokens: [batch, blocks, sb] positions; a request with fewer blocks, or with a
    # last block that is not full, has its last one or last token again in the places left over
    blocks = (s["most"] - 1) // sb + 2
    block = torch.minimum(((lens - m) // sb)[:, None] + torch.arange(blocks, device=DEV), ((lens - 1) // sb)[:, None])
    t = torch.minimum(block[..., None] * sb + torch.arange(sb, device=DEV), (lens - 1)[:, None, None])
    back = t - (lens - m)[:, None, None]                                           # below zero: cached before
    pages = torch.gather(s["table"].long(), 1, (t // page).view(batch, -1)).view(t.shape)
    row = starts[:-1, None, None] + back.clamp(min=0)
    at_scale = (t % page) // sb
    for cache, scales, x in ((s["k_cache"], s["k_scales"], _rotated(s["new_k"], t_row, c["rope"])), (s["v_cache"], s["v_scales"], s["new_v"].float())):
        codes, scales = cache.view(torch.uint8).transpose(1, 2), scales.transpose(1, 2)   # [pages, slots, hkv, d], [pages, scales, hkv]
        was = codes[pages, t % page].view(torch.float8_e4m3fn).float() * scales[pages, at_scale][..., None]
        y = torch.where((back >= 0)[..., None, None], x[row], was)                 # [batch, blocks, sb, hkv, d]
        scale = _scale_of(y.abs().amax((2, 4)))                                    # [batch, blocks, hkv]
        codes[pages, t % page] = (y / scale[:, :, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        scales[pages[..., 0], at_scale[..., 0]] = scale
    return _appended(s)


def _plain_logprob(s):
    c = s["case"]
    x = s["logits"][:, :c["vocab"]].float()
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    z = e.sum(1, keepdim=True)
    lse = top + torch.log(z)
    entropy = torch.log(z[:, 0]) - (e * (x - top)).sum(1) / z[:, 0]
    # the largest logits first, the lowest id first among equals: one whole number orders both
    bits = x.view(torch.int32).long()
    key = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF)) * 2 ** 24 - torch.arange(c["vocab"], device=DEV)
    ids = torch.topk(key, c["top"], dim=1).indices
    skip = s["tokens"] < 0
    logprobs = (torch.gather(x, 1, s["tokens"].long().clamp(min=0)[:, None]) - lse)[:, 0]
    return {"logprobs": logprobs.masked_fill(skip, math.nan), "entropy": entropy.masked_fill(skip, math.nan),
            "top_ids": ids.int().masked_fill(skip[:, None], -1), "top_logprobs": (torch.gather(x, 1, ids) - lse).masked_fill(skip[:, None], math.nan)}


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "logprob":
        rows = case["rows"] - sum(_skips(case))
        return {"bytes": rows * case["vocab"] * size + case["rows"] * (4 + 4 + 4 + 8 * case["top"]), "flops": 6 * rows * case["vocab"]}
    lens, m = _lens(case)
    hq, hkv, d, sb = case["hq"], case["hkv"], case["d"], case["sb"]
    if case["op"] == "attn":
        cache = 2 * hkv * (d * sum(lens) + 4 * sum(-(-n // sb) for n in lens))
        seen = sum(k * (n - k) + k * (k + 1) // 2 for n, k in zip(lens, m))
        return {"bytes": cache + sum(m) * hq * (2 * d * size + 4), "flops": 4 * hq * d * seen}
    # new rows in, their codes out; the older tokens of each first block in; scales in and out; queries in and out
    old = sum((n - k) % sb for n, k in zip(lens, m))
    blocks = sum((n - 1) // sb - (n - k) // sb + 1 for n, k in zip(lens, m))
    return {"bytes": 2 * hkv * (d * (size * sum(m) + sum(m) + old) + 8 * blocks) + 2 * sum(m) * hq * d * size, "flops": 3 * sum(m) * d * (hq + hkv)}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "append": _exact_append, "logprob": _exact_logprob}[case["op"]](case, s)


def _exact_tokens(case, cache, scales, pages, n):
    """The first n cached tokens of a request in 64 bits: [n, hkv, d]."""
    codes = cache.view(torch.uint8)[pages].view(torch.float8_e4m3fn).double()
    codes = codes.permute(0, 2, 1, 3).reshape(-1, case["hkv"], case["d"])[:n]
    per_token = scales[pages].double().permute(0, 2, 1).reshape(-1, case["hkv"])
    return codes * per_token.repeat_interleave(case["sb"], dim=0)[:n, :, None]


def _exact_attn(case, s):
    lens, m = _lens(case)
    hq, hkv, d, q0 = case["hq"], case["hkv"], case["d"], 0
    if sum(lens) * hkv * d > 2 ** 30:
        return None
    outs, lses = [], []
    for r, (n, k) in enumerate(zip(lens, m)):
        pages = s["table"][r, : -(-n // case["page"])].long()
        keys = _exact_tokens(case, s["k_cache"], s["k_scales"], pages, n)
        values = _exact_tokens(case, s["v_cache"], s["v_scales"], pages, n)
        q = s["q"][q0:q0 + k].double().view(k, hkv, hq // hkv, d)
        x = torch.einsum("jghd,tgd->jght", q, keys) / math.sqrt(d)
        hidden = torch.arange(n, device=DEV)[None] > torch.arange(n - k, n, device=DEV)[:, None]
        x.masked_fill_(hidden[:, None, None], -math.inf)
        lse = torch.logsumexp(x, -1)
        outs.append(torch.einsum("jght,tgd->jghd", torch.exp(x - lse[..., None]), values).reshape(k, hq, d))
        lses.append(lse.reshape(k, hq))
        q0 += k
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_turn(x, t, base):
    half = x.shape[-1] // 2
    angle = t.double()[:, None, None] * (float(base) ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half))
    z = torch.complex(x[..., :half].double(), x[..., half:].double()) * torch.polar(torch.ones_like(angle), angle)
    return torch.cat((z.real, z.imag), -1)


def _exact_append(case, s):
    lens, m = _lens(case)
    page, sb, q0 = case["page"], case["sb"], 0
    if sum(m) // sb + 2 * len(m) > 4000:
        return None
    limit = torch.tensor(448.0, dtype=torch.float64, device=DEV)
    turned = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for r, (n, k) in enumerate(zip(lens, m)):
        where = torch.arange(n - k, n, device=DEV)
        turned[q0:q0 + k] = _exact_turn(s["q"][q0:q0 + k], where, case["rope"])
        new = {"k": _exact_turn(s["new_k"][q0:q0 + k], where, case["rope"]), "v": s["new_v"][q0:q0 + k].double()}
        table = s["table"][r].tolist()
        for b in range((n - k) // sb, (n - 1) // sb + 1):
            t0, t1 = b * sb, min(n, b * sb + sb)
            p, slot = table[t0 // page], t0 % page
            for which in ("k", "v"):
                codes, scales = s[which + "_cache"], s[which + "_scales"]
                held = codes.view(torch.uint8)[p, :, slot:slot + t1 - t0].view(torch.float8_e4m3fn).double() * scales[p, :, slot // sb].double()[:, None, None]
                y = held.transpose(0, 1).clone()                                    # [tokens, hkv, d]
                a = max(t0, n - k)
                y[a - t0:] = new[which][a - (n - k):t1 - (n - k)].float().double()
                peak = y.abs().amax((0, 2))
                scale = torch.where(peak > 0, torch.exp2(torch.ceil(torch.log2(peak / limit) - 1e-12)), 1.0)
                codes.view(torch.uint8)[p, :, slot:slot + t1 - t0] = (y / scale[:, None]).float().to(torch.float8_e4m3fn).view(torch.uint8).transpose(0, 1)
                scales[p, :, slot // sb] = scale.float()
        q0 += k
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "k_scales": s["k_scales"].double(), "v_scales": s["v_scales"].double(), "q": turned}


def _exact_logprob(case, s):
    n, top = case["rows"], case["top"]
    out = {"logprobs": torch.full((n,), math.nan, dtype=torch.float64, device=DEV), "entropy": torch.full((n,), math.nan, dtype=torch.float64, device=DEV),
           "top_ids": None, "top_logprobs": torch.full((n, top), math.nan, dtype=torch.float64, device=DEV)}
    tokens = s["tokens"].tolist()
    for i, token in enumerate(tokens):
        if token < 0:
            continue
        lp = torch.log_softmax(s["logits"][i, : case["vocab"]].double(), 0)
        out["logprobs"][i] = lp[token]
        out["entropy"][i] = -(lp.exp() * lp).sum()
        out["top_logprobs"][i] = torch.sort(lp, descending=True).values[:top]
    return out
