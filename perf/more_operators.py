"""Cases and plain forms of three operators that bring prompts into the paged cache and share them:

  prompt  causal attention of whole prompts, or of chunks of them, packed one behind the other, over the
          paged cache that their rows have entered (any number of query rows a request);
  prefix  verify attention of requests that share a long prefix: the prefix is read once for its group;
  append  K/V and query rows rotated to positions of several axes (time, height, width) as they enter
          the cache, prompts as well as single tokens.

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
def _prompt(name, batch, mlo, mhi, hlo, hhi, hq, hkv, d, page, pool="rows", dtype="bf16", layout="HND"):
    """batch requests of mlo..mhi new tokens behind hlo..hhi cached ones."""
    return {"name": name, "op": "prompt", "batch": batch, "mlo": mlo, "mhi": mhi, "hlo": hlo, "hhi": hhi, "hq": hq, "hkv": hkv,
            "d": d, "page": page, "sb": page, "pool": pool, "dtype": dtype, "layout": layout}


def _prefix(name, groups, size, plo, phi, lo, hi, ks, hq, hkv, d, page, pool="rows", dtype="bf16", layout="HND"):
    """groups of `size` requests; plo..phi shared tokens, lo..hi of their own, k draft tokens among them."""
    return {"name": name, "op": "prefix", "groups": groups, "size": size, "plo": plo, "phi": phi, "lo": lo, "hi": hi, "ks": ks,
            "hq": hq, "hkv": hkv, "d": d, "page": page, "sb": page, "pool": pool, "dtype": dtype, "layout": layout}


def _append(name, batch, mlo, mhi, hist, hq, hkv, d, page, sections, interleaved=False, rope=1000000.0, pool="rows", dtype="bf16",
            layout="HND"):
    return {"name": name, "op": "append", "batch": batch, "mlo": mlo, "mhi": mhi, "hist": hist, "hq": hq, "hkv": hkv, "d": d,
            "page": page, "sb": page, "sections": sections, "interleaved": interleaved, "rope": rope, "pool": pool, "dtype": dtype,
            "layout": layout}


def listed():
    return [
        # the fp32 configuration's heads: four short prompts, exact arithmetic
        _prompt("prompt-tiny-f32", 4, 1, 200, 0, 60, 8, 2, 64, 16, dtype="f32"),
        # one short question on the Llama-3-8B layer shape: latency counts
        _prompt("prompt-short", 1, 97, 97, 0, 0, 32, 8, 128, 16),
        # a ragged batch of prompts, some of a single token, seven query heads per kv head, pool in token order
        _prompt("prompt-ragged", 24, 1, 2000, 0, 0, 28, 4, 128, 16, layout="NHD"),
        # a chunk of a long prompt behind what is cached of it: few rows, a long axis
        _prompt("prompt-chunk", 1, 500, 500, 30000, 30000, 32, 8, 128, 32),
        # prompts that entered an 8-bit cache
        _prompt("prompt-8bit", 6, 1000, 4000, 0, 0, 32, 8, 128, 16, pool="e4m3"),
        # two whole prompts of 8192 tokens on the Llama-3-8B layer shape: the largest case
        _prompt("prompt-long", 2, 8192, 8192, 0, 0, 32, 8, 128, 32),
        # the fp32 configuration: twelve requests behind one prompt, five positions each
        _prefix("prefix-tiny-f32", 1, 12, 300, 300, 5, 100, "4", 8, 2, 64, 16, dtype="f32"),
        # the Llama-3-8B layer shape's verify step behind one system prompt
        _prefix("prefix-8b", 1, 64, 4096, 4096, 100, 1000, "5", 32, 8, 128, 16),
        # eight tenants of sixteen requests with prompts of their own, 8-bit cache, mixed draft counts, Llama-3-70B heads
        _prefix("prefix-tenants-8bit", 8, 16, 500, 4000, 16, 800, "0,2,4", 64, 8, 128, 32, pool="e4m3"),
        # one new token for each of four image requests, fp32 rows
        _append("append-one-f32", 4, 1, 1, 256, 8, 2, 64, 16, "8,12,12", rope=10000.0, dtype="f32"),
        # prompts with images entering the cache, sections interleaved
        _append("append-image", 5, 200, 3000, 100, 28, 4, 128, 16, "24,20,20", interleaved=True, layout="NHD"),
        # video prompts entering an 8-bit cache
        _append("append-video-8bit", 4, 2000, 6000, 0, 32, 8, 128, 32, "16,24,24", pool="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_FLOPS = 4 * 32 * 128 * 8192 * 8193     # of the largest listed case
MOST_CACHE = 2 ** 28                        # elements of all requests' K, each padded to the longest


def draw(rng):
    while True:
        case = _draw(rng)
        if case is not None:
            del case["name"]
            return case


def _draw(rng):
    op = rng.choice(["prompt", "prompt", "prefix", "prefix", "append"])
    hq, hkv, d = rng.choice([(32, 8, 128), (64, 8, 128), (8, 2, 64), (16, 16, 64), (28, 4, 128), (12, 4, 128), (8, 1, 64)])
    page = rng.choice([8, 16, 32, 64, 128])
    layout = rng.choice(["HND", "NHD"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    pool = rng.choice(["rows", "rows", "e4m3"])
    if op == "prompt":
        batch = _log_int(rng, 1, 48)
        mhi = _log_int(rng, 1, 8192 if dtype == "bf16" else 1500)
        mlo = rng.randint(1, mhi)
        hhi = rng.choice([0, 0, _log_int(rng, 1, 30000 if dtype == "bf16" else 4000)])
        case = _prompt("", batch, mlo, mhi, rng.randint(0, hhi), hhi, hq, hkv, d, page, pool, dtype, layout)
        wide = batch * (mhi + hhi)
        most = MOST_FLOPS if dtype == "bf16" else MOST_FLOPS // 16
    elif op == "prefix":
        groups = _log_int(rng, 1, 12)
        size = _log_int(rng, 2, 128 // groups if groups < 9 else 14)
        phi = _log_int(rng, 64, 16384 if dtype == "bf16" else 2000)
        hi = _log_int(rng, 1, 2000)
        most_k = min(15, 128 // (hq // hkv) - 1)
        ks = rng.choice([str(rng.randint(0, most_k)), "0", ",".join(str(k) for k in (0, 2, 4, 6) if k <= most_k)])
        case = _prefix("", groups, size, rng.randint(16, phi), phi, rng.randint(1, hi), hi, ks, hq, hkv, d, page, pool, dtype, layout)
        wide = groups * size * (phi + hi + 16)
        most = MOST_FLOPS if dtype == "bf16" else MOST_FLOPS // 16
    else:
        batch = _log_int(rng, 1, 128)
        mhi = _log_int(rng, 1, max(2, 20000 // batch)) if rng.random() < 0.6 else rng.randint(1, 16)
        interleaved = rng.choice([False, True])
        if interleaved:   # every axis but the first has at most its turns
            b, c = rng.randint(1, d // 6), rng.randint(1, d // 6)
            sections = rng.choice([f"{d // 2 - b - c},{b},{c}", {128: "24,20,20", 64: "12,10,10"}[d], f"{d // 2 - b},{b}"])
        else:
            b = rng.randint(1, d // 2 - 2)
            c = rng.randint(1, d // 2 - 1 - b)
            sections = rng.choice([f"{d // 2 - b - c},{b},{c}", {128: "16,24,24", 64: "8,12,12"}[d], f"{b},{d // 2 - b}", str(d // 2)])
        hist = _log_int(rng, 1, 2000)
        case = _append("", batch, rng.randint(1, mhi), mhi, hist, hq, hkv, d, page, sections, interleaved,
                       rng.choice([10000.0, 1000000.0]), pool, dtype, layout)
        wide, most = batch * (mhi + hist), MOST_FLOPS
    if wide * hkv * d > MOST_CACHE or work(case)["flops"] > most:
        return None
    return case


# ------------------------------------------------------------------------------------------------
# what a program has in hand
# ------------------------------------------------------------------------------------------------
def _fixed(case):
    """Lengths go by the case alone, so that work() can count them."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lens(case):
    """Per request: cached tokens with the new ones, new positions; per group: shared tokens (of `prefix` cases)."""
    rng = _fixed(case)
    if case["op"] == "prompt":
        m = [rng.randint(case["mlo"], case["mhi"]) for _ in range(case["batch"])]
        return [x + rng.randint(case["hlo"], case["hhi"]) for x in m], m, []
    if case["op"] == "append":
        m = [rng.randint(case["mlo"], case["mhi"]) for _ in range(case["batch"])]
        return [x + rng.randint(0, case["hist"]) for x in m], m, []
    shared = [rng.randint(case["plo"], case["phi"]) for _ in range(case["groups"])]
    ks = [int(k) for k in case["ks"].split(",")]
    lens, m = [], []
    for p in shared:
        for _ in range(case["size"]):
            m.append(rng.choice(ks) + 1)
            # the shared tokens end inside a page at times: its rest is each request's own, and so is the page
            lens.append(p + max(m[-1], rng.randint(case["lo"], case["hi"])))
    return lens, m, shared


def _positions(case, lens, m, rng):
    """Positions of the new rows on every axis: text counts all axes up together, an image or a frame of a
    video lies on a grid of rows and columns behind them."""
    axes = len(case["sections"].split(","))
    out = [[] for _ in range(axes)]
    for n, k in zip(lens, m):
        at, left = n - k, k
        while left:
            text = min(left, rng.randint(1, 60))
            for axis in out:
                axis.extend(range(at, at + text))
            at, left = at + text, left - text
            frames, high, wide = rng.choice([1, 1, 4]), rng.randint(4, 32), rng.randint(4, 32)
            cells = [(f, h, w) for f in range(frames) for h in range(high) for w in range(wide)][:left]
            for cell in cells:
                for axis, place in zip(out, cell):
                    axis.append(at + place)
            at, left = at + max([max(cell) for cell in cells], default=-1) + 1, left - len(cells)
    return out


def _scale_of(amax):
    """2^e with the smallest e for which amax <= 448 * 2^e; 1 for an amax of zero."""
    f, x = torch.frexp(amax)
    e = torch.where(f > 0.875, x - 8, x - 9).clamp(-126, 120)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def _pool(case, num_pages, gen):
    """A pool [pages, heads, slots, d], of the rows' type or of 8-bit floats with their scales."""
    hkv, d, page, sb = case["hkv"], case["d"], case["page"], case["sb"]
    x = torch.randn(num_pages, hkv, page, d, generator=gen, device=DEV)
    scale = None
    if case["pool"] == "e4m3":
        x = (x * torch.exp(0.5 * torch.randn(hkv, 1, d, generator=gen, device=DEV))).view(num_pages, hkv, page // sb, sb, d)
        scale = _scale_of(x.abs().amax((3, 4)))
        x = x.div_(scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(num_pages, hkv, page, d)
    else:
        x = x.to(TYPES[case["dtype"]])
    if case["layout"] == "NHD":
        x = x.transpose(1, 2).contiguous().transpose(1, 2)
    return (x.view(torch.float8_e4m3fn) if scale is not None else x), scale


def prepare(case, seed):
    gen = torch.Generator(DEV).manual_seed(seed)
    rng = random.Random(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    lens, m, shared = _lens(case)
    page, hkv, hq, d = case["page"], case["hkv"], case["hq"], case["d"]
    # block-table rows: the whole pages of a group's prefix, then the request's own
    common = [shared[r // case["size"]] // page for r in range(len(lens))] if shared else [0] * len(lens)
    need = [-(-n // page) for n in lens]
    firsts = [p // page for p in shared]
    num_pages = sum(need) - sum(common) + sum(firsts)
    order = list(range(num_pages))
    rng.shuffle(order)
    at = 0
    heads = []
    for n in firsts:
        heads.append(order[at:at + n])
        at += n
    table = []
    for r, (n, c) in enumerate(zip(need, common)):
        table.append((heads[r // case["size"]] if shared else []) + order[at:at + n - c] + [-1] * (max(need) - n))
        at += n - c
    starts = [0]
    for x in m:
        starts.append(starts[-1] + x)
    total, kind = starts[-1], TYPES[case["dtype"]]
    k_cache, k_scales = _pool(case, num_pages, gen)
    v_cache, v_scales = _pool(case, num_pages, gen)
    s = {"case": case, "k_cache": k_cache, "v_cache": v_cache, "k_scales": k_scales, "v_scales": v_scales, "num_pages": num_pages,
         "strides": (k_cache.stride(0), k_cache.stride(1), k_cache.stride(2)), "table": ints(table), "lens": ints(lens), "starts": ints(starts),
         "n": lens, "m": m, "most": max(m), "q": torch.randn(total, hq, d, generator=gen, device=DEV).to(kind),
         "out": torch.empty(total, hq, d, dtype=kind, device=DEV), "ws": None}
    if case["op"] == "append":
        s |= {"status": torch.zeros(1, dtype=torch.int32, device=DEV), "positions": ints(_positions(case, lens, m, rng)),
              "sections": [int(x) for x in case["sections"].split(",")], "new_k": torch.randn(total, hkv, d, generator=gen, device=DEV).to(kind),
              "new_v": torch.randn(total, hkv, d, generator=gen, device=DEV).to(kind)}
    else:
        s["lse"] = torch.empty(total, hq, dtype=torch.float32, device=DEV)
    if shared:
        s |= {"groups": ints([g * case["size"] for g in range(len(shared) + 1)]), "prefix_lens": ints(shared)}
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2609_34370_b200 as spx
        return {"prompt": _own_prompt, "prefix": _own_prefix, "append": _own_append}[op](spx, state)
    return {"prompt": _plain_attention, "prefix": _plain_attention, "append": _plain_append}[op](state)


def _own_prompt(spx, s):
    c = s["case"]
    out, lse, s["ws"] = spx.prompt_attention(
        s["q"], s["k_cache"], s["v_cache"], s["strides"], s["table"], s["lens"], s["starts"], c["hkv"], c["page"], s["num_pages"],
        out=s["out"], lse=s["lse"], ws=s["ws"], k_scales=s["k_scales"], v_scales=s["v_scales"])
    return {"out": out, "lse": lse}


def _own_prefix(spx, s):
    c = s["case"]
    out, lse, s["ws"] = spx.verify_attention(
        s["q"], s["k_cache"], s["v_cache"], s["strides"], s["table"], s["lens"], s["starts"], c["hkv"], c["page"], s["num_pages"],
        out=s["out"], lse=s["lse"], max_q_len=s["most"], ws=s["ws"], k_scales=s["k_scales"], v_scales=s["v_scales"],
        group_indptr=s["groups"], prefix_lens=s["prefix_lens"])
    return {"out": out, "lse": lse}


def _own_append(spx, s):
    c = s["case"]
    spx.kv_append(s["new_k"], s["new_v"], s["k_cache"], s["v_cache"], s["strides"], s["table"], s["lens"], s["starts"], c["page"],
                  s["num_pages"], status=s["status"], rope_base=c["rope"], q_rows=s["q"], q_out=s["out"], k_scales=s["k_scales"],
                  v_scales=s["v_scales"], positions=s["positions"], rope_sections=s["sections"],
                  rope_interleaved=c["interleaved"])
    return _appended(s)


def _appended(s):
    out = {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "q": s["out"]}
    if s["k_scales"] is not None:
        out |= {"k_scales": s["k_scales"], "v_scales": s["v_scales"]}
    return out


def _tokens(c, s, cache, scales, r, n):
    """The first n cached tokens of request r as [hkv, n, d] floats."""
    pages = s["table"][r, : -(-n // c["page"])].long()
    if scales is None:
        x = cache[pages].float()
    else:
        x = cache.view(torch.uint8)[pages].view(torch.float8_e4m3fn).float()
        x = x * scales[pages].repeat_interleave(c["sb"], dim=2)[..., None]
    return x.transpose(0, 1).reshape(c["hkv"], -1, c["d"])[:, :n]


def _plain_attention(s):
    """Request by request, the query rows in blocks that keep the scores below 2^28 numbers."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    group, q0 = hq // hkv, 0
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    for r, (n, m) in enumerate(zip(s["n"], s["m"])):
        k, v = _tokens(c, s, s["k_cache"], s["k_scales"], r, n), _tokens(c, s, s["v_cache"], s["v_scales"], r, n)
        step = max(1, 2 ** 28 // (hq * n))
        for j in range(0, m, step):
            rows = min(step, m - j)
            seen = n - m + j + rows                                                  # tokens the last of these rows sees
            q = s["q"][q0 + j:q0 + j + rows].float().view(rows, hkv, group, d).permute(1, 0, 2, 3).reshape(hkv, rows * group, d)
            x = torch.matmul(q, k[:, :seen].transpose(1, 2)).view(hkv, rows, group, seen) * (1.0 / math.sqrt(d))
            hidden = torch.arange(seen, device=DEV) > torch.arange(n - m + j, seen, device=DEV)[:, None]
            x.masked_fill_(hidden[:, None], -math.inf)
            top = x.amax(-1, keepdim=True)
            p = torch.exp(x - top)
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(hkv, rows * group, seen), v[:, :seen]).view(hkv, rows, group, d) / total
            out[q0 + j:q0 + j + rows] = o.permute(1, 0, 2, 3).reshape(rows, hq, d)
            lse[q0 + j:q0 + j + rows] = (top + torch.log(total)).squeeze(-1).permute(1, 0, 2).reshape(rows, hq)
        q0 += m
    return {"out": out, "lse": lse}


def _axis_of_pairs(c):
    """The axis each pair of elements turns by: sections one behind the other, or dealt out in turn, where an axis
    but the first has no pairs behind its section and the first has what is left."""
    sections = [int(x) for x in c["sections"].split(",")]
    if not c["interleaved"]:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    axes = len(sections)
    return [i % axes if i < axes * sections[i % axes] else 0 for i in range(c["d"] // 2)]


def _angles(s):
    """[rows, d / 2] in 64 bits."""
    c = s["case"]
    f = torch.pow(c["rope"], -2.0 * torch.arange(c["d"] // 2, device=DEV, dtype=torch.float64) / c["d"])
    return s["positions"][torch.tensor(_axis_of_pairs(c), device=DEV)].t().double() * f


def _rotated(x, angles):
    """x [rows, heads, d] turned, rounded once to 32 bits."""
    half, a = x.shape[-1] // 2, angles[:, None]
    lo, hi = x[..., :half].double(), x[..., half:].double()
    return torch.cat((lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()), -1).float()


def _plain_append(s):
    c = s["case"]
    page, sb, hkv, d, batch = c["page"], c["sb"], c["hkv"], c["d"], c["batch"]
    lens, starts = s["lens"].long(), s["starts"].long()
    m = starts[1:] - starts[:-1]
    angles = _angles(s)
    s["out"].copy_(_rotated(s["q"], angles))
    new = ((s["k_cache"], s["k_scales"], _rotated(s["new_k"], angles)), (s["v_cache"], s["v_scales"], s["new_v"].float()))
    if c["pool"] == "rows":
        r = torch.repeat_interleave(torch.arange(batch, device=DEV), m, output_size=s["q"].shape[0])
        t = (lens - m - starts[:-1])[r] + torch.arange(s["q"].shape[0], device=DEV)
        pages = s["table"].long()[r, t // page]
        for cache, _, x in new:
            cache.transpose(1, 2)[pages, t % page] = x.to(cache.dtype)
        return _appended(s)
    # the scale blocks that hold new tokens: [batch, blocks, sb] positions; a request with fewer blocks, or with a
    # last block that is not full, has its last one or last token again in the places left over
    blocks = (max(s["m"]) - 1) // sb + 2
    block = torch.minimum(((lens - m) // sb)[:, None] + torch.arange(blocks, device=DEV), ((lens - 1) // sb)[:, None])
    t = torch.minimum(block[..., None] * sb + torch.arange(sb, device=DEV), (lens - 1)[:, None, None])
    back = t - (lens - m)[:, None, None]                                           # below zero: cached before
    pages = torch.gather(s["table"].long(), 1, (t // page).view(batch, -1)).view(t.shape)
    row = starts[:-1, None, None] + back.clamp(min=0)
    at_scale = (t % page) // sb
    for cache, scales, x in new:
        codes, scales = cache.view(torch.uint8).transpose(1, 2), scales.transpose(1, 2)   # [pages, slots, hkv, d], [pages, scales, hkv]
        was = codes[pages, t % page].view(torch.float8_e4m3fn).float() * scales[pages, at_scale][..., None]
        y = torch.where((back >= 0)[..., None, None], x[row], was)                 # [batch, blocks, sb, hkv, d]
        scale = _scale_of(y.abs().amax((2, 4)))                                    # [batch, blocks, hkv]
        codes[pages, t % page] = (y / scale[:, :, None, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        scales[pages[..., 0], at_scale[..., 0]] = scale
    return _appended(s)


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    kept = 1 if case["pool"] == "e4m3" else size                                    # bytes of a cached element
    lens, m, shared = _lens(case)
    hq, hkv, d, sb = case["hq"], case["hkv"], case["d"], case["sb"]
    if case["op"] == "append":
        # new rows in, stored out; query rows in and out; positions; 8-bit pools: older tokens of each first block in, scales in and out
        rows = sum(m)
        extra = 0
        if case["pool"] == "e4m3":
            old = sum((n - k) % sb for n, k in zip(lens, m))
            extra = 2 * hkv * (d * old + 8 * sum((n - 1) // sb - (n - k) // sb + 1 for n, k in zip(lens, m)))
        axes = len(case["sections"].split(","))
        return {"bytes": 2 * hkv * d * rows * (size + kept) + 2 * rows * hq * d * size + 4 * axes * rows + extra, "flops": 3 * rows * d * (hq + hkv)}
    tokens = sum(lens) - (case["size"] - 1) * sum(shared) if shared else sum(lens)  # a shared token is read once
    scales = 4 * (tokens // sb) if case["pool"] == "e4m3" else 0
    seen = sum(k * (n - k) + k * (k + 1) // 2 for n, k in zip(lens, m))
    return {"bytes": 2 * hkv * (d * kept * tokens + scales) + sum(m) * hq * (2 * d * size + 4), "flops": 4 * hq * d * seen}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(case, s) if case["op"] == "append" else _exact_attention(case, s)


def _exact_rows(case, cache, scales, table, n):
    """The first n tokens of the pages of a block-table row in 64 bits: [n, hkv, d]."""
    pages = table[: (n + case["page"] - 1) // case["page"]].long()
    if scales is None:
        held = cache[pages].double()
    else:
        held = cache.view(torch.uint8)[pages].view(torch.float8_e4m3fn).double()
        held = held.view(len(pages), case["hkv"], -1, case["sb"], case["d"]) * scales[pages].double()[..., None, None]
        held = held.view(len(pages), case["hkv"], case["page"], case["d"])
    return held.permute(0, 2, 1, 3).reshape(-1, case["hkv"], case["d"])[:n]


def _exact_attention(case, s):
    if work(case)["flops"] > 2 * MOST_FLOPS:
        return None
    lens, m, _ = _lens(case)
    hq, hkv, d, q0 = case["hq"], case["hkv"], case["d"], 0
    outs, lses = [], []
    for r, (n, k) in enumerate(zip(lens, m)):
        keys = _exact_rows(case, s["k_cache"], s["k_scales"], s["table"][r], n)
        values = _exact_rows(case, s["v_cache"], s["v_scales"], s["table"][r], n)
        for g in range(hkv):
            heads = slice(g * (hq // hkv), (g + 1) * (hq // hkv))
            for j in range(0, k, 1024):
                q = s["q"][q0 + j:q0 + min(k, j + 1024), heads].double()
                x = torch.einsum("jhd,td->jht", q, keys[:, g]) / math.sqrt(d)
                last = n - k + j + torch.arange(q.shape[0], device=DEV)
                x = x.masked_fill((torch.arange(n, device=DEV)[None] > last[:, None])[:, None], -math.inf)
                lse = torch.logsumexp(x, -1)
                outs.append((r, g, j, torch.einsum("jht,td->jhd", torch.exp(x - lse[..., None]), values[:, g])))
                lses.append(lse)
        q0 += k
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    total = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    base = [sum(m[:r]) for r in range(len(m))]
    for (r, g, j, o), lse in zip(outs, lses):
        rows = slice(base[r] + j, base[r] + j + o.shape[0])
        heads = slice(g * (hq // hkv), (g + 1) * (hq // hkv))
        out[rows, heads], total[rows, heads] = o, lse
    return {"out": out, "lse": total}


def _exact_turn(case, x, places):
    """x [rows, heads, d] as complex numbers times e^(i angle); places [axes, rows]."""
    half = x.shape[-1] // 2
    sections = [int(n) for n in case["sections"].split(",")]
    axes = len(sections)
    angle = torch.empty(x.shape[0], half, dtype=torch.float64, device=DEV)
    for i in range(half):
        if case["interleaved"]:
            axis = i % axes
            if axis and i >= axes * sections[axis] or not axis:
                axis = 0
        else:
            axis = next(a for a in range(axes) if i < sum(sections[: a + 1]))
        angle[:, i] = places[axis].double() * float(case["rope"]) ** (-i / half)
    z = torch.complex(x[..., :half].double(), x[..., half:].double()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat((z.real, z.imag), -1)


def _exact_append(case, s):
    lens, m, _ = _lens(case)
    page, sb, q0 = case["page"], case["sb"], 0
    if sum(m) // sb + 2 * len(m) > 6000:
        return None
    turned = _exact_turn(case, s["q"], s["positions"])
    new_k, new_v = _exact_turn(case, s["new_k"], s["positions"]), s["new_v"].double()
    if case["pool"] == "rows":
        pools = {w: s[w + "_cache"].double() for w in "kv"}
        for r, (n, k) in enumerate(zip(lens, m)):
            t = torch.arange(n - k, n, device=DEV)
            pages = s["table"][r].long()[t // page]
            pools["k"].transpose(1, 2)[pages, t % page] = new_k[q0:q0 + k]
            pools["v"].transpose(1, 2)[pages, t % page] = new_v[q0:q0 + k]
            q0 += k
        return {"k_cache": pools["k"], "v_cache": pools["v"], "q": turned}
    limit = torch.tensor(448.0, dtype=torch.float64, device=DEV)
    for r, (n, k) in enumerate(zip(lens, m)):
        table = s["table"][r].tolist()
        for b in range((n - k) // sb, (n - 1) // sb + 1):
            t0, t1 = b * sb, min(n, b * sb + sb)
            p, slot = table[t0 // page], t0 % page
            for which, rows in (("k", new_k), ("v", new_v)):
                codes, scales = s[which + "_cache"], s[which + "_scales"]
                held = codes.view(torch.uint8)[p, :, slot:slot + t1 - t0].view(torch.float8_e4m3fn).double() * scales[p, :, slot // sb].double()[:, None, None]
                y = held.transpose(0, 1).clone()                                    # [tokens, hkv, d]
                a = max(t0, n - k)
                y[a - t0:] = rows[q0 + a - (n - k):q0 + t1 - (n - k)].float().double()
                peak = y.abs().amax((0, 2))
                scale = torch.where(peak > 0, torch.exp2(torch.ceil(torch.log2(peak / limit) - 1e-12)), 1.0)
                codes.view(torch.uint8)[p, :, slot:slot + t1 - t0] = (y / scale[:, None]).float().to(torch.float8_e4m3fn).view(torch.uint8).transpose(0, 1)
                scales[p, :, slot // sb] = scale.float()
        q0 += k
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "q": turned, "k_scales": s["k_scales"].double(), "v_scales": s["v_scales"].double()}
