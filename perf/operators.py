"""The paged-cache and token-scoring operators as cases that can be timed and
compared: a key/value cache quantised as it is written and read back, decode
attention over it, decode attention of a batch whose rows share a prefix that
is stored once, and log probabilities of given tokens with entropy and the most
likely alternatives.

listed() and draw() give cases (dicts of plain values), prepare() what a decoder
holds before the call, run() one pass (plain torch in 32 bits, or with `own` the
library's entry points), work() what a pass cannot do without, exact() the same
results in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 64  # tokens of a page
NEG = -math.inf


def listed():
    return [
        # one decode step of the 768 px workload, batch 8: a token per head joins its list
        dict(name="cache_token_b8_int8", kind="cache", type="int8", lists=8, heads=32, dim=128,
             tokens=1, start=2400, ragged=False),
        # one decode step of 256 guided class-conditional sequences, heads of 64
        dict(name="cache_token_b256_fp4", kind="cache", type="fp4", lists=256, heads=20, dim=64,
             tokens=1, start=576, ragged=False),
        # whole images (2352 tokens and shorter ones) enter an empty cache and are read back
        dict(name="cache_image_b16_int8", kind="cache", type="int8", lists=16, heads=32, dim=128,
             tokens=2352, start=0, ragged=True),
        # one image at a time at the 768 px shape: 32 heads, local ones with a window of two rows
        dict(name="attn_768_b1_int8", kind="attn", type="int8", batch=1, heads=32, group=1,
             dim=128, lo=300, hi=2480, window=98, prefixes=0, prefix=0, shared_share=0),
        # batch 64 with lengths from 64 to 1024, the spread of the stress workload
        dict(name="attn_768_b64_int8", kind="attn", type="int8", batch=64, heads=32, group=1,
             dim=128, lo=64, hi=1024, window=0, prefixes=0, prefix=0, shared_share=0),
        # grouped query heads over long caches (interleaved text and images) in 4 bits
        dict(name="attn_gqa_b32_fp4", kind="attn", type="fp4", batch=32, heads=8, group=4,
             dim=128, lo=1500, hi=16384, window=0, prefixes=0, prefix=0, shared_share=0),
        # a short prompt and eight images at its start: latency
        dict(name="shared_b8_c128_bf16", kind="attn", type="bf16", batch=8, heads=32, group=1,
             dim=128, lo=1, hi=98, window=0, prefixes=1, prefix=128, shared_share=8),
        # 64 images of one prompt that holds an image
        dict(name="shared_b64_c2048_int8", kind="attn", type="int8", batch=64, heads=32, group=1,
             dim=128, lo=64, hi=1024, window=0, prefixes=1, prefix=2048, shared_share=64),
        # 64 guidance pairs (every other row unconditional), grouped heads, a document as the prompt
        dict(name="shared_cfg_b128_c16384_fp4", kind="attn", type="fp4", batch=128, heads=8,
             group=4, dim=128, lo=0, hi=576, window=0, prefixes=2, prefix=16384, shared_share=128),
        # the sampled tokens of one decode step, image vocabulary of 16384
        dict(name="score_b8_v16384", kind="score", type="bf16", rows=8, vocab=16384, top=5,
             masked=0, temperature=1.0),
        # a large step over a text and image vocabulary, text tokens masked, 20 alternatives
        dict(name="score_b256_v65536_top20", kind="score", type="bf16", rows=256, vocab=65536,
             top=20, masked=57344, temperature=0.7),
        # eight whole images re-scored to rank them
        dict(name="score_images_v16384_f32", kind="score", type="f32", rows=18816, vocab=16384,
             top=1, masked=0, temperature=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("cache", "attn", "attn", "shared", "shared", "score"))
    kv = rng.choice(("int8", "fp4", "int8", "fp4", "bf16"))
    dim = rng.choice((64, 128, 128))
    if kind == "score":
        vocab = _log(rng, 1000, 131072)
        rows = max(1, min(_log(rng, 1, 20000), 300_000_000 // vocab))
        return dict(kind=kind, type=rng.choice(("bf16", "bf16", "f32")), rows=rows, vocab=vocab,
                    top=rng.choice((0, 1, 5, 20, 32)),
                    masked=rng.choice((0, 0, vocab // 2, vocab - 40)),
                    temperature=rng.choice((1.0, 0.7, 1.3)))
    heads = rng.choice((1, 2, 4, 5, 8, 20, 32))
    if kind == "cache":
        tokens = rng.choice((1, 1, _log(rng, 2, 2352)))
        lists = max(1, min(_log(rng, 1, 256), 100_000_000 // (tokens * heads * dim)))
        ragged = tokens > 1 and rng.random() < 0.5
        return dict(kind=kind, type=kv, lists=lists, heads=heads, dim=dim, tokens=tokens,
                    start=0 if ragged else _log(rng, 1, 2400), ragged=ragged)
    group = rng.choice((1, 1, 2, 3, 4, 7, 8))
    hi = _log(rng, 1, 16384)
    lo = rng.choice((0, 1, max(1, hi // 8), hi))
    most = 250_000_000 // (heads * dim)  # elements of one row's lists and of the shared ones
    case = dict(kind="attn", type=kv, batch=max(1, min(_log(rng, 1, 128), most // hi)),
                heads=heads, group=group, dim=dim, lo=lo, hi=hi,
                window=rng.choice((0, 0, 98, 1)), prefixes=0, prefix=0, shared_share=0)
    if kind == "shared":
        case["prefixes"] = rng.choice((1, 1, 2, 3))
        rows = case["batch"] * heads * group * case["prefixes"]
        case["prefix"] = min(_log(rng, 1, 16384), 60_000_000_000 // (rows * dim) // 16)
        case["shared_share"] = rng.choice((case["batch"], max(1, case["batch"] - 1)))
    return case


# ------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _pattern(n, lo, hi, salt):
    """Integers of [lo, hi], spread over their logarithm: a property of the case, not of a seed."""
    if lo >= hi:
        return torch.full((n,), hi, dtype=torch.int32)
    g = torch.Generator().manual_seed(1000 + salt)
    u = torch.rand(n, generator=g, dtype=torch.float64)
    x = torch.exp(math.log(lo + 1) + u * (math.log(hi + 1) - math.log(lo + 1))) - 1
    x = x.round().to(torch.int32).clamp(lo, hi)
    x[0], x[n // 2] = hi, lo if n > 1 else hi
    return x


def _lens(case):
    """len and first of every (batch row, head): a windowed head attends its newest tokens."""
    n = case["batch"] * case["heads"]
    shape = (case["batch"], case["heads"])
    length = _pattern(n, case["lo"], case["hi"], 1).view(shape)
    first = torch.zeros_like(length)
    if case["window"]:
        local = torch.arange(n).view(shape) % 5 < 2  # two heads of five
        first = torch.where(local, (length - case["window"]).clamp(min=0), first)
    return length, first


def _rows(shape, g):
    """Keys or values: normal, some channels of a head larger, as a trained model's are."""
    scale = torch.exp(0.5 * torch.randn((shape[-2], shape[-1]), generator=g, device="cuda"))
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 26) // max(1, out[0].numel()))
    for i in range(0, shape[0], step):
        part = out[i:i + step]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * scale)
    return out


def _codes(x, kind):
    """A quantised cache in its plain form: code values (int8; for fp4 twice the 4-bit value) and
    the scales they are multiplied by, of x [..., d] in bf16."""
    if kind == "bf16":
        return x, None
    code = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    scale = torch.empty((*x.shape[:-1], 1 if kind == "int8" else x.shape[-1] // 32),
                        dtype=torch.float32, device=x.device)
    step = max(1, (1 << 26) // max(1, x[0].numel()))
    for i in range(0, x.shape[0], step):
        code[i:i + step], scale[i:i + step] = _quantise(x[i:i + step], kind)
    return code, scale


def _pages(n_lists, heads, tokens, seed):
    """Page numbers in no order, as an allocator in use gives them: [lists][heads][pages]."""
    per = max(1, -(-tokens // PAGE))
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = n_lists * heads * per
    return torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(n_lists, heads, per)


class State:
    pass


def prepare(case, seed):
    s = State()
    s.case = case
    g = _generator(seed)
    if case["kind"] == "score":
        rows, vocab = case["rows"], case["vocab"]
        dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
        s.logits = torch.empty((rows, vocab), dtype=dtype, device="cuda")
        s.tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
        # the most likely tokens of a row are often sampled, others now and then
        step = max(1, (1 << 26) // vocab)
        for i in range(0, rows, step):
            x = 2.5 * torch.randn((min(step, rows - i), vocab), generator=g, device="cuda")
            if case["masked"]:
                x[:, :case["masked"]] = NEG
            s.logits[i:i + step] = x
            noise = torch.empty_like(x).exponential_(generator=g).log_()
            s.tokens[i:i + step] = (x - noise).argmax(1)
        return s
    if case["kind"] == "cache":
        n, heads, d, tokens = case["lists"], case["heads"], case["dim"], case["tokens"]
        s.k = _rows((n, tokens, heads, d), g)
        s.v = _rows((n, tokens, heads, d), g)
        if case["ragged"]:
            s.counts = _pattern(n, 0, tokens, 2).cuda()
            s.len = torch.zeros((n, heads), dtype=torch.int32, device="cuda")
        else:
            s.counts = None
            s.len = _pattern(n * heads, 0, case["start"], 3).view(n, heads).cuda()
        if own:  # the cache and its page table
            from paper_2605_20600_amd.paged import PagedKV
            most = case["start"] + tokens
            pages = _pages(n, heads, most, seed)
            s.cache = PagedKV(case["type"], d, heads, pages.numel(), page_tokens=PAGE)
            s.lists = s.cache.lists(pages, s.len, max_len=case["start"])
            after = s.len + (tokens if s.counts is None else s.counts[:, None])
            s.after = s.cache.lists(pages, after.to(torch.int32), max_len=most)
            s.out = torch.empty_like(s.k), torch.empty_like(s.v)
        return s
    b, heads, d = case["batch"], case["heads"], case["dim"]
    s.q = (1.5 * torch.randn((b, heads * case["group"], d), generator=g,
                             device="cuda")).bfloat16()
    length, first = _lens(case)
    s.len, s.first = length.cuda(), first.cuda()
    kv = [(b, case["hi"], s.len)]
    s.share = None
    if case["prefixes"]:
        # every other row its own list in turn (guidance pairs); the last rows may share none
        share = torch.arange(b) % case["prefixes"]
        share[case["shared_share"]:] = -1
        s.share = share.to(torch.int32).cuda()
        s.prefix_len = torch.tensor([[case["prefix"] - i % 2] * heads
                                     for i in range(case["prefixes"])],
                                    dtype=torch.int32, device="cuda")
        kv.append((case["prefixes"], case["prefix"], s.prefix_len))
    raw = [(_rows((n, most, heads, d), g), _rows((n, most, heads, d), g)) for n, most, _ in kv]
    if own:  # the cache, filled as a decoder fills it
        from paper_2605_20600_amd.paged import PagedKV
        tables = [_pages(n, heads, most, seed + i) for i, (n, most, _) in enumerate(kv)]
        if len(tables) > 1:
            tables[1] += tables[0].numel()
        s.cache = PagedKV(case["type"], d, heads, sum(t.numel() for t in tables),
                          page_tokens=PAGE, group=case["group"])
        s.lists = []
        for table, (k, v), (n, most, ln) in zip(tables, raw, kv):
            empty = torch.zeros_like(ln)
            s.cache.write(s.cache.lists(table, empty, max_len=0), k, v)
            s.lists.append(s.cache.lists(table, ln, max_len=most,
                                         first=s.first if not s.lists else None))
        s.out = torch.empty((b, heads * case["group"], d), device="cuda")
        s.lse = torch.empty((b, heads * case["group"]), device="cuda")
    else:  # the same cache in its plain form: codes and scales [lists][heads][tokens][d]
        s.kv = [[_codes(x.transpose(1, 2).contiguous(), case["type"]) for x in pair]
                for pair in raw]
    return s


# --------------------------------------------------------------------- pass
def run(state):
    case = state.case
    if case["kind"] == "cache":
        return _run_cache_own(state) if own else _run_cache_plain(state)
    if case["kind"] == "attn":
        return _run_attn_own(state) if own else _run_attn_plain(state)
    return _run_score_own(state) if own else _run_score_plain(state)


def _run_cache_own(s):
    s.cache.write(s.lists, s.k, s.v, counts=s.counts)
    tokens = s.k.shape[1]
    s.cache.read(s.after, tokens, begin=0 if s.case["ragged"] else -tokens, k=s.out[0],
                 v=s.out[1])
    return {"k": s.out[0], "v": s.out[1]}


def _run_attn_own(s):
    shared = s.lists[1] if s.share is not None else None
    s.cache.attn(s.lists[0], s.q, shared=shared, share=s.share, out=s.out, lse=s.lse)
    return {"out": s.out, "lse": s.lse}


def _run_score_own(s):
    from paper_2605_20600_amd.paged import token_logprobs
    return token_logprobs(s.logits, s.tokens, top=s.case["top"],
                          temperature=s.case["temperature"])


def _quantise(x, kind):
    """Codes and scales of x [..., d] (bf16), 32-bit arithmetic."""
    x = x.float()
    if kind == "int8":
        top = x.abs().amax(-1, keepdim=True)
        scale = (top / torch.full_like(top, 127)).bfloat16().float()
        code = torch.where(scale > 0, x / scale, torch.zeros_like(x)).round().clamp(-127, 127)
        return code.to(torch.int8), scale
    y = x.view(*x.shape[:-1], x.shape[-1] // 32, 32)
    bits = y.abs().amax(-1, keepdim=True).bfloat16().view(torch.int16).int()
    power = ((((bits + 63) >> 7) - 2).clamp(min=1) << 23).view(torch.float32)
    y = y / power
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    code = 2 * torch.copysign((a / step).round() * step, y)
    return code.view(x.shape).to(torch.int8), 0.5 * power.squeeze(-1)


def _value(code, scale):
    """32-bit values of codes [..., d] with scales [..., d or d / 32 or 1 per row]."""
    if scale is None:
        return code.float()
    n = scale.shape[-1]
    x = code.float().view(*code.shape[:-1], n, code.shape[-1] // n)
    return (x * scale[..., None]).view(code.shape)


def _run_cache_plain(s):
    tokens = s.k.shape[1]
    out = {}
    for name, x in (("k", s.k), ("v", s.v)):
        y = x if s.case["type"] == "bf16" else _value(*_quantise(x, s.case["type"])).bfloat16()
        if s.counts is not None:
            there = torch.arange(tokens, device="cuda") < s.counts[:, None]
            y = torch.where(there[..., None, None], y, torch.zeros_like(y))
        out[name] = y
    return out


def _run_attn_plain(s):
    case = s.case
    b, heads, group, d = case["batch"], case["heads"], case["group"], case["dim"]
    (kc, ks), (vc, vs) = s.kv[0]
    q = s.q.float().view(b, heads, group, d) * (1 / math.sqrt(d))
    at = torch.arange(case["hi"], device="cuda")
    there = (at < s.len[..., None]) & (at >= s.first[..., None])
    sc = torch.matmul(q, _value(kc, ks).transpose(2, 3))
    sc = sc.masked_fill(~there[:, :, None], NEG)
    if s.share is not None:
        (pkc, pks), (pvc, pvs) = s.kv[1]
        n, c = case["prefixes"], case["prefix"]
        # every row against every shared list, the one that it shares kept
        qh = q.permute(1, 0, 2, 3).reshape(heads, b * group, d)
        ps = torch.matmul(qh[None], _value(pkc, pks).transpose(2, 3))
        ps = ps.view(n, heads, b, group, c)
        mine = s.share[None] == torch.arange(n, device="cuda")[:, None]  # [n][b]
        seen = torch.arange(c, device="cuda") < s.prefix_len[..., None]  # [n][heads][c]
        seen = mine[:, None, :, None] & seen[:, :, None]                 # [n][heads][b][c]
        ps = ps.masked_fill(~seen[:, :, :, None], NEG)
        top = torch.maximum(sc.amax(-1), ps.amax((0, -1)).transpose(0, 1))
    else:
        top = sc.amax(-1)
    low = torch.where(top == NEG, torch.zeros_like(top), top)
    w = torch.exp(sc - low[..., None])
    total = w.sum(-1)
    out = torch.matmul(w, _value(vc, vs))
    if s.share is not None:
        pw = torch.exp(ps - low.transpose(0, 1)[None, ..., None])
        total = total + pw.sum((0, -1)).transpose(0, 1)
        po = torch.matmul(pw.view(n, heads, b * group, c), _value(pvc, pvs)).sum(0)
        out = out + po.view(heads, b, group, d).transpose(0, 1)
    out = out / torch.where(total > 0, total, torch.ones_like(total))[..., None]
    return {"out": out.reshape(b, heads * group, d),
            "lse": (low + torch.log(total)).reshape(b, heads * group)}


def _run_score_plain(s):
    case = s.case
    x = s.logits.float()
    scale = 1.0 / case["temperature"]
    top = x.amax(1, keepdim=True)
    y = (x - top) * scale
    e = torch.exp(y)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    mine = x.gather(1, s.tokens.long()[:, None])
    weighted = torch.where(e > 0, e * y, torch.zeros_like(y)).sum(1)
    out = {"logprob": ((mine - top) * scale - log_total)[:, 0],
           "entropy": log_total[:, 0] - weighted / total[:, 0],
           "rank": (x > mine).sum(1).to(torch.int32)}
    if case["top"]:
        best, index = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_logprob"] = (best[:, :case["top"]] - top) * scale - log_total
        out["top_index"] = index[:, :case["top"]].to(torch.int32)
    return out


# --------------------------------------------------------------------- work
ROW = {"bf16": lambda d: 2 * d, "int8": lambda d: d + 2, "fp4": lambda d: d // 2 + d // 32}


def work(case):
    if case["kind"] == "score":
        rows, vocab = case["rows"], case["vocab"]
        size = 2 if case["type"] == "bf16" else 4
        return {"bytes": rows * (vocab * size + 16 + 8 * case["top"]), "flops": 5 * rows * vocab}
    d = case["dim"]
    row = ROW[case["type"]](d)
    if case["kind"] == "cache":
        n, tokens = case["lists"], case["tokens"]
        there = int(_pattern(n, 0, tokens, 2).sum()) if case["ragged"] else n * tokens
        # inputs read, rows stored and read back, values written (zeros past the end too)
        return {"bytes": 2 * case["heads"] * (there * (2 * d + 2 * row) + n * tokens * 2 * d),
                "flops": 2 * case["heads"] * there * d * 4}
    length, first = _lens(case)
    tokens = int((length - first).sum())
    heads = case["batch"] * case["heads"] * case["group"]
    pairs = tokens * case["group"]
    if case["prefixes"]:
        used = min(case["prefixes"], case["shared_share"])
        at = [case["prefix"] - i % 2 for i in range(case["prefixes"])]
        tokens += sum(at[:used]) * case["heads"]
        pairs += sum(at[i % case["prefixes"]] for i in range(case["shared_share"])) * (
            case["heads"] * case["group"])
    return {"bytes": tokens * 2 * row + heads * (2 * d + 4 * d + 4), "flops": 4 * d * pairs}


# -------------------------------------------------------------------- exact
def _exact_value(x, kind):
    """What a cache of this kind holds for x, in 64 bits, from the format's definition."""
    x = x.double()
    if kind == "bf16":
        return x
    if kind == "int8":
        scale = (x.abs().amax(-1, keepdim=True) / 127).bfloat16().double()
        n = torch.nan_to_num(x / scale, nan=0.0, posinf=0.0, neginf=0.0).round().clamp(-127, 127)
        return n * scale
    y = x.view(*x.shape[:-1], -1, 32)
    mant, ex = torch.frexp(y.abs().amax(-1, keepdim=True))  # amax = mant * 2^ex, mant < 1
    power = torch.where(mant <= 0.75, ex - 3, ex - 2).clamp(min=-126).double()
    y = torch.ldexp(y, -power)
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64,
                        device=x.device)
    a = y.abs().clamp(max=6.0)
    up = torch.bucketize(a, grid).clamp(max=7)  # the first value that is not below
    down = (up - 1).clamp(min=0)
    below, above = a - grid[down], grid[up] - a
    pick = torch.where(below < above, down, torch.where(below > above, up, down + down % 2))
    return torch.ldexp(grid[pick] * torch.sign(y), power).view(x.shape)


def exact(case, seed):
    g = _generator(seed)
    if case["kind"] == "score":
        return _exact_score(case, seed)
    d, heads = case["dim"], case["heads"]
    if case["kind"] == "cache":
        n, tokens = case["lists"], case["tokens"]
        res = {}
        for name in ("k", "v"):
            x = _rows((n, tokens, heads, d), g)
            res[name] = torch.stack([_exact_value(x[i], case["type"]) for i in range(n)])
        if case["ragged"]:
            counts = _pattern(n, 0, tokens, 2)
            for i in range(n):
                for x in res.values():
                    x[i, int(counts[i]):] = 0
        return res
    b, group = case["batch"], case["group"]
    q = (1.5 * torch.randn((b, heads * group, d), generator=g, device="cuda")).bfloat16().double()
    length, first = _lens(case)
    k, v = (_rows((b, case["hi"], heads, d), g) for _ in range(2))
    pk = pv = None
    if case["prefixes"]:
        shape = (case["prefixes"], case["prefix"], heads, d)
        pk, pv = (_exact_value(_rows(shape, g), case["type"]) for _ in range(2))
    out = torch.zeros((b, heads * group, d), dtype=torch.float64, device="cuda")
    lse = torch.full((b, heads * group), NEG, dtype=torch.float64, device="cuda")
    for i in range(b):
        ki, vi = (_exact_value(x[i], case["type"]) for x in (k, v))  # [tokens][heads][d]
        shares = case["prefixes"] and i < case["shared_share"]
        at = torch.arange(case["hi"], device="cuda")[None]
        gone = ((at >= length[i].cuda()[:, None]) | (at < first[i].cuda()[:, None]))
        if shares:
            j = i % case["prefixes"]
            c = case["prefix"] - j % 2
            ki, vi = torch.cat((pk[j, :c], ki)), torch.cat((pv[j, :c], vi))
            gone = torch.cat((gone.new_zeros(heads, c), gone), 1)
        qi = q[i].view(heads, group, d)
        s = torch.bmm(qi, ki.permute(1, 2, 0).contiguous()) / math.sqrt(d)
        s = s.masked_fill(gone[:, None], NEG)
        lse[i] = torch.logsumexp(s, -1).view(-1)
        w = torch.nan_to_num(torch.softmax(s, -1), nan=0.0)
        out[i] = torch.bmm(w, vi.transpose(0, 1).contiguous()).view(heads * group, d)
    return {"out": out, "lse": lse}


def _exact_score(case, seed):
    s = prepare(case, seed)
    parts = []
    step = max(1, (1 << 25) // case["vocab"])
    for i in range(0, case["rows"], step):
        x = s.logits[i:i + step].double()
        t = s.tokens[i:i + step].long()
        lp = torch.log_softmax(x / case["temperature"], 1)
        p = lp.exp()
        res = {"logprob": lp.gather(1, t[:, None])[:, 0],
               "entropy": -torch.where(p > 0, p * lp, 0.0).sum(1)}
        if case["top"]:
            res["top_logprob"] = torch.topk(lp, case["top"], dim=1).values
        parts.append(res)
    res = {key: torch.cat([p[key] for p in parts]) for key in parts[0]}
    res["rank"] = None
    if case["top"]:
        res["top_index"] = None
    return res
