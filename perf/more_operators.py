"""The operators of a decode step with several drafted tokens per row, on paged
caches, as cases that can be timed and compared: norms of queries and keys with
rotary positions, also straight into the cache; attention of several new tokens of
each row; verification of drafted tokens against the target's probabilities; page
tables, windows and the start order brought up to date on the GPU.

listed() and draw() give cases (dicts of plain values), prepare() what a decoder
holds before the call, run() one pass (plain torch, or with `own` the library's
entry points), work() what a pass cannot do without, exact() the same results in
64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 64  # tokens of a page
NEG = -math.inf


def listed():
    return [
        # one decode step of the 768 px workload, batch 8, heads normalised one by one: the
        # queries come back, keys and values join the cache
        dict(name="rope_token_b8_int8", kind="rope", cache="int8", rows=8, tokens=1, q_heads=32,
             kv_heads=32, dim=128, rot=128, layout="half", axes=1, norm="layer", base=10000.0,
             scaling="none", far=2480, ragged=False),
        # five drafted tokens of 256 guided class-conditional sequences, positions of two axes
        dict(name="rope_draft_b256_2d_fp4", kind="rope", cache="fp4", rows=256, tokens=5,
             q_heads=20, kv_heads=20, dim=64, rot=64, layout="pairs", axes=2, norm="none",
             base=10000.0, scaling="none", far=24, ragged=False),
        # 16 prompts of up to 2352 tokens (an image and shorter ones) enter an empty cache
        dict(name="rope_prompt_b16_int8", kind="rope", cache="int8", rows=16, tokens=2352,
             q_heads=32, kv_heads=32, dim=128, rot=128, layout="half", axes=1, norm="rms",
             base=10000.0, scaling="none", far=0, ragged=True),
        # two long documents, grouped heads, half of a head turned, scaled to eight times the
        # trained length; no cache
        dict(name="rope_long_b2_gqa", kind="rope", cache="", rows=2, tokens=16384, q_heads=32,
             kv_heads=8, dim=128, rot=64, layout="half", axes=1, norm="rms", base=500000.0,
             scaling="bands", far=65536, ragged=False),
        # five drafted tokens for each of eight images, 32 heads, local ones with a window of two
        # rows: latency
        dict(name="attn_draft_b8_int8", kind="attn", type="int8", rows=8, tokens=5, heads=32,
             group=1, dim=128, lo=300, hi=2480, window=98, ragged=False, prefix=0),
        # the same for 64 images of one prompt that holds an image
        dict(name="attn_draft_b64_c2048_int8", kind="attn", type="int8", rows=64, tokens=5,
             heads=32, group=1, dim=128, lo=64, hi=1024, window=0, ragged=False, prefix=2048),
        # prompts in pieces of 256 tokens behind what is already there, grouped heads, 4 bits
        dict(name="attn_prompt_b4_t256_fp4", kind="attn", type="fp4", rows=4, tokens=256, heads=8,
             group=4, dim=128, lo=0, hi=2048, window=0, ragged=True, prefix=0),
        # four drafts of one image, image vocabulary of 16384: latency
        dict(name="verify_b1_v16384_f32", kind="verify", type="f32", rows=1, drafts=4,
             vocab=16384, masked=0, model=True, ragged=False, temperature=1.0),
        # a large step over a text and image vocabulary, text tokens masked
        dict(name="verify_b128_v65536", kind="verify", type="bf16", rows=128, drafts=4,
             vocab=65536, masked=49152, model=True, ragged=True, temperature=0.7),
        # eight tokens each guessed without a model (copied from the row above)
        dict(name="verify_b256_v16384_copied", kind="verify", type="bf16", rows=256, drafts=8,
             vocab=16384, masked=0, model=False, ragged=False, temperature=1.0),
        # a drafted step of eight images, one layer's lists
        dict(name="pages_step_b8_l1", kind="pages", rows=8, layers=1, heads=32, length=2480,
             window=98, tokens=5, ends=0, scarce=False),
        # 64 images, all 32 layers at once; every eighth image ends and another prompt begins
        dict(name="pages_step_b64_l32", kind="pages", rows=64, layers=32, heads=32, length=2480,
             window=98, tokens=5, ends=8, scarce=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "rope", "attn", "attn", "verify", "pages"))
    kv = rng.choice(("int8", "fp4", "bf16"))
    if kind == "rope":
        dim = rng.choice((64, 128, 128))
        axes = rng.choice((1, 1, 2))
        kv_heads = rng.choice((1, 2, 5, 8, 20, 32))
        q_heads = kv_heads * rng.choice((1, 1, 2, 4))
        tokens = rng.choice((1, rng.randint(2, 9), _log(rng, 10, 4000)))
        per = tokens * (q_heads + 2 * kv_heads) * dim
        rows = max(1, min(_log(rng, 1, 256), 300_000_000 // per))
        cache = rng.choice((kv, kv, ""))
        ragged = tokens > 1 and rng.random() < 0.5
        return dict(kind=kind, cache=cache, rows=rows, tokens=tokens, q_heads=q_heads,
                    kv_heads=kv_heads, dim=dim,
                    rot=rng.choice((dim, dim, dim // 2, 3 * dim // 4, 16 * axes)),
                    layout=rng.choice(("half", "half", "pairs")), axes=axes,
                    norm=rng.choice(("none", "rms", "layer")),
                    base=rng.choice((10000.0, 500000.0)),
                    scaling=rng.choice(("none", "linear", "base", "bands")),
                    far=rng.choice((0, _log(rng, 1, 1000000))), ragged=ragged)
    if kind == "attn":
        dim = rng.choice((64, 128, 128))
        heads, group = rng.choice((1, 2, 8, 20, 32)), rng.choice((1, 1, 2, 3, 4, 8))
        tokens = rng.choice((1, rng.randint(2, 9), rng.randint(2, 9), _log(rng, 10, 256)))
        hi = _log(rng, 1, 8192)
        prefix = rng.choice((0, 0, _log(rng, 1, 4096)))
        most = min(250_000_000 // (heads * dim * (hi + tokens)),
                   60_000_000 // (heads * group * tokens * (hi + tokens + prefix)))
        return dict(kind=kind, type=kv, rows=max(1, min(_log(rng, 1, 64), most)), tokens=tokens,
                    heads=heads, group=group, dim=dim, lo=rng.choice((0, 1, max(1, hi // 8), hi)),
                    hi=hi, window=rng.choice((0, 0, 98, 1)),
                    ragged=tokens > 1 and rng.random() < 0.4, prefix=prefix)
    if kind == "verify":
        vocab, drafts = _log(rng, 1000, 131072), rng.choice((1, 2, 4, 5, 8))
        rows = max(1, min(_log(rng, 1, 256), 75_000_000 // (vocab * (2 * drafts + 1))))
        return dict(kind=kind, type=rng.choice(("bf16", "bf16", "f32")), rows=rows, drafts=drafts,
                    vocab=vocab, masked=rng.choice((0, 0, vocab // 2, vocab - 40)),
                    model=rng.random() < 0.7, ragged=rng.random() < 0.4,
                    temperature=rng.choice((1.0, 0.7, 1.3, 0.0)))
    rows, heads = _log(rng, 1, 64), rng.choice((1, 4, 8, 20, 32))
    return dict(kind=kind, rows=rows, layers=rng.choice((1, 1, 4, 32)), heads=heads,
                length=_log(rng, 1, 2480), window=rng.choice((0, 98, 1)),
                tokens=rng.choice((1, 5, 9, 300)), ends=rng.choice((0, 1, 3, 8)),
                scarce=rng.random() < 0.3)


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


def _normal(shape, g, dtype=torch.bfloat16):
    """Normal values, some channels of a head larger, as a trained model's are."""
    scale = torch.exp(0.5 * torch.randn(shape[-1], generator=g, device="cuda"))
    out = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 26) // max(1, out[0].numel()))
    for i in range(0, shape[0], step):
        part = out[i:i + step]
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * scale)
    return out


def _tables(lists, heads, tokens, g):
    """Page numbers in no order, as an allocator in use gives them: [lists][heads][pages]."""
    n = lists * heads * max(1, -(-tokens // PAGE))
    return torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(lists, heads, -1)


class State:
    pass


def prepare(case, seed):
    s = State()
    s.case = case
    _PREPARE[case["kind"]](s, case, _generator(seed))
    return s


SCALED = dict(factor=8.0, original=8192, low=1.0, high=4.0)  # of "bands"


def _prepare_rope(s, case, g):
    rows, tokens, d = case["rows"], case["tokens"], case["dim"]
    qh, kh = case["q_heads"], case["kv_heads"]
    # a projection's output: queries, keys and values of a token beside each other
    x = _normal((rows, tokens, (qh + (2 if case["cache"] else 1) * kh) * d), g)
    s.q, s.k, *v = x.split([qh * d, kh * d] + ([kh * d] if case["cache"] else []), dim=2)
    s.q, s.k = (t.unflatten(2, (-1, d)) for t in (s.q, s.k))
    s.v = v[0].unflatten(2, (-1, d)) if v else None
    first = torch.randint(0, case["far"] + 1, (rows, 1, case["axes"]), generator=g, device="cuda")
    steps = torch.arange(tokens, device="cuda")[:, None]
    if case["axes"] == 2:  # row and column of an image of 24 columns
        steps = torch.cat((steps // 24, steps % 24), 1)
    s.positions = (first + steps).to(torch.int32).contiguous()
    s.q_weight = s.k_weight = s.q_bias = s.k_bias = None
    if case["norm"] != "none":  # one for every head
        s.q_weight = 1 + 0.1 * torch.randn((qh, d), generator=g, device="cuda")
        s.k_weight = 1 + 0.1 * torch.randn((kh, d), generator=g, device="cuda")
    if case["norm"] == "layer":
        s.q_bias = 0.1 * torch.randn((qh, d), generator=g, device="cuda")
        s.k_bias = 0.1 * torch.randn((kh, d), generator=g, device="cuda")
    s.counts = _pattern(rows, 0, tokens, 2).cuda() if case["ragged"] else None
    if own:
        from paper_2605_20600_amd.paged import PagedKV
        from paper_2605_20600_amd.rotary import NormWeights, Rotary
        scaling = {"none": None, "linear": ("linear", SCALED["factor"]),
                   "base": ("base", SCALED["factor"]),
                   "bands": ("bands", SCALED["factor"], SCALED["original"], SCALED["low"],
                             SCALED["high"])}[case["scaling"]]
        s.rotary = Rotary(d, case["rot"], layout=case["layout"], axes=case["axes"],
                          norm=None if case["norm"] == "none" else case["norm"], eps=1e-6,
                          base=case["base"], scaling=scaling)
        s.weights = NormWeights(s.q_weight, s.q_bias, s.k_weight, s.k_bias)
        s.q_out = torch.zeros((rows, tokens, qh, d), dtype=torch.bfloat16, device="cuda")
        s.k_out = torch.zeros((rows, tokens, kh, d), dtype=torch.bfloat16, device="cuda")
        if case["cache"]:
            start = 0 if case["ragged"] else case["far"] % 2500
            length = _pattern(rows * kh, 0, start, 3).view(rows, kh).cuda()
            pages = _tables(rows, kh, start + tokens, g)
            s.cache = PagedKV(case["cache"], d, kh, pages.numel(), page_tokens=PAGE,
                              group=qh // kh)
            s.lists = s.cache.lists(pages, length, max_len=start)
            after = length + (tokens if s.counts is None else s.counts[:, None])
            s.after = s.cache.lists(pages, after.to(torch.int32), max_len=start + tokens)
            s.v_out = torch.zeros_like(s.k_out)


def _lens(case):
    """len and window of every (row, head), the new tokens not counted: two heads of five are
    local."""
    shape = (case["rows"], case["heads"])
    n = shape[0] * shape[1]
    length = _pattern(n, case["lo"], case["hi"], 1).view(shape)
    local = torch.arange(n).view(shape) % 5 < 2
    window = torch.where(local, case["window"], 0).to(torch.int32)
    return length, window


def _counts(case):
    n, most = case["rows"], case["tokens"]
    return _pattern(n, 0, most, 2) if case["ragged"] else torch.full((n,), most, dtype=torch.int32)


def _prepare_attn(s, case, g):
    b, heads, d, tokens = case["rows"], case["heads"], case["dim"], case["tokens"]
    s.q = (1.5 * torch.randn((b, tokens, heads * case["group"], d), generator=g,
                             device="cuda")).bfloat16()
    s.len, s.window = (t.cuda() for t in _lens(case))
    s.counts = _counts(case).cuda()
    most = case["hi"] + tokens
    kv = [(_normal((b, most, heads, d), g), _normal((b, most, heads, d), g))]
    if case["prefix"]:  # one list for all rows
        kv.append((_normal((1, case["prefix"], heads, d), g),
                   _normal((1, case["prefix"], heads, d), g)))
    if own:  # the cache, the new tokens in it
        from paper_2605_20600_amd.paged import PagedKV
        tables = [_tables(k.shape[0], heads, k.shape[1], g) for k, _ in kv]
        if len(tables) > 1:
            tables[1] += tables[0].numel()
        s.cache = PagedKV(case["type"], d, heads, sum(t.numel() for t in tables),
                          page_tokens=PAGE, group=case["group"])
        s.lists, s.share = [], None
        for table, (k, v) in zip(tables, kv):
            none = torch.zeros(table.shape[:2], dtype=torch.int32, device="cuda")
            s.cache.write(s.cache.lists(table, none, max_len=0), k, v)
            if not s.lists:
                s.lists.append(s.cache.lists(table, s.len, max_len=case["hi"]))
            else:
                s.lists.append(s.cache.lists(table, none + case["prefix"],
                                             max_len=case["prefix"]))
                s.share = torch.zeros(b, dtype=torch.int32, device="cuda")
        s.out = torch.zeros((b, tokens, heads * case["group"], d), device="cuda")
        s.lse = torch.zeros((b, tokens, heads * case["group"]), device="cuda")
        s.some = s.counts if case["ragged"] else None
        s.local = s.window if case["window"] else None
    else:  # the same cache in its plain form: codes and scales [lists][heads][tokens][d]
        s.kv = [[_codes(x.transpose(1, 2).contiguous(), case["type"]) for x in pair]
                for pair in kv]


def _prepare_verify(s, case, g):
    rows, drafts, vocab = case["rows"], case["drafts"], case["vocab"]
    dtype = torch.bfloat16 if case["type"] == "bf16" else torch.float32
    s.logits = torch.empty((rows, drafts + 1, vocab), dtype=dtype, device="cuda")
    s.draft = torch.empty((rows, drafts, vocab), dtype=dtype, device="cuda") if case["model"] \
        else None
    s.tokens = torch.empty((rows, drafts), dtype=torch.int32, device="cuda")
    t = case["temperature"] or 1.0
    step = max(1, (1 << 26) // (vocab * (drafts + 1)))
    for i in range(0, rows, step):
        x = 2.5 * torch.randn((min(step, rows - i), drafts + 1, vocab), generator=g, device="cuda")
        if case["masked"]:
            x[..., :case["masked"]] = NEG
        s.logits[i:i + step] = x
        x = x[:, :drafts]
        if case["model"]:  # a smaller model's, near the target's
            x = x + 0.7 * torch.randn(x.shape, generator=g, device="cuda")
            s.draft[i:i + step] = x
        noise = torch.empty_like(x).exponential_(generator=g).log_()
        sharp = 1.0 if case["model"] else 3.0  # guesses hit the likely tokens often
        s.tokens[i:i + step] = (sharp * x / t - noise).argmax(2)
    s.uniforms = torch.rand((rows, drafts + 1), generator=g, device="cuda")
    s.counts = _pattern(rows, 0, drafts, 4).cuda() if case["ragged"] else None


def _prepare_pages(s, case, g):
    rows, layers, heads, w = case["rows"], case["layers"], case["heads"], case["window"]
    lists, tokens = rows * layers, case["tokens"]
    prompt = max(1, case["length"] // 4)
    s.tokens = max(tokens, prompt if case["ends"] else 0)
    s.max_pages = -(-(case["length"] + s.tokens + 1) // PAGE)
    # images at different steps, the heads of a list as far on as each other
    at = torch.randint(0, case["length"] + 1, (rows,), generator=g, device="cuda")
    length = at.repeat(layers)[:, None].expand(lists, heads)
    local = torch.rand((lists, heads), generator=g, device="cuda") < 0.4
    window = torch.where(local, w, 0)
    first = torch.where(window > 0, (length + 1 - window).clamp(min=0), 0)
    # what the last step left: pages of the window and of the tokens that it had room for
    p = torch.arange(s.max_pages, device="cuda")
    held = (p >= (first // PAGE)[..., None]) & (p < (-(-(length + tokens) // PAGE))[..., None])
    s.num_pages = held.numel()
    numbers = torch.randperm(s.num_pages, generator=g, device="cuda")
    place = (held.flatten().cumsum(0) - 1).view(held.shape)
    used = held.sum()
    pages = torch.where(held, numbers[place.clamp(min=0)], -1)
    free = s.num_pages - used
    if case["scarce"]:  # pages for some of what will be asked for
        free = free.clamp(max=max(1, lists * heads // 100))
    # the ring: free pages from a place of its own on
    head = torch.randint(0, s.num_pages, (1,), generator=g, device="cuda")
    ring = numbers[(used + torch.arange(s.num_pages, device="cuda") - head) % s.num_pages]
    ring_state = torch.zeros(4, dtype=torch.int64, device="cuda")
    ring_state[0:1], ring_state[1] = head, free
    s.start = dict(pages=pages, len=length, first=first, free_pages=ring, free_state=ring_state)
    s.start = {k: t.to(torch.int32).contiguous() for k, t in s.start.items()}
    s.window = window.to(torch.int32)
    # tokens that the rows have gained, -1: ended, and those that come next
    s.advance = torch.randint(1, max(2, min(tokens, 6)), (rows,), generator=g,
                              device="cuda").to(torch.int32)
    s.counts = torch.full((rows,), tokens, dtype=torch.int32, device="cuda")
    if case["ends"]:
        over = torch.arange(rows, device="cuda") % case["ends"] == 0
        s.advance[over], s.counts[over] = -1, prompt
    if own:
        from paper_2605_20600_amd.page_tables import PageTables
        s.tables = PageTables(heads, s.max_pages, s.num_pages, rows=rows, layers=layers,
                              page_tokens=PAGE, window=s.window)
        for name, t in s.start.items():
            getattr(s.tables, name).copy_(t)
        s.begin = s.tables.buffer.clone()


_PREPARE = dict(rope=_prepare_rope, attn=_prepare_attn, verify=_prepare_verify,
                pages=_prepare_pages)


# --------------------------------------------------------------------- pass
def run(state):
    kind = state.case["kind"]
    if own:
        return {"rope": _rope_own, "attn": _attn_own, "verify": _verify_own,
                "pages": _pages_own}[kind](state)
    return {"rope": _rope_plain, "attn": _attn_plain, "verify": _verify_plain,
            "pages": _pages_plain}[kind](state)


def _rope_own(s):
    if not s.case["cache"]:
        s.rotary(s.q, s.k, s.positions, weights=s.weights, counts=s.counts, q_out=s.q_out,
                 k_out=s.k_out)
        return {"q": s.q_out, "k": s.k_out}
    s.cache.write_rotary(s.lists, s.rotary, s.q, s.k, s.v, s.positions, weights=s.weights,
                         counts=s.counts, q_out=s.q_out)
    tokens = s.k.shape[1]  # what the cache holds now
    s.cache.read(s.after, tokens, begin=0 if s.case["ragged"] else -tokens, k=s.k_out, v=s.v_out)
    return {"q": s.q_out, "k": s.k_out, "v": s.v_out}


def _attn_own(s):
    s.cache.attn_tokens(s.lists[0], s.q, counts=s.some, window=s.local,
                        shared=s.lists[1] if s.share is not None else None, share=s.share,
                        out=s.out, lse=s.lse)
    return {"out": s.out, "lse": s.lse}


def _verify_own(s):
    from paper_2605_20600_amd.drafts import verify_drafts
    return verify_drafts(s.logits, s.tokens, s.uniforms, draft_logits=s.draft, counts=s.counts,
                         temperature=s.case["temperature"])


def _pages_own(s):
    s.tables.buffer.copy_(s.begin)  # a pass begins where the last one did
    s.tables.extend(s.tokens, advance=s.advance, counts=s.counts)
    t = s.tables
    return {"pages": t.pages, "len": t.len, "first": t.first, "order": t.order,
            "free_pages": t.free_pages, "free_state": t.free_state}


def _frequencies(case, device):
    """Radians a position, of each pair, in 64 bits."""
    n = case["rot"] // case["axes"]
    j = torch.arange(n // 2, dtype=torch.float64, device=device)
    f, base = SCALED["factor"], case["base"]
    if case["scaling"] == "base":  # the slowest pair as slow as if positions were divided
        base = base * f ** (n / (n - 2.0))
    omega = base ** (-2 * j / n)
    if case["scaling"] == "linear":
        omega = omega / f
    if case["scaling"] == "bands":  # pairs that turn often in the trained length stay
        often = SCALED["original"] * omega / (2 * math.pi)
        share = ((often - SCALED["low"]) / (SCALED["high"] - SCALED["low"])).clamp(0, 1)
        omega = omega / f * (1 - share) + omega * share
    return omega


def _turned(x, case, cos, sin, weight, bias):
    """Norm and rotation of x [rows][tokens][heads][d], 32-bit arithmetic."""
    x = x.float()
    if case["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    if case["norm"] != "none":
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
    if case["norm"] == "layer":
        x = x + bias
    r = case["rot"]
    turned, rest = x[..., :r], x[..., r:]
    if case["layout"] == "half":
        a, b = turned[..., :r // 2], turned[..., r // 2:]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        y = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((y, rest), -1).bfloat16()


def _rope_plain(s):
    case = s.case
    per_axis = _frequencies(case, "cuda")
    angle = (s.positions.double()[..., None] * per_axis).flatten(2)[:, :, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = {"q": _turned(s.q, case, cos, sin, s.q_weight, s.q_bias),
           "k": _turned(s.k, case, cos, sin, s.k_weight, s.k_bias)}
    if case["cache"]:
        out["v"] = s.v
        if case["cache"] != "bf16":
            for name in ("k", "v"):
                out[name] = _value(*_codes(out[name], case["cache"])).bfloat16()
    if s.counts is not None:
        there = torch.arange(s.q.shape[1], device="cuda") < s.counts[:, None]
        out = {name: torch.where(there[..., None, None], x, torch.zeros_like(x))
               for name, x in out.items()}
    return out


def _codes(x, kind):
    """Codes and scales of x [..., d] (bf16) in a cache of this kind, 32-bit arithmetic: int8, for
    fp4 twice the 4-bit value."""
    if kind == "bf16":
        return x, None
    x = x.float()
    if kind == "int8":
        scale = (x.abs().amax(-1, keepdim=True) / 127.0).bfloat16().float()
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
    """32-bit values of codes [..., d] with scales [..., d / 32 or 1]."""
    if scale is None:
        return code.float()
    n = scale.shape[-1]
    x = code.float().view(*code.shape[:-1], n, code.shape[-1] // n)
    return (x * scale[..., None]).view(code.shape)


def _attn_plain(s):
    case = s.case
    b, tokens, heads, group, d = (case[n] for n in ("rows", "tokens", "heads", "group", "dim"))
    (kc, ks), (vc, vs) = s.kv[0]
    q = s.q.float().view(b, tokens, heads, group, d).permute(0, 2, 1, 3, 4) * (1 / math.sqrt(d))
    q = q.reshape(b, heads, tokens * group, d)
    at = torch.arange(kc.shape[2], device="cuda")
    i = torch.arange(tokens, device="cuda")
    end = s.len[..., None] + i + 1                       # [b][heads][tokens]
    first = torch.where(s.window[..., None] > 0, end - s.window[..., None], torch.zeros_like(end))
    seen = (at < end[..., None]) & (at >= first[..., None])
    seen = seen[:, :, :, None].expand(-1, -1, -1, group, -1).reshape(b, heads, tokens * group, -1)
    sc = torch.matmul(q, _value(kc, ks).transpose(2, 3)).masked_fill(~seen, NEG)
    top = sc.amax(-1, keepdim=True)
    if case["prefix"]:
        (pkc, pks), (pvc, pvs) = s.kv[1]
        qh = q.transpose(0, 1).reshape(heads, b * tokens * group, d)
        ps = torch.matmul(qh, _value(pkc, pks)[0].transpose(1, 2))
        ptop = ps.amax(-1).view(heads, b, -1, 1).transpose(0, 1)
        top = torch.maximum(top, ptop)
    w = torch.exp(sc - top)
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w, _value(vc, vs))
    if case["prefix"]:
        pw = torch.exp(ps - top.transpose(0, 1).reshape(heads, -1, 1))
        total = total + pw.sum(-1).view(heads, b, -1, 1).transpose(0, 1)
        po = torch.matmul(pw, _value(pvc, pvs)[0])
        out = out + po.view(heads, b, -1, d).transpose(0, 1)
    out, lse = out / total, (top + torch.log(total))[..., 0]
    out = out.view(b, heads, tokens, group, d).transpose(1, 2).reshape(b, tokens, -1, d)
    lse = lse.view(b, heads, tokens, group).transpose(1, 2).reshape(b, tokens, -1)
    there = (i < s.counts[:, None])[..., None]
    return {"out": torch.where(there[..., None], out, torch.zeros_like(out)),
            "lse": torch.where(there, lse, torch.zeros_like(lse))}


def _shares(x, temperature):
    """softmax(x / temperature) over the last axis, 64 bits: a draft is accepted, and the next
    token found, by comparisons that values next to a border must not turn."""
    x = x.double()
    if temperature == 0:  # all on the largest, the first of equal ones
        return torch.zeros_like(x).scatter_(-1, x.argmax(-1, keepdim=True), 1.0)
    e = torch.exp((x - x.amax(-1, keepdim=True)) / temperature)
    return e / e.sum(-1, keepdim=True)


def _verify_plain(s):
    rows, drafts = s.tokens.shape
    t = s.case["temperature"]
    given = s.counts.long() if s.counts is not None else torch.full((rows,), drafts, device="cuda")
    i = torch.arange(drafts, device="cuda")
    p = _shares(s.logits, t)
    x = s.tokens.long()[..., None]
    px = p[:, :drafts].gather(2, x)[..., 0]
    q = torch.zeros_like(p[:, :drafts])
    if s.draft is not None and t > 0:
        q = _shares(s.draft, t)
    elif t > 0:  # a guess is all that its source would have said
        q = q.scatter_(2, x, 1.0)
    # (t = 0: the target's largest, whoever drafted it)
    good = s.uniforms[:, :drafts].double() * q.gather(2, x)[..., 0] < px
    good &= i < given[:, None]
    accepted = good.long().cumprod(1).sum(1)
    # the row of the first draft that is not taken, or the one behind them all
    r = torch.arange(rows, device="cuda")
    pr = p[r, accepted]
    qr = q[r, accepted.clamp(max=drafts - 1)]
    qr = torch.where((accepted < given)[:, None], qr, torch.zeros_like(qr))
    rest = (pr - qr).clamp(min=0)
    up_to = rest.cumsum(1)
    want = s.uniforms[:, drafts].double() * up_to[:, -1]
    following = (up_to <= want[:, None]).sum(1)
    place = torch.arange(drafts + 1, device="cuda")
    here = place == accepted[:, None]
    tokens = torch.cat((s.tokens.long(), s.tokens.new_zeros((rows, 1)).long()), 1)
    tokens = torch.where(here, following[:, None], tokens)
    there = place <= accepted[:, None]
    tokens = torch.where(there, tokens, -1)
    logprob = torch.log(p.gather(2, tokens.clamp(min=0)[..., None])[..., 0])
    return {"tokens": tokens.to(torch.int32), "count": (accepted + 1).to(torch.int32),
            "logprob": torch.where(there, logprob, torch.zeros_like(logprob)).float()}


def _order_key(n):
    """Tokens in eighths of their octave: what the start order goes by."""
    e = torch.frexp(n.clamp(min=8).double())[1].long() - 1
    return torch.where(n < 8, n, (e - 2) * 8 + ((n.long() >> (e - 3)) & 7))


def _pages_plain(s):
    c = s.case
    n, most = s.num_pages, s.max_pages * PAGE
    t = {k: v.long() for k, v in s.start.items()}
    advance = s.advance.long().repeat(c["layers"])[:, None]
    counts = s.counts.long().clamp(0, s.tokens).repeat(c["layers"])[:, None]
    ended = advance < 0
    length = torch.where(ended, 0, (t["len"] + advance).clamp(max=most))
    before = torch.where(ended, 0, t["first"])
    w = s.window.long()
    first = torch.where(w > 0, torch.maximum(before, length + 1 - w), before)
    p = torch.arange(s.max_pages, device="cuda")
    pages = t["pages"]
    held = (pages >= 0) & (pages < n)
    gone = (p >= (before // PAGE)[..., None]) & (p < (first // PAGE)[..., None])
    gone = held & (gone | ended[..., None])
    pages = torch.where(gone | ended[..., None], -1, pages)
    # freed pages join the ring's end, in the table's order
    head, free = t["free_state"][0], t["free_state"][1]
    k = gone.flatten().cumsum(0)
    at = torch.where(gone.flatten(), (head + free + k - 1) % n, n)
    ring = torch.cat((t["free_pages"], t["free_pages"].new_zeros(1)))
    ring = ring.scatter(0, at, t["pages"].flatten())[:n]
    ring_has = free + k[-1]
    # new ones leave at its head
    need = (p >= (-(-length // PAGE))[..., None]) & (p < (-(-(length + counts) // PAGE))[..., None])
    need &= ~(held & ~gone)
    k = need.flatten().cumsum(0)
    given = (need.flatten() & (k <= ring_has)).view(need.shape)
    pages = torch.where(given, ring[(head + k - 1) % n].view(need.shape), pages)
    gave = torch.minimum(k[-1], ring_has)
    state = torch.stack(((head + gave) % n, ring_has - gave, k[-1] - gave, k[-1] * 0))
    key = _order_key((length + counts - first).clamp(min=0)).view(c["layers"], -1)
    order = torch.sort(key, dim=1, descending=True, stable=True)[1]
    res = dict(pages=pages, len=length, first=first, order=order, free_pages=ring,
               free_state=state)
    return {k: v.to(torch.int32) for k, v in res.items()}


# --------------------------------------------------------------------- work
ROW = {"bf16": lambda d: 2 * d, "int8": lambda d: d + 2, "fp4": lambda d: d // 2 + d // 32}


def work(case):
    kind = case["kind"]
    if kind == "rope":
        d, qh, kh = case["dim"], case["q_heads"], case["kv_heads"]
        n = case["rows"] * case["tokens"]
        there = int(_pattern(case["rows"], 0, case["tokens"], 2).sum()) if case["ragged"] else n
        size = there * (qh + kh) * 4 * d
        if case["cache"]:  # stored, read back, returned (zeros past the end too)
            size = there * (qh * 4 * d + 2 * kh * (2 * d + 2 * ROW[case["cache"]](d)))
            size += n * kh * 4 * d
        return {"bytes": size, "flops": there * (qh + kh) * d * 8}
    if kind == "attn":
        d, group = case["dim"], case["group"]
        length, window = _lens(case)
        counts = _counts(case)[:, None].expand_as(length)
        end = length + counts
        first = torch.where(window > 0, (length + 1 - window).clamp(min=0), 0)
        kv = int(torch.where(counts > 0, end - first, 0).sum())
        # (row, token, head) times the tokens each sees, on average
        seen = torch.where(window > 0, torch.minimum(window, end), length + (counts + 1) // 2)
        pairs = int((seen.long() * counts).sum()) * group
        queries = int(counts.sum()) * group
        kv += case["prefix"] * case["heads"]
        pairs += queries * case["prefix"]
        return {"bytes": kv * 2 * ROW[case["type"]](d) + queries * (2 * d + 4 * d + 4),
                "flops": 4 * d * pairs}
    if kind == "verify":
        size = 2 if case["type"] == "bf16" else 4
        drafts = case["drafts"]
        n = case["rows"] * case["vocab"] * (drafts + 1 + (drafts if case["model"] else 0))
        return {"bytes": n * size + case["rows"] * (drafts + 1) * 16, "flops": 5 * n}
    lists = case["rows"] * case["layers"] * case["heads"]
    # length, first, window and order of each, length and first written, a page's number moved
    return {"bytes": lists * 6 * 4 + (lists // 8) * 16, "flops": 0}


# -------------------------------------------------------------------- exact
def exact(case, seed):
    if case["kind"] == "pages":  # whole numbers
        return None
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    return dict(rope=_exact_rope, attn=_exact_attn, verify=_exact_verify)[case["kind"]](s, case,
                                                                                       seed)


def _exact_rope(s, case, seed):
    """Rows as complex numbers that are multiplied by the unit ones of their angles."""
    rows, tokens, d, r = case["rows"], case["tokens"], case["dim"], case["rot"]
    n = r // case["axes"]
    base = case["base"]
    if case["scaling"] == "base":
        base *= SCALED["factor"] ** (n / (n - 2))
    omega = []
    for j in range(n // 2):
        w = math.exp(-2 * j / n * math.log(base))
        turns = SCALED["original"] / (2 * math.pi / w)  # in the trained length
        if case["scaling"] == "linear" or (case["scaling"] == "bands" and turns <= SCALED["low"]):
            w /= SCALED["factor"]
        elif case["scaling"] == "bands" and turns < SCALED["high"]:
            t = (turns - SCALED["low"]) / (SCALED["high"] - SCALED["low"])
            w = t * w + (1 - t) * w / SCALED["factor"]
        omega.append(w)
    omega = torch.tensor(omega, dtype=torch.float64, device="cuda")
    out = {}
    for name, x, weight, bias in (("q", s.q, s.q_weight, s.q_bias),
                                  ("k", s.k, s.k_weight, s.k_bias)):
        res = torch.zeros(x.shape, dtype=torch.float64 if name == "q" or not case["cache"]
                          else torch.bfloat16, device="cuda")
        for i in range(rows):
            y = x[i].double()
            if case["norm"] == "rms":
                y = y * (y.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * weight.double()
            elif case["norm"] == "layer":
                var, mean = torch.var_mean(y, -1, keepdim=True, correction=0)
                y = (y - mean) * (var + 1e-6).rsqrt() * weight.double() + bias.double()
            phase = [torch.outer(s.positions[i, :, a].double(), omega) for a in range(case["axes"])]
            phase = torch.cat(phase, 1)[:, None]
            unit = torch.complex(phase.cos(), phase.sin())
            if case["layout"] == "half":
                z = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous())
                z = z * unit
                y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
            else:
                z = torch.view_as_complex(y[..., :r].contiguous().view(tokens, -1, r // 2, 2))
                y[..., :r] = torch.view_as_real(z * unit).flatten(-2)
            res[i] = y
        out[name] = res
    if case["cache"]:
        out["v"] = s.v
        for name in ("k", "v"):
            out[name] = torch.stack([_exact_value(out[name][i], case["cache"])
                                     for i in range(rows)])
    if s.counts is not None:
        for x in out.values():
            for i, c in enumerate(s.counts.tolist()):
                x[i, c:] = 0
    return out


def _exact_value(x, kind):
    """What a cache of this kind holds for x (bf16), in 64 bits, from the format's definition."""
    x = x.double()
    if kind == "bf16":
        return x
    if kind == "int8":
        scale = (x.abs().amax(-1, keepdim=True) / 127).bfloat16().double()
        n = torch.nan_to_num(x / scale, nan=0.0, posinf=0.0, neginf=0.0).round().clamp(-127, 127)
        return n * scale
    y = x.unflatten(-1, (-1, 32))
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


def _exact_attn(s, case, seed):
    b, tokens, heads, group, d = (case[n] for n in ("rows", "tokens", "heads", "group", "dim"))
    g = _generator(seed)
    q = (1.5 * torch.randn((b, tokens, heads * group, d), generator=g, device="cuda")).bfloat16()
    k, v = (_normal((b, case["hi"] + tokens, heads, d), g) for _ in range(2))
    before = [x[0] for x in (k[:1, :0], v[:1, :0])]
    if case["prefix"]:
        before = [_normal((1, case["prefix"], heads, d), g)[0] for _ in range(2)]
    c = before[0].shape[0]
    before = [_exact_value(x, case["type"]) for x in before]
    length, window = _lens(case)
    counts = _counts(case).tolist()
    out = torch.zeros((b, tokens, heads * group, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((b, tokens, heads * group), dtype=torch.float64, device="cuda")
    at = torch.arange(case["hi"] + tokens, device="cuda")
    for row in range(b):
        n = counts[row]
        ki, vi = (torch.cat((x, _exact_value(y[row], case["type"])))
                  for x, y in zip(before, (k, v)))
        for h in range(heads):
            ln, w = int(length[row, h]), int(window[row, h])
            mine = q[row, :n, h * group:(h + 1) * group].double().reshape(n * group, d)
            score = mine @ ki[:, h].T.contiguous() / math.sqrt(d)
            end = ln + 1 + torch.arange(n, device="cuda")[:, None]
            gone = (at >= end) | ((at < end - w) if w else False)
            gone = torch.cat((gone.new_zeros((n, c)), gone), 1).repeat_interleave(group, 0)
            score = score.masked_fill(gone, NEG)
            o = torch.softmax(score, -1) @ vi[:, h].contiguous()
            out[row, :n, h * group:(h + 1) * group] = o.view(n, group, d)
            lse[row, :n, h * group:(h + 1) * group] = torch.logsumexp(score, -1).view(n, group)
    return {"out": out, "lse": lse}


def _exact_verify(s, case, seed):
    """Draft by draft; only the log probabilities are computed numbers."""
    rows, drafts = s.tokens.shape
    t = case["temperature"]
    res = torch.zeros((rows, drafts + 1), dtype=torch.float64, device="cuda")
    if t == 0:  # what is certain
        return {"tokens": None, "count": None, "logprob": res}
    tokens, uniforms = s.tokens.tolist(), s.uniforms.tolist()
    given = [drafts] * rows if s.counts is None else s.counts.tolist()
    for r in range(rows):
        for i in range(drafts + 1):
            lp = torch.log_softmax(s.logits[r, i].double() / t, 0)
            rest = lp.exp()
            if i < given[r]:
                x = tokens[r][i]
                other = torch.zeros_like(rest)
                if s.draft is None:
                    other[x] = 1.0
                else:
                    other = torch.softmax(s.draft[r, i].double() / t, 0)
                p, q = torch.stack((rest[x], other[x])).tolist()
                if uniforms[r][i] * q < p:
                    res[r, i] = lp[x]
                    continue
                rest = torch.relu(rest - other)
            up_to = torch.cumsum(rest, 0)
            found = torch.searchsorted(up_to, uniforms[r][drafts] * up_to[-1:], right=True)
            res[r, i] = lp[found[0]]
            break
    return {"tokens": None, "count": None, "logprob": res}
