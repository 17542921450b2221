"""Cases of the quantised key-value cache where not every row is read for every sequence: a prefix that a batch shares, and
pages that a cheap score chooses.

The cache holds one fp32 norm and one symbol per coordinate for every (token, head) row of keys and of values; a symbol is
2 * (index of a level) + sign, in 4 or 8 bits, and stands for the signed level times the norm.  A page of the cache is int32
words: for each head the keys' rows of all its tokens, the values' rows, the keys' norms and the values' norms.  A row has
head_dim symbols, little endian, and zeros up to 64, 128 or 256 of them.

Operators ("op" of a case):
  shared   one new token a sequence, over the tokens of a prefix that all sequences share and then those of its own pages:
           softmax(scale * q K^T) V and the log of the softmax's denominator
  bounds   for each page of a list and each head: the largest and the least value of every coordinate of its keys, in whole
           numbers of 8 bits with one scale
  chosen   one new token a sequence and head of the cache, over the pages whose bounds give the highest scores: the pages, how
           many tokens they hold, softmax(scale * q K^T) V over those and the log of the denominator

Bounds: N is the largest norm of the page's keys, inv = 127 / N, and coordinate d has ceil(max v_d * inv) and floor(min v_d * inv)
within [-127, 127], with the scale N / 127; a page whose N is below 2^-100 has zeros and scale 0.  Scores: a query becomes whole
numbers i_d = rint(q_d * (127 / max |q|)) with the scale max |q| / 127, and page p scores (sum_d max(i_d upper_d, i_d lower_d)) *
(query's scale) * (page's scale); a head's score is the largest of its queries'.  Of a sequence's pages the first and the last ones
are kept always, of the others those with the highest scores, of equal ones the first, all in their order.

Plain forms compute in 32 bits; rotary tables are inputs, made in 64.  What stands beside a border between two whole numbers, or
two pages' scores, is a 32-bit number by definition: rotated coordinates (each product and their sum), the quotients, and each
product above.
"""
import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SEED = 20250514


def _case(name, op, **over):
    c = dict(name=name, op=op, batch=1, prefix=0, tokens=1, kv_heads=8, group=4, dim=128, bits_k=3, bits_v=3, type="bf16",
             page=64, rotary=0, interleaved=False, ragged=False, keep=0, first=1, last=1)
    c.update(over)
    return c


def listed():
    return [
        # two answers to one short prompt, just begun: latency is all
        _case("shared-two-answers", "shared", batch=2, prefix=700, tokens=20, rotary=128),
        # a serving step: one instruction text before all requests, each with some turns of its own
        _case("shared-serving", "shared", batch=32, prefix=4096, tokens=600, ragged=True, rotary=128),
        # many samples of one long document's question
        _case("shared-many-samples", "shared", batch=128, prefix=16384, tokens=900, ragged=True, rotary=128),
        # fine symbols, small heads of which two serve all queries, a prompt of a whole book's chapter
        _case("shared-fine", "shared", batch=16, prefix=32768, tokens=333, kv_heads=2, group=8, dim=64, bits_k=7, bits_v=7,
              type="fp16", page=16),
        # the odd heads of the Transformer-XL shapes of this repository in the framework's own type
        _case("shared-odd-heads", "shared", batch=24, prefix=2050, tokens=150, kv_heads=10, group=1, dim=41, type="fp32",
              ragged=True, page=32),
        # a long prompt has been written: the bounds of all its pages
        _case("bounds-prompt", "bounds", tokens=16384),
        # a decoding step of 64 sequences: the pages that it has filled, a quarter of the batch
        _case("bounds-step", "bounds", batch=64, dim=80, bits_k=7, page=16),
        # a context of middle length, small pages: latency
        _case("chosen-short", "chosen", tokens=900, page=16, keep=16, rotary=128),
        # one sequence, a very long context
        _case("chosen-long", "chosen", tokens=130001, keep=64, first=1, last=4, rotary=128),
        # serving many sequences of all lengths, some shorter than what is kept, one empty slot among them
        _case("chosen-batch", "chosen", batch=64, tokens=32768, keep=32, ragged=True, rotary=128),
        # finer symbols, eight queries a head, small pages
        _case("chosen-fine", "chosen", batch=16, tokens=16000, kv_heads=4, group=8, dim=64, bits_k=7, bits_v=7, type="fp16",
              page=16, keep=128, last=2),
        # the odd heads in the framework's own type
        _case("chosen-odd-heads", "chosen", batch=32, tokens=4100, kv_heads=10, group=1, dim=41, type="fp32", ragged=True,
              page=32, keep=20, first=0),
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["shared", "shared", "bounds", "chosen", "chosen"])
    dim = rng.choice([41, 64, 80, 128, 128, 256, rng.randint(8, 256)])
    c = _case("", op, kv_heads=rng.choice([1, 2, 4, 8, 8, 10]), group=rng.choice([1, 2, 4, 4, 7, 8, 16]), dim=dim,
              bits_k=rng.choice([3, 7]), bits_v=rng.choice([3, 7]), type=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
              page=rng.choice([16, 32, 64, 128]))
    del c["name"]
    row = c["kv_heads"] * _padded(dim)
    if op == "bounds":
        if rng.random() < 0.5:
            c["tokens"] = _log_uniform(rng, 16, max(16, min(100000, (1 << 24) // row)))
        else:
            c["batch"] = _log_uniform(rng, 1, 256)
        return c
    if rng.random() < 0.6:
        c["rotary"] = 2 * rng.randint(4, dim // 2)
        c["interleaved"] = rng.random() < 0.5
    c["ragged"] = rng.random() < 0.6
    if op == "shared":
        c["batch"] = _log_uniform(rng, 1, 128)
        c["tokens"] = _log_uniform(rng, 1, max(1, min(2000, (1 << 26) // (row * c["batch"]))))
        # (rows of a head times tokens of the prefix times heads times coordinates: the work of the largest listed case)
        most = (1 << 33) // (c["batch"] * c["group"] * row)
        c["prefix"] = _log_uniform(rng, 1, max(1, min(32768, most)))
        return c
    c["batch"] = _log_uniform(rng, 1, 128)
    c["tokens"] = _log_uniform(rng, 16, max(16, min(131072, (1 << 28) // (row * c["batch"]))))
    pages = -(-c["tokens"] // c["page"])
    c["first"], c["last"] = rng.randint(0, 2), rng.randint(1, 3)
    c["keep"] = max(c["first"] + c["last"], _log_uniform(rng, 4, max(4, min(256, pages))))
    return c


# ---- sizes -------------------------------------------------------------------------------------------------

def _padded(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def _row_words(case):
    p = _padded(case["dim"])
    return p * (case["bits_k"] + 1) // 32, p * (case["bits_v"] + 1) // 32


def _head_words(case):
    return case["page"] * (sum(_row_words(case)) + 2)


def _lengths(case):
    """Tokens of every sequence: all equal, or spread down to one, with an empty one in larger batches."""
    if not case["ragged"]:
        return [case["tokens"]] * case["batch"]
    r = random.Random(case["tokens"] * 1009 + case["batch"])
    n = [_log_uniform(r, max(1, case["tokens"] // 64), case["tokens"]) for _ in range(case["batch"])]
    n[0] = case["tokens"]
    if case["batch"] > 16:
        n[case["batch"] // 2] = 0
    return n


def _filled(case):
    """Pages whose bounds are wanted, and the list's entries."""
    if case["batch"] > 1 or case["tokens"] == 1:
        return (case["batch"] + 3) // 4, case["batch"]
    n = max(1, case["tokens"] // case["page"])
    return n, n


def work(case):
    """Bytes: inputs and outputs once, a cache row and a page's bounds once.  flops: what the definition adds and multiplies."""
    e = TYPES[case["type"]].itemsize
    h, d, page = case["kv_heads"], case["dim"], case["page"]
    row = h * (4.0 * sum(_row_words(case)) + 8.0)
    if case["op"] == "bounds":
        n, entries = _filled(case)
        return {"bytes": n * h * (page * (4.0 * _row_words(case)[0] + 4) + 2 * d + 4) + 4.0 * entries, "flops": 3.0 * n * h * page * d}
    q, lengths = h * case["group"], _lengths(case)
    rows = case["batch"] * (2.0 * q * d * e + 4 * q)
    if case["op"] == "shared":
        seen = float(case["prefix"] * case["batch"] + sum(lengths))
        return {"bytes": (case["prefix"] + sum(lengths)) * row + rows + 4.0 * sum(-(-n // page) for n in lengths),
                "flops": seen * q * 4.0 * d}
    scored = seen = 0.0
    for n in lengths:
        pages = -(-n // page)
        scored += max(0, pages - case["first"] - case["last"]) if pages > case["keep"] else 0
        seen += n - max(0, pages - case["keep"]) * page
    return {"bytes": seen * row + scored * (h * (2.0 * d + 4) + 4) + rows + case["batch"] * h * (case["keep"] + 1) * 4.0,
            "flops": seen * q * 4.0 * d + scored * q * 2.0 * d}


# ---- inputs ------------------------------------------------------------------------------------------------

def _levels(bits, power, device):
    """0 = l_0 < ... < l_{n-1} = 1, finer near zero; numbers of 11 bits, as the cache keeps them."""
    n = 1 << bits
    return torch.tensor([(j / (n - 1)) ** power for j in range(n)], dtype=torch.float64).half().float().to(device)


def _rotary_table(positions, dim):
    """[positions][dim]: cosines of the dim / 2 angles, then sines."""
    f = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def _random_pages(case, num_pages, levels_k, levels_v, gen):
    """Pages of quantised normal values: symbols by nearest rounding of |z| / 3.5, norms around 3."""
    h, page, p = case["kv_heads"], case["page"], _padded(case["dim"])
    pages = torch.empty((num_pages, h, _head_words(case)), dtype=torch.int32, device="cuda")
    some = max(1, (1 << 26) // (h * page * p))
    for at in range(0, num_pages, some):
        n = min(some, num_pages - at)
        parts = []
        for bits, levels in ((case["bits_k"], levels_k), (case["bits_v"], levels_v)):
            z = torch.randn((n, h, page, p), generator=gen, device="cuda")
            middles = ((levels[1:] + levels[:-1]) * 1.75).contiguous()
            sym = torch.bucketize(z.abs(), middles, out_int32=True) * 2 + (z < 0)
            sym[..., case["dim"]:] = 0
            if bits == 3:
                sym = sym[..., 0::2] + 16 * sym[..., 1::2]
            parts.append(sym.to(torch.uint8).view(torch.int32).reshape(n, h, -1))
        norms = (torch.randn((n, h, 2 * page), generator=gen, device="cuda") * 0.2 + 1.1).exp()
        pages[at: at + n] = torch.cat([*parts, norms.view(torch.int32)], dim=2)
    return pages.view(num_pages, -1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = random.Random(seed)
    h, d, page = case["kv_heads"], case["dim"], case["page"]
    power = 1.2 + 0.2 * host.random()
    s = dict(case=case, levels_k=_levels(case["bits_k"], power, "cuda"), levels_v=_levels(case["bits_v"], power, "cuda"))
    if own:
        import paper_2505_14371_b200 as lq
        s["cache"] = lq.Cache(num_layers=1, kv_heads=h, head_dim=d, page_size=page, bits=(case["bits_k"], case["bits_v"]),
                              seed=SEED + seed)
        s["cache"].lq_cache_set_levels(0, "keys", s["levels_k"].tolist())
        s["cache"].lq_cache_set_levels(0, "values", s["levels_v"].tolist())
    if case["op"] == "bounds":
        n, entries = _filled(case)
        s["pages"] = _random_pages(case, n + 3, s["levels_k"], s["levels_v"], gen)
        s["which"] = torch.full((entries,), -1, dtype=torch.int32, device="cuda")
        s["which"][torch.randperm(entries, generator=gen, device="cuda")[:n]] = torch.randperm(n + 3, generator=gen, device="cuda")[:n].int()
        if own:
            s["bounds"] = s["cache"].empty_bounds(n + 3)
        else:
            s["upper"], s["lower"] = (torch.zeros((n + 3, h, d), dtype=torch.int8, device="cuda") for _ in range(2))
            s["scales"] = torch.zeros((n + 3, h), device="cuda")
        return s
    lengths, shared = _lengths(case), -(-case["prefix"] // page)
    width = max(1, max(-(-n // page) for n in lengths))
    num_pages = shared + sum(-(-n // page) for n in lengths) + 3
    order = torch.randperm(num_pages, generator=gen, device="cuda").to(torch.int32)
    s["prefix"] = order[:shared].contiguous()
    s["table"] = torch.full((case["batch"], width), -1, dtype=torch.int32, device="cuda")
    at = shared
    for b, n in enumerate(lengths):
        k = -(-n // page)
        s["table"][b, :k] = order[at: at + k]
        at += k
    s["prefix_length"] = torch.tensor([case["prefix"]], dtype=torch.int32, device="cuda")
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["pages"] = _random_pages(case, num_pages, s["levels_k"], s["levels_v"], gen)
    s["queries"] = torch.randn((case["batch"], h * case["group"], d), generator=gen, device="cuda").to(TYPES[case["type"]])
    if case["rotary"]:
        s["rotary"] = _rotary_table(max(case["prefix"] + max(lengths), 1), case["rotary"])
        s["positions"] = (s["lengths"].long() - 1).clamp(min=0)
    if case["op"] == "chosen":
        # the bounds of the pages, which the program keeps beside them as they fill
        if own:
            s["bounds"] = s["cache"].empty_bounds(num_pages)
            s["cache"].lq_cache_bounds(0, s["pages"], torch.arange(num_pages, dtype=torch.int32, device="cuda"), s["bounds"])
        else:
            parts = [_bounds_of(case, s["pages"][i: i + 1024], s["levels_k"]) for i in range(0, num_pages, 1024)]
            s["upper"], s["lower"], s["scales"] = (torch.cat(x) for x in zip(*parts))
    return s


# ---- plain forms -------------------------------------------------------------------------------------------

def _rotated(x, table, interleaved):
    """x [..., dim] in 32 bits, table rows [..., 2 * pairs]: every pair turned by its angle."""
    n = table.shape[-1] // 2
    c, s = table[..., :n], table[..., n:]
    a, b = (x[..., 0: 2 * n: 2], x[..., 1: 2 * n: 2]) if interleaved else (x[..., :n], x[..., n: 2 * n])
    y, z = a * c - b * s, b * c + a * s
    pair = torch.stack([y, z], dim=-1).flatten(-2) if interleaved else torch.cat([y, z], dim=-1)
    return torch.cat([pair, x[..., 2 * n:]], dim=-1)


def _symbol_values(levels):
    """The signed level of every symbol, or of both symbols of a byte where they have 4 bits: [256][symbols]."""
    both = torch.stack([levels, -levels], dim=1).reshape(-1)
    if both.numel() == 256:
        return both[:, None]
    return torch.stack([both.repeat(16), both.repeat_interleave(16)], dim=1)


def _unpacked(codes, norms, levels, dim):
    """codes int32 [..., words], norms fp32 [...] -> values [..., dim] in 32 bits."""
    v = _symbol_values(levels)[codes.view(torch.uint8).int()].flatten(-2)[..., :dim]
    return v * norms[..., None]


def _parts(case, pages):
    """Views of pages [..., words of a page]: keys' and values' codes [..., heads, page, row words], norms [..., heads, page]."""
    page, (rk, rv) = case["page"], _row_words(case)
    w = pages.unflatten(-1, (case["kv_heads"], _head_words(case)))
    ck, cv, nk, nv = w.split([page * rk, page * rv, page, page], dim=-1)
    return ck.unflatten(-1, (page, rk)), cv.unflatten(-1, (page, rv)), nk.view(torch.float32), nv.view(torch.float32)


def _bounds_of(case, pages, levels):
    """Upper and lower bounds [pages][heads][dim] int8 and scales [pages][heads] of the keys of whole pages."""
    ck, _, nk, _ = _parts(case, pages)
    k = _unpacked(ck.contiguous(), nk, levels, case["dim"])
    n = nk.amax(-1)
    kept = (n >= 2.0 ** -100) & (n < math.inf)
    inv = torch.where(kept, 127.0 / n, torch.zeros_like(n))[..., None]
    upper = (k.amax(2) * inv).ceil().clamp(-127, 127)
    lower = (k.amin(2) * inv).floor().clamp(-127, 127)
    return upper.to(torch.int8), lower.to(torch.int8), torch.where(kept, n / 127.0, torch.zeros_like(n))


def _bounds(s):
    which = s["which"][s["which"] >= 0].long()
    s["upper"][which], s["lower"][which], s["scales"][which] = _bounds_of(s["case"], s["pages"][which], s["levels_k"])
    return {"upper": s["upper"], "lower": s["lower"], "scales": s["scales"]}


def _queries(s, positions):
    """Queries in 32 bits, rotated by their positions: [batch][heads of the cache][group][dim]."""
    case, q = s["case"], s["queries"].float()
    if case["rotary"]:
        q = _rotated(q, s["rotary"][positions][:, None, :], case["interleaved"])
    return q.view(case["batch"], case["kv_heads"], case["group"], case["dim"])


def _tokens(case, pages, levels_k, levels_v):
    """pages [..., n, words]: keys and values [..., heads, n * page, dim] in 32 bits."""
    out = []
    for codes, norms, levels in zip(*(lambda ck, cv, nk, nv: ((ck, cv), (nk, nv)))(*_parts(case, pages)), (levels_k, levels_v)):
        codes, norms = codes.transpose(-4, -3).flatten(-3, -2), norms.transpose(-3, -2).flatten(-2, -1)
        out.append(_unpacked(codes.contiguous(), norms, levels, case["dim"]))
    return out


def _weighed(scores, top):
    return (scores - top.clamp(min=-1e30)).exp()


def _shared(s):
    case = s["case"]
    b, h, g, d = case["batch"], case["kv_heads"], case["group"], case["dim"]
    length, lengths = s["prefix_length"].long(), s["lengths"].long()
    q = _queries(s, (length + lengths - 1).clamp(min=0)) * d ** -0.5
    kp, vp = _tokens(case, s["pages"][s["prefix"].long()], s["levels_k"], s["levels_v"])            # [heads][prefix][dim]
    rows = q.transpose(0, 1).reshape(h, b * g, d)
    sp = rows @ kp.transpose(1, 2)
    sp = sp.masked_fill(torch.arange(sp.shape[-1], device=q.device) >= length, -math.inf)
    ko, vo = _tokens(case, s["pages"][s["table"].clamp(min=0).long()], s["levels_k"], s["levels_v"])    # [batch][heads][own][dim]
    so = q @ ko.transpose(2, 3)
    so = so.masked_fill((torch.arange(so.shape[-1], device=q.device) >= lengths[:, None])[:, None, None], -math.inf)
    tp = sp.amax(-1, keepdim=True) if sp.shape[-1] else sp.new_full((h, b * g, 1), -math.inf)
    tp = tp.view(h, b, g, 1).transpose(0, 1)
    top = torch.maximum(tp, so.amax(-1, keepdim=True))
    wp, wo = _weighed(sp, top.transpose(0, 1).reshape(h, b * g, 1)), _weighed(so, top)
    total = wp.sum(-1, keepdim=True).view(h, b, g, 1).transpose(0, 1) + wo.sum(-1, keepdim=True)
    out = (wp @ vp).view(h, b, g, d).transpose(0, 1) + wo @ vo
    out = out / torch.where(total > 0, total, torch.ones_like(total))
    return {"out": out.reshape(b, h * g, d).to(TYPES[case["type"]]), "lse": (top + total.log()).reshape(b, h * g)}


def _chosen(s):
    case = s["case"]
    b, h, g, d, page, keep = (case[x] for x in ("batch", "kv_heads", "group", "dim", "page", "keep"))
    lengths, table = s["lengths"].long(), s["table"].clamp(min=0).long()
    q = _queries(s, s["positions"] if case["rotary"] else None)
    # the queries as whole numbers, and the scores of all pages of the tables
    top = q.abs().amax(-1, keepdim=True)
    kept = (top >= 2.0 ** -100) & (top < math.inf)
    whole = torch.where(kept, (q * torch.where(kept, 127.0 / top, top)).round(), torch.zeros_like(q))
    per = torch.where(kept, top / 127.0, torch.zeros_like(top))
    # (sums of whole numbers below 2^24: exact in 32 bits)
    upper, lower = (x[table].float().permute(0, 2, 3, 1) for x in (s["upper"], s["lower"]))        # [batch][heads][dim][pages]
    score = (whole.clamp(min=0) @ upper + whole.clamp(max=0) @ lower) * per
    score = (score * s["scales"][table].permute(0, 2, 1)[:, :, None]).amax(2)                       # [batch][heads][pages]
    pages = (lengths + page - 1) // page
    at = torch.arange(table.shape[1], device=q.device)
    must = (at < case["first"]) | (at >= pages[:, None] - case["last"])
    score = score.masked_fill(must[:, None], math.inf).masked_fill((at >= pages[:, None])[:, None], -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    best = torch.nn.functional.pad(best, (0, keep - best.shape[-1]), value=table.shape[1])
    best = torch.where(best < pages[:, None, None], best, torch.full_like(best, table.shape[1])).sort(dim=-1).values
    there = best < pages[:, None, None]
    numbers = table[:, None].expand(-1, h, -1).gather(2, best.clamp(max=table.shape[1] - 1))
    chosen = torch.where(there, numbers, torch.full_like(numbers, -1)).int()
    seen = (lengths - (pages - keep).clamp(min=0) * page)[:, None].expand(-1, h)
    # every head's own pages: [batch][heads][keep][head words]
    words = s["pages"].view(-1, h, _head_words(case))[numbers, torch.arange(h, device=q.device)[:, None]]
    one = dict(case, kv_heads=1)
    k, v = (x[:, :, 0] for x in _tokens(one, words, s["levels_k"], s["levels_v"]))
    scores = (q * d ** -0.5) @ k.transpose(2, 3)
    scores = scores.masked_fill((torch.arange(keep * page, device=q.device) >= seen[..., None])[:, :, None], -math.inf)
    most = scores.amax(-1, keepdim=True)
    w = _weighed(scores, most)
    total = w.sum(-1, keepdim=True)
    out = (w @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return {"chosen": chosen, "seen": seen.int(), "out": out.reshape(b, h * g, d).to(TYPES[case["type"]]),
            "lse": (most + total.log()).reshape(b, h * g)}


# ---- one pass ----------------------------------------------------------------------------------------------

def _own(s):
    case, cache = s["case"], s["cache"]
    h, d = case["kv_heads"], case["dim"]
    if case["op"] == "bounds":
        cache.lq_cache_bounds(0, s["pages"], s["which"], s["bounds"])
        values = s["bounds"][:, : h * _padded(d) // 2].view(torch.int8).unflatten(1, (h, 2, _padded(d)))
        scales = s["bounds"][:, h * _padded(d) // 2: h * _padded(d) // 2 + h].view(torch.float32)
        return {"upper": values[:, :, 0, :d], "lower": values[:, :, 1, :d], "scales": scales}
    layout = "interleaved" if case["interleaved"] else "half"
    out = torch.empty_like(s["queries"])
    lse = torch.empty(out.shape[:2], dtype=torch.float32, device=out.device)
    if case["op"] == "shared":
        cache.lq_cache_attend_shared(0, s["queries"], s["pages"], s["prefix"], s["prefix_length"], s["table"], s["lengths"], out,
                                     lse=lse, rotary=s.get("rotary"), layout=layout)
        return {"out": out, "lse": lse}
    chosen = torch.empty((case["batch"], h, case["keep"]), dtype=torch.int32, device=out.device)
    seen = torch.empty((case["batch"], h), dtype=torch.int32, device=out.device)
    turn = dict(rotary=s.get("rotary"), positions=s.get("positions"), layout=layout)
    cache.lq_cache_choose(s["queries"], s["bounds"], s["table"], s["lengths"], chosen, seen, first=case["first"], last=case["last"],
                          **turn)
    cache.lq_cache_attend_chosen(0, s["queries"], s["pages"], chosen, seen, out, lse=lse, **turn)
    return {"chosen": chosen, "seen": seen, "out": out, "lse": lse}


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    return _shared(s) if op == "shared" else _bounds(s) if op == "bounds" else _chosen(s)


# ---- the definition in 64 bits -----------------------------------------------------------------------------

def _turned(x, angles, interleaved, rounded):
    """x [..., dim] in 64 bits with its pairs turned by the table's angles; `rounded`: with the 32-bit numbers of the keys'
    definition."""
    n = angles.shape[-1] // 2
    pairs = [slice(0, 2 * n, 2), slice(1, 2 * n, 2)] if interleaved else [slice(0, n), slice(n, 2 * n)]
    f = (lambda v: v.float().double()) if rounded else (lambda v: v)
    re, im, cos, sin = x[..., pairs[0]], x[..., pairs[1]], angles[..., :n].double(), angles[..., n:].double()
    y = x.clone()
    y[..., pairs[0]] = f(f(re * cos) - f(im * sin))
    y[..., pairs[1]] = f(f(re * sin) + f(im * cos))
    return y


def _exact_cached(case, words, norms, levels):
    """Symbols of [tokens][heads][words] by shifts, and the values that they stand for."""
    bits = 4 if levels.numel() == 8 else 8
    shifts = torch.arange(0, 32, bits, device=words.device, dtype=torch.int32)
    sym = ((words[..., None] >> shifts) & ((1 << bits) - 1)).flatten(-2)[..., :case["dim"]].long()
    return levels.double()[sym >> 1] * (1 - 2 * (sym & 1)) * norms.double()[..., None]


def _exact_tokens(case, s, slots):
    """Keys and values of slots in 64 bits, [tokens][heads][dim]."""
    page, (rk, rv), hw = case["page"], _row_words(case), _head_words(case)
    w = s["pages"].view(-1, case["kv_heads"], hw)
    at, row = slots // page, slots % page

    def section(begin, words):
        cols = begin + row[:, None] * words + torch.arange(words, device=slots.device)
        return w[at].gather(2, cols[:, None, :].expand(-1, case["kv_heads"], -1))

    nk, nv = (section(page * (rk + rv) + i * page, 1)[..., 0].contiguous().view(torch.float32) for i in (0, 1))
    return (_exact_cached(case, section(0, rk), nk, s["levels_k"]),
            _exact_cached(case, section(page * rk, rv), nv, s["levels_v"]))


def _exact_bounds(case, s, number):
    """Bounds of the keys of one page: whole numbers [heads][dim] twice, scales [heads], all held in 64 bits."""
    slots = number * case["page"] + torch.arange(case["page"], device="cuda")
    h, page, rk = case["kv_heads"], case["page"], _row_words(case)[0]
    v = _exact_tokens(case, s, slots)[0].float().double()               # a value is the rounded product of level and norm
    w = s["pages"].view(-1, h, _head_words(case))[number]
    norms = w[:, page * sum(_row_words(case)): page * (sum(_row_words(case)) + 1)].contiguous().view(torch.float32).double()
    n = norms.max(1).values
    bad = ~((n >= 2.0 ** -100) & (n < math.inf))
    inv = (127.0 / n.masked_fill(bad, 1.0)).float().double()[:, None]
    upper = torch.ceil((v.max(0).values * inv).float().double()).clamp(-127, 127)
    lower = torch.floor((v.min(0).values * inv).float().double()).clamp(-127, 127)
    return (upper.masked_fill(bad[:, None], 0), lower.masked_fill(bad[:, None], 0),
            (n / 127.0).float().double().masked_fill(bad, 0.0))


def _exact_shared(case, s):
    h, g, d, page, length = case["kv_heads"], case["group"], case["dim"], case["page"], case["prefix"]
    out = torch.zeros((case["batch"], h * g, d), dtype=torch.float64, device="cuda")
    lse = torch.full((case["batch"], h * g), -math.inf, dtype=torch.float64, device="cuda")

    def tokens(pages, n):
        ids = torch.arange(n, device="cuda")
        parts = [_exact_tokens(case, s, pages.long()[x // page] * page + x % page) for x in ids.split(8192)]
        return torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])

    before = tokens(s["prefix"], length) if length else None
    for b, n in enumerate(_lengths(case)):
        if length + n == 0:
            continue
        q = s["queries"][b].double()
        if case["rotary"]:
            q = _turned(q, s["rotary"][length + n - 1][None, :].expand(h * g, -1), case["interleaved"], False)
        q = q.view(h, g, d) / math.sqrt(d)
        parts = ([before] if length else []) + ([tokens(s["table"][b], n)] if n else [])
        z = torch.cat([torch.einsum("hgd,thd->hgt", q, k) for k, _ in parts], dim=2)
        p = torch.softmax(z, -1).split([k.shape[0] for k, _ in parts], dim=2)
        out[b] = sum(torch.einsum("hgt,thd->hgd", w, v) for w, (_, v) in zip(p, parts)).reshape(h * g, d)
        lse[b] = torch.logsumexp(z, -1).reshape(-1)
    return {"out": out, "lse": lse}


def _exact_chosen(case, s):
    b, h, g, d, page, keep = (case[x] for x in ("batch", "kv_heads", "group", "dim", "page", "keep"))
    result = {"chosen": torch.full((b, h, keep), -1, dtype=torch.int32, device="cuda"),
              "seen": torch.zeros((b, h), dtype=torch.int32, device="cuda"),
              "out": torch.zeros((b, h * g, d), dtype=torch.float64, device="cuda"),
              "lse": torch.full((b, h * g), -math.inf, dtype=torch.float64, device="cuda")}
    for i, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        q = plain = s["queries"][i].double()
        if case["rotary"]:
            angles = s["rotary"][n - 1][None, :].expand(h * g, -1)
            q, plain = (_turned(plain, angles, case["interleaved"], r) for r in (True, False))
        count = -(-n // page)
        kept = [list(range(count))] * h
        middle = list(range(case["first"], count - case["last"]))
        if count > keep:
            big = q.abs().max(1).values
            whole = torch.round((q * (127.0 / big).float().double()[:, None]).float().double()).view(h, g, 1, d)
            per = (big / 127.0).float().double().view(h, g, 1)
            some = [_exact_bounds(case, s, x) for x in s["table"][i, middle].tolist()]
            upper, lower, scales = (torch.stack([x[j] for x in some], dim=1) for j in range(3))     # [heads][pages][dim]
            dots = torch.maximum(whole * upper[:, None], whole * lower[:, None]).sum(-1)
            score = ((dots * per).float().double() * scales[:, None]).float().max(1).values.tolist()
            kept = [sorted(list(range(case["first"])) + list(range(count - case["last"], count)) +
                           sorted(middle, key=lambda x: (-score[j][x - case["first"]], x))[:keep - case["first"] - case["last"]])
                    for j in range(h)]
        for j in range(h):
            numbers = s["table"][i, kept[j]]
            result["chosen"][i, j, :len(kept[j])] = numbers
            seen = n - max(0, count - keep) * page
            result["seen"][i, j] = seen
            at = torch.arange(seen, device="cuda")
            k, v = (x[:, j] for x in _exact_tokens(case, s, numbers.long()[at // page] * page + at % page))
            z = plain.view(h, g, d)[j] @ k.T / math.sqrt(d)
            result["out"][i, j * g: (j + 1) * g] = torch.softmax(z, -1) @ v
            result["lse"][i, j * g: (j + 1) * g] = torch.logsumexp(z, -1)
    return result


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "shared":
        return _exact_shared(case, s)
    if case["op"] == "chosen":
        return _exact_chosen(case, s)
    n, h, d = s["pages"].shape[0], case["kv_heads"], case["dim"]
    upper, lower = (torch.zeros((n, h, d), dtype=torch.int8, device="cuda") for _ in range(2))
    scales = torch.zeros((n, h), dtype=torch.float64, device="cuda")
    for number in s["which"].tolist():
        if number >= 0:
            u, v, scales[number] = _exact_bounds(case, s, number)
            upper[number], lower[number] = u.to(torch.int8), v.to(torch.int8)
    return {"upper": upper, "lower": lower, "scales": scales}
