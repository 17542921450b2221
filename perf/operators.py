"""Cases of the quantised key-value cache: rows stored and read back, rows read back, attention of one new token.

The cache holds one fp32 norm and one symbol per coordinate for every (token, head) row of keys and of values: the row's
L^q norm N, and for each coordinate 2 * (index of a level) + sign, where the level is one of the two neighbours of
u = min(|x| * (1 / N), 1) in the level set of the (layer, keys or values).  A symbol has 4 or 8 bits.

A page of the cache is int32 words: for each head the keys' rows of all its tokens, the values' rows, the keys' norms and
the values' norms.  A row has head_dim symbols, little endian, and zeros up to 64, 128 or 256 of them.

Operators ("op" of a case):
  store    rows of keys (rotated by their positions where the case has a rotary dimension) and values quantised into their
           slots, and read back from there, as a prompt's later attention over whole rows does
  read     rows of many slots read back: the context of a request that goes on
  attend   one new token a sequence against its pages: softmax(scale * q K^T) V and the log of the softmax's denominator

Plain forms compute in 32 bits: the rotary tables are inputs, made in 64; norms are summed in 64.  What stands beside a
border between two levels is a 32-bit number by definition: a rotated coordinate (each product and their sum), u (one product
of |x| with the rounded reciprocal of the norm), and the product that the stochastic rounding compares with.
"""
import math
import random

import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SEED = 20250514


def _case(name, op, **over):
    c = dict(name=name, op=op, batch=1, tokens=1, kv_heads=8, group=4, dim=128, bits_k=3, bits_v=3, norm=0, type="bf16",
             page=64, rotary=0, interleaved=False, step=-1, ragged=False, window=0)
    c.update(over)
    return c


def listed():
    return [
        # one sequence is served: the new token's rows go into the cache; latency is all
        _case("store-one-token", "store", tokens=1, rotary=128),
        # a decoding step of 256 sequences, each at a place of its own; small heads, fine symbols
        _case("store-decoding-step", "store", tokens=256, dim=64, bits_k=7, bits_v=7, norm=2, type="fp16", page=16,
              rotary=32, interleaved=True),
        # a long prompt, in coarse symbols
        _case("store-prompt", "store", tokens=16384, rotary=128),
        # segments of a training run's recurrent memory, 10 heads of 41 as in the Transformer-XL shapes of this repository,
        # unbiased rounding
        _case("store-segments-unbiased", "store", tokens=9600, kv_heads=10, dim=41, bits_k=7, bits_v=7, norm=2, type="fp32",
              page=32, step=7),
        # a short prefix that a new request shares
        _case("read-prefix", "read", tokens=777, type="fp16", dim=64, bits_k=7, bits_v=7, page=16),
        # the whole context of a long conversation
        _case("read-context", "read", tokens=100003),
        # the start of an answer: few tokens so far
        _case("attend-short", "attend", tokens=200, rotary=128),
        # one sequence, a very long context: the cache's length has to be split
        _case("attend-long", "attend", tokens=130001, rotary=128),
        # serving many sequences of all lengths, some just begun, one empty slot among them
        _case("attend-batch-ragged", "attend", batch=64, tokens=16384, ragged=True, rotary=128),
        # finer symbols for both, eight queries a head
        _case("attend-batch-fine", "attend", batch=32, tokens=4096, group=8, bits_k=7, bits_v=7, type="fp16"),
        # one head of keys for all queries, wide heads, only the last tokens seen
        _case("attend-one-head-window", "attend", batch=24, tokens=9000, kv_heads=1, group=16, dim=256, bits_k=7, window=4096,
              ragged=True),
        # the odd heads of the Transformer-XL shapes in the framework's own type
        _case("attend-odd-heads", "attend", batch=48, tokens=2050, kv_heads=10, group=1, dim=41, type="fp32", ragged=True,
              page=32),
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["store", "read", "attend", "attend"])
    dim = rng.choice([41, 64, 80, 128, 128, 256, rng.randint(8, 256)])
    c = _case("", op, kv_heads=rng.choice([1, 2, 4, 8, 8, 10, 16]), group=rng.choice([1, 2, 4, 4, 7, 8, 16]), dim=dim,
              bits_k=rng.choice([3, 7]), bits_v=rng.choice([3, 7]), norm=rng.choice([0, 0, 1, 2]),
              type=rng.choice(["bf16", "bf16", "fp16", "fp32"]), page=rng.choice([16, 32, 64, 128]))
    del c["name"]
    if op != "read" and rng.random() < 0.6:
        c["rotary"] = 2 * rng.randint(4, dim // 2)
        c["interleaved"] = rng.random() < 0.5
    row = c["kv_heads"] * _padded(dim)
    if op == "attend":
        c["batch"] = _log_uniform(rng, 1, 256)
        # (the padded rows of a batch in 32 bits are what the plain form takes memory for)
        c["tokens"] = _log_uniform(rng, 16, max(16, min(131072, (1 << 28) // (row * c["batch"]))))
        c["ragged"] = rng.random() < 0.6
        c["window"] = rng.choice([0, 0, 0, max(1, c["tokens"] // 3)])
    else:
        c["tokens"] = _log_uniform(rng, 1, max(1, min(100000, (1 << 23 if op == "store" else 1 << 26) // row)))
        if op == "store" and rng.random() < 0.4:
            c["step"] = rng.randint(0, 1000)
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


def work(case):
    """Bytes: inputs and outputs once, a cache row once (written, or read).  flops: what the definition adds and multiplies."""
    e = TYPES[case["type"]].itemsize
    h, d = case["kv_heads"], case["dim"]
    row = h * (4.0 * sum(_row_words(case)) + 8.0)
    t = float(case["tokens"])
    if case["op"] == "store":
        return {"bytes": t * (2 * h * d * e + row + 2 * h * d * e + 8 + 8 * bool(case["rotary"]) + 4 * case["rotary"]),
                "flops": t * h * (2 * 8 * d + 3 * case["rotary"])}
    if case["op"] == "read":
        return {"bytes": t * (row + 2 * h * d * e + 8), "flops": t * 2 * h * d}
    seen = float(sum(min(n, case["window"] or n) for n in _lengths(case)))
    q = h * case["group"]
    return {"bytes": seen * row + case["batch"] * (2 * q * d * e + 4 * q), "flops": seen * q * 4.0 * d}


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
    op, h, d, page, t = case["op"], case["kv_heads"], case["dim"], case["page"], case["tokens"]
    dtype = TYPES[case["type"]]
    power = 1.2 + 0.2 * host.random()
    s = dict(case=case, levels_k=_levels(case["bits_k"], power, "cuda"), levels_v=_levels(case["bits_v"], power, "cuda"),
             seed=SEED + seed)
    if own:
        import paper_2505_14371_b200 as lq
        s["cache"] = lq.Cache(num_layers=1, kv_heads=h, head_dim=d, page_size=page, bits=(case["bits_k"], case["bits_v"]),
                              q=case["norm"], seed=s["seed"])
        s["cache"].lq_cache_set_levels(0, "keys", s["levels_k"].tolist())
        s["cache"].lq_cache_set_levels(0, "values", s["levels_v"].tolist())
    if op == "attend":
        lengths = _lengths(case)
        width = max(1, max(-(-n // page) for n in lengths))
        num_pages = sum(-(-n // page) for n in lengths) + 3
        order = torch.randperm(num_pages, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((case["batch"], width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(lengths):
            k = -(-n // page)
            table[b, :k] = order[at: at + k]
            at += k
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["table"] = table
        s["pages"] = _random_pages(case, num_pages, s["levels_k"], s["levels_v"], gen)
        s["queries"] = torch.randn((case["batch"], h * case["group"], d), generator=gen, device="cuda").to(dtype)
        if case["rotary"]:
            s["rotary"] = _rotary_table(max(max(lengths), 1), case["rotary"])
        return s
    num_pages = -(-t // page) + 3
    if op == "read":
        # whole pages in any order, as a sequence's table lists them
        order = torch.randperm(num_pages, generator=gen, device="cuda")
        s["slots"] = (order[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)[:t].contiguous()
        s["pages"] = _random_pages(case, num_pages, s["levels_k"], s["levels_v"], gen)
        return s
    # keys and values as the projection before them leaves them: parts of one row a token, beside its queries
    heads = h * (case["group"] + 2)
    z = torch.randn((t, heads, d), generator=gen, device="cuda")
    loud = torch.rand((1, heads, d), generator=gen, device="cuda") < 0.03      # a few coordinates are larger in every token
    rows = torch.where(loud, z * 5.0, z).to(dtype)
    s["keys"], s["values"] = rows[:, h * case["group"]: h * (case["group"] + 1)], rows[:, h * (case["group"] + 1):]
    order = torch.randperm(num_pages * page, generator=gen, device="cuda") if t <= 256 else (
        torch.randperm(num_pages, generator=gen, device="cuda")[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)
    s["slots"] = order[:t].contiguous()
    s["pages"] = torch.zeros((num_pages, h * _head_words(case)), dtype=torch.int32, device="cuda")
    if case["rotary"]:
        s["rotary"] = _rotary_table(32768, case["rotary"])
        first = host.randint(0, 32768 - t) if t > 256 else 0
        s["positions"] = torch.arange(first, first + t, device="cuda") if t > 256 else torch.randint(
            0, 32768, (t,), generator=gen, device="cuda")
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


def _mulhilo(a, b):
    """High and low 32 bits of the product of two 32-bit numbers held in int64."""
    lo = (a & 0xFFFF) * b
    hi = (a >> 16) * b + (lo >> 16)
    return hi >> 16, ((hi & 0xFFFF) << 16) | (lo & 0xFFFF)


def _philox_uniform(seed, slots, heads, dim, which, step):
    """[tokens][heads][dim] uniforms on the 2^-23 grid: Philox4x32-10, counter (coordinate / 4, which, slot, step), where a
    head's coordinates start at a multiple of its padded size."""
    device, p = slots.device, _padded(dim)
    c0 = (torch.arange(heads * p, device=device)[::4] // 4)[None, :] + 0 * slots[:, None]
    c1 = torch.full_like(c0, which)
    c2 = slots[:, None] + 0 * c0
    c3 = torch.full_like(c0, step)
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        h0, l0 = _mulhilo(torch.full_like(c0, 0xD2511F53), c0)
        h1, l1 = _mulhilo(torch.full_like(c0, 0xCD9E8D57), c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack([c0, c1, c2, c3], dim=-1).view(slots.shape[0], heads, p)[..., :dim]
    return (words >> 9).float() * 2.0 ** -23


def _quantised(x, levels, q, uniform):
    """The values that rows x [..., dim] in 32 bits are kept as."""
    a = x.abs()
    n = a.amax(-1) if q == 0 else (a.double().sum(-1) if q == 1 else a.double().square().sum(-1).sqrt()).float()
    n = torch.where((n >= 2.0 ** -126) & (n < math.inf), n, torch.zeros_like(n))[..., None]
    u = (a * torch.where(n > 0, 1.0 / n, n)).clamp(max=1.0)
    at = torch.bucketize(u, levels[1:-1].contiguous(), right=True)
    low, high = levels[at], levels[at + 1]
    taken = torch.where(uniform * (high - low) < u - low, high, low)
    return torch.where(x < 0, -taken, taken) * n


def _store(s):
    case = s["case"]
    k, v = s["keys"].float(), s["values"].float()
    if case["rotary"]:
        k = _rotated(k, s["rotary"][s["positions"]][:, None, :], case["interleaved"])
    uk = uv = 0.5
    if case["step"] >= 0:
        uk, uv = (_philox_uniform(s["seed"], s["slots"], case["kv_heads"], case["dim"], w, case["step"]) for w in (0, 1))
    dtype = TYPES[case["type"]]
    return {"keys": _quantised(k, s["levels_k"], case["norm"], uk).to(dtype),
            "values": _quantised(v, s["levels_v"], case["norm"], uv).to(dtype)}


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


def _read(s):
    case, slots = s["case"], s["slots"]
    ck, cv, nk, nv = _parts(case, s["pages"])
    at, row, dtype = slots // case["page"], slots % case["page"], TYPES[case["type"]]
    return {"keys": _unpacked(ck[at, :, row].contiguous(), nk[at, :, row], s["levels_k"], case["dim"]).to(dtype),
            "values": _unpacked(cv[at, :, row].contiguous(), nv[at, :, row], s["levels_v"], case["dim"]).to(dtype)}


def _attend(s):
    case = s["case"]
    h, g, d = case["kv_heads"], case["group"], case["dim"]
    q, lengths = s["queries"].float(), s["lengths"].long()
    if case["rotary"]:
        q = _rotated(q, s["rotary"][(lengths - 1).clamp(min=0)][:, None, :], case["interleaved"])
    ck, cv, nk, nv = _parts(case, s["pages"][s["table"].clamp(min=0).long()])
    # [batch][page of the table][heads][token] -> [batch][heads][tokens]
    k = _unpacked(ck.transpose(1, 2).flatten(2, 3).contiguous(), nk.transpose(1, 2).flatten(2, 3), s["levels_k"], d)
    scores = (q.view(-1, h, g, d) * d ** -0.5) @ k.transpose(2, 3)
    del k
    place = torch.arange(scores.shape[-1], device=q.device)
    seen = place < lengths[:, None]
    if case["window"]:
        seen &= place >= lengths[:, None] - case["window"]
    scores = scores.masked_fill(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = (scores - top.clamp(min=-1e30)).exp()
    total = p.sum(-1, keepdim=True)
    v = _unpacked(cv.transpose(1, 2).flatten(2, 3).contiguous(), nv.transpose(1, 2).flatten(2, 3), s["levels_v"], d)
    out = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return {"out": out.reshape(-1, h * g, d).to(TYPES[case["type"]]), "lse": (top + total.log()).view(-1, h * g)}


# ---- one pass ----------------------------------------------------------------------------------------------

def _own(s):
    case, cache = s["case"], s["cache"]
    layout = "interleaved" if case["interleaved"] else "half"
    if case["op"] == "attend":
        out = torch.empty_like(s["queries"])
        lse = torch.empty(out.shape[:2], dtype=torch.float32, device=out.device)
        cache.lq_cache_attend(0, s["queries"], s["pages"], s["table"], s["lengths"], out, lse=lse, window=case["window"],
                              rotary=s.get("rotary"), layout=layout)
        return {"out": out, "lse": lse}
    if case["op"] == "store":
        cache.lq_cache_write(0, s["keys"], s["values"], s["slots"], s["pages"],
                             step=case["step"] if case["step"] >= 0 else None, rotary=s.get("rotary"),
                             positions=s.get("positions"), layout=layout)
    shape = (case["tokens"], case["kv_heads"], case["dim"])
    keys = torch.empty(shape, dtype=TYPES[case["type"]], device="cuda")
    values = torch.empty_like(keys)
    cache.lq_cache_read(0, s["pages"], s["slots"], keys, values)
    return {"keys": keys, "values": values}


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    return _store(s) if op == "store" else _read(s) if op == "read" else _attend(s)


# ---- the definition in 64 bits -----------------------------------------------------------------------------

def _exact_rows(x, levels, q, rho):
    """x [rows][dim] in 64 bits; N, 1 / N and u as the 32-bit numbers that they are by definition."""
    a = x.abs()
    n = (a.max(1).values if q == 0 else a.pow(q).sum(1).pow(1.0 / q)).float().double()
    u = torch.minimum((a * (1.0 / n).float().double()[:, None]).float().double(), torch.ones((), dtype=torch.float64, device=x.device))
    lv = levels.double()
    at = (torch.searchsorted(lv, u, right=True) - 1).clamp(max=lv.numel() - 2)
    gap = lv[at + 1] - lv[at]
    up = (rho * gap).float().double() < u - lv[at]
    return torch.sign(x) * lv[at + up.long()] * n[:, None]


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


def exact(case, seed):
    s = prepare(case, seed)
    h, g, d, page = case["kv_heads"], case["group"], case["dim"], case["page"]
    if case["op"] == "store":
        k, v = s["keys"].double(), s["values"].double()
        if case["rotary"]:
            k = _turned(k, s["rotary"][s["positions"]][:, None, :].expand(-1, h, -1), case["interleaved"], True)
        rho = [torch.full((), 0.5, dtype=torch.float64, device=k.device)] * 2
        if case["step"] >= 0:
            rho = [_philox_uniform(s["seed"], s["slots"], h, d, w, case["step"]).double().reshape(-1, d) for w in (0, 1)]
        return {n: _exact_rows(x.reshape(-1, d), lv, case["norm"], r).view(x.shape)
                for n, x, lv, r in (("keys", k, s["levels_k"], rho[0]), ("values", v, s["levels_v"], rho[1]))}
    if case["op"] == "read":
        some = max(1, (1 << 24) // (h * _padded(d)))
        parts = [_exact_tokens(case, s, x) for x in s["slots"].split(some)]
        return {"keys": torch.cat([p[0] for p in parts]), "values": torch.cat([p[1] for p in parts])}
    out = torch.zeros((case["batch"], h * g, d), dtype=torch.float64, device="cuda")
    lse = torch.full((case["batch"], h * g), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case)):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            continue
        q = s["queries"][b].double()
        if case["rotary"]:
            q = _turned(q, s["rotary"][n - 1][None, :].expand(h * g, -1), case["interleaved"], False)
        ids = torch.arange(first, n, device="cuda")
        parts = [_exact_tokens(case, s, s["table"][b].long()[x // page] * page + x % page) for x in ids.split(8192)]
        k, v = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
        z = torch.einsum("hgd,thd->hgt", q.view(h, g, d), k) / math.sqrt(d)
        out[b] = torch.einsum("hgt,thd->hgd", torch.softmax(z, -1), v).reshape(h * g, d)
        lse[b] = torch.logsumexp(z, -1).reshape(-1)
    return {"out": out, "lse": lse}
