"""Pages chosen by bounds of their keys on the GPU: bounds and choices number for number as defined, attention over what was chosen in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

import cache_choice_reference as S
import cache_reference as R
from test_gpu_cache import TYPES, filled, make, rows, sections

pytestmark = pytest.mark.gpu


def words(t):
    return t.cpu().numpy().view(np.uint32)


def bounds_of(c, pages):
    b = c.empty_bounds(pages.shape[0])
    c.lq_cache_bounds(0, pages, torch.arange(pages.shape[0], dtype=torch.int32, device="cuda"), b)
    return b


# ---- bounds --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,dim,page,bits", [(1, 1, 16, 3), (8, 128, 64, 3), (3, 41, 32, 7), (2, 64, 16, 7), (5, 65, 128, 7), (2, 256, 16, 3),
                                                 (1, 200, 1024, 7), (10, 96, 256, 3), (7, 8, 512, 3), (1, 256, 64, 7)])
def test_bounds_are_those_of_the_definition(heads, dim, page, bits):
    c = make(heads, dim, page, (bits, 3))
    gen = torch.Generator("cuda").manual_seed(dim)
    n = 23
    pages = filled(c, n, gen)
    which = torch.tensor([4, -1, 0, 22, -2 ** 31, 7, 9, 4, 13], dtype=torch.int32, device="cuda")
    b = torch.full((n, c.bounds_words), 0x5a5a5a5a, dtype=torch.int32, device="cuda")
    c.lq_cache_bounds(0, pages, which, b)
    assert c.lq_cache_status() == 0
    got = S.unpacked(words(b), heads, R.padded(dim))
    want = S.bounds(words(pages), heads, dim, page, c.bits, c.lq_cache_get_levels(0, "keys"))
    asked = sorted(set(int(x) for x in which.tolist() if x >= 0))
    for g, w in zip(got, want):
        assert np.array_equal(g[asked], w[asked])
    others = [i for i in range(n) if i not in asked]
    assert (b[others] == 0x5a5a5a5a).all()


def test_bounds_of_norms_that_are_none():
    """Norms of zero, below 2^-100, at it, of any size, infinite and NaN (a page may hold whatever was copied into it)."""
    import paper_2505_14371_b200 as lq
    for bits in (3, 7):
        c = make(2, 70, 16, (bits, 7))
        gen = torch.Generator("cuda").manual_seed(5)
        pages = filled(c, 12, gen)
        p = R.padded(70)
        at = c.page_size * (p * (bits + 1) // 32 + p // 4)
        norms = pages.view(12, 2, -1)[:, :, at: at + 16].view(torch.float32)
        norms[0] = 0
        norms[1] = 2.0 ** -101
        norms[2] = 2.0 ** -101; norms[2, 0, 3] = 2.0 ** -100
        norms[3, 1, 15] = float("inf")
        norms[4, 0, 0] = float("nan")
        norms[5] = 3.4e38
        norms[6] *= 1e30
        norms[7] *= 1e-25
        norms[8] = 0; norms[8, 1, 7] = 1
        b = bounds_of(c, pages)
        got = S.unpacked(words(b), 2, p)
        want = S.bounds(words(pages), 2, 70, 16, c.bits, c.lq_cache_get_levels(0, "keys"))
        for g, w in zip(got, want):
            assert np.array_equal(g, w)
        assert not got[2][0].any() and not got[2][1].any() and got[2][2, 0] > 0 and got[2][3, 1] == 0 and got[2][4, 0] == 0
        assert c.lq_cache_status() == 0
        c.lq_cache_bounds(0, pages, torch.tensor([12, 3], dtype=torch.int32, device="cuda"), b)
        assert c.lq_cache_status() == lq.CACHE_BAD_PAGE


# ---- choice --------------------------------------------------------------------------------------------------

def numbers(c, q, table=None, positions=None, interleaved=False):
    """Queries as the fp32 numbers that are scored, [batch][heads][group][dim]."""
    x = q.float().cpu().numpy()
    if table is not None:
        x = R.rotate(x, table.cpu().numpy()[positions], interleaved)
    return x.reshape(x.shape[0], c.kv_heads, -1, c.head_dim)


def check_choice(c, b, table, lengths, x, chosen, seen, first, last):
    up, low, scale = S.unpacked(words(b), c.kv_heads, R.padded(c.head_dim))
    got, got_seen, keep = chosen.cpu().numpy(), seen.cpu().numpy(), chosen.shape[2]
    for i, n in enumerate(lengths):
        pages = -(-n // c.page_size)
        t = table[i, :pages].cpu().numpy()
        there = (t >= 0) & (t < len(up))
        for h in range(c.kv_heads):
            w, per = S.whole(x[i, h])
            at = np.where(there, t, 0)
            s = np.where(there, S.scores(w, per, up[at, h, : c.head_dim], low[at, h, : c.head_dim], scale[at, h]), -np.inf)
            kept = S.choose(s, pages, first, last, keep)
            want = np.full(keep, -1)
            want[: len(kept)] = t[kept]
            assert np.array_equal(got[i, h], want), (i, h, n)
            assert got_seen[i, h] == n - max(0, pages - keep) * c.page_size


CHOICES = [
    # heads, group, dim, page, bits, type, rotary, interleaved, keep, first, last, lengths
    (1, 1, 1, 16, 3, "fp32", 0, False, 1, 0, 1, [0, 1, 16, 17, 300]),
    (8, 4, 128, 16, 3, "bf16", 128, False, 16, 1, 1, [900]),
    (2, 4, 128, 16, 3, "bf16", 64, True, 8, 2, 3, [0, 1, 15, 16, 17, 127, 128, 129, 400, 1000]),
    (3, 7, 41, 32, 7, "fp16", 0, False, 5, 0, 2, [31, 32, 160, 161, 700, 2000]),
    (2, 17, 64, 16, 7, "fp32", 0, False, 20, 1, 1, [333, 1500]),               # more queries than are scored at a time
    (1, 33, 256, 16, 3, "fp16", 256, False, 3, 1, 2, [40, 48, 49, 640]),
    (1, 2, 200, 16, 3, "bf16", 0, False, 300, 1, 1, [40000, 20, 4801]),        # several CTAs a head
    (4, 2, 64, 16, 3, "bf16", 0, False, 1000, 3, 7, [33333]),
    (1, 1, 64, 16, 3, "bf16", 0, False, 64, 1, 4, [250000, 3]),                # more pages than a CTA keeps
]


@pytest.mark.parametrize("heads,group,dim,page,bits,kind,rot,inter,keep,first,last,lengths", CHOICES)
def test_choice(heads, group, dim, page, bits, kind, rot, inter, keep, first, last, lengths):
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(keep * 7 + dim)
    c = make(heads, dim, page, (bits, 3))
    pages = filled(c, 61, gen)
    b = bounds_of(c, pages)
    width = max(1, max(-(-n // page) for n in lengths)) + 2
    table = torch.randint(0, 61, (len(lengths), width), generator=gen, device="cuda", dtype=torch.int32)    # (a page may stand twice: equal scores)
    ln = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = rows(len(lengths), heads * group, dim, TYPES[kind], gen, 3)
    chosen = torch.full((len(lengths), heads, keep), 77, dtype=torch.int32, device="cuda")
    seen = torch.full((len(lengths), heads), 77, dtype=torch.int32, device="cuda")
    t = lq.lq_rotary_table(2100, rot) if rot else None
    c.lq_cache_choose(q, b, table, ln, chosen, seen, first=first, last=last, rotary=t, layout="interleaved" if inter else "half")
    assert c.lq_cache_status() == 0
    at = [max(n - 1, 0) for n in lengths]
    check_choice(c, b, table, lengths, numbers(c, q, t, at, inter), chosen, seen, first, last)
    if rot:                                                     # at positions of their own
        at = torch.randint(0, 2100, (len(lengths),), generator=gen, device="cuda")
        c.lq_cache_choose(q, b, table, ln, chosen, seen, first=first, last=last, rotary=t, positions=at, layout="interleaved" if inter else "half")
        check_choice(c, b, table, lengths, numbers(c, q, t, at.cpu().numpy(), inter), chosen, seen, first, last)


def test_equal_scores_go_to_the_first():
    c = make(2, 64, 16, (3, 3))
    gen = torch.Generator("cuda").manual_seed(1)
    pages = filled(c, 3, gen)
    b = bounds_of(c, pages)
    q = torch.randn((1, 2, 64), generator=gen, device="cuda")
    for pattern in ([0] * 400, [1] + [0] * 399, [0, 1] * 200, [2, 1, 0, 0] * 100):
        table = torch.tensor([pattern], dtype=torch.int32, device="cuda")
        for keep in (2, 3, 57, 199, 200, 201, 399):
            chosen, seen = torch.empty((1, 2, keep), dtype=torch.int32, device="cuda"), torch.empty((1, 2), dtype=torch.int32, device="cuda")
            c.lq_cache_choose(q, b, table, torch.tensor([6400], dtype=torch.int32, device="cuda"), chosen, seen)
            check_choice(c, b, table, [6400], numbers(c, q), chosen, seen, 1, 1)


@pytest.mark.parametrize("value", [0.0, 1e-35, 2.0 ** -100, 1e38, float("inf"), float("nan")])
def test_queries_that_score_nothing(value):
    """Of zeros, too small, too large, infinite or not a number: every page alike, or in order as far as fp32 tells."""
    c = make(1, 64, 16, (3, 3))
    gen = torch.Generator("cuda").manual_seed(2)
    pages = filled(c, 40, gen)
    b = bounds_of(c, pages)
    table = torch.randperm(40, generator=gen, device="cuda").to(torch.int32)[None]
    q = torch.zeros((1, 2, 64), device="cuda")
    q[0, 0, 5] = value
    q[0, 1] = value
    chosen, seen = torch.empty((1, 1, 9), dtype=torch.int32, device="cuda"), torch.empty((1, 1), dtype=torch.int32, device="cuda")
    c.lq_cache_choose(q, b, table, torch.tensor([639], dtype=torch.int32, device="cuda"), chosen, seen, first=0, last=2)
    check_choice(c, b, table, [639], numbers(c, q), chosen, seen, 0, 2)


def test_choice_with_bad_data():
    import paper_2505_14371_b200 as lq
    c = make(2, 64, 16, (3, 3))
    gen = torch.Generator("cuda").manual_seed(3)
    pages = filled(c, 40, gen)
    b = bounds_of(c, pages)
    table = torch.randint(0, 40, (4, 30), generator=gen, device="cuda", dtype=torch.int32)
    table[0, 3] = -1; table[0, 7] = 40; table[1, 9] = 2 ** 31 - 1; table[1, 0] = -5
    lengths = torch.tensor([480, 479, -3, 481], dtype=torch.int32, device="cuda")
    q = torch.randn((4, 4, 64), generator=gen, device="cuda")
    chosen, seen = torch.empty((4, 2, 29), dtype=torch.int32, device="cuda"), torch.empty((4, 2), dtype=torch.int32, device="cuda")
    c.lq_cache_choose(q, b, table, lengths, chosen, seen)
    assert c.lq_cache_status() == lq.CACHE_BAD_LENGTH
    check_choice(c, b, table, [480, 479, 0, 480], numbers(c, q), chosen, seen, 1, 1)
    t = lq.lq_rotary_table(100, 64)
    c.lq_cache_choose(q, b, table, lengths, chosen, seen, rotary=t, positions=torch.tensor([5, 100, 3, -1], device="cuda"))
    assert c.lq_cache_status() == lq.CACHE_BAD_LENGTH | lq.CACHE_BAD_POSITION
    x = numbers(c, q, t, [5, 0, 3, 0])
    x[1] = x[3] = 0                                             # (a query that cannot be turned scores nothing)
    check_choice(c, b, table, [480, 479, 0, 480], x, chosen, seen, 1, 1)


# ---- attention over what was chosen --------------------------------------------------------------------------

def check_chosen(c, pages, chosen, seen, q, out, lse, turned=None):
    sec = sections(c, pages)
    kk, vv = (R.values_of(sec[i], sec[2 + i], c.lq_cache_get_levels(0, n))[..., : c.head_dim] for i, n in ((0, "keys"), (1, "values")))
    half = torch.finfo(out.dtype).eps / 2
    w_error = 2.0 ** -20 if out.dtype == torch.float32 else 2.0 ** -11
    group = q.shape[1] // c.kv_heads
    qq = (q if turned is None else turned).double().cpu().numpy()
    got, got_lse, pg, n = out.double().cpu().numpy(), lse.double().cpu().numpy(), chosen.cpu().numpy(), seen.cpu().numpy()
    for b in range(q.shape[0]):
        for h in range(q.shape[1]):
            at = np.arange(max(n[b, h // group], 0))
            p = pg[b, h // group][at // c.page_size]
            ok = (p >= 0) & (p < pages.shape[0])
            p, place = p[ok], at[ok] % c.page_size
            o, l, bound, lse_bound = R.attend(qq[b, h], kk[p, h // group, place], vv[p, h // group, place], c.head_dim ** -0.5, 2.0 ** -21, w_error)
            assert np.all(np.abs(got[b, h] - o) <= bound + half * (np.abs(o) + bound)), (b, h, n[b, h // group])
            assert got_lse[b, h] == l if np.isinf(l) else abs(got_lse[b, h] - l) <= lse_bound, (b, h)


CHOSEN = [
    # heads, group, dim, page, bits, type, rotary, keep, batch
    (1, 1, 1, 16, (3, 3), "fp32", 0, 4, 3),
    (8, 4, 128, 64, (3, 3), "bf16", 128, 16, 5),
    (3, 3, 64, 16, (7, 3), "fp16", 32, 9, 33),
    (10, 1, 41, 32, (3, 7), "fp32", 0, 3, 12),
    (2, 9, 200, 16, (7, 7), "fp16", 0, 40, 4),
    (1, 16, 256, 128, (3, 3), "bf16", 0, 5, 2),
    (4, 2, 96, 16, (3, 3), "bf16", 0, 1, 300),
    (2, 1, 64, 16, (3, 3), "fp32", 64, 700, 1),
]


@pytest.mark.parametrize("heads,group,dim,page,bits,kind,rot,keep,batch", CHOSEN)
def test_attention_over_pages_of_each_head(heads, group, dim, page, bits, kind, rot, keep, batch):
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(keep + dim)
    c = make(heads, dim, page, bits)
    pages = filled(c, 37, gen, 2.0)
    chosen = torch.randint(0, 37, (batch, heads, keep), generator=gen, device="cuda", dtype=torch.int32)
    seen = torch.randint(0, keep * page + 1, (batch, heads), generator=gen, device="cuda", dtype=torch.int32)
    seen[0, 0] = keep * page
    if batch > 1:
        seen[1, heads - 1] = 0
        seen[1, 0] = min(1, heads - 1)
    q = rows(batch, heads * group, dim, TYPES[kind], gen, 1)
    wide = torch.full((batch, heads * group + 1, dim + 4), 9.0, dtype=TYPES[kind], device="cuda")
    out = wide[:, 1:, 4:]
    lse = torch.empty((batch, heads * group), device="cuda")
    t = at = turned = None
    if rot:
        t, at = lq.lq_rotary_table(999, rot), torch.randint(0, 999, (batch,), generator=gen, device="cuda")
        turned = torch.from_numpy(R.rotate(q.float().cpu().numpy(), t.cpu().numpy()[at.cpu().numpy()], False))
    c.lq_cache_attend_chosen(0, q, pages, chosen, seen, out, lse=lse, rotary=t, positions=at)
    assert c.lq_cache_status() == 0
    check_chosen(c, pages, chosen, seen, q, out, lse, turned)
    assert (wide[:, 0] == 9).all() and (wide[..., :4] == 9).all()


def test_the_same_pages_for_all_heads_give_the_same_bits():
    gen = torch.Generator("cuda").manual_seed(8)
    c = make(4, 128, 16, (3, 7))
    pages = filled(c, 30, gen)
    table = torch.randint(0, 30, (6, 5), generator=gen, device="cuda", dtype=torch.int32)
    lengths = torch.tensor([0, 1, 80, 33, 64, 17], dtype=torch.int32, device="cuda")
    q = torch.randn((6, 16, 128), generator=gen, device="cuda").half()
    a, b = torch.empty_like(q), torch.empty_like(q)
    c.lq_cache_attend(0, q, pages, table, lengths, a)
    c.lq_cache_attend_chosen(0, q, pages, table[:, None].repeat(1, 4, 1), lengths[:, None].repeat(1, 4), b)
    assert torch.equal(a, b)


def test_chosen_pages_that_are_not_there():
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(9)
    c = make(2, 64, 16, (3, 3))
    pages = filled(c, 10, gen)
    chosen = torch.randint(0, 10, (2, 2, 4), generator=gen, device="cuda", dtype=torch.int32)
    chosen[0, 1, 2] = -1; chosen[1, 0] = 10
    seen = torch.tensor([[64, 60], [33, -4]], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 2, 64), generator=gen, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((2, 2), device="cuda")
    c.lq_cache_attend_chosen(0, q, pages, chosen, seen, out, lse=lse)
    assert c.lq_cache_status() == lq.CACHE_BAD_PAGE | lq.CACHE_BAD_LENGTH
    check_chosen(c, pages, chosen, seen, q, out, lse)
    assert not out[1].any() and torch.isneginf(lse[1]).all()


# ---- together ------------------------------------------------------------------------------------------------

def step(c, s, stream=None):
    """One new token a sequence: written, its page's bounds where it is full, pages chosen, attended to."""
    c.lq_cache_write(0, s["k"], s["v"], s["slots"], s["pages"], rotary=s["turn"], positions=s["positions"])
    c.lq_cache_bounds(0, s["pages"], s["full"], s["bounds"])
    c.lq_cache_choose(s["q"], s["bounds"], s["table"], s["lengths"], s["chosen"], s["seen"], first=1, last=1, rotary=s["turn"])
    c.lq_cache_attend_chosen(0, s["q"], s["pages"], s["chosen"], s["seen"], s["out"], lse=s["lse"], rotary=s["turn"], positions=s["positions"])


@pytest.mark.parametrize("graph", [False, True])
def test_steps_of_a_batch(graph):
    """Decoding steps over pages that fill up, on a stream of their own, launched or captured once and replayed: every step as defined."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(10)
    c = make(2, 64, 16, (3, 7))
    batch, width, keep, n = 5, 12, 4, [100, 15, 16, 1, 190]
    s = dict(pages=filled(c, batch * width, gen), table=torch.randperm(batch * width, generator=gen, device="cuda").view(batch, width).int())
    s["bounds"] = bounds_of(c, s["pages"])
    s.update(turn=lq.lq_rotary_table(256, 64), chosen=torch.empty((batch, 2, keep), dtype=torch.int32, device="cuda"),
             seen=torch.empty((batch, 2), dtype=torch.int32, device="cuda"), out=torch.empty((batch, 8, 64), dtype=torch.bfloat16, device="cuda"),
             lse=torch.empty((batch, 8), device="cuda"), q=torch.empty((batch, 8, 64), dtype=torch.bfloat16, device="cuda"),
             k=torch.empty((batch, 2, 64), dtype=torch.bfloat16, device="cuda"), v=torch.empty((batch, 2, 64), dtype=torch.bfloat16, device="cuda"),
             slots=torch.empty(batch, dtype=torch.int64, device="cuda"), positions=torch.empty(batch, dtype=torch.int64, device="cuda"),
             lengths=torch.empty(batch, dtype=torch.int32, device="cuda"), full=torch.empty(batch, dtype=torch.int32, device="cuda"))

    def ready(i):
        at = [x + i for x in n]                                 # the new token's place
        pg = [int(s["table"][j, a // 16]) for j, a in enumerate(at)]
        s["slots"].copy_(torch.tensor([p * 16 + a % 16 for p, a in zip(pg, at)]))
        s["positions"].copy_(torch.tensor(at))
        s["lengths"].copy_(torch.tensor([a + 1 for a in at]))
        s["full"].copy_(torch.tensor([p if a % 16 == 15 else -1 for p, a in zip(pg, at)]))
        for name in "qkv":
            s[name].copy_(torch.randn(s[name].shape, generator=gen, device="cuda"))
        return at

    side = torch.cuda.Stream()
    ready(0)
    torch.cuda.synchronize()
    kept = s["pages"].clone(), s["bounds"].clone()
    if graph:
        with torch.cuda.stream(side):
            step(c, s)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=side):
            step(c, s)
        s["pages"].copy_(kept[0]); s["bounds"].copy_(kept[1])
    for i in range(2):
        at = ready(i)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay() if graph else step(c, s)
        side.synchronize()
        want = S.bounds(words(s["pages"]), 2, 64, 16, c.bits, c.lq_cache_get_levels(0, "keys"))
        got = S.unpacked(words(s["bounds"]), 2, 64)
        full = [p for p in s["full"].tolist() if p >= 0]
        for x, w in zip(got, want):
            assert np.array_equal(x[full], w[full])
        x = numbers(c, s["q"], s["turn"], at)
        check_choice(c, s["bounds"], s["table"], [a + 1 for a in at], x, s["chosen"], s["seen"], 1, 1)
        check_chosen(c, s["pages"], s["chosen"], s["seen"], s["q"], s["out"], s["lse"], torch.from_numpy(x.reshape(batch, 8, 64)))
    assert c.lq_cache_status() == 0


# ---- refusals ------------------------------------------------------------------------------------------------

def test_refusals():
    import paper_2505_14371_b200 as lq
    c = make(2, 64, 16, (3, 3))
    pages, b = c.empty_pages(4), c.empty_bounds(4)
    i32 = dict(dtype=torch.int32, device="cuda")
    which, table, lengths = torch.zeros(3, **i32), torch.zeros((2, 4), **i32), torch.zeros(2, **i32)
    chosen, seen = torch.zeros((2, 2, 3), **i32), torch.zeros((2, 2), **i32)
    q = torch.zeros((2, 4, 64), device="cuda")
    out = torch.zeros_like(q)
    bad = [
        lambda: c.lq_cache_bounds(1, pages, which, b),
        lambda: c.lq_cache_bounds(0, pages, which.long(), b),
        lambda: c.lq_cache_bounds(0, pages, which, b[:3]),
        lambda: c.lq_cache_bounds(0, pages, which, b[:, :-1]),
        lambda: c.lq_cache_bounds(0, pages, which.cpu(), b),
        lambda: c.lq_cache_choose(q, b, table, lengths, chosen, seen, first=-1),
        lambda: c.lq_cache_choose(q, b, table, lengths, chosen, seen, last=0),
        lambda: c.lq_cache_choose(q, b, table, lengths, chosen, seen, first=2, last=2),
        lambda: c.lq_cache_choose(q, b, table, lengths, chosen[:1], seen),
        lambda: c.lq_cache_choose(q, b, table, lengths, chosen[:, :1], seen),
        lambda: c.lq_cache_choose(q, b, table[:1], lengths, chosen, seen),
        lambda: c.lq_cache_choose(q, b, table, lengths[:1], chosen, seen),
        lambda: c.lq_cache_choose(q[:, :3], b, table, lengths, chosen, seen),
        lambda: c.lq_cache_choose(q[..., :63], b, table, lengths, chosen, seen),
        lambda: c.lq_cache_choose(q.double(), b, table, lengths, chosen, seen),
        lambda: c.lq_cache_choose(q, b, table, lengths, chosen.long(), seen),
        lambda: c.lq_cache_choose(q, b, table, lengths, chosen, seen, positions=torch.zeros(2, dtype=torch.int64, device="cuda")),
        lambda: c.lq_cache_choose(q, b, table, lengths, chosen, seen, layout="pairs"),
        lambda: c.lq_cache_choose(q.clone().requires_grad_(), b, table, lengths, chosen, seen),
        lambda: c.lq_cache_attend_chosen(0, q, pages, chosen, seen, out.half()),
        lambda: c.lq_cache_attend_chosen(0, q, pages, chosen[:, :1], seen, out),
        lambda: c.lq_cache_attend_chosen(0, q, pages, chosen, seen[:1], out),
        lambda: c.lq_cache_attend_chosen(0, q[:1], pages, chosen, seen, out[:1]),
        lambda: c.lq_cache_attend_chosen(0, q, pages, chosen, seen, out, scale=float("nan")),
        lambda: c.lq_cache_attend_chosen(0, q, pages, chosen, seen, out, rotary=lq.lq_rotary_table(9, 64)),     # no positions
        lambda: c.lq_cache_attend_chosen(0, q, pages, chosen, seen, out[:, :1].expand(-1, 4, -1)),
        lambda: c.lq_cache_attend_chosen(0, q, pages, chosen, seen, out, lse=torch.zeros((2, 3), device="cuda")),
        lambda: c.lq_cache_attend_chosen(0, q, pages, chosen, seen, out.clone().requires_grad_()),
    ]
    for call in bad:
        with pytest.raises(lq.LqError):
            call()
    lib = lq.load_library()
    assert lib.lq_cache_bounds(c._h, 0, pages.data_ptr(), 4, which.data_ptr(), 3, b.data_ptr() + 4, None) == -1
    assert lib.lq_cache_bounds(c._h, 0, pages.data_ptr(), 4, None, 3, b.data_ptr(), None) == -1
    assert lib.lq_cache_bounds(c._h, 0, pages.data_ptr(), 4, which.data_ptr(), -1, b.data_ptr(), None) == -1
    assert lib.lq_cache_choose_workspace(c._h, 1 << 24, 10) == -1 and lib.lq_cache_choose_workspace(c._h, 3, 12289) == 3 * 2 * 12289 * 4
    assert lib.lq_cache_choose_workspace(c._h, 3, 12288) == 0
    assert c.lq_cache_status() == 0 and not b.any() and not out.any()
    # nothing to do
    c.lq_cache_bounds(0, pages, which[:0], b)
    c.lq_cache_choose(q[:0], b, table[:0], lengths[:0], chosen[:0], seen[:0])
    c.lq_cache_attend_chosen(0, q[:0], pages, chosen[:0], seen[:0], out[:0])
    c.lq_cache_attend_chosen(0, q, pages, chosen[..., :0].contiguous(), seen, out)      # (no page can be seen)
    assert not out.any() and c.lq_cache_status() == 0
