"""The quantised key-value cache on the GPU: rows written bit for bit as defined, read back, attended to, against numpy in 64 bits."""
import numpy as np
import pytest
import torch

import cache_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SEED = 0x5EED0DA12345


def make(heads, dim, page=16, bits=(3, 3), q=0, layers=1, curve=1.3):
    import paper_2505_14371_b200 as lq
    c = lq.Cache(layers, heads, dim, page, bits, q, SEED)
    for m in range(layers):
        for kind, b in zip(("keys", "values"), bits):
            n = 1 << b
            c.lq_cache_set_levels(m, kind, [(j / (n - 1)) ** (curve + 0.1 * m + (0.2 if kind == "values" else 0)) for j in range(n)])
    return c


def sections(c, pages):
    return R.head_sections(pages.cpu().numpy().view(np.uint32), c.kv_heads, c.head_dim, c.page_size, c.bits)


def rows(tokens, heads, dim, dtype, gen, pad=0):
    """Rows as a part of wider ones (strides), `pad` elements off their start."""
    wide = torch.randn((tokens, heads + 2, dim + pad), generator=gen, device="cuda").to(dtype)
    return wide[:, 1: heads + 1, pad:]


# ---- writing -------------------------------------------------------------------------------------------------

WRITES = [
    # tokens, heads, dim, page, bits, q, type, pad, step, rotary dim, interleaved
    (1, 1, 1, 16, (3, 3), 0, "fp32", 0, None, 0, False),
    (1, 8, 128, 64, (3, 3), 0, "bf16", 0, None, 128, False),
    (37, 3, 41, 16, (3, 7), 2, "fp32", 0, 5, 0, False),
    (64, 2, 64, 32, (7, 7), 1, "fp16", 0, None, 64, True),
    (129, 5, 65, 16, (7, 3), 2, "bf16", 3, 0, 22, True),
    (33, 1, 256, 128, (3, 3), 0, "fp16", 8, 4294967295, 100, False),
    (1000, 4, 200, 16, (7, 7), 0, "fp32", 4, None, 200, False),
    (77, 10, 96, 1024, (3, 7), 1, "bf16", 1, 9, 96, False),
    (50, 2, 8, 16, (3, 3), 0, "fp16", 0, None, 2, True),
]


@pytest.mark.parametrize("tokens,heads,dim,page,bits,q,kind,pad,step,rot,inter", WRITES)
def test_rows_are_written_bit_for_bit(tokens, heads, dim, page, bits, q, kind, pad, step, rot, inter):
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(tokens * 31 + dim)
    c = make(heads, dim, page, bits, q, layers=2)
    n = -(-tokens // page) + 2
    pages = torch.randint(-2 ** 31, 2 ** 31 - 1, (n, c.page_words), generator=gen, device="cuda", dtype=torch.int32)
    before = pages.clone()
    k, v = (rows(tokens, heads, dim, TYPES[kind], gen, pad) for _ in range(2))
    slots = torch.randperm(n * page, generator=gen, device="cuda")[:tokens]
    if tokens > 3:
        slots[2] = -1
        k[1, 0] = 0                                           # a row of zeros
    table = pos = None
    if rot:
        table = lq.lq_rotary_table(5000, rot)
        pos = torch.randint(0, 5000, (tokens,), generator=gen, device="cuda")
    c.lq_cache_write(1, k, v, slots, pages, step=step, rotary=table, positions=pos, layout="interleaved" if inter else "half")
    assert c.lq_cache_status() == 0
    got, was = sections(c, pages), sections(c, before)
    sl = slots.cpu().numpy()
    live = sl >= 0
    for i, x in enumerate((k, v)):
        x = x.float().cpu().numpy()
        if rot and i == 0:
            x = R.rotate(x, table.cpu().numpy()[pos.cpu().numpy()], inter)
        rho = np.float32(0.5) if step is None else R.uniforms(SEED, 1, i, np.maximum(sl, 0), heads, dim, step)
        sym, norm = R.quantise(x, c.lq_cache_get_levels(1, ("keys", "values")[i]), q, rho)
        gs, gn = got[i], got[2 + i]
        at, place = sl[live] // page, sl[live] % page
        g_sym, g_norm = gs[at, :, place], gn[at, :, place]
        # the sum of a norm is rounded once from 64 bits; its terms' order can move it by one unit in the last place, hardly ever
        same = g_norm == norm[live]
        assert np.all(np.abs(g_norm - norm[live]) <= 2.0 ** -23 * norm[live]) and same.mean() > 0.99
        assert np.array_equal(g_sym[..., :dim][same], sym[live][same])
        assert not g_sym[..., dim:].any()
        untouched = np.ones((n * page,), bool)
        untouched[sl[live]] = False
        keep = lambda a: np.moveaxis(a, 2, 1).reshape(n * page, heads, -1)[untouched]
        assert np.array_equal(keep(gs), keep(was[i]))
        assert np.array_equal(keep(gn).view(np.uint32), keep(was[2 + i]).view(np.uint32))


def crowded(n):
    """Levels of which most are neighbours among the numbers of 11 bits, just above 1/2 and just above 2^-14."""
    near = [0.5 + j * 2.0 ** -11 for j in range(n // 2)] + [2.0 ** -14 + j * 2.0 ** -24 for j in range(n - 2 - n // 2)]
    return [0.0] + sorted(near) + [1.0]


@pytest.mark.parametrize("bits,levels", [(3, None), (7, None), (3, crowded(8)), (7, crowded(128)), (7, [j / 127 for j in range(128)]),
                                         (3, [0, 2.0 ** -24, 2.0 ** -23, 2.0 ** -20, 2.0 ** -16, 2.0 ** -8, 0.25, 1])])
@pytest.mark.parametrize("step", [None, 3])
def test_values_on_and_beside_every_border(bits, levels, step):
    """Rows of one large value (the norm is 1) and values at levels, at the middles between them, and one step off either."""
    c = make(1, 256, 16, (bits, bits), 0)
    if levels:
        for kind in ("keys", "values"):
            c.lq_cache_set_levels(0, kind, levels)
    lv = np.array(c.lq_cache_get_levels(0, "keys"), np.float32)
    pts = np.concatenate([lv, (lv[1:] + lv[:-1]) / 2]).astype(np.float32)
    pts = np.concatenate([pts, np.nextafter(pts, np.float32(0)), np.nextafter(pts, np.float32(2)), -pts, [np.float32(1e-42), 0, -0.0]])
    pts = pts[np.abs(pts) <= 1]
    per = 255
    count = -(-len(pts) // per)
    x = np.zeros((count, 1, 256), np.float32)
    x[:, 0, 0] = 1
    for i in range(count):
        part = pts[i * per: (i + 1) * per]
        x[i, 0, 1: 1 + len(part)] = part
    k = torch.from_numpy(x).cuda()
    pages = c.empty_pages(-(-count // 16))
    c.lq_cache_write(0, k, k, torch.arange(count, device="cuda"), pages, step=step)
    got = sections(c, pages)
    for kind, name in ((0, "keys"), (1, "values")):
        rho = np.float32(0.5) if step is None else R.uniforms(SEED, 0, kind, np.arange(count), 1, 256, step)
        sym, norm = R.quantise(x, c.lq_cache_get_levels(0, name), 0, rho)
        g = np.moveaxis(got[kind], 2, 1).reshape(-1, 1, 256)[:count]
        assert np.array_equal(g, sym)


def test_rows_that_cannot_be_kept():
    import paper_2505_14371_b200 as lq
    for q in (0, 1, 2):
        c = make(2, 70, 16, (7, 3), q)
        k = torch.randn((6, 2, 70), device="cuda")
        v = torch.randn((6, 2, 70), device="cuda")
        pages = c.empty_pages(1)
        slots = torch.arange(6, device="cuda")
        c.lq_cache_write(0, k, v, slots, pages)
        assert c.lq_cache_status() == 0
        k[0, 0, 69] = float("nan"); k[1, 1, 0] = float("inf"); v[2, 0, 33] = float("-inf")
        k[3, 0] = 0; v[3, 1] = 1e-39; k[4, 0] = 3e38
        c.lq_cache_write(0, k, v, slots, pages)
        assert c.lq_cache_status() == lq.CACHE_NONFINITE and c.lq_cache_status() == 0
        sk, sv, nk, nv = sections(c, pages)
        zero = [(sk, nk, 0, 0), (sk, nk, 1, 1), (sv, nv, 2, 0), (sk, nk, 3, 0)] + ([(sk, nk, 4, 0)] if q else [])
        if q == 0:
            zero.append((sv, nv, 3, 1))
        for s, n, token, head in zero:
            assert not s[0, head, token].any() and n[0, head, token] == 0
        assert nk[0, 1, 0] > 0 and nv[0, 0, 0] > 0                     # their neighbours are kept


def test_bad_slots_and_positions_are_skipped_and_flagged():
    import paper_2505_14371_b200 as lq
    c = make(1, 64)
    pages = c.empty_pages(2)
    k = torch.ones((4, 1, 64), device="cuda")
    table = lq.lq_rotary_table(10, 64)
    pos = torch.tensor([0, 10, -1, 9], device="cuda")
    c.lq_cache_write(0, k, k, torch.tensor([0, 1, 2, 3], device="cuda"), pages, rotary=table, positions=pos)
    assert c.lq_cache_status() == lq.CACHE_BAD_POSITION
    norms = sections(c, pages)[2][0, 0]
    assert norms[0] > 0 and norms[1] == 0 and norms[2] == 0 and norms[3] > 0
    c.lq_cache_write(0, k, k, torch.tensor([32, 2 ** 40, -7, 31], device="cuda"), pages)
    assert c.lq_cache_status() == lq.CACHE_BAD_SLOT
    assert sections(c, pages)[3][1, 0, 15] > 0
    out = torch.full((4, 1, 64), 7.0, device="cuda")
    other = out.clone()
    c.lq_cache_read(0, pages, torch.tensor([32, -1, 31, 0], device="cuda"), out, other)
    assert c.lq_cache_status() == lq.CACHE_BAD_SLOT
    assert not out[:2].any() and out[2].all() and other[3].all()


def test_unbiased_rounding_averages_to_the_row():
    c = make(2, 41, 16, (3, 7), 2)
    gen = torch.Generator("cuda").manual_seed(1)
    k = torch.randn((5, 2, 41), generator=gen, device="cuda")
    pages, slots = c.empty_pages(1), torch.arange(5, device="cuda") * 3
    a, b, draws = torch.zeros_like(k, dtype=torch.float64), torch.zeros_like(k, dtype=torch.float64), 600
    x, y = torch.empty_like(k), torch.empty_like(k)
    for step in range(draws):
        c.lq_cache_write(0, k, k, slots, pages, step=step)
        c.lq_cache_read(0, pages, slots, x, y)
        a += x; b += y
    norm = k.double().norm(dim=2, keepdim=True)
    for mean, name in ((a / draws, "keys"), (b / draws, "values")):
        lv = torch.tensor(c.lq_cache_get_levels(0, name), dtype=torch.float64)
        gap = float((lv[1:] - lv[:-1]).max())
        # a draw's spread is at most half a gap times the norm: 6 standard errors
        assert ((mean - k.double()).abs() <= 6 * 0.5 * gap * norm / draws ** 0.5).all()


# ---- reading -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,dim,page,bits,kind,pad", [(1, 1, 16, (3, 7), "fp32", 0), (3, 41, 16, (7, 3), "bf16", 1), (8, 128, 64, (3, 3), "fp16", 0),
                                                          (2, 250, 32, (7, 7), "fp32", 2), (5, 64, 16, (3, 3), "bf16", 0)])
def test_rows_are_read_back(heads, dim, page, bits, kind, pad):
    gen = torch.Generator("cuda").manual_seed(dim)
    c = make(heads, dim, page, bits)
    pages = c.empty_pages(7)
    x = torch.randn((7 * page, heads, dim), generator=gen, device="cuda")
    c.lq_cache_write(0, x, x * 2, torch.arange(7 * page, device="cuda"), pages)
    slots = torch.randint(0, 7 * page, (251,), generator=gen, device="cuda")      # the same one twice, any order
    slots[5] = -3
    wide = [torch.full((251, heads + 1, dim + pad), 9.0, device="cuda", dtype=TYPES[kind]) for _ in range(2)]
    c.lq_cache_read(0, pages, slots, wide[0][:, 1:, pad:], wide[1][:, 1:, pad:])
    sec = sections(c, pages)
    sl = slots.cpu().numpy()
    for i, name in enumerate(("keys", "values")):
        want = R.values_of(sec[i], sec[2 + i], c.lq_cache_get_levels(0, name))[sl // page, :, sl % page][..., :dim]
        want[5] = 0
        # one rounding to fp32, one to the type
        assert torch.equal(wide[i][:, 1:, pad:].cpu(), torch.from_numpy(want.astype(np.float32)).to(TYPES[kind]))
        assert (wide[i][:, 0] == 9).all() and (wide[i][..., :pad] == 9).all()


# ---- attention -----------------------------------------------------------------------------------------------

def filled(c, num_pages, gen, scale=1.0):
    pages = torch.empty((num_pages, c.page_words), dtype=torch.int32, device="cuda")
    n = num_pages * c.page_size
    k = torch.randn((n, c.kv_heads, c.head_dim), generator=gen, device="cuda") * scale
    v = torch.randn((n, c.kv_heads, c.head_dim), generator=gen, device="cuda") * torch.randn((n, 1, 1), generator=gen, device="cuda").mul_(2).exp_()
    c.lq_cache_write(0, k, v, torch.arange(n, device="cuda"), pages)
    return pages


def check_attention(c, pages, table, lengths, q, out, lse, window=0, scale=None, turned=None, missing=()):
    sec = sections(c, pages)
    kk, vv = (R.values_of(sec[i], sec[2 + i], c.lq_cache_get_levels(0, n))[..., :c.head_dim] for i, n in ((0, "keys"), (1, "values")))
    scale = c.head_dim ** -0.5 if scale is None else scale
    half = torch.finfo(out.dtype).eps / 2
    # fp32 queries and rotated ones are taken with 22 bits, others as they are; weights with 11 bits, 22 for fp32 outputs
    q_error = 2.0 ** -21
    w_error = 2.0 ** -20 if out.dtype == torch.float32 else 2.0 ** -11
    group = q.shape[1] // c.kv_heads
    qq = (q if turned is None else turned).double().cpu().numpy()
    got, got_lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
    for b, n in enumerate(lengths):
        ids = np.arange(max(0, n - window) if window else 0, max(n, 0))
        pg = table[b].cpu().numpy()[ids // c.page_size] if len(ids) else ids
        seen = ~np.isin(pg, missing) if len(missing) else np.ones(len(ids), bool)
        pg, place = pg[seen], ids[seen] % c.page_size
        for h in range(q.shape[1]):
            o, l, bound, lse_bound = R.attend(qq[b, h], kk[pg, h // group, place], vv[pg, h // group, place], scale, q_error, w_error)
            assert np.all(np.abs(got[b, h] - o) <= bound + half * (np.abs(o) + bound)), (b, h, n, np.abs(got[b, h] - o).max())
            if lse is not None:
                assert got_lse[b, h] == l if np.isinf(l) else abs(got_lse[b, h] - l) <= lse_bound, (b, h, n)


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 33, 127, 128, 129, 300]
ATTENDS = [
    # heads, group, dim, page, bits, type, window, rotary, interleaved, lengths
    (1, 1, 1, 16, (3, 3), "fp32", 0, 0, False, LENGTHS),
    (2, 4, 128, 16, (3, 3), "bf16", 0, 0, False, LENGTHS),
    (2, 4, 128, 64, (3, 3), "bf16", 0, 128, False, LENGTHS),
    (1, 8, 128, 32, (7, 7), "fp16", 0, 0, False, LENGTHS),
    (3, 3, 64, 16, (3, 7), "fp16", 40, 32, True, LENGTHS),
    (2, 1, 41, 32, (3, 3), "fp32", 0, 40, False, LENGTHS),
    (1, 9, 65, 16, (7, 3), "fp32", 17, 0, False, LENGTHS),
    (1, 16, 256, 128, (7, 3), "bf16", 100, 64, True, LENGTHS),
    (2, 5, 200, 16, (7, 7), "fp32", 0, 200, False, LENGTHS),
    (1, 17, 250, 16, (3, 7), "fp16", 1, 0, False, LENGTHS),
    (1, 2, 64, 16, (7, 7), "bf16", 0, 0, False, LENGTHS),
    (1, 3, 256, 16, (3, 3), "fp16", 0, 0, False, LENGTHS),
    (1, 1, 64, 16, (3, 3), "bf16", 0, 0, False, [1]),
    (1, 7, 128, 16, (3, 3), "bf16", 0, 0, False, [20000]),                 # one sequence over many CTAs
    (4, 2, 64, 16, (3, 7), "fp16", 0, 16, False, [5000, 3, 0, 9000, 129]),
    (1, 1, 128, 1024, (3, 3), "fp32", 3000, 0, False, [12345, 2999, 3001]),
    (1, 4, 16, 16, (3, 3), "bf16", 0, 0, False, [5, 0, 17] * 230),          # more sequences than threads of a CTA
    (1, 1, 64, 16, (3, 3), "fp16", 0, 0, False, [0] * 40),                  # nothing to see at all
]


@pytest.mark.parametrize("heads,group,dim,page,bits,kind,window,rot,inter,lengths", ATTENDS)
def test_attention_of_a_new_token(heads, group, dim, page, bits, kind, window, rot, inter, lengths):
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim * 7 + heads)
    c = make(heads, dim, page, bits)
    width = max(1, max(-(-n // page) for n in lengths)) + 1
    num_pages = min(3 * width, 2500)
    pages = filled(c, num_pages, gen)
    table = torch.randint(0, num_pages, (len(lengths), width), generator=gen, device="cuda", dtype=torch.int32)
    for b, n in enumerate(lengths):
        table[b, -(-n // page):] = 1 << 30                                   # never looked at
    q = rows(len(lengths), heads * group, dim, TYPES[kind], gen, 3) * 3
    q = rows(len(lengths), heads * group, dim, TYPES[kind], gen, 3).copy_(q)
    out = torch.full((len(lengths), heads * group + 1, dim + 1), 5.0, dtype=TYPES[kind], device="cuda")
    lse = torch.empty((len(lengths), heads * group), device="cuda")
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    angles = turned = None
    if rot:
        angles = lq.lq_rotary_table(max(lengths) + 1, rot)
        at = (n.long() - 1).clamp(min=0).cpu().numpy()
        turned = torch.from_numpy(R.rotate(q.float().cpu().numpy(), angles.cpu().numpy()[at], inter))
    c.lq_cache_attend(0, q, pages, table, n, out[:, :-1, 1:], lse=lse, window=window, rotary=angles, layout="interleaved" if inter else "half")
    assert c.lq_cache_status() == 0
    assert (out[:, -1] == 5).all() and (out[..., 0] == 5).all()
    check_attention(c, pages, table, lengths, q, out[:, :-1, 1:], lse, window, turned=turned)


def test_what_a_page_holds_past_the_end_does_not_matter():
    gen = torch.Generator("cuda").manual_seed(3)
    c = make(2, 128, 16, (3, 7))
    pages = filled(c, 8, gen)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    lengths = [20, 50]
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    q = torch.randn((2, 8, 128), generator=gen, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((2, 8), device="cuda")
    c.lq_cache_attend(0, q, pages, table, n, out, lse=lse)
    check_attention(c, pages, table, lengths, q, out, lse)
    bad = pages.clone().view(8, 2, -1)
    rk, rv = 128 * 4 // 32, 128 * 8 // 32
    for value in (float("nan"), float("inf"), -1.0):
        norms = bad[..., 16 * (rk + rv):].view(torch.float32).view(8, 2, 2, 16)
        norms[1, :, :, 4:] = value; norms[2:4] = value; norms[7, :, :, 2:] = value
        bad[1, :, rk * 4: rk * 16] = -1
        o2, l2 = torch.empty_like(q), torch.empty_like(lse)
        c.lq_cache_attend(0, q, bad.view(8, -1), table, n, o2, lse=l2)
        assert torch.equal(o2, out) and torch.equal(l2, lse)


def test_missing_pages_and_lengths_out_of_range():
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(4)
    c = make(1, 64, 16, (7, 7))
    pages = filled(c, 12, gen)
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4)
    table[0, 1] = -1; table[1, :3] = 12; table[1, 3] = 2 ** 31 - 1
    q = torch.randn((3, 4, 64), generator=gen, device="cuda").half()
    out, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
    lengths = [60, 64, 64]
    c.lq_cache_attend(0, q, pages, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), out, lse=lse)
    assert c.lq_cache_status() == lq.CACHE_BAD_PAGE
    check_attention(c, pages, table, lengths, q, out, lse, missing=(-1, 12, 2 ** 31 - 1))
    table = torch.arange(12, dtype=torch.int32, device="cuda").view(3, 4)
    c.lq_cache_attend(0, q, pages, table, torch.tensor([-5, 65, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), out, lse=lse)
    assert c.lq_cache_status() == lq.CACHE_BAD_LENGTH
    check_attention(c, pages, table, [0, 64, 64], q, out, lse)
    # a table without columns: nothing to see
    c.lq_cache_attend(0, q, pages, table[:, :0].contiguous(), torch.zeros(3, dtype=torch.int32, device="cuda"), out, lse=lse)
    assert not out.any() and torch.isneginf(lse).all() and c.lq_cache_status() == 0


def test_positions_of_queries():
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(5)
    c = make(2, 128, 16)
    pages = filled(c, 4, gen)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    n = torch.tensor([30, 30], dtype=torch.int32, device="cuda")
    q = torch.randn((2, 2, 128), generator=gen, device="cuda")
    angles = lq.lq_rotary_table(100, 64)
    out, lse = torch.empty_like(q), torch.empty((2, 2), device="cuda")
    pos = torch.tensor([99, 3], device="cuda")
    c.lq_cache_attend(0, q, pages, table, n, out, lse=lse, rotary=angles, positions=pos, layout="interleaved")
    turned = torch.from_numpy(R.rotate(q.cpu().numpy(), angles.cpu().numpy()[[99, 3]], True))
    check_attention(c, pages, table, [30, 30], q, out, lse, turned=turned)
    assert c.lq_cache_status() == 0
    good = out.clone()
    c.lq_cache_attend(0, q, pages, table, n, out, rotary=angles, positions=torch.tensor([100, 3], device="cuda"), layout="interleaved")
    assert c.lq_cache_status() == lq.CACHE_BAD_POSITION
    assert torch.isnan(out[0]).all() and torch.equal(out[1], good[1])


def test_queries_of_any_size_and_kind():
    gen = torch.Generator("cuda").manual_seed(6)
    for kind in ("fp32", "bf16", "fp16"):
        c = make(1, 128, 16)
        pages = filled(c, 4, gen)
        table = torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4)
        n = torch.tensor([57], dtype=torch.int32, device="cuda")
        q = torch.randn((1, 8, 128), generator=gen, device="cuda").to(TYPES[kind])
        q[0, 0] = 0
        q[0, 1] *= 1e-3
        q[0, 2, 0] = 300
        if kind != "fp16":
            q[0, 3] *= 1e-30
        q[0, 4, 77] = float("nan")
        out, lse = torch.empty_like(q), torch.empty((1, 8), device="cuda")
        c.lq_cache_attend(0, q, pages, table, n, out, lse=lse)
        assert torch.isnan(out[0, 4]).all() and torch.isnan(lse[0, 4])
        for h in (0, 1, 2, 3, 5, 6, 7):
            check_attention(c, pages, table, [57], q[:, h: h + 1], out[:, h: h + 1], lse[:, h: h + 1])
    # scores far apart, weights that follow the values' norms over many orders of magnitude
    c = make(1, 64, 16, (7, 7))
    x = torch.randn((64, 1, 64), generator=gen, device="cuda")
    v = x * torch.logspace(-12, 12, 64, device="cuda")[torch.randperm(64, device="cuda", generator=gen)].view(64, 1, 1)
    pages = c.empty_pages(4)
    c.lq_cache_write(0, x * 4, v, torch.arange(64, device="cuda"), pages)
    q = torch.randn((1, 8, 64), generator=gen, device="cuda") * 4
    out, lse = torch.empty_like(q), torch.empty((1, 8), device="cuda")
    c.lq_cache_attend(0, q, pages, table, torch.tensor([64], dtype=torch.int32, device="cuda"), out, lse=lse)
    check_attention(c, pages, table, [64], q, out, lse)
    c.lq_cache_attend(0, q, pages, table, torch.tensor([64], dtype=torch.int32, device="cuda"), out, lse=lse, scale=0.0)
    check_attention(c, pages, table, [64], q, out, lse, scale=0.0)


def test_pages_past_32_bits_of_offset():
    """A layer of more than 2^32 bytes and 2^31 words: rows at its far end."""
    c = make(8, 128, 128, (7, 7))
    num_pages = (1 << 31) // c.page_words + 40
    pages = torch.empty((num_pages, c.page_words), dtype=torch.int32, device="cuda")
    assert pages.numel() > 1 << 31
    gen = torch.Generator("cuda").manual_seed(7)
    k, v = (torch.randn((200, 8, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    first = (num_pages - 2) * 128
    slots = torch.arange(first, first + 200, device="cuda")
    c.lq_cache_write(0, k, v, slots, pages)
    x, y = torch.empty_like(k), torch.empty_like(v)
    c.lq_cache_read(0, pages, slots, x, y)
    few = pages[-2:].clone()
    table = torch.tensor([[num_pages - 2, num_pages - 1]], dtype=torch.int32, device="cuda")
    n = torch.tensor([200], dtype=torch.int32, device="cuda")
    q = torch.randn((1, 16, 128), generator=gen, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty((1, 16), device="cuda")
    c.lq_cache_attend(0, q, pages, table, n, out, lse=lse)
    assert c.lq_cache_status() == 0
    del pages
    check_attention(c, few, table - (num_pages - 2), [200], q, out, lse)
    a, b = torch.empty_like(k), torch.empty_like(v)
    c.lq_cache_read(0, few, slots - first, a, b)
    assert torch.equal(a, x) and torch.equal(b, y)


# ---- calls at once, recorded, in a row -------------------------------------------------------------------------

def test_two_graphs_replayed_at_the_same_time():
    """Both split one long sequence over many CTAs and join it; neither sees the other's partial sums."""
    gen = torch.Generator("cuda").manual_seed(8)
    c = make(2, 128, 64)
    pages = filled(c, 200, gen)
    state = []
    for i in range(2):
        table = torch.randperm(200, generator=gen, device="cuda").to(torch.int32).view(1, 200)
        n = torch.tensor([12800 - 100 * i], dtype=torch.int32, device="cuda")
        q = torch.randn((1, 8, 128), generator=gen, device="cuda")
        want, out = torch.empty_like(q), torch.zeros_like(q)
        c.lq_cache_attend(0, q, pages, table, n, want)
        state.append((table, n, q, want, out, torch.cuda.Stream(), torch.cuda.CUDAGraph()))
    torch.cuda.synchronize()
    for table, n, q, want, out, stream, graph in state:
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(20):
                c.lq_cache_attend(0, q, pages, table, n, out)
    for _ in range(5):
        for s in state:
            with torch.cuda.stream(s[5]):
                s[6].replay()
    torch.cuda.synchronize()
    for table, n, q, want, out, stream, graph in state:
        assert torch.equal(out, want)


def test_a_run_from_fitted_levels_to_answers():
    """Levels fitted to samples of keys and values by the plan's own fit (buckets of 128), a prompt written, read back, then tokens written
    and attended to one by one from a recorded graph."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(9)
    heads, dim, prompt, steps = 4, 128, 100, 40
    x = [torch.randn((1000, heads, dim), generator=gen, device="cuda") * s for s in (1.0, 0.2)]
    plan = lq.Plan([x[0].numel(), x[1].numel()], 3, 2, 1, 0)
    plan.lq_set_norm_scope("bucket")
    grads = torch.zeros((1, plan.padded_elems), device="cuda")
    for off, t in zip(plan.elem_offsets, x):
        grads[0, off: off + t.numel()] = t.reshape(-1)
    packed, norms, hist = plan.empty_packed(), plan.empty_norms(), plan.zero_hist()
    plan.lq_quantize_pack(grads, 1, packed, norms, hist=hist)
    plan.lq_fit_levels(hist, norms, 1)
    c = lq.Cache(1, heads, dim, 16, 3, 2, SEED)
    uniform = lq.Cache(1, heads, dim, 16, 3, 2, SEED)
    for m, kind in enumerate(("keys", "values")):
        c.lq_cache_set_levels(0, kind, plan.lq_get_levels(m))
    n_pages = 12
    pages, flat = c.empty_pages(n_pages), uniform.empty_pages(n_pages)
    k, v = (torch.randn((prompt + steps, heads, dim), generator=gen, device="cuda") * s for s in (1.0, 0.2))
    angles = lq.lq_rotary_table(1000, dim)
    order = torch.randperm(n_pages, generator=gen, device="cuda")
    slots = (order[:, None] * 16 + torch.arange(16, device="cuda")).reshape(-1)
    pos = torch.arange(prompt + steps, device="cuda")
    c.lq_cache_write(0, k[:prompt], v[:prompt], slots[:prompt], pages, rotary=angles, positions=pos[:prompt])
    uniform.lq_cache_write(0, k[:prompt], v[:prompt], slots[:prompt], flat, rotary=angles, positions=pos[:prompt])
    back = [torch.empty_like(v[:prompt]) for _ in range(4)]
    c.lq_cache_read(0, pages, slots[:prompt], back[0], back[1])
    uniform.lq_cache_read(0, flat, slots[:prompt], back[2], back[3])
    # what fitting is for: values are kept closer than by uniform levels
    assert (back[1] - v[:prompt]).norm() < (back[3] - v[:prompt]).norm()
    # one token at a time: the recorded step takes its inputs from buffers
    table = order.to(torch.int32).view(1, -1).contiguous()
    nk, nv, nq = torch.empty((1, heads, dim), device="cuda"), torch.empty((1, heads, dim), device="cuda"), torch.empty((1, 8, dim), device="cuda")
    at, slot, length = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(nq), torch.empty((1, 8), device="cuda")
    slot.copy_(slots[prompt: prompt + 1])

    def step():
        c.lq_cache_write(0, nk, nv, slot, pages, rotary=angles, positions=at)
        c.lq_cache_attend(0, nq, pages, table, length, out, lse=lse, rotary=angles)

    nk.zero_(); nv.zero_(); nq.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    qs = torch.randn((steps, 8, dim), generator=gen, device="cuda")
    for i in range(prompt, prompt + steps):
        nk.copy_(k[i: i + 1]); nv.copy_(v[i: i + 1]); nq.copy_(qs[i - prompt: i - prompt + 1])
        at.fill_(i); slot.copy_(slots[i: i + 1]); length.fill_(i + 1)
        graph.replay()
        if i % 13 == 0 or i == prompt + steps - 1:
            turned = torch.from_numpy(R.rotate(nq.cpu().numpy(), angles.cpu().numpy()[[i]], False))
            check_attention(c, pages, table, [i + 1], nq, out, lse, turned=turned)
    assert c.lq_cache_status() == 0


def test_calls_that_are_refused():
    import paper_2505_14371_b200 as lq
    c = make(2, 64, 16)
    pages = c.empty_pages(4)
    k = torch.randn((3, 2, 64), device="cuda")
    slots = torch.arange(3, device="cuda")
    q = torch.randn((2, 4, 64), device="cuda")
    table, n = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    angles = lq.lq_rotary_table(10, 64)
    out = torch.empty_like(q)
    write, read, attend = c.lq_cache_write, c.lq_cache_read, c.lq_cache_attend
    refused = [
        lambda: write(1, k, k, slots, pages), lambda: write(-1, k, k, slots, pages), lambda: write(0, k[:2], k, slots, pages),
        lambda: write(0, k, k.half(), slots, pages), lambda: write(0, k.double(), k.double(), slots, pages), lambda: write(0, k.cpu(), k, slots, pages),
        lambda: write(0, k, k, slots.int(), pages), lambda: write(0, k, k, slots, pages[:, 1:]), lambda: write(0, k, k, slots, pages.view(2, -1)),
        lambda: write(0, k.transpose(1, 2).contiguous().transpose(1, 2), k, slots, pages), lambda: write(0, k, k, slots, pages, step=-1),
        lambda: write(0, k, k, slots, pages, step=1 << 32), lambda: write(0, k, k, slots, pages, rotary=angles),
        lambda: write(0, k, k, slots, pages, positions=slots), lambda: write(0, k, k, slots, pages, rotary=angles, positions=slots[:2]),
        lambda: write(0, k, k, slots, pages, rotary=torch.zeros((4, 66), device="cuda"), positions=slots),
        lambda: write(0, k, k, slots, pages, rotary=torch.zeros((4, 3), device="cuda"), positions=slots),
        lambda: write(0, k, k, slots, pages, rotary=torch.zeros((0, 4), device="cuda"), positions=slots),
        lambda: read(0, pages, slots, k[:1].expand(3, 2, 64), k.clone()), lambda: read(0, pages, slots, k[:, :1].expand(3, 2, 64), k.clone()),
        lambda: attend(0, q[:, :3], pages, table, n, out[:, :3]), lambda: attend(0, q, pages, table, n, out.half()),
        lambda: attend(0, q, pages, table[:1], n, out), lambda: attend(0, q, pages, table.long(), n, out), lambda: attend(0, q, pages, table, n.long(), out),
        lambda: attend(0, q, pages, table, n, out, window=-1), lambda: attend(0, q, pages, table, n, out, scale=float("nan")),
        lambda: attend(0, q, pages, table, n, out[:1].expand(2, 4, 64)), lambda: attend(0, q, pages, table, n, out, lse=torch.empty((2, 3), device="cuda")),
        lambda: attend(0, q, pages, table, n, out, rotary=angles, positions=slots),
        lambda: c.lq_cache_set_levels(0, "keys", [0, 0.5, 1]), lambda: c.lq_cache_set_levels(0, "keys", [j / 8 for j in range(8)]),
        lambda: c.lq_cache_set_levels(0, "keys", [0, 0.125, 0.12501, 0.3, 0.4, 0.5, 0.6, 1]),       # one number after rounding
        lambda: c.lq_cache_set_levels(0, "keys", [0, 0.1, float("nan"), 0.3, 0.4, 0.5, 0.6, 1]), lambda: c.lq_cache_set_levels(2, "keys", [j / 7 for j in range(8)]),
    ]
    before = pages.clone()
    for i, call in enumerate(refused):
        with pytest.raises(lq.LqError):
            call()
            pytest.fail(f"call {i} was not refused")
    assert torch.equal(pages, before)
    # nothing to do is done
    write(0, k[:0], k[:0], slots[:0], pages)
    read(0, pages, slots[:0], k[:0], k[:0])
    attend(0, q[:0], pages, table[:0], n[:0], out[:0])
    # the C entry points check a workspace that torch would always size right
    lib, rows_t = lq.load_library(), lq.binding.Rows
    r = rows_t(q.data_ptr(), 256, 64, 0)
    o = rows_t(out.data_ptr(), 256, 64, 0)
    space = torch.empty(64, dtype=torch.uint8, device="cuda")
    wide = torch.zeros((2, 100), dtype=torch.int32, device="cuda")
    for window in (0, 1500):
        assert lib.lq_cache_workspace(c._h, 100, window) > 64
        rc = lib.lq_cache_attend(c._h, 0, r, 2, 4, pages.data_ptr(), 4, wide.data_ptr(), 100, n.data_ptr(), 1.0, window, None, o, None, space.data_ptr(), 64, None)
        assert rc == -1 and b"workspace" in lib.lq_last_error()
    # sequences that cannot be split need none
    assert lib.lq_cache_workspace(c._h, 2, 0) == 0 and lib.lq_cache_workspace(c._h, 100, 60) == 0
    assert lib.lq_cache_attend(c._h, 0, r, 2, 4, pages.data_ptr(), 4, table.data_ptr(), 2, n.data_ptr(), 1.0, 0, None, o, None, None, 0, None) == 0
    assert lib.lq_cache_workspace(c._h, -1, 0) == -1 and lib.lq_cache_workspace(c._h, 1, -1) == -1
    torch.cuda.synchronize()
    c.close()
    for call in (lambda: write(0, k, k, slots, pages), lambda: attend(0, q, pages, table, n, out), lambda: c.lq_cache_status()):
        with pytest.raises(lq.LqError):
            call()
