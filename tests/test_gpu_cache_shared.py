"""Attention over a prefix that a batch shares, on the GPU against numpy in 64 bits."""
import numpy as np
import pytest
import torch

import cache_reference as R
from test_gpu_cache import TYPES, filled, make, rows, sections

pytestmark = pytest.mark.gpu


def check(c, pages, prefix, length, table, lengths, q, out, lse, turned=None, scale=None, some=None):
    """Every row, or `some` of them."""
    sec = sections(c, pages)
    kk, vv = (R.values_of(sec[i], sec[2 + i], c.lq_cache_get_levels(0, n))[..., : c.head_dim] for i, n in ((0, "keys"), (1, "values")))
    half = torch.finfo(out.dtype).eps / 2
    w_error = 2.0 ** -20 if out.dtype == torch.float32 else 2.0 ** -11
    group = q.shape[1] // c.kv_heads
    qq = (q if turned is None else turned).double().cpu().numpy()
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    first, rest = prefix.cpu().numpy(), table.cpu().numpy()
    every = [(b, h) for b in range(q.shape[0]) for h in range(q.shape[1])]
    for b, h in every if some is None else [every[i] for i in some]:
        at, own = np.arange(length), np.arange(max(lengths[b], 0))
        pg = np.concatenate([first[at // c.page_size], rest[b][own // c.page_size]]).astype(np.int64)
        place = np.concatenate([at, own]) % c.page_size
        ok = (pg >= 0) & (pg < pages.shape[0])
        pg, place = pg[ok], place[ok]
        o, l, bound, lse_bound = R.attend(qq[b, h], kk[pg, h // group, place], vv[pg, h // group, place], c.head_dim ** -0.5 if scale is None else scale,
                                          2.0 ** -21, w_error)
        assert np.all(np.abs(got[b, h] - o) <= bound + half * (np.abs(o) + bound)), (b, h, lengths[b], np.abs(got[b, h] - o).max())
        assert got_lse[b, h] == l if np.isinf(l) else abs(got_lse[b, h] - l) <= lse_bound, (b, h, lengths[b])


def setting(c, length, lengths, gen, scale=1.0, more=2):
    page = c.page_size
    shared, width = -(-length // page), max(1, max((-(-n // page) for n in lengths), default=1)) + 1
    pages = filled(c, shared + 19, gen, scale)
    order = torch.randperm(shared + 19, generator=gen, device="cuda").int()
    prefix = torch.cat([order[:shared], torch.full((more,), -1, dtype=torch.int32, device="cuda")])     # (more room than the prefix takes)
    table = order[torch.randint(0, shared + 19, (len(lengths), width), generator=gen, device="cuda")]
    return pages, prefix, torch.tensor([length], dtype=torch.int32, device="cuda"), table, torch.tensor(lengths, dtype=torch.int32, device="cuda")


SHARED = [
    # heads, group, dim, page, bits, type, rotary, interleaved, prefix, lengths
    (1, 1, 64, 16, (3, 3), "bf16", 0, False, 64, [0]),
    (1, 1, 64, 16, (3, 3), "bf16", 0, False, 1, [0, 1]),
    (2, 4, 128, 64, (3, 3), "bf16", 0, False, 200, [0, 5, 64, 65]),
    (2, 4, 128, 16, (3, 3), "bf16", 128, False, 700, [20, 0, 1, 100]),
    (1, 8, 128, 32, (7, 7), "fp16", 0, False, 1000, [3] * 5),
    (3, 3, 64, 16, (3, 7), "fp16", 32, True, 333, [0, 7, 40]),
    (2, 1, 41, 32, (3, 3), "fp32", 0, False, 2050, list(range(9))),
    (1, 9, 65, 16, (7, 3), "fp32", 60, False, 129, [17] * 15),                  # 135 rows: two blocks, one with few
    (1, 16, 256, 128, (7, 3), "bf16", 64, True, 777, [100] * 9),                # 144 rows of 256
    (2, 5, 200, 16, (7, 7), "fp32", 200, False, 65, [1, 2, 3]),
    (1, 2, 256, 16, (3, 3), "fp16", 0, False, 500, [30]),
    (1, 4, 128, 16, (3, 3), "bf16", 128, False, 640, [11] * 64),                # 256 rows: a pair of blocks
    (2, 3, 128, 16, (3, 7), "fp16", 0, False, 450, [9] * 100),                  # 300 rows: a pair and one alone
    (1, 4, 64, 16, (7, 3), "bf16", 0, False, 63, [2] * 96),                     # 384 rows
    (1, 5, 96, 1024, (3, 3), "fp32", 96, True, 5000, [0, 100]),
    (1, 1, 8, 16, (3, 3), "bf16", 8, False, 15, [5, 0, 3]),
]


@pytest.mark.parametrize("heads,group,dim,page,bits,kind,rot,inter,length,lengths", SHARED)
def test_attention_with_a_shared_prefix(heads, group, dim, page, bits, kind, rot, inter, length, lengths):
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(length + dim)
    c = make(heads, dim, page, bits)
    pages, prefix, n, table, ln = setting(c, length, lengths, gen, 2.0)
    batch = len(lengths)
    q = rows(batch, heads * group, dim, TYPES[kind], gen, 1)
    wide = torch.full((batch, heads * group + 1, dim + 8), 9.0, dtype=TYPES[kind], device="cuda")
    out = wide[:, 1:, 8:]
    lse = torch.empty((batch, heads * group), device="cuda")
    t = lq.lq_rotary_table(length + 110, rot) if rot else None
    layout = "interleaved" if inter else "half"
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse, rotary=t, layout=layout)
    assert c.lq_cache_status() == 0
    some = None if batch * heads * group <= 64 else list(range(0, batch * heads * group, 7)) + [batch * heads * group - 1]
    turned = None
    if rot:
        turned = torch.from_numpy(R.rotate(q.float().cpu().numpy(), t.cpu().numpy()[[max(length + x - 1, 0) for x in lengths]], inter))
    check(c, pages, prefix, length, table, lengths, q, out, lse, turned, some=some)
    assert (wide[:, 0] == 9).all() and (wide[..., :8] == 9).all()
    again = torch.empty_like(out)
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, again, rotary=t, layout=layout)
    assert torch.equal(out, again)                              # the same call, the same bits


@pytest.mark.parametrize("length", [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 191, 192, 193])
@pytest.mark.parametrize("heads,group,dim,kind", [(1, 3, 64, "bf16"), (2, 2, 128, "fp32"), (1, 4, 256, "fp16")])
def test_prefixes_of_every_size(length, heads, group, dim, kind):
    gen = torch.Generator("cuda").manual_seed(length)
    c = make(heads, dim, 16, (3, 7))
    lengths = [0, 1, 33]
    pages, prefix, n, table, ln = setting(c, length, lengths, gen, more=0)
    q = torch.randn((3, heads * group, dim), generator=gen, device="cuda").to(TYPES[kind])
    out, lse = torch.full_like(q, 7), torch.full((3, heads * group), 7.0, device="cuda")
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse)
    check(c, pages, prefix, length, table, lengths, q, out, lse)
    # without a page of its own for any sequence
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table[:, :0], ln * 0, out, lse=lse)
    check(c, pages, prefix, length, table, [0, 0, 0], q, out, lse)
    if length == 0:
        assert not out.any() and torch.isneginf(lse).all()
    assert c.lq_cache_status() == 0


@pytest.mark.parametrize("rot", [0, 64])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("heads,group,dim,batch", [(40, 1, 64, 3), (37, 2, 128, 5), (75, 1, 200, 1), (20, 3, 128, 60), (80, 2, 64, 130), (30, 4, 250, 40)])
def test_many_tiles_a_share(heads, group, dim, batch, kind, rot):
    """So many heads that a CTA goes through dozens of tiles: few rows of a block (warps without any), one block, two, three."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim + batch)
    c = make(heads, dim, 64, (3, 7))
    length, lengths = 3001, [(7 * i) % 50 for i in range(batch)]
    pages, prefix, n, table, ln = setting(c, length, lengths, gen)
    q = torch.randn((batch, heads * group, dim), generator=gen, device="cuda").to(TYPES[kind])
    out, lse = torch.empty_like(q), torch.empty((batch, heads * group), device="cuda")
    t = turned = None
    if rot:
        t = lq.lq_rotary_table(3100, rot)
        turned = torch.from_numpy(R.rotate(q.float().cpu().numpy(), t.cpu().numpy()[[length + x - 1 for x in lengths]], False))
    rows = batch * heads * group
    for _ in range(3):
        out.fill_(7), lse.fill_(7)
        c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse, rotary=t)
        check(c, pages, prefix, length, table, lengths, q, out, lse, turned, some=sorted(set(list(range(0, rows, max(1, rows // 25))) + [rows - 1])))
    assert c.lq_cache_status() == 0


def test_it_is_the_plain_call_on_longer_tables():
    """With the prefix's pages before each sequence's own (a prefix of whole pages): the same numbers up to their rounding."""
    gen = torch.Generator("cuda").manual_seed(4)
    c = make(2, 128, 16, (3, 3))
    pages, prefix, n, table, ln = setting(c, 512, [0, 1, 40, 64], gen, more=0)
    q = torch.randn((4, 16, 128), generator=gen, device="cuda")
    a, b, la, lb = torch.empty_like(q), torch.empty_like(q), torch.empty((4, 16), device="cuda"), torch.empty((4, 16), device="cuda")
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, a, lse=la)
    c.lq_cache_attend(0, q, pages, torch.cat([prefix.expand(4, -1), table], dim=1).contiguous(), ln + 512, b, lse=lb)
    check(c, pages, prefix, 512, table, [0, 1, 40, 64], q, a, la)
    check(c, pages, prefix, 512, table, [0, 1, 40, 64], q, b, lb)


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("size,spread", [(30.0, 0.0), (1.0, 20.0), (1e-6, 8.0), (300.0, 3.0)])
def test_large_scores_and_norms_of_any_size(kind, size, spread):
    """Scores of hundreds, norms of the values over many powers of two: no weight loses bits that its row would show."""
    gen = torch.Generator("cuda").manual_seed(6)
    c = make(1, 64, 16, (3, 7))
    lengths = [0, 3, 20]
    pages, prefix, n, table, ln = setting(c, 700, lengths, gen)
    at = c.page_size * (64 * 4 // 32 + 64 * 8 // 32)
    norms = pages[:, at:].view(torch.float32)
    norms[:, 16:32] = torch.exp2(torch.randn(norms[:, 16:32].shape, generator=gen, device="cuda") * spread)
    norms[:, 16] = 0
    q = (torch.randn((3, 4, 64), generator=gen, device="cuda") * size).to(TYPES[kind])
    out, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse)
    sec = sections(c, pages)
    kk, vv = (R.values_of(sec[i], sec[2 + i], c.lq_cache_get_levels(0, x))[..., :64] for i, x in ((0, "keys"), (1, "values")))
    half = torch.finfo(out.dtype).eps / 2
    w_error = 2.0 ** -20 if kind == "fp32" else 2.0 ** -11
    for b, own in enumerate(lengths):
        at, mine = np.arange(700), np.arange(own)
        pg = np.concatenate([prefix.cpu().numpy()[at // 16], table[b].cpu().numpy()[mine // 16]])
        place = np.concatenate([at, mine]) % 16
        for h in range(4):
            v = vv[pg, 0, place]
            x = q[b, h].double().cpu().numpy()
            o, l, bound, lse_bound = R.attend(x, kk[pg, 0, place], v, 0.125, 2.0 ** -21, w_error)
            # (R.attend's bound holds weights to 2^-31 of the largest; here the largest weight times norm counts, which it knows nothing of)
            s = 0.125 * (kk[pg, 0, place] @ x)
            p = np.exp(s - s.max())
            bound = bound + len(p) * 2.0 ** -31 * (p[:, None] * np.abs(v)).max() / p.sum() + 2.0 ** -149
            low = np.finfo(np.float16).tiny * 2.0 ** -11 if kind == "fp16" else 0.0      # (an output below fp16's normal numbers: half its last bit)
            most = 65504.0 if kind == "fp16" else np.inf
            fits = np.abs(o) + bound < most
            g = out[b, h].double().cpu().numpy()
            assert np.all((np.abs(g - o) <= bound + half * (np.abs(o) + bound) + low)[fits]), (b, h, np.abs(g - o).max(), np.abs(o).max())
            assert abs(float(lse[b, h]) - l) <= lse_bound


def test_queries_that_are_not_finite():
    gen = torch.Generator("cuda").manual_seed(7)
    c = make(1, 64, 16, (3, 3))
    pages, prefix, n, table, ln = setting(c, 100, [0, 0, 4], gen)
    q = torch.randn((3, 2, 64), generator=gen, device="cuda")
    q[0, 0, 3] = float("nan")
    q[1, 1, 0] = float("inf")
    out, lse = torch.empty_like(q), torch.empty((3, 2), device="cuda")
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse)
    assert out[0, 0].isnan().all() and out[1, 1].isnan().all() and lse[0, 0].isnan() and lse[1, 1].isnan()
    good = torch.tensor([[False, True], [True, False], [True, True]], device="cuda")
    assert out[good].isfinite().all() and lse[good].isfinite().all()
    check(c, pages, prefix, 100, table, [0, 0, 4], q, out, lse, some=[1, 2, 4, 5])
    # nothing to see: zeros, whatever the query
    c.lq_cache_attend_shared(0, q, pages, prefix, n * 0, table, ln * 0, out, lse=lse)
    assert not out.any() and torch.isneginf(lse).all()


def test_bad_data():
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(8)
    c = make(2, 64, 16, (3, 3))
    pages, prefix, n, table, ln = setting(c, 320, [5, 16, 33], gen, more=0)
    q = torch.randn((3, 4, 64), generator=gen, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
    prefix[3] = -1; prefix[9] = pages.shape[0]; prefix[19] = 2 ** 31 - 1
    prefix[4: 8] = -7                                           # (a whole tile without a page)
    table[1, 0] = -2
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse)
    assert c.lq_cache_status() == lq.CACHE_BAD_PAGE
    check(c, pages, prefix, 320, table, [5, 16, 33], q, out, lse)
    prefix[:] = -1
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse)
    assert c.lq_cache_status() == lq.CACHE_BAD_PAGE
    check(c, pages, prefix, 320, table, [5, 16, 33], q, out, lse)
    assert not out[1].any() and torch.isneginf(lse[1]).all()
    # lengths past their tables are the tables', negative ones 0
    pages, prefix, n, table, ln = setting(c, 320, [5, 16, 33], gen, more=0)
    for given, taken in ((321, 320), (2 ** 31 - 1, 320), (-1, 0), (-2 ** 31, 0)):
        c.lq_cache_attend_shared(0, q, pages, prefix, n * 0 + given, table, ln, out, lse=lse)
        assert c.lq_cache_status() == lq.CACHE_BAD_LENGTH
        check(c, pages, prefix, taken, table, [5, 16, 33], q, out, lse)
    t = lq.lq_rotary_table(352, 64)
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse, rotary=t)          # the third one stands at 352
    assert c.lq_cache_status() == lq.CACHE_BAD_POSITION
    assert out[2].isnan().all()
    turned = torch.from_numpy(R.rotate(q.float().cpu().numpy(), t.cpu().numpy()[[324, 335, 0]], False))
    check(c, pages, prefix, 320, table, [5, 16, 33], q, out, lse, turned, some=range(8))
    at = torch.tensor([7, 351, 0], device="cuda")
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse, rotary=t, positions=at)
    assert c.lq_cache_status() == 0
    turned = torch.from_numpy(R.rotate(q.float().cpu().numpy(), t.cpu().numpy()[[7, 351, 0]], False))
    check(c, pages, prefix, 320, table, [5, 16, 33], q, out, lse, turned)


def test_captured_and_replayed_with_other_lengths():
    """One graph on a stream of its own, another call on the current stream at the same time; lengths, queries and pages change between replays."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(9)
    c = make(2, 128, 16, (3, 3))
    pages, prefix, n, table, ln = setting(c, 640, [30, 30, 30], gen, more=0)
    t = lq.lq_rotary_table(700, 128)
    q = torch.randn((3, 8, 128), generator=gen, device="cuda").to(torch.bfloat16)
    outs, lses = [torch.empty_like(q) for _ in range(3)], [torch.empty((3, 8), device="cuda") for _ in range(3)]

    def call(i):
        c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, outs[i], lse=lses[i], rotary=t)

    side, graphs = torch.cuda.Stream(), []
    call(0)
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(i)
        graphs.append(g)
    for length, lengths in ((640, [30, 1, 0]), (1, [0, 2, 3]), (333, [7, 30, 29]), (0, [0, 1, 30])):
        n.fill_(length)
        ln.copy_(torch.tensor(lengths))
        q.copy_(torch.randn(q.shape, generator=gen, device="cuda"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[0].replay()
        graphs[1].replay()
        call(2)
        torch.cuda.synchronize()
        turned = torch.from_numpy(R.rotate(q.float().cpu().numpy(), t.cpu().numpy()[[max(length + x - 1, 0) for x in lengths]], False))
        check(c, pages, prefix, length, table, lengths, q, outs[0], lses[0], turned)
        for i in (1, 2):
            assert torch.equal(outs[0], outs[i]) and torch.equal(lses[0], lses[i])
    assert c.lq_cache_status() == 0


def test_refusals():
    import paper_2505_14371_b200 as lq
    c = make(2, 64, 16, (3, 3))
    pages = c.empty_pages(4)
    i32 = dict(dtype=torch.int32, device="cuda")
    prefix, n, table, ln = torch.zeros(3, **i32), torch.zeros(1, **i32), torch.zeros((2, 4), **i32), torch.zeros(2, **i32)
    q = torch.zeros((2, 4, 64), device="cuda")
    out = torch.zeros_like(q)
    good = dict(layer=0, queries=q, pages=pages, prefix=prefix, prefix_length=n, table=table, lengths=ln, out=out)
    for bad in (dict(layer=1), dict(layer=-1), dict(queries=q[:1]), dict(queries=q[:, :3], out=out[:, :3]), dict(queries=q.half()), dict(queries=q.double()),
                dict(pages=pages[:, :-1]), dict(pages=pages.float()), dict(prefix=prefix.long()), dict(prefix=prefix[None]), dict(prefix=prefix.cpu()),
                dict(prefix_length=torch.zeros(2, **i32)), dict(prefix_length=n.long()), dict(prefix_length=5), dict(table=table[:1]),
                dict(table=table.t()), dict(lengths=ln.long()), dict(lengths=ln[:1]), dict(out=out[:, :1].expand(-1, 4, -1)), dict(out=out[..., ::2]),
                dict(lse=torch.zeros((2, 3), device="cuda")), dict(lse=torch.zeros((2, 4), device="cuda").half()), dict(scale=float("inf")), dict(scale="a"),
                dict(positions=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(rotary=lq.lq_rotary_table(9, 66)), dict(layout="none"),
                dict(queries=q.clone().requires_grad_()), dict(out=out.clone().requires_grad_())):
        with pytest.raises((lq.LqError, TypeError)):
            c.lq_cache_attend_shared(**{**good, **bad})
    lib = lq.load_library()
    assert lib.lq_cache_shared_workspace(c._h, -1, 4, 3, 4, 0, 0) == -1 and lib.lq_cache_shared_workspace(c._h, 2, 3, 3, 4, 0, 0) == -1
    assert lib.lq_cache_shared_workspace(c._h, 2, 4, -1, 4, 0, 0) == -1 and lib.lq_cache_shared_workspace(c._h, 2, 4, 3, 4, 3, 0) == -1
    assert lib.lq_cache_shared_workspace(c._h, 1 << 24, 8, 3, 4, 0, 0) == -1
    assert lib.lq_cache_shared_workspace(c._h, 0, 4, 3, 4, 0, 0) >= 0
    assert c.lq_cache_status() == 0 and not out.any()
    c.lq_cache_attend_shared(0, q[:0], pages, prefix, n, table[:0], ln[:0], out[:0])
    c.lq_cache_attend_shared(**good)
    assert c.lq_cache_status() == 0 and not out.any()
