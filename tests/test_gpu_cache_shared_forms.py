"""Attention over a shared prefix where the sequences' own tokens are split, where blocks of rows are left over, and in calls queued behind one
another."""
import numpy as np
import pytest
import torch

import cache_reference as R
from test_gpu_cache import TYPES, make, sections
from test_gpu_cache_shared import check, setting

pytestmark = pytest.mark.gpu


def turned_of(lq, q, length, lengths, rot, inter=False):
    t = lq.lq_rotary_table(length + max(lengths) + 1, rot)
    at = [max(length + x - 1, 0) for x in lengths]
    return t, torch.from_numpy(R.rotate(q.float().cpu().numpy(), t.cpu().numpy()[at], inter))


# ---- own tokens that several teams have --------------------------------------------------------------------

OWN = [
    # heads, group, dim, page, bits, type, rotary, prefix, own lengths
    (1, 1, 64, 16, (3, 3), "bf16", 0, 100, [3000]),
    (2, 4, 128, 64, (3, 3), "bf16", 128, 700, [2500, 0, 129, 300]),
    (2, 4, 128, 64, (3, 7), "fp16", 0, 333, [1, 2000, 777]),
    (1, 3, 128, 16, (7, 3), "fp32", 64, 1100, [4000, 17]),
    (1, 9, 41, 32, (3, 3), "fp32", 0, 65, [5000, 256, 257]),                    # two blocks of queries, one with one of them
    (2, 2, 256, 128, (3, 3), "bf16", 0, 500, [1500, 128, 129]),
    (1, 5, 200, 16, (7, 7), "fp16", 200, 40, [900, 901]),
    (1, 12, 256, 16, (3, 7), "fp32", 0, 0, [1000]),
    (3, 1, 64, 1024, (7, 7), "fp16", 0, 2000, [6000, 5, 1025]),
]


@pytest.mark.parametrize("heads,group,dim,page,bits,kind,rot,length,lengths", OWN)
def test_own_tokens_of_several_teams(heads, group, dim, page, bits, kind, rot, length, lengths):
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(length + dim)
    c = make(heads, dim, page, bits)
    pages, prefix, n, table, ln = setting(c, length, lengths, gen, 2.0)
    q = torch.randn((len(lengths), heads * group, dim), generator=gen, device="cuda").to(TYPES[kind])
    out, lse = torch.full_like(q, 7), torch.full(q.shape[:2], 7.0, device="cuda")
    t, turned = turned_of(lq, q, length, lengths, rot) if rot else (None, None)
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse, rotary=t)
    assert c.lq_cache_status() == 0
    check(c, pages, prefix, length, table, lengths, q, out, lse, turned)
    again = torch.empty_like(out)
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, again, rotary=t)
    assert torch.equal(out, again)


# ---- blocks of 128 rows that are left over -----------------------------------------------------------------

@pytest.mark.parametrize("length", [1, 64, 65, 129, 200, 1000, 3001])
@pytest.mark.parametrize("heads,group,batch", [(1, 4, 96), (1, 5, 65), (40, 4, 72), (2, 4, 160), (1, 4, 127), (30, 3, 130), (2, 8, 94)])
def test_a_block_that_is_left_over(heads, group, batch, length):
    """Rotated bf16 queries of rows of 128 in three blocks and five, whose last has no other beside it, and in four and six; last blocks of few rows."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(length + batch)
    c = make(heads, 128, 64, (3, 7))
    lengths = [(5 * i) % 23 for i in range(batch)]
    pages, prefix, n, table, ln = setting(c, length, lengths, gen)
    q = torch.randn((batch, heads * group, 128), generator=gen, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    t, turned = turned_of(lq, q, length, lengths, 128)
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse, rotary=t)
    assert c.lq_cache_status() == 0
    rows = batch * heads * group
    check(c, pages, prefix, length, table, lengths, q, out, lse, turned, some=sorted(set(list(range(0, rows, max(1, rows // 40))) + list(range(rows - 9, rows)))))


# ---- fp16 outputs: weights of 22 bits ----------------------------------------------------------------------

def within(got, o, bound):
    """Outputs that are fp16 numbers, half a step of their own (not of the binade's end) beside what 32-bit arithmetic may be off."""
    step = np.spacing(np.abs(o).astype(np.float16)).astype(np.float64)
    return np.abs(got - o) <= bound + np.maximum(step, np.spacing((np.abs(o) + bound).astype(np.float16)).astype(np.float64)) / 2


@pytest.mark.parametrize("rot", [0, 64])
@pytest.mark.parametrize("dim,group,batch", [(64, 3, 4), (64, 8, 40), (128, 4, 4), (128, 4, 70), (256, 2, 5)])
@pytest.mark.parametrize("length,own", [(2, 0), (3, 0), (17, 0), (40, 3), (64, 0), (130, 1)])
def test_weights_of_fp16_outputs_have_22_bits(dim, group, batch, rot, length, own):
    """Few tokens, so that roundings do not even out: with weights of 11 bits (which the oracle shows) some outputs would be a step off."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim + length)
    c = make(1, dim, 16, (7, 7))
    lengths = [own] * batch
    pages, prefix, n, table, ln = setting(c, length, lengths, gen)
    q = torch.randn((batch, group, dim), generator=gen, device="cuda").half()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    t, turned = turned_of(lq, q, length, lengths, rot) if rot else (None, q)
    c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse, rotary=t)
    sec = sections(c, pages)
    kk, vv = (R.values_of(sec[i], sec[2 + i], c.lq_cache_get_levels(0, x))[..., :dim] for i, x in ((0, "keys"), (1, "values")))
    at, mine = np.arange(length), np.arange(own)
    place = np.concatenate([at, mine]) % 16
    got, qq = out.double().cpu().numpy(), turned.double().cpu().numpy()
    coarse = 0
    for b in range(0, batch, max(1, batch // 8)):
        pg = np.concatenate([prefix.cpu().numpy()[at // 16], table[b].cpu().numpy()[mine // 16]])
        k, v = kk[pg, 0, place], vv[pg, 0, place]
        for h in range(group):
            o, _, bound, _ = R.attend(qq[b, h], k, v, dim ** -0.5, 2.0 ** -21, 2.0 ** -20)
            assert np.all(within(got[b, h], o, bound)), (b, h, (np.abs(got[b, h] - o) - bound).max())
            s = dim ** -0.5 * (k @ qq[b, h])
            w = np.exp(s - s.max()) * np.abs(v).max(-1)         # (level times norm: the norm is part of a weight)
            r = w.astype(np.float16).astype(np.float64) / np.abs(v).max(-1)
            coarse += not np.all(within(((r @ v) / np.exp(s - s.max()).sum()).astype(np.float16).astype(np.float64), o, bound))
    assert coarse > 0


# ---- calls queued behind one another -----------------------------------------------------------------------

@pytest.mark.parametrize("heads,dim,page,bits,kind,rot,batch", [(8, 128, 64, (3, 3), "bf16", 128, 3), (2, 128, 32, (3, 7), "bf16", 0, 70), (2, 41, 16, (7, 7), "fp32", 0, 2),
                                                                (1, 64, 16, (7, 3), "fp16", 20, 40), (2, 256, 32, (3, 7), "bf16", 256, 4)])
def test_rows_lengths_and_queries_of_the_call_before(heads, dim, page, bits, kind, rot, batch):
    """Every round writes rows of the prefix and of the sequences anew, and lengths, and attends to them; nothing but the calls on the stream, so each kernel
    starts beside its predecessor, and every call takes the workspace that the one before it had.  A result that is late by a call is another round's."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim + batch)
    rounds, dtype, tokens, own = 60, TYPES[kind], 400, 50
    c = make(heads, dim, page, bits)
    shared, each = -(-tokens // page), -(-own // page)
    num = shared + batch * each
    k, v = (torch.randn((rounds, num * page, heads, dim), generator=gen, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((rounds, batch, heads * 4, dim), generator=gen, device="cuda").to(dtype)
    slots = torch.randperm(num * page, generator=gen, device="cuda")
    prefix = torch.arange(shared, dtype=torch.int32, device="cuda")
    table = torch.arange(shared, num, dtype=torch.int32, device="cuda").view(batch, each)
    lengths = torch.randint(0, own + 1, (rounds, batch), generator=gen, device="cuda", dtype=torch.int32)
    first = torch.randint(0, tokens + 1, (rounds, 1), generator=gen, device="cuda", dtype=torch.int32)
    angles = lq.lq_rotary_table(tokens + own, rot) if rot else None
    now, n = torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(wait):
        pages, out, lse = c.empty_pages(num), torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
        torch.cuda.synchronize()
        for i in range(rounds):
            for call in (lambda: now.copy_(lengths[i]), lambda: n.copy_(first[i]), lambda: c.lq_cache_write(0, k[i], v[i], slots, pages),
                         lambda: c.lq_cache_attend_shared(0, q[i], pages, prefix, n, table, now, out[i], lse=lse[i], rotary=angles),
                         lambda: c.lq_cache_attend_shared(0, out[i], pages, prefix, n, table, now, q2[i], rotary=angles)):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return out, lse, q2.clone()

    q2 = torch.empty_like(q)
    want = run(True)
    for _ in range(3):
        for got, w in zip(run(False), want):
            assert torch.equal(got, w)
    assert c.lq_cache_status() == 0
    assert not torch.equal(want[0][0], want[0][1]) and want[0].isfinite().all()


@pytest.mark.parametrize("heads,dim,page,bits,kind,rot,batch", [(8, 128, 16, (3, 3), "bf16", 128, 3), (2, 41, 16, (7, 7), "fp32", 0, 40), (1, 64, 16, (7, 3), "fp16", 20, 1)])
def test_bounds_and_choices_of_the_call_before(heads, dim, page, bits, kind, rot, batch):
    """The same for bounds, a choice by them and attention over what was chosen."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim + batch)
    rounds, dtype, tokens, keep = 60, TYPES[kind], 700, 6
    c = make(heads, dim, page, bits)
    each = -(-tokens // page)
    num = batch * each
    k, v = (torch.randn((rounds, num * page, heads, dim), generator=gen, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((rounds, batch, heads * 4, dim), generator=gen, device="cuda").to(dtype)
    slots, which = torch.randperm(num * page, generator=gen, device="cuda"), torch.arange(num, dtype=torch.int32, device="cuda")
    table = torch.randperm(num, generator=gen, device="cuda").int().view(batch, each)
    lengths = torch.randint(1, tokens + 1, (rounds, batch), generator=gen, device="cuda", dtype=torch.int32)
    angles = lq.lq_rotary_table(tokens, rot) if rot else None
    now, at = torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.zeros(batch, dtype=torch.int64, device="cuda")

    def run(wait):
        pages, bounds, out, lse = c.empty_pages(num), c.empty_bounds(num), torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
        chosen = torch.empty((rounds, batch, heads, keep), dtype=torch.int32, device="cuda")
        seen = torch.empty((rounds, batch, heads), dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        for i in range(rounds):
            for call in (lambda: now.copy_(lengths[i]), lambda: at.copy_(lengths[i] - 1), lambda: c.lq_cache_write(0, k[i], v[i], slots, pages),
                         lambda: c.lq_cache_bounds(0, pages, which, bounds), lambda: c.lq_cache_choose(q[i], bounds, table, now, chosen[i], seen[i], rotary=angles),
                         lambda: c.lq_cache_attend_chosen(0, q[i], pages, chosen[i], seen[i], out[i], lse=lse[i], rotary=angles, positions=at if rot else None)):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        return chosen, seen, out, lse

    want = run(True)
    for _ in range(3):
        for got, w in zip(run(False), want):
            assert torch.equal(got, w)
    assert c.lq_cache_status() == 0
    assert not torch.equal(want[2][0], want[2][1]) and want[2].isfinite().all()
