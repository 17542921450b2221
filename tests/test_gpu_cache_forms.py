"""Every form that the cache's attention is compiled for, the joined split at all row sizes, and rows in orders other than tokens first."""
import pytest
import torch

import cache_reference as R
from test_gpu_cache import TYPES, check_attention, filled, make

pytestmark = pytest.mark.gpu

# type, queries a head, rotated: one of each way in which queries and weights are rounded
WAYS = [("bf16", 8, False), ("bf16", 7, True), ("bf16", 3, True), ("fp16", 4, True), ("fp16", 6, False), ("fp16", 5, True), ("fp32", 2, True), ("fp32", 9, True)]


def attend_and_check(c, pages, lengths, group, kind, rot, gen, window=0, inter=False):
    import paper_2505_14371_b200 as lq
    width = max(1, max(-(-n // c.page_size) for n in lengths))
    table = torch.randint(0, pages.shape[0], (len(lengths), width), generator=gen, device="cuda", dtype=torch.int32)
    q = (torch.randn((len(lengths), c.kv_heads * group, c.head_dim), generator=gen, device="cuda") * 2).to(TYPES[kind])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    angles = turned = None
    if rot:
        angles = lq.lq_rotary_table(max(lengths) + 1, c.head_dim // 2 * 2)
        at = (n.long() - 1).clamp(min=0).cpu().numpy()
        turned = torch.from_numpy(R.rotate(q.float().cpu().numpy(), angles.cpu().numpy()[at], inter))
    c.lq_cache_attend(0, q, pages, table, n, out, lse=lse, window=window, rotary=angles, layout="interleaved" if inter else "half")
    assert c.lq_cache_status() == 0
    check_attention(c, pages, table, lengths, q, out, lse, window, turned=turned)


@pytest.mark.parametrize("dim", [64, 50, 128, 256, 136])
@pytest.mark.parametrize("bits", [(3, 3), (3, 7), (7, 3), (7, 7)])
@pytest.mark.parametrize("kind,group,rot", WAYS)
def test_every_compiled_form(dim, bits, kind, group, rot):
    gen = torch.Generator("cuda").manual_seed(dim + group)
    c = make(2, dim, 32, bits)
    attend_and_check(c, filled(c, 30, gen), [0, 1, 16, 37, 259, 700], group, kind, rot, gen, inter=group % 2 == 1)


@pytest.mark.parametrize("dim,bits", [(64, (7, 7)), (128, (3, 3)), (128, (7, 3)), (256, (3, 3)), (256, (7, 7)), (200, (3, 7))])
@pytest.mark.parametrize("kind,group,rot", WAYS)
def test_long_sequences_are_split_and_joined(dim, bits, kind, group, rot):
    """One sequence over all teams, several units each; then a few of which some teams have an end and a beginning."""
    gen = torch.Generator("cuda").manual_seed(dim + group)
    c = make(1, dim, 64, bits)
    pages = filled(c, 600, gen)
    attend_and_check(c, pages, [77777], group, kind, rot, gen)
    attend_and_check(c, pages, [9001, 3, 20011, 0, 4097], group, kind, rot, gen, window=8191 if group % 2 else 0)


@pytest.mark.parametrize("dim,kind,group", [(128, "bf16", 4), (41, "fp32", 3), (64, "fp16", 8), (256, "fp32", 1)])
def test_rows_with_heads_outermost_and_rows_that_are_shared(dim, kind, group):
    """Views [heads][tokens][dim] turned round, every second token, and inputs whose tokens or heads are one row (a stride of 0)."""
    heads, tokens, page = 3, 100, 16
    gen = torch.Generator("cuda").manual_seed(dim)
    dtype = TYPES[kind]
    c = make(heads, dim, page, (3, 7))
    slots = torch.randperm(7 * page, generator=gen, device="cuda")[:tokens]
    base = torch.randn((heads, 2 * tokens, dim), generator=gen, device="cuda").to(dtype)
    views = [base.transpose(0, 1)[:tokens], base.transpose(0, 1)[::2], base[:1, :1].transpose(0, 1).expand(tokens, heads, dim), base[:, :1].transpose(0, 1).expand(tokens, heads, dim),
             base[:1].transpose(0, 1)[:tokens].expand(tokens, heads, dim)]
    for k in views:
        for v in (views[0], views[2]):
            one, two = c.empty_pages(7), c.empty_pages(7)
            c.lq_cache_write(0, k, v, slots, one)
            c.lq_cache_write(0, k.contiguous(), v.contiguous(), slots, two)
            assert torch.equal(one, two)
    want = [torch.empty((tokens, heads, dim), dtype=dtype, device="cuda") for _ in range(2)]
    wide = [torch.full((heads, 2 * tokens, dim), 9.0, dtype=dtype, device="cuda") for _ in range(2)]
    c.lq_cache_read(0, one, slots, *want)
    c.lq_cache_read(0, one, slots, *(w.transpose(0, 1)[::2] for w in wide))
    for w, x in zip(wide, want):
        assert torch.equal(w.transpose(0, 1)[::2], x) and (w[:, 1::2] == 9).all()
    batch = 5
    table = torch.arange(7, dtype=torch.int32, device="cuda").repeat(batch, 1)
    n = torch.tensor([112, 1, 0, 60, 111], dtype=torch.int32, device="cuda")
    q = torch.randn((heads * group, 2 * batch, dim), generator=gen, device="cuda").to(dtype).transpose(0, 1)
    for mine in (q[:batch], q[::2], q[:1].expand(batch, heads * group, dim), q[:batch, :1].expand(batch, heads * group, dim)):
        out, lse = torch.empty((batch, heads * group, dim), dtype=dtype, device="cuda"), torch.empty((batch, heads * group), device="cuda")
        c.lq_cache_attend(0, mine.contiguous(), one, table, n, out, lse=lse)
        check_attention(c, one, table, n.tolist(), mine.contiguous(), out, lse)
        turned = torch.full((heads * group, 2 * batch, dim), 9.0, dtype=dtype, device="cuda")
        again = torch.empty_like(lse)
        c.lq_cache_attend(0, mine, one, table, n, turned.transpose(0, 1)[::2], lse=again)
        assert torch.equal(turned.transpose(0, 1)[::2], out) and torch.equal(again, lse) and (turned[:, 1::2] == 9).all()
    # in place: every query's place takes its output
    mine = q[:batch].contiguous()
    out = torch.empty_like(mine)
    c.lq_cache_attend(0, mine, one, table, n, out)
    c.lq_cache_attend(0, mine, one, table, n, mine)
    assert torch.equal(mine, out) and c.lq_cache_status() == 0
