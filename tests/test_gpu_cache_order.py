"""Calls of the cache queued one behind the other, each reading what the one before it writes: every result as when the device is waited
for between them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.mark.parametrize("heads,dim,page,bits,kind,rot", [(8, 128, 64, (3, 3), "bf16", 128), (2, 41, 16, (7, 7), "fp32", 0), (1, 64, 16, (7, 3), "fp16", 20),
                                                          (2, 256, 32, (3, 7), "bf16", 256)])
@pytest.mark.parametrize("tokens", [1, 333])
def test_rows_pages_and_sums_of_the_call_before(heads, dim, page, bits, kind, rot, tokens):
    """New rows in the same slots every round: written, read back, the rows read written to a second cache, and that attended to; nothing
    but the calls on the stream, so each starts beside its predecessor.  A result that is late by a call is another round's."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(tokens + dim)
    rounds, dtype = 120, TYPES[kind]
    a, b = (lq.Cache(1, heads, dim, page, bits, 0, 7) for _ in range(2))
    num = -(-tokens // page) + 1
    k, v = (torch.randn((rounds, tokens, heads, dim), generator=gen, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn((rounds, 1, heads * 4, dim), generator=gen, device="cuda").to(dtype)
    slots = torch.randperm(num * page, generator=gen, device="cuda")[:tokens].contiguous()
    ordered = torch.arange(tokens, device="cuda")
    table = torch.arange(num, dtype=torch.int32, device="cuda").view(1, num)
    length = torch.tensor([tokens], dtype=torch.int32, device="cuda")
    angles = lq.lq_rotary_table(tokens, rot) if rot else None

    def run(wait):
        p, r = a.empty_pages(num), b.empty_pages(num)
        x, y = torch.empty_like(k), torch.empty_like(v)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
        torch.cuda.synchronize()
        calls = []
        for i in range(rounds):
            calls += [lambda i=i: a.lq_cache_write(0, k[i], v[i], slots, p, rotary=angles, positions=ordered if rot else None),
                      lambda i=i: a.lq_cache_read(0, p, slots, x[i], y[i]),
                      lambda i=i: b.lq_cache_write(0, x[i], y[i], ordered, r),
                      lambda i=i: b.lq_cache_attend(0, q[i], r, table, length, out[i], lse=lse[i], rotary=angles)]
        for call in calls:
            call()
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return x, y, out, lse

    want = run(True)
    for _ in range(3):
        for got, w in zip(run(False), want):
            assert torch.equal(got, w)
    assert a.lq_cache_status() == 0 and b.lq_cache_status() == 0
    # the rounds do differ
    assert not torch.equal(want[0][0], want[0][1]) and not torch.equal(want[3][0], want[3][1])


@pytest.mark.parametrize("dim,group,kind", [(128, 1, "bf16"), (128, 3, "fp32"), (128, 5, "bf16"), (64, 7, "fp32"), (64, 3, "fp16"), (256, 5, "bf16"), (256, 9, "fp16"), (41, 2, "fp32")])
def test_the_same_call_gives_the_same_bits(dim, group, kind):
    """Rotated queries in blocks that they do not fill, whatever ran before: the places without a query have no say in when the running
    references move, by which weights are rounded."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim + group)
    heads, tokens, page = 2, 4001, 32
    c = lq.Cache(1, heads, dim, page, (3, 7), 0, 7)
    num = -(-tokens // page)
    # scores that grow along the sequence: references move all the way
    grow = torch.linspace(0.1, 8.0, num * page, device="cuda").view(-1, 1, 1)
    k, v = (torch.randn((num * page, heads, dim), generator=gen, device="cuda") for _ in range(2))
    pages = c.empty_pages(num)
    c.lq_cache_write(0, k * grow, v, torch.arange(num * page, device="cuda"), pages)
    table = torch.arange(num, dtype=torch.int32, device="cuda").view(1, num)
    length = torch.tensor([tokens], dtype=torch.int32, device="cuda")
    q = torch.randn((1, heads * group, dim), generator=gen, device="cuda").to(TYPES[kind])
    angles = lq.lq_rotary_table(tokens, dim // 2 * 2)
    first = None
    others = [lambda: None, lambda: torch.randn(1 << 22, generator=gen, device="cuda").mul_(1e30).exp_(),
              lambda: torch.full((4096, 4096), 3e38, device="cuda") @ torch.ones((4096, 4096), device="cuda"),
              lambda: (torch.randn((2048, 2048), generator=gen, device="cuda").half() * 100) @ torch.randn((2048, 2048), generator=gen, device="cuda").half(),
              lambda: torch.randint(-2 ** 31, 2 ** 31 - 1, (1 << 22,), generator=gen, device="cuda").sort(),
              lambda: c.lq_cache_read(0, pages, torch.arange(64, device="cuda"), torch.empty_like(k[:64]), torch.empty_like(k[:64])),
              lambda: torch.randn((64, 64, 64), generator=gen, device="cuda", dtype=torch.float64).cumsum(0)]
    for i in range(6 * len(others)):
        others[i % len(others)]()
        out, lse = torch.empty_like(q), torch.empty((1, heads * group), device="cuda")
        c.lq_cache_attend(0, q, pages, table, length, out, lse=lse, rotary=angles)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), i


@pytest.mark.parametrize("dim,group,kind,bits", [(128, 1, "bf16", (3, 3)), (128, 5, "bf16", (7, 7)), (64, 3, "fp32", (3, 7)), (64, 7, "fp16", (3, 3)), (256, 5, "fp32", (3, 3)),
                                                 (256, 2, "bf16", (7, 3))])
def test_other_sequences_of_a_batch_leave_no_trace(dim, group, kind, bits):
    """The queries of every second sequence are other ones: the bits of those between them stay (lengths, and with them the split, are the same)."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim + group)
    heads, page, batch, most = 3, 16, 400, 700
    c = lq.Cache(1, heads, dim, page, bits, 0, 7)
    per = most // page + 1
    grow = torch.linspace(0.1, 8.0, per * page, device="cuda").repeat(4).view(-1, 1, 1)
    k, v = (torch.randn((4 * per * page, heads, dim), generator=gen, device="cuda") for _ in range(2))
    pages = c.empty_pages(4 * per)
    c.lq_cache_write(0, k * grow, v * torch.randn_like(v[:, :1, :1]).mul_(3).exp_(), torch.arange(4 * per * page, device="cuda"), pages)
    table = (torch.arange(batch, device="cuda")[:, None] % 4 * per + torch.arange(per, device="cuda")).to(torch.int32)
    lengths = torch.randint(1, most, (batch,), generator=gen, device="cuda", dtype=torch.int32)
    q = torch.randn((batch, heads * group, dim), generator=gen, device="cuda").to(TYPES[kind])
    angles = lq.lq_rotary_table(most, dim // 2 * 2)
    first = None
    for factor in (1.0, 50.0, 0.0, -3.0):
        mine = q.clone()
        mine[1::2] *= factor
        out, lse = torch.empty_like(q), torch.empty((batch, heads * group), device="cuda")
        c.lq_cache_attend(0, mine, pages, table, lengths, out, lse=lse, rotary=angles)
        first = first or (out[::2].clone(), lse[::2].clone())
        assert torch.equal(out[::2], first[0]) and torch.equal(lse[::2], first[1]), factor


def test_no_flag_is_lost_to_another_threads_status():
    """One thread makes calls that set a flag, each after the last flag was seen; another asks for the flags all the time.  (A flag that is set
    between their copy and their clearing has to stay.)"""
    import random
    import threading
    import time
    import paper_2505_14371_b200 as lq
    c = lq.Cache(1, 1, 64, 16, 3, 0, 7)
    pages = c.empty_pages(1)
    k, bad = torch.ones((1, 1, 64), device="cuda"), torch.tensor([1000], device="cuda")
    seen, stop, failed = [0], threading.Event(), []

    def ask():
        try:
            while not stop.is_set():
                if c.lq_cache_status() & lq.CACHE_BAD_SLOT:
                    seen[0] += 1
        except Exception as e:                      # (reported by the test's thread)
            failed.append(e)

    asking = threading.Thread(target=ask)
    torch.cuda.synchronize()
    asking.start()
    try:
        rng, stream, lost = random.Random(1), torch.cuda.Stream(), None
        with torch.cuda.stream(stream):
            for i in range(1500):
                before, until = seen[0], time.perf_counter() + rng.random() * 60e-6
                while time.perf_counter() < until:
                    pass
                c.lq_cache_write(0, k, k, bad, pages)
                until = time.perf_counter() + 1.0
                while seen[0] == before and not failed and time.perf_counter() < until:
                    time.sleep(0)
                if seen[0] == before:
                    lost = i
                    break
    finally:
        stop.set()
        asking.join()
    assert not failed and lost is None, (failed, lost)


def test_gradients_are_not_cut_off_silently():
    import paper_2505_14371_b200 as lq
    c = lq.Cache(1, 2, 64, 16, 3, 0, 7)
    pages = c.empty_pages(1)
    k, q, slots = torch.randn((4, 2, 64), device="cuda"), torch.randn((1, 4, 64), device="cuda"), torch.arange(4, device="cuda")
    table, n = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.tensor([4], dtype=torch.int32, device="cuda")
    kept = k.clone().requires_grad_()
    c.lq_cache_write(0, kept, kept * 2, slots, pages)               # what is stored is numbers
    out, lse = torch.empty_like(q), torch.empty((1, 4), device="cuda")
    c.lq_cache_attend(0, q, pages, table, n, out, lse=lse)
    want = q.clone().requires_grad_()
    for mine in (want, want * 1.0):
        with pytest.raises(lq.LqError, match="queries.*gradient"):
            c.lq_cache_attend(0, mine, pages, table, n, out)
    with pytest.raises(lq.LqError, match="out.*gradient"):
        c.lq_cache_attend(0, q, pages, table, n, out.clone().requires_grad_())
    with pytest.raises(lq.LqError, match="lse.*gradient"):
        c.lq_cache_attend(0, q, pages, table, n, out, lse=lse.clone().requires_grad_())
    with pytest.raises(lq.LqError, match="keys.*gradient"):
        c.lq_cache_read(0, pages, slots, kept, k.clone())
    with pytest.raises(lq.LqError, match="values.*gradient"):
        c.lq_cache_read(0, pages, slots, k.clone(), kept)
    other = torch.empty_like(out)
    with torch.no_grad():
        c.lq_cache_attend(0, want, pages, table, n, other)
    assert torch.equal(other, out)
    c.lq_cache_attend(0, want.detach(), pages, table, n, other)
    assert torch.equal(other, out) and c.lq_cache_status() == 0
