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
