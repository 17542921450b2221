"""Waits inside the attention over a shared prefix that run out: the call ends, says so, and leaves nothing behind that the next one meets."""
import pytest
import torch

from test_gpu_cache import TYPES, make
from test_gpu_cache_shared import check, setting

pytestmark = pytest.mark.gpu

# heads, group, dim, batch, type, rotary: every form of the prefix's kernel, one block of rows, two and three
FORMS = [(2, 2, 64, 3, "bf16", 0), (2, 2, 64, 3, "bf16", 64), (2, 2, 64, 3, "fp16", 0), (2, 2, 64, 70, "fp32", 0), (3, 4, 128, 5, "bf16", 0), (3, 4, 128, 5, "bf16", 128),
         (1, 4, 128, 64, "bf16", 128), (1, 4, 128, 96, "bf16", 128), (1, 4, 128, 128, "bf16", 128), (2, 3, 128, 50, "fp16", 0), (2, 3, 128, 50, "fp32", 0), (2, 1, 256, 4, "bf16", 0),
         (2, 1, 256, 4, "bf16", 256), (2, 2, 256, 70, "fp16", 0), (2, 1, 256, 4, "fp32", 0)]


@pytest.mark.parametrize("heads,group,dim,batch,kind,rot", FORMS)
def test_a_call_that_gives_up(heads, group, dim, batch, kind, rot):
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim + batch)
    c = make(heads, dim, 16, (3, 7))
    length, lengths = 5001, [i % 20 for i in range(batch)]
    pages, prefix, n, table, ln = setting(c, length, lengths, gen)
    q = torch.randn((batch, heads * group, dim), generator=gen, device="cuda").to(TYPES[kind])
    want, got = torch.empty_like(q), torch.empty_like(q)
    lse, lse_got = torch.empty((batch, heads * group), device="cuda"), torch.empty((batch, heads * group), device="cuda")
    t = lq.lq_rotary_table(5100, rot) if rot else None

    def call(out, l):
        c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=l, rotary=t)

    call(want, lse)
    assert c.lq_cache_status() == 0
    if not rot:
        check(c, pages, prefix, length, table, lengths, q, want, lse, some=range(0, batch * heads * group, 17))
    for cycles in (0, 1, 300, 1000, 3000):
        for _ in range(3):
            c.lq_cache_wait(cycles)
            call(got, lse_got)
            flags = c.lq_cache_status()
            assert flags == lq.CACHE_GAVE_UP if cycles == 0 else flags in (0, lq.CACHE_GAVE_UP)
            if flags == 0:
                assert torch.equal(got, want) and torch.equal(lse_got, lse)
            c.lq_cache_wait()
            call(got, lse_got)
            assert c.lq_cache_status() == 0
            assert torch.equal(got, want) and torch.equal(lse_got, lse)


def test_limits():
    import paper_2505_14371_b200 as lq
    c = make(1, 64)
    with pytest.raises(lq.LqError, match="negative"):
        c.lq_cache_wait(-1)
    c.lq_cache_wait(1 << 62)                                    # (taken as the most)
    assert lq.load_library().lq_cache_wait(None, 5) == -1
