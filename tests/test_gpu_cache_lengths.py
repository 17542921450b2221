"""Lengths of the calls over a shared prefix that no table holds."""
import pytest
import torch

from test_gpu_cache import filled, make
from test_gpu_cache_shared import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width", [0, 2])
@pytest.mark.parametrize("prefix_width", [0, 3])
def test_lengths_that_no_table_holds(width, prefix_width):
    """Negative ones and ones past their tables are reported and taken as 0 or the table's, whether there is a table or not."""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(width)
    c = make(2, 64, 16, (3, 3))
    pages = filled(c, 9, gen)
    i32 = dict(dtype=torch.int32, device="cuda")
    prefix, table = torch.arange(prefix_width, **i32), torch.randint(0, 9, (3, width), generator=gen, device="cuda", dtype=torch.int32)
    q = torch.randn((3, 4, 64), generator=gen, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((3, 4), device="cuda")
    most = 16 * prefix_width
    for lengths, length, flags in (([0, 0, 0], most, 0), ([0, -1, 0], most, 1), ([0, 0, 16 * width + 1], most, 1), ([2 ** 31 - 1, 0, -2 ** 31], 0, 1), ([0, 0, 0], most + 1, 1),
                                   ([0, 0, 0], -1, 1), ([0, 0, 0], 0, 0)):
        n, ln = torch.tensor([length], **i32), torch.tensor(lengths, **i32)
        c.lq_cache_attend_shared(0, q, pages, prefix, n, table, ln, out, lse=lse)
        assert c.lq_cache_status() == (lq.CACHE_BAD_LENGTH if flags else 0), (lengths, length)
        check(c, pages, prefix, min(max(length, 0), most), table, [min(max(x, 0), 16 * width) for x in lengths], q, out, lse)
