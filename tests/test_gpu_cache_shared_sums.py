"""Sums of the attention over a shared prefix where many small terms make them up, against 64 bits: denominators whose terms have small values or
none, and weights that a type's own rounding does not hide."""
import numpy as np
import pytest
import torch

import cache_reference as R
from test_gpu_cache import TYPES, make

pytestmark = pytest.mark.gpu


def plain_rows(c, size_k, size_v):
    """A layer's pages whose rows are size_k and size_v [tokens] times ones, the same for every head: levels of 1, so that they are those numbers."""
    tokens = len(size_k)
    pages = c.empty_pages(-(-tokens // c.page_size))
    k, v = (torch.tensor(x, dtype=torch.float32, device="cuda")[:, None].expand(-1, c.head_dim).contiguous()[:, None].expand(-1, c.kv_heads, -1) for x in (size_k, size_v))
    c.lq_cache_write(0, k, v, torch.arange(tokens, device="cuda"), pages)
    return pages


@pytest.mark.parametrize("kind,batch", [("bf16", 1), ("fp16", 1), ("fp32", 1), ("bf16", 65), ("fp16", 65)])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -110, 2.0 ** -60, 2.0 ** -50, 2.0 ** -39, 2.0 ** -30])
@pytest.mark.parametrize("first", [True, False])
def test_small_values_count_in_the_denominator(kind, batch, small, first):
    """Two valued tokens and 65534 with small values or none, 26 powers of two below them: 0.0005 of the denominator, in tiles that hold nothing
    else.  148 heads: a CTA has all tiles (fp32: sixteen of them)."""
    c = make(148, 64, 1024)
    tokens, scale = 65536, 2.0 ** -6
    # a score is scale * 64 * (a query's coordinate, 1) * (a key's): the key's coordinate, in powers of two 26.05 apart
    low = -13.05 * np.log(2)
    k, v = np.full(tokens, np.float32(low), np.float64), np.full(tokens, small)
    at = [0, 64] if first else [tokens - 1, tokens - 65]
    k[at], v[at] = np.float32(13 * np.log(2)), 0.75
    pages = plain_rows(c, k, v)
    i32 = dict(dtype=torch.int32, device="cuda")
    prefix, n = torch.arange(pages.shape[0], **i32), torch.tensor([tokens], **i32)
    q = torch.ones((batch, 148 * (2 if batch > 1 else 1), 64), device="cuda", dtype=TYPES[kind])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    c.lq_cache_attend_shared(0, q, pages, prefix, n, torch.zeros((batch, 0), **i32), torch.zeros(batch, **i32), out, lse=lse, scale=scale)
    assert c.lq_cache_status() == 0
    o, l, bound, lse_bound = R.attend(np.ones(64), np.repeat(k[:, None], 64, 1), np.repeat(v[:, None], 64, 1), scale, 0.0, 2.0 ** -11 if kind == "bf16" else 2.0 ** -20)
    assert lse_bound < 1e-4                                     # (what is left out would show)
    half = torch.finfo(out.dtype).eps / 2
    assert (lse.double().cpu() - l).abs().max() <= lse_bound, (float(lse[0, 0]) - l, lse_bound)
    assert np.all(np.abs(out.double().cpu().numpy() - o) <= bound + half * (np.abs(o) + bound))


@pytest.mark.parametrize("kind,tokens,heads", [("fp16", 524288, 148), ("bf16", 1048576, 148), ("fp32", 65536, 148), ("fp16", 100003, 150), ("fp16", 40000, 3)])
def test_sums_of_many_tokens(kind, tokens, heads):
    """Values of one sign, so that a sum grows all the way and what the matrix unit cuts off each of its steps adds up; so many heads that each has a CTA to
    itself.  A split ends a sum where that would come to a quarter of half a step of the outputs at worst: 2^-14, 2^-11 and (fp32, by 1024 tokens) 2^-17 of it."""
    c = make(heads, 64, 1024)
    rng = np.random.default_rng(tokens)
    k, v = rng.uniform(-1, 1, tokens).astype(np.float32), rng.uniform(0.5, 1, tokens).astype(np.float32)
    pages = plain_rows(c, k, v)
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.ones((1, heads, 64), device="cuda", dtype=TYPES[kind])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    c.lq_cache_attend_shared(0, q, pages, torch.arange(pages.shape[0], **i32), torch.tensor([tokens], **i32), torch.zeros((1, 0), **i32), torch.zeros(1, **i32), out,
                             lse=lse, scale=2.0 ** -6)
    p = np.exp(k.astype(np.float64))
    o, l = (p @ v) / p.sum(), np.log(p.sum())
    # scores of up to 1 and their exponentials: 2^-20 together; weights of 11 or 22 bits; sums of parts in fp32
    cut = {"fp16": 2.0 ** -14, "bf16": 2.0 ** -11, "fp32": 2.0 ** -17}[kind]
    bound = o * (2.0 ** -20 + (2.0 ** -12 if kind == "bf16" else 2.0 ** -21) + cut + 2.0 ** -19)
    step = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "fp32": 2.0 ** -24}[kind]        # of a number from 1/2 to 1
    assert 0.5 < o < 1 and (out.double().cpu() - o).abs().max() <= bound + step / 2, (float(out[0, 0, 0]), o)
    assert (lse.double().cpu() - l).abs().max() <= 2.0 ** -19 + 2.0 ** -22 * l
