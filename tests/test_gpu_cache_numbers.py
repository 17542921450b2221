"""The cache's attention where numbers are large, small or many: scores past 1e30, norms of every size, weights of a long context."""
import numpy as np
import pytest
import torch

import cache_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def in_order(heads, dim, k, v, page=16, bits=(3, 3), q=0):
    """A cache whose slots 0, 1, ... hold k and v [tokens][heads][dim], its pages, and the table of the one sequence that they are."""
    import paper_2505_14371_b200 as lq
    c = lq.Cache(1, heads, dim, page, bits, q, 7)
    num = -(-k.shape[0] // page)
    pages = c.empty_pages(num)
    c.lq_cache_write(0, k, v, torch.arange(k.shape[0], device="cuda"), pages)
    assert c.lq_cache_status() == 0
    return c, pages, torch.arange(num, dtype=torch.int32, device="cuda").view(1, num)


def kept(c, pages, tokens):
    """What the cache holds of its first tokens, in 64 bits: keys and values [heads][tokens][dim]."""
    sec = R.head_sections(pages.cpu().numpy().view(np.uint32), c.kv_heads, c.head_dim, c.page_size, c.bits)
    got = [R.values_of(sec[i], sec[2 + i], c.lq_cache_get_levels(0, n))[..., : c.head_dim] for i, n in ((0, "keys"), (1, "values"))]
    return [np.moveaxis(x, 0, 1).reshape(c.kv_heads, -1, c.head_dim)[:, :tokens] for x in got]


def attended(c, pages, table, q, tokens, **more):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    c.lq_cache_attend(0, q, pages, table, torch.tensor([tokens], dtype=torch.int32, device="cuda"), out, lse=lse, **more)
    assert c.lq_cache_status() == 0
    return out, lse


@pytest.mark.parametrize("norm", [1e-30, 1e-12, 1e-6, 1.0, 1e6, 1e12, 1e30])
@pytest.mark.parametrize("group,dim,bits", [(2, 64, (3, 3)), (6, 128, (3, 7)), (3, 200, (7, 3)), (8, 41, (7, 7))])
def test_weights_are_as_exact_for_values_of_any_size(norm, group, dim, bits):
    """fp32, small scores, all values' norms of one size, nothing that cancels: a factor that all weights share would show."""
    gen = torch.Generator("cuda").manual_seed(dim)
    tokens = 100
    k = torch.randn((tokens, 2, dim), generator=gen, device="cuda")
    v = (torch.rand((tokens, 2, dim), generator=gen, device="cuda") + 0.1) * (torch.rand((tokens, 2, 1), generator=gen, device="cuda") + 1) * norm
    c, pages, table = in_order(2, dim, k, v, bits=bits)
    q = torch.randn((1, 2 * group, dim), generator=gen, device="cuda")
    out, lse = attended(c, pages, table, q, tokens, scale=1e-4)
    keys, values = kept(c, pages, tokens)
    for h in range(2 * group):
        s = 1e-4 * (keys[h // group] @ q[0, h].double().cpu().numpy())
        assert np.abs(s).max() < 0.01
        p = np.exp(s - s.max())
        want = p @ values[h // group] / p.sum()
        # in units of 2^-24: exp2 of a weight and of p 4 each, significand 1, a weight as two numbers 2, a sum of 100 tokens in products of 16
        # (truncated: 2 each, 2 of them a warp) and 8 warps 4 + 8 in both, the quotient 2; scores below 0.01 have errors below 1 together
        assert np.all(np.abs(out[0, h].double().cpu().numpy() - want) <= 36 * 2.0 ** -24 * want)
        assert abs(float(lse[0, h]) - (s.max() + np.log(p.sum()))) <= 36 * 2.0 ** -24 + 2.0 ** -23 * np.log(tokens)


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("group,dim,bits", [(4, 128, (3, 3)), (6, 64, (7, 3)), (16, 256, (3, 7))])
@pytest.mark.parametrize("size", [30.0, 1e3, 1e5, 1e7])
def test_large_scores_leave_the_values_norms_alone(kind, group, dim, bits, size):
    """All tokens have the same key, so the same score, however large: the output is the mean of values of many sizes."""
    gen = torch.Generator("cuda").manual_seed(dim)
    tokens = 333
    k = torch.randn((1, 1, dim), generator=gen, device="cuda").expand(tokens, 1, dim)
    v = (torch.rand((tokens, 1, dim), generator=gen, device="cuda") + 0.1) * torch.randn((tokens, 1, 1), generator=gen, device="cuda").exp_()
    c, pages, table = in_order(1, dim, k, v, bits=bits)
    q = torch.randn((1, group, dim), generator=gen, device="cuda").to(TYPES[kind])
    keys, values = kept(c, pages, tokens)
    # every query's score about `size`, with either sign
    raw = q[0].double().cpu().numpy() @ keys[0, 0]
    want = values[0].mean(0)
    for sign in (1, -1):
        scale = sign * size / float(np.abs(raw).max())
        out, lse = attended(c, pages, table, q, tokens, scale=scale)
        got = out[0].double().cpu().numpy()
        # weights: a logarithm and an exponential of 2^-21 each, then 11 bits (two of them for fp32); sums of 333 tokens; the output's rounding
        half = torch.finfo(TYPES[kind]).eps / 2
        assert np.all(np.abs(got - want) <= (2.0 ** -18 + (0 if kind == "fp32" else 2.0 ** -11 + half)) * want)
        s = scale * raw
        assert np.all(np.abs(lse[0].double().cpu().numpy() - (s + np.log(tokens))) <= 2.0 ** -18 * (np.abs(s) + abs(scale) * np.abs(q[0].double().cpu().numpy()) @ np.abs(keys[0, 0]) + 6))


def test_a_score_of_nothing_times_a_large_norm():
    """Queries of 2^100 and keys' norms of 2^50 whose products are all with the level 0: scores are 0, not 0 times infinity."""
    k = torch.zeros((50, 1, 64), device="cuda")
    k[..., 1:] = 2.0 ** 50
    v = torch.rand((50, 1, 64), generator=torch.Generator("cuda").manual_seed(3), device="cuda") + 0.1
    c, pages, table = in_order(1, 64, k, v)
    q = torch.zeros((1, 3, 64), device="cuda")
    q[..., 0] = 2.0 ** 100
    out, lse = attended(c, pages, table, q, 50)
    want = kept(c, pages, 50)[1][0].mean(0)
    assert np.all(np.abs(out[0].double().cpu().numpy() - want) <= 2.0 ** -18 * want)
    assert np.all(np.abs(lse.double().cpu().numpy() - np.log(50)) <= 2.0 ** -20)


@pytest.mark.parametrize("tokens", [5, 40, 3000])
@pytest.mark.parametrize("sign", [-1, 1])
def test_scores_of_any_finite_size(tokens, sign):
    """Scores of 1e35 times 1, 2, 3, ...: the softmax is one at the largest, also where all are below -1e30."""
    dim = 64
    u = torch.zeros((tokens, 1, dim), device="cuda")
    size = torch.arange(1, tokens + 1, device="cuda", dtype=torch.float32).view(-1, 1, 1)
    order = torch.randperm(tokens, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    u[..., 0] = 1e15
    v = torch.randn((tokens, 1, dim), generator=torch.Generator("cuda").manual_seed(tokens), device="cuda")
    c, pages, table = in_order(1, dim, (u * size)[order], v)
    q = torch.zeros((1, 2, dim), device="cuda")
    q[..., 0] = sign * 1e20 / tokens
    out, lse = attended(c, pages, table, q, tokens, scale=1.0)
    keys, values = kept(c, pages, tokens)
    scores = keys[0] @ q[0, 0].double().cpu().numpy()
    top = scores.argmax()
    assert np.abs(scores).max() < 3e38 and abs(np.sort(scores)[-1]) > 1e30
    # the one weight is 1, as a sum of two numbers of 11 bits exactly; the sum of weights is 1
    assert np.all(np.abs(out[0].double().cpu().numpy() - values[0, top]) <= 2.0 ** -20 * np.abs(values[0, top]))
    assert np.all(np.abs(lse.double().cpu().numpy() - scores[top]) <= 2.0 ** -20 * abs(scores[top]))


@pytest.mark.parametrize("group,dim,bits,rot", [(1, 128, (3, 3), 0), (4, 64, (3, 7), 0), (4, 128, (3, 3), 128), (3, 256, (7, 7), 0), (6, 128, (7, 7), 0), (8, 128, (3, 3), 0),
                                                (8, 64, (7, 3), 64), (16, 256, (3, 7), 0), (7, 200, (3, 3), 100), (5, 41, (7, 7), 0)])
def test_fp16_outputs_are_off_by_their_own_rounding_alone(group, dim, bits, rot):
    """Over many short sequences, the error against 64 bits is that of rounding the exact output to fp16.  (Weights of 11 bits add a fifth
    and more.)"""
    import paper_2505_14371_b200 as lq
    gen = torch.Generator("cuda").manual_seed(dim + group)
    heads, batch, tokens = 2, 300, 5
    k, v = (torch.randn((16 * batch, heads, dim), generator=gen, device="cuda") for _ in range(2))
    c, pages, _ = in_order(heads, dim, k, v * torch.randn((16 * batch, heads, 1), generator=gen, device="cuda").exp_(), bits=bits)
    table = torch.arange(batch, dtype=torch.int32, device="cuda").view(batch, 1)
    q = torch.randn((batch, heads * group, dim), generator=gen, device="cuda").half()
    out = torch.empty_like(q)
    angles = lq.lq_rotary_table(tokens, rot) if rot else None
    scale = 0.2 / dim
    c.lq_cache_attend(0, q, pages, table, torch.full((batch,), tokens, dtype=torch.int32, device="cuda"), out, scale=scale, rotary=angles)
    keys, values = (x.reshape(heads, batch, 16, dim)[:, :, :tokens] for x in kept(c, pages, 16 * batch))
    x = q.float().cpu().numpy()
    if rot:
        x = R.rotate(x, np.repeat(angles[tokens - 1:].cpu().numpy(), batch, 0), False)
    x = x.astype(np.float64).reshape(batch, heads, group, dim)
    s = scale * np.einsum("bhgd,hbtd->bhgt", x, keys)
    assert (scale * np.einsum("bhgd,hbtd->bhgt", np.abs(x), np.abs(keys))).max() < 0.5
    p = np.exp(s)
    p /= p.sum(-1, keepdims=True)
    want = np.einsum("bhgt,hbtd->bhgd", p, values).reshape(out.shape)
    own = np.linalg.norm(torch.from_numpy(want).half().double().numpy() - want)
    # before the rounding, in units of 2^-24 of sum p |v|: exp2 twice 8, the norm's logarithm (below 8 in size) 22 and its sum 1, two numbers 2,
    # one product of 16 tokens 2, the quotient 2, scores whose terms add up to 0.5 at most: 18 * 2 * 0.5 twice.  A rounding that
    # tips over because of it is off by twice as much more.
    before = 73 * 2.0 ** -24 * np.linalg.norm(np.einsum("bhgt,hbtd->bhgd", p, np.abs(values)))
    assert before < 0.06 * own
    assert np.linalg.norm(out.double().cpu().numpy() - want) <= own + 2 * before


def test_scales_at_the_end_of_fp32():
    """2^126 is a scale; above 2^127 the factor of base 2 would be infinite, and a score of 0 no number."""
    import paper_2505_14371_b200 as lq
    k = torch.zeros((20, 1, 64), device="cuda")
    k[..., 1:] = 1.0
    v = torch.rand((20, 1, 64), generator=torch.Generator("cuda").manual_seed(3), device="cuda") + 0.1
    c, pages, table = in_order(1, 64, k, v)
    q = torch.zeros((1, 3, 64), device="cuda")
    q[..., 0] = 1.0
    want = kept(c, pages, 20)[1][0].mean(0)
    for scale in (2.0 ** 126, -(2.0 ** 126)):
        out, _ = attended(c, pages, table, q, 20, scale=scale)
        assert np.all(np.abs(out[0].double().cpu().numpy() - want) <= 2.0 ** -18 * want)
    for scale in (3e38, -3e38, float("inf"), 1e300):
        with pytest.raises(lq.LqError, match="scale"):
            attended(c, pages, table, q, 20, scale=scale)


@pytest.mark.parametrize("group,dim", [(4, 64), (8, 128), (2, 256)])
def test_small_weights_keep_their_bits_down_to_the_bound(group, dim):
    """Two tokens whose values share no coordinate, fp16: what the second adds is off by 2^-31 of the first's weight beside the output's own
    rounding, wherever the first's norm lies between two powers of two."""
    batch = 64
    k, v = torch.zeros((16 * batch, 1, dim), device="cuda"), torch.zeros((16 * batch, 1, dim), device="cuda")
    norm = 2.0 ** torch.linspace(14.0, 15.5, batch, device="cuda")
    k[::16, 0, 0] = 1.0
    v[::16, 0, 0] = norm
    v[1::16, 0, 1] = norm
    c, pages, _ = in_order(1, dim, k, v)
    table = torch.arange(batch, dtype=torch.int32, device="cuda").view(batch, 1)
    q = torch.zeros((batch, group, dim), device="cuda")
    q[..., 0] = torch.linspace(8, 20, batch * group, device="cuda")[torch.randperm(batch * group, generator=torch.Generator("cuda").manual_seed(5), device="cuda")].view(batch, group)
    q = q.half()
    out = torch.empty_like(q)
    c.lq_cache_attend(0, q, pages, table, torch.full((batch,), 2, dtype=torch.int32, device="cuda"), out, scale=1.0)
    p = np.exp(-q[..., 0].double().cpu().numpy())
    values = kept(c, pages, 16 * batch)[1][0].reshape(batch, 16, dim)
    big, small = values[:, 0, 0][:, None], values[:, 1, 1][:, None]
    got = out.double().cpu().numpy()
    # a weight's exponent: a score below 20 as one product (2^-20), exp2 and log2 below 16 in size (2^-18)
    for at, want in ((0, big / (1 + p)), (1, small * p / (1 + p))):
        assert np.all(np.abs(got[..., at] - want) <= want * (2.0 ** -11 + 2.0 ** -17) + 2.0 ** -31 * big + 2.0 ** -25)
    assert not got[..., 2:].any()
