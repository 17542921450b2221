"""The cache's calls over parts of the tokens: what is refused before any device is looked at."""
import pytest

from test_cache_names import unopened


def test_calls_without_a_cache():
    import paper_2505_14371_b200 as lq
    lib = lq.load_library()
    assert lib.lq_cache_bounds_words(None) == -1 and lib.lq_cache_choose_workspace(None, 1, 1) == -1
    assert lib.lq_cache_shared_workspace(None, 1, 1, 1, 1, 0, 0) == -1
    assert lib.lq_cache_bounds(None, 0, None, 0, None, 0, None, None) == -1
    assert lib.lq_cache_choose(None, None, 0, 1, None, 0, None, 0, None, 0, 1, None, None, 1, None, None, 0, None) == -1
    assert lib.lq_cache_attend_chosen(None, 0, None, 0, 1, None, 0, None, 0, None, 1.0, None, None, None, None, 0, None) == -1
    assert lib.lq_cache_attend_shared(None, 0, None, 0, 1, None, 0, None, 0, None, None, 0, None, 1.0, None, None, None, None, 0, None) == -1
    assert b"cache is NULL" in lib.lq_last_error()


@pytest.mark.parametrize("name", ["halves", "", None, True, ["half"]])
def test_layouts(name):
    import paper_2505_14371_b200 as lq
    lq.load_library()
    for call in (lambda c: c.lq_cache_attend_shared(0, *[None] * 7, layout=name), lambda c: c.lq_cache_choose(*[None] * 6, layout=name),
                 lambda c: c.lq_cache_attend_chosen(0, *[None] * 5, layout=name)):
        with pytest.raises(lq.LqError, match="layout .* is not one of half, interleaved"):
            call(unopened())


def test_the_references_agree_on_a_bound():
    """A page's score is at least the product of the query, as it was rounded, with any of its keys."""
    import numpy as np

    import cache_choice_reference as S
    import cache_reference as R
    rng = np.random.default_rng(0)
    page, dim = 16, 40
    lv = np.array([(j / 7) ** 1.3 for j in range(8)], np.float16).astype(np.float32)
    k = rng.standard_normal((6 * page, 1, dim)).astype(np.float32)
    sym, n = R.quantise(k, lv, 0, np.float32(0.5))
    values = R.values_of(sym, n, lv).reshape(6, page, dim)
    p = R.padded(dim)
    words = np.zeros((6, 1, page, p // 8), np.uint32)
    full = np.zeros((6, 1, page, p), np.uint32)
    full[..., :dim] = sym.reshape(6, 1, page, dim)
    for i in range(8):
        words |= full[..., i::8] << np.uint32(4 * i)
    norms = n.reshape(6, 1, page).view(np.uint32)
    pages = np.concatenate([words.reshape(6, -1), np.zeros((6, page * p // 8), np.uint32), norms.reshape(6, -1), np.zeros((6, page), np.uint32)], axis=1)
    up, low, scale = S.bounds(pages, 1, dim, page, (3, 3), lv)
    assert not up[..., dim:].any() and not low[..., dim:].any()
    q = rng.standard_normal((3, dim)).astype(np.float32)
    i, per = S.whole(q)
    assert np.abs(i * per[:, None] - q).max() <= 0.5001 * per.max()
    s = S.scores(i, per, up[:, 0, :dim], low[:, 0, :dim], scale[:, 0])
    dots = np.einsum("gd,ptd->gpt", i * per[:, None].astype(np.float64), values).max((0, 2))
    # max(i u, i l) is between i v and 127 |i|; scales and the reciprocal are off by 2^-24 each, of what a sum's terms are together
    most = (np.abs(i) * per[:, None].astype(np.float64)).sum(1).max() * n.reshape(6, page).max(1)
    assert np.all(s >= dots - 8 * 2.0 ** -24 * most) and np.all(s <= most * (1 + 8 * 2.0 ** -24))
    assert S.choose(s, 6, 1, 1, 3) == [0, 1 + int(np.argmax(s[1:5])), 5] and S.choose(s, 6, 1, 1, 6) == list(range(6))
