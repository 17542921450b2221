"""Names that the cache's calls do not know are refused as everything else is, before any device is looked at."""
import pytest


def unopened():
    import paper_2505_14371_b200 as lq
    c = lq.Cache.__new__(lq.Cache)
    c._h = c._addr = None
    c.bits, c.head_dim = (3, 7), 64
    return c


@pytest.mark.parametrize("name", ["key", "", None, 0, ["keys"]])
def test_kinds(name):
    import paper_2505_14371_b200 as lq
    with pytest.raises(lq.LqError, match="kind .* is not one of keys, values"):
        unopened().lq_cache_set_levels(0, name, [0.0, 1.0])
    with pytest.raises(lq.LqError, match="kind .* is not one of keys, values"):
        unopened().lq_cache_get_levels(0, name)


@pytest.mark.parametrize("name", ["halves", "", None, True, ["half"]])
def test_layouts(name):
    import paper_2505_14371_b200 as lq
    with pytest.raises(lq.LqError, match="layout .* is not one of half, interleaved"):
        unopened().lq_cache_write(0, None, None, None, None, layout=name)
    with pytest.raises(lq.LqError, match="layout .* is not one of half, interleaved"):
        unopened().lq_cache_attend(0, None, None, None, None, None, layout=name)


def test_the_known_names_are_taken():
    import paper_2505_14371_b200 as lq
    for kind in ("keys", "values"):
        with pytest.raises(lq.LqError, match="NULL"):
            unopened().lq_cache_get_levels(0, kind)
    for layout in ("half", "interleaved"):
        with pytest.raises(lq.LqError, match="NULL"):
            unopened().lq_cache_write(0, None, None, None, None, layout=layout)
