"""What of the key-value cache needs no GPU: refusals before anything is allocated, tables of angles, the reference itself."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import cache_reference as R


@pytest.fixture(scope="module")
def lib():
    import paper_2505_14371_b200 as lq
    return lq.load_library()


@pytest.mark.parametrize("args,word", [((0, 1, 64, 16, 3, 3, 0), b"num_layers"), ((4097, 1, 64, 16, 3, 3, 0), b"num_layers"), ((1, 0, 64, 16, 3, 3, 0), b"kv_heads"), ((1, 1, 0, 16, 3, 3, 0), b"head_dim"),
                                       ((1, 1, 257, 16, 3, 3, 0), b"head_dim"), ((1, 1, 64, 8, 3, 3, 0), b"page_size"), ((1, 1, 64, 48, 3, 3, 0), b"page_size"),
                                       ((1, 1, 64, 2048, 3, 3, 0), b"page_size"), ((1, 1, 64, 16, 4, 3, 0), b"bits"), ((1, 1, 64, 16, 3, 8, 0), b"bits"),
                                       ((1, 1, 64, 16, 3, 3, 3), b"q must"), ((1, 1, 64, 16, 3, 3, -1), b"q must")])
def test_shapes_that_are_refused(lib, args, word):
    h = C.c_void_p(5)
    assert lib.lq_cache_create(C.byref(h), *args, 0) == -1 and word in lib.lq_last_error() and not h.value


def test_calls_without_a_cache(lib):
    assert lib.lq_cache_destroy(None) == 0
    assert lib.lq_cache_page_words(None) == -1 and lib.lq_cache_workspace(None, 1, 0) == -1
    assert lib.lq_cache_status(None, C.byref(C.c_uint32())) == -1
    assert lib.lq_cache_write(None, 0, None, None, 0, None, None, 0, -1, None, None) == -1
    assert lib.lq_cache_read(None, 0, None, 0, 0, None, None, None, None) == -1
    assert lib.lq_cache_attend(None, 0, None, 0, 1, None, 0, None, 0, None, 1.0, 0, None, None, None, None, 0, None) == -1


def test_angles():
    import paper_2505_14371_b200 as lq
    t = lq.lq_rotary_table(1000001, 6, device="cpu").double().numpy()
    for p, i in ((0, 0), (1, 1), (999999, 0), (1000000, 2)):
        a = p * 10000.0 ** (-2 * i / 6)
        assert abs(t[p, i] - math.cos(a)) <= 2.0 ** -24 and abs(t[p, 3 + i] - math.sin(a)) <= 2.0 ** -24
    long = lq.lq_rotary_table(64, 8, stretch=4.0, device="cpu")
    assert torch.equal(long[::4], lq.lq_rotary_table(16, 8, device="cpu"))
    # fast pairs keep their angles, slow ones are divided, amplitudes multiply
    parts = lq.lq_rotary_table(10, 64, stretch=8.0, trained=2000, amplitude=1.25, device="cpu").double() / 1.25
    plain, slow = lq.lq_rotary_table(10, 64, device="cpu").double(), lq.lq_rotary_table(10, 64, stretch=8.0, device="cpu").double()
    turns = [2000 * 10000.0 ** (-2 * i / 64) / (2 * math.pi) for i in range(32)]
    for i, n in enumerate(turns):
        want = plain if n >= 32 else slow if n <= 1 else None
        if want is not None:
            assert (parts[:, i] - want[:, i]).abs().max() <= 2.0 ** -23
        else:
            assert ((parts[1, i] < slow[1, i]) and (parts[1, i] > plain[1, i]))
    for bad in (dict(dim=5), dict(dim=0), dict(positions=0), dict(stretch=0.5), dict(base=0.0), dict(slow=4.0, fast=2.0)):
        with pytest.raises(lq.LqError):
            lq.lq_rotary_table(**{"positions": 4, "dim": 4, "device": "cpu", **bad})


def test_the_reference_keeps_what_it_should():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 3, 41)).astype(np.float32)
    lv = (np.arange(128) / 127.0) ** 1.3
    for q in (0, 1, 2):
        sym, n = R.quantise(x, lv, q, np.float32(0.5))
        back = R.values_of(sym, n, lv.astype(np.float32))
        u = np.abs(x) / n[..., None]
        gap = np.diff(lv)[np.minimum(np.searchsorted(lv, u, side="right") - 1, 126)]
        assert np.all(np.abs(back - x) <= (0.5 * gap + 1e-6) * n[..., None])
    k0 = R.philox_words(0, np.uint64(0), np.uint64(0), np.uint64(0), np.uint64(0))
    assert [int(w) for w in k0] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    o, l, b, _ = R.attend(rng.standard_normal(8), rng.standard_normal((5, 8)), rng.standard_normal((5, 8)), 0.3, 0, 0)
    assert o.shape == (8,) and np.isfinite(l) and (b >= 0).all()
