"""Sizes of the 8-bit paged cache whose arithmetic would not fit: refused on
the host (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2507_09252_amd import tppsd as tp
from test_cache_host import ARG, cfg, make


@pytest.fixture(scope="module")
def lib():
    return tp.lib()


def refused(lib, **kw):
    c, n, h = cfg(**kw), ctypes.c_size_t(), ctypes.c_void_p()
    codes = (lib.tppsd_cache_bytes(ctypes.byref(c), ctypes.byref(n)),
             lib.tppsd_cache_entry(ctypes.byref(c), 0, None, None),
             lib.tppsd_cache_create(ctypes.byref(c), ctypes.c_void_p(1 << 30), (1 << 64) - 1, ctypes.byref(h)))
    if not codes[2]:
        lib.tppsd_cache_destroy(h)
    return codes == (ARG,) * 3


# A plan sums pages over its rows in 32 bits: at most max_seqs ceil(max_events /
# 64) of them, whatever the pool holds (a call of 4 million positions asks for
# 65000 a row, 33000 rows for more than 2^31).
@pytest.mark.parametrize("seqs,events,fits", [(33000, 65001 * 64, False), (1 << 20, 1 << 30, False),
                                              (1 << 10, (1 << 20) * 64 + 1, False), (1 << 10, (1 << 20) * 64, True),
                                              (1 << 20, (1 << 10) * 64, True)])
def test_tables_that_a_plan_cannot_sum(lib, seqs, events, fits):
    assert refused(lib, max_seqs=seqs, max_events=min(events, 1 << 30), n_pages=100) is not fits


# bytes that pass 64 bits, or come near: 2 x 64 d_head a page, layer and head
@pytest.mark.parametrize("kw", [dict(n_layers=65534, n_heads=65535, n_kv_heads=65535, d_head=128, n_pages=1 << 26),
                                dict(n_layers=32768, n_heads=32768, n_kv_heads=32768, d_head=128, n_pages=1 << 20),
                                dict(n_layers=32768, n_heads=32768, n_kv_heads=32768, d_head=128, n_pages=1,
                                     max_seqs=1 << 20, max_events=64)],
                         ids=["pages", "pages-wrap", "tails"])
def test_workspaces_past_64_bits(lib, kw):
    assert refused(lib, **kw)


def test_states_of_split_rows_fit(lib):
    """The partial states of split rows are sized without passing 64 bits: 2^15
    heads and 2^25 groups of query rows are 2^40 states a page."""
    base = dict(n_layers=1, n_heads=32768, n_kv_heads=32768, d_head=16, prec=1, n_pages=1)
    n = [ctypes.c_size_t(), ctypes.c_size_t()]
    for x, events in zip(n, (1 << 20, 1 << 30)):
        assert lib.tppsd_cache_bytes(ctypes.byref(cfg(**base, max_seqs=8, max_events=events)), ctypes.byref(x)) == 0
    assert n[1].value >= n[0].value                      # a longer table, the same states


def test_scale_whose_base_two_form_overflows(lib):
    """Scores are taken to base 2: scale log2 e has to be a number too."""
    h = make(lib)
    if torch.cuda.is_available():
        pytest.skip("marks a cache over a made-up address as reset")
    p = ctypes.c_void_p(1 << 20)
    rows = tp.CacheRowsC(p, p, p, p, 128, 64, 64, 128)
    assert lib.tppsd_cache_reset(h, None) == 5
    assert lib.tppsd_cache_begin(h, 1, 1, None, None, None) == 5
    for scale, code in ((3e38, ARG), (2e38, 5)):
        assert lib.tppsd_cache_attend(h, 0, ctypes.byref(rows), scale, 0, None) == code
    lib.tppsd_cache_destroy(h)
