"""Sizes of the 8-bit paged cache whose arithmetic would not fit: refused on
the host (no GPU needed)."""
import ctypes

import pytest

from paper_2507_09252_amd import tppsd as tp
from test_cache_host import ARG, cfg


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
