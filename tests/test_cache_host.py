"""The 8-bit paged cache's entry points: what the host refuses, before
anything is enqueued (no GPU needed), and the reference's own rounding."""
import ctypes

import numpy as np
import pytest
import torch

from cache_reference import e4m3
from paper_2507_09252_amd import tppsd as tp

ARG, CONFIG, WORKSPACE, ORDER = 1, 2, 3, 4


def cfg(**kw):
    base = dict(n_layers=2, n_heads=4, n_kv_heads=2, d_head=32, prec=1, max_seqs=3, max_events=200, n_pages=0)
    return tp.CacheCfgC(*{**base, **kw}.values())


def make(lib, **kw):
    """A handle over an address that nothing is done with."""
    h, n = ctypes.c_void_p(), ctypes.c_size_t()
    c = cfg(**kw)
    assert lib.tppsd_cache_bytes(ctypes.byref(c), ctypes.byref(n)) == 0
    assert lib.tppsd_cache_create(ctypes.byref(c), ctypes.c_void_p(1 << 30), n.value, ctypes.byref(h)) == 0
    return h


@pytest.fixture(scope="module")
def lib():
    return tp.lib()


@pytest.mark.parametrize("bad,code", [
    (dict(n_layers=0), CONFIG), (dict(n_heads=3), CONFIG), (dict(n_kv_heads=0), CONFIG), (dict(n_heads=0), CONFIG),
    (dict(d_head=48), CONFIG), (dict(d_head=256), CONFIG), (dict(prec=2), CONFIG), (dict(n_layers=70000), CONFIG),
    (dict(max_seqs=0), ARG), (dict(max_events=0), ARG), (dict(n_pages=-1), ARG), (dict(max_seqs=1 << 21), ARG),
    (dict(max_events=1 << 30, max_seqs=1 << 20), ARG), (dict(n_pages=(1 << 26) + 1), ARG)],
    ids=lambda x: "-".join(f"{k}{v}" for k, v in x.items()) if isinstance(x, dict) else None)
def test_configurations_refused(lib, bad, code):
    n, h = ctypes.c_size_t(), ctypes.c_void_p()
    c = cfg(**bad)
    assert lib.tppsd_cache_bytes(ctypes.byref(c), ctypes.byref(n)) == code
    assert lib.tppsd_cache_create(ctypes.byref(c), ctypes.c_void_p(1 << 30), 1 << 50, ctypes.byref(h)) == code
    assert lib.tppsd_cache_entry(ctypes.byref(c), 0, None, None) == code
    assert len(lib.tppsd_last_error()) > 0


def test_workspace(lib):
    c, n, h = cfg(), ctypes.c_size_t(), ctypes.c_void_p()
    assert lib.tppsd_cache_bytes(None, ctypes.byref(n)) == ARG
    assert lib.tppsd_cache_bytes(ctypes.byref(c), None) == ARG
    assert lib.tppsd_cache_bytes(ctypes.byref(c), ctypes.byref(n)) == 0
    for ws, size, code in ((1 << 30, n.value - 1, WORKSPACE), ((1 << 30) + 8, n.value, WORKSPACE), (0, n.value, ARG),
                           (1 << 30, n.value, 0)):
        assert lib.tppsd_cache_create(ctypes.byref(c), ctypes.c_void_p(ws), size, ctypes.byref(h)) == code
    lib.tppsd_cache_destroy(h)
    lib.tppsd_cache_destroy(None)
    names, offs = [], []
    while True:
        name, off = ctypes.c_char_p(), ctypes.c_size_t()
        if lib.tppsd_cache_entry(ctypes.byref(c), len(names), ctypes.byref(name), ctypes.byref(off)):
            break
        names.append(name.value.decode())
        offs.append(off.value)
    assert names == ["pages", "scales", "tails", "table", "lens", "refs"]
    assert all(o % 256 == 0 for o in offs) and sorted(offs) == offs and offs[-1] < n.value
    # 2 layers x 3 sequences x 4 pages x 2 heads x 64 positions x 2 x 32 bytes
    assert offs[1] == 2 * 12 * 2 * 64 * 2 * 32


def test_calls_refused(lib):
    h, other, wide = make(lib), make(lib, max_events=1000), make(lib, d_head=64)
    p, q = ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 8)
    rows = tp.CacheRowsC(p, p, p, p, 128, 64, 64, 128)
    r = ctypes.byref(rows)
    # before a reset
    assert lib.tppsd_cache_begin(h, 1, 1, None, None, None) == ORDER
    assert lib.tppsd_cache_append(h, 0, r, None) == ORDER
    assert lib.tppsd_cache_attend(h, 0, r, 1.0, 0, None) == ORDER
    assert lib.tppsd_cache_commit(h, None, None) == ORDER
    assert lib.tppsd_cache_truncate(h, 1, p, None, None) == ORDER
    assert lib.tppsd_cache_fork(h, 1, p, p, None) == ORDER
    assert lib.tppsd_cache_copy(h, other, 1, p, p, None) == ORDER
    assert lib.tppsd_cache_read(h, 0, 1, p, None, 1, p, p, None) == ORDER
    assert lib.tppsd_cache_status(h, None, None) == ORDER
    for f in (lib.tppsd_cache_reset, ):
        assert f(None, None) == ARG
    assert lib.tppsd_cache_begin(None, 1, 1, None, None, None) == ARG
    assert lib.tppsd_cache_status(None, None, None) == ARG
    if torch.cuda.is_available():
        pytest.skip("the rest marks caches over made-up addresses as reset")
    for c in (h, other, wide):
        assert lib.tppsd_cache_reset(c, None) == 5          # no device; the handle's own state moves on
    # without a plan
    assert lib.tppsd_cache_append(h, 0, r, None) == ORDER
    assert lib.tppsd_cache_attend(h, 0, r, 1.0, 0, None) == ORDER
    assert lib.tppsd_cache_commit(h, None, None) == ORDER
    for B, n in ((0, 1), (4, 1), (1, 0), (1, 201), (-1, 5)):
        assert lib.tppsd_cache_begin(h, B, n, None, None, None) == ARG, (B, n)
    assert lib.tppsd_cache_begin(h, 2, 5, None, None, None) == 5
    # groups of query rows are a grid dimension: 8 positions of 8 heads a group of 64 rows
    many = make(lib, n_heads=16, max_events=1 << 20)
    assert lib.tppsd_cache_reset(many, None) == 5
    wide_rows = tp.CacheRowsC(p, p, p, p, 512, 64, 64, 512)
    for n, code in ((1 << 19, ARG), (1 << 18, 5)):
        assert lib.tppsd_cache_begin(many, 1, n, None, None, None) == 5
        assert lib.tppsd_cache_attend(many, 0, ctypes.byref(wide_rows), 1.0, 0, None) == code
    lib.tppsd_cache_destroy(many)
    for layer in (-1, 2):
        assert lib.tppsd_cache_append(h, layer, r, None) == ARG
        assert lib.tppsd_cache_attend(h, layer, r, 1.0, 0, None) == ARG
        assert lib.tppsd_cache_read(h, layer, 1, None, None, 1, p, p, None) == ARG
    assert lib.tppsd_cache_append(h, 0, None, None) == ARG
    for kw in (dict(k=None), dict(v=None), dict(k=q), dict(v=q), dict(ldk=63), dict(ldv=56), dict(ldk=68), dict(ldk=-64)):
        vals = {**dict(q=p, k=p, v=p, o=p, ldq=128, ldk=64, ldv=64, ldo=128), **kw}
        bad = tp.CacheRowsC(*vals.values())
        assert lib.tppsd_cache_append(h, 0, ctypes.byref(bad), None) == ARG, kw
        assert lib.tppsd_cache_attend(h, 0, ctypes.byref(bad), 1.0, 0, None) == ARG, kw
    for kw in (dict(q=None), dict(o=None), dict(q=q), dict(o=q), dict(ldq=120), dict(ldo=132)):
        vals = {**dict(q=p, k=p, v=p, o=p, ldq=128, ldk=64, ldv=64, ldo=128), **kw}
        bad = tp.CacheRowsC(*vals.values())
        assert lib.tppsd_cache_attend(h, 0, ctypes.byref(bad), 1.0, 0, None) == ARG, kw
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert lib.tppsd_cache_attend(h, 0, r, scale, 0, None) == ARG
    for n in (0, -1, (1 << 20) + 1):
        assert lib.tppsd_cache_truncate(h, n, p, None, None) == ARG
    for n in (0, 4, -1):
        assert lib.tppsd_cache_fork(h, n, p, p, None) == ARG
        assert lib.tppsd_cache_copy(h, other, n, p, p, None) == ARG
    assert lib.tppsd_cache_truncate(h, 1, None, None, None) == ARG
    assert lib.tppsd_cache_fork(h, 1, None, p, None) == ARG
    assert lib.tppsd_cache_fork(h, 1, p, None, None) == ARG
    assert lib.tppsd_cache_copy(h, h, 1, p, p, None) == ARG
    assert lib.tppsd_cache_copy(h, wide, 1, p, p, None) == CONFIG
    assert lib.tppsd_cache_read(h, 0, 0, None, None, 1, p, p, None) == ARG
    assert lib.tppsd_cache_read(h, 0, 4, None, None, 1, p, p, None) == ARG
    assert lib.tppsd_cache_read(h, 0, 1, None, None, 0, p, p, None) == ARG
    assert lib.tppsd_cache_read(h, 0, 1, None, None, 1, None, p, None) == ARG
    assert lib.tppsd_cache_read(h, 0, 1, None, None, 1, p, q, None) == ARG
    for c in (h, other, wide):
        lib.tppsd_cache_destroy(c)


def test_reference_rounding():
    """The reference's e4m3 is the type's: torch's conversion of the scaled block."""
    rng = np.random.default_rng(0)
    for f in (1.0, 1e-3, 300.0, 448.0, 1e20):
        x = (rng.standard_normal((64, 2, 16)) * f).astype(np.float32).astype(np.float64)
        x[3, 0, 2] = 0.0
        top = np.abs(x).max(axis=(0, 2))
        for h in range(2):
            e = int(np.ceil(np.log2(top[h] / 448.0)))
            t = torch.from_numpy(x[:, h] * 2.0 ** -e).float().to(torch.float8_e4m3fn).double().numpy() * 2.0 ** e
            assert np.array_equal(e4m3(x)[:, h], t)
