"""Host side of the paged 4-bit cache: sizes, refusals (nothing is launched, so no GPU is needed) and the plain form's own pins."""
import ctypes
import math

import numpy as np
import pytest
import torch

from cache_plain import SCALES, PlainCache, bf16, decode, encode
from paper_2601_15305_b200 import binding as gsa, build

GEO = dict(B=2, n_pages=10, page_tokens=16, max_pages=5, n_kv=2, d_h=64, dI=32)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return gsa.lib()


def test_struct_layout_matches_header():
    assert ctypes.sizeof(gsa.gsa_cache_t) == 4 * 8 + 7 * 4 + 4


@pytest.mark.parametrize("n_kv,d_h,dI,T", [(8, 128, 64, 64), (1, 64, 32, 16), (2, 64, 64, 128), (1, 128, 32, 32)])
def test_sizes(lib, n_kv, d_h, dI, T):
    c = gsa.cache_geometry(B=3, n_pages=7, page_tokens=T, max_pages=4, n_kv=n_kv, d_h=d_h, dI=dI)
    assert gsa.gsa_cache_page_bytes(c) == PlainCache(3, 7, T, 4, n_kv, d_h, dI).page_bytes
    assert gsa.gsa_cache_workspace_bytes(c) >= 256 + 12 * 7


@pytest.mark.parametrize("over,rc", [(dict(B=0), -1), (dict(n_pages=0), -1), (dict(max_pages=0), -1), (dict(B=4097), -2),
                                     (dict(n_pages=(1 << 20) + 1), -2), (dict(page_tokens=48), -2), (dict(page_tokens=256), -2),
                                     (dict(n_kv=3), -2), (dict(n_kv=16), -2), (dict(d_h=96), -2), (dict(dI=16), -2),
                                     (dict(max_pages=1 << 20), -2), (dict(n_kv=8, d_h=128, dI=64, page_tokens=64, n_pages=1 << 20), -2)])
def test_geometries_that_are_refused(lib, over, rc):
    c = gsa.cache_geometry(**{**GEO, **over})
    n = ctypes.c_size_t(0)
    assert lib.gsa_cache_page_bytes(ctypes.byref(c), ctypes.byref(n)) == rc
    assert lib.gsa_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(n)) == rc


def _call(lib, name, c, *args):
    return getattr(lib, name)(ctypes.byref(c) if c is not None else None, *args)


def test_arguments_that_are_refused(lib):
    """Host memory stands in for device memory: every call below is refused before anything is enqueued."""
    n0 = gsa.gsa_launch_count()
    mem = torch.zeros(1 << 16, dtype=torch.uint8)
    base = (mem.data_ptr() + 255) // 256 * 256
    P = lambda off=0: ctypes.c_void_p(base + off)  # noqa: E731
    c = gsa.cache_geometry(**GEO)
    c.pool, c.table, c.lens, c.refs = P(), P(), P(), P()
    big, small, L = ctypes.c_size_t(1 << 40), ctypes.c_size_t(255), ctypes.c_int32
    p = gsa.make_params(B=2, Lq=1, Lk=80, n_h=4, n_kv=2, d_h=64, HI=2, dI=32, k_base=8, k_min=1, k_max=16)
    pp, N, st = ctypes.byref(p), ctypes.c_void_p(0), ctypes.c_void_p(0)
    good = {
        "gsa_cache_reserve": [P(), P(64)], "gsa_cache_append": [L(4), P(), P(), P(), P(), P(), P(64)], "gsa_cache_read": [L(4), P(), P(), P()],
        "gsa_cache_fork": [P(), L(1)], "gsa_cache_release": [P()], "gsa_cache_compact": [P()],
        "gsa_cache_indexer_scores": [pp, P(), P(), P(), P(), ctypes.c_int64(80)],
        "gsa_cache_topk": [pp, P(), ctypes.c_int64(80), P(), P(), P()], "gsa_cache_attn_fwd": [pp, P(), P(), P(), P(), P()],
    }
    for name, args in good.items():
        assert _call(lib, name, c, *args, N, big, st) == -3, name                    # no workspace
        assert _call(lib, name, c, *args, P(), small, st) == -3, name                # too small
        assert _call(lib, name, c, *args, P(8), big, st) == -3, name                 # not aligned
        assert _call(lib, name, None, *args, P(), big, st) == -1, name
        for field in ("pool", "table", "lens", "refs"):
            d = gsa.cache_geometry(**GEO)
            d.pool, d.table, d.lens, d.refs = c.pool, c.table, c.lens, c.refs
            setattr(d, field, None)
            assert _call(lib, name, d, *args, P(), small, st) == -1, (name, field)
        d = gsa.cache_geometry(**GEO)
        d.pool, d.table, d.lens, d.refs = P(16), c.table, c.lens, c.refs
        assert _call(lib, name, d, *args, P(), small, st) == -1, name                # the pool is read 32 bytes at a time

    def refused(name, at, value, rc=-1):
        args = list(good[name])
        args[at] = value
        assert _call(lib, name, c, *args, P(), big, st) == rc, (name, at)

    for name, at in (("gsa_cache_reserve", 0), ("gsa_cache_reserve", 1), ("gsa_cache_append", 1), ("gsa_cache_append", 2), ("gsa_cache_append", 4),
                     ("gsa_cache_append", 5), ("gsa_cache_append", 6), ("gsa_cache_fork", 0), ("gsa_cache_release", 0), ("gsa_cache_compact", 0),
                     ("gsa_cache_indexer_scores", 1), ("gsa_cache_indexer_scores", 2), ("gsa_cache_indexer_scores", 4), ("gsa_cache_topk", 1),
                     ("gsa_cache_topk", 3), ("gsa_cache_topk", 4), ("gsa_cache_attn_fwd", 1), ("gsa_cache_attn_fwd", 2), ("gsa_cache_attn_fwd", 3),
                     ("gsa_cache_attn_fwd", 4), ("gsa_cache_attn_fwd", 5)):
        refused(name, at, N)
    refused("gsa_cache_reserve", 1, P())                                             # start and n_new are the same array
    for v in (0, -1, 81):
        refused("gsa_cache_append", 0, L(v))
        refused("gsa_cache_read", 0, L(v))
    for at in (1, 2, 3):
        refused("gsa_cache_append", at, P(16))
    refused("gsa_cache_append", 4, P(8))
    refused("gsa_cache_read", 1, P(16))
    assert _call(lib, "gsa_cache_read", c, L(4), N, N, N, P(), big, st) == -1
    for stride in (79, 81, 82):
        refused("gsa_cache_indexer_scores", 5, ctypes.c_int64(stride))
        refused("gsa_cache_topk", 2, ctypes.c_int64(stride))
    for over in (dict(B=3), dict(n_kv=1), dict(d_h=128), dict(dI=64), dict(Lk=81)):
        q = gsa.make_params(**{**dict(B=2, Lq=1, Lk=80, n_h=4, n_kv=2, d_h=64, HI=2, dI=32, k_base=8, k_min=1, k_max=16), **over})
        for name in ("gsa_cache_indexer_scores", "gsa_cache_topk", "gsa_cache_attn_fwd"):
            refused(name, 0, ctypes.byref(q))
    assert gsa.gsa_launch_count() == n0
    assert lib.gsa_status_string(-8).decode().startswith("the cache")


def test_calls_through_the_extension(lib):
    """The same function by ctypes and by the extension; what it does not take."""
    address = gsa._address("gsa_cache_page_bytes")
    c, n, m = gsa.cache_geometry(**GEO), ctypes.c_size_t(0), ctypes.c_size_t(0)
    assert lib.gsa_cache_page_bytes(ctypes.byref(c), ctypes.byref(n)) == 0
    assert gsa._call(address, ctypes.addressof(c), ctypes.addressof(m)) == 0 and m.value == n.value > 0
    assert gsa._call(address, ctypes.addressof(c), None) == -1 and gsa._call(address, None, None) == -1
    # negative integers, and every argument in its place: reserve .. attn take up to ten
    big, st = 1 << 40, 0
    assert gsa._call(gsa._address("gsa_cache_append"), ctypes.addressof(c), -1, 0, 0, 0, 0, 0, 0, 0, big, st) == -1
    for bad in ((), (0,), (address, 1.5), (address, "x"), (address,) + (0,) * 17):
        with pytest.raises((TypeError, ValueError)):
            gsa._call(*bad)


def test_binding_checks_shapes_and_places():
    t = lambda *s, dtype=torch.int32: torch.zeros(*s, dtype=dtype)  # noqa: E731
    with pytest.raises(gsa.GsaError):
        gsa.make_cache(t(100, dtype=torch.uint8), t(2, 5), t(3), t(10), page_tokens=16, n_kv=2, d_h=64, dI=32)
    with pytest.raises(gsa.GsaError, match="pool has"):
        gsa.make_cache(t(100, dtype=torch.uint8), t(2, 5), t(2), t(10), page_tokens=16, n_kv=2, d_h=64, dI=32)
    n = gsa.gsa_cache_page_bytes(gsa.cache_geometry(**GEO)) * 10
    with pytest.raises(gsa.GsaError, match="GPU"):
        gsa.make_cache(t(n, dtype=torch.uint8), t(2, 5), t(2), t(10), page_tokens=16, n_kv=2, d_h=64, dI=32)


def test_binding_refuses_calls_without_tensors():
    c = gsa.cache_geometry(**GEO)
    c.device = 0
    x = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    n = torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(1024, dtype=torch.uint8)
    for call in (lambda: gsa.gsa_cache_append(c, x, x, None, None, n, n, ws), lambda: gsa.gsa_cache_append(c, x, x, None, x, n, n, ws),
                 lambda: gsa.gsa_cache_read(c, None, None, None, ws), lambda: gsa.gsa_cache_read(c, n, None, None, ws)):
        with pytest.raises(gsa.GsaError):
            call()


# ---- the plain form itself ---------------------------------------------------------------------------------------------------
def test_plain_rounding_to_bf16():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(20000, generator=g, dtype=torch.float64) * torch.exp(8 * torch.randn(20000, generator=g, dtype=torch.float64))
    assert np.array_equal(bf16(x.float().double().numpy()), x.float().to(torch.bfloat16).double().numpy())
    half = 1 + 2.0 ** -8                                        # halfway between two bf16 numbers: to even
    assert bf16(np.array([half])).item() == 1.0 and bf16(np.array([half + 2.0 ** -20])).item() == 1 + 2.0 ** -7


def test_plain_format():
    assert SCALES[0] == 2.0 ** -20 and SCALES[160] == 1.0 and SCALES[254] == 1.75 * 2.0 ** 11
    x = np.linspace(-1, 1, 16)[None]
    u, b = encode(x)
    s = SCALES[b[0, 0]]
    assert abs(1 / 7 - s) <= (SCALES[b[0, 0] + 1] - SCALES[b[0, 0] - 1]) / 4
    assert (np.abs(decode(u, b) - x) <= s / 2 + 1e-15).all()
    u, b = encode(np.zeros((1, 16)))
    assert (u == 8).all() and b[0, 0] == 0
    x[0, 3] = math.inf
    u, b = encode(x)
    assert b[0, 0] == 255 and np.isnan(decode(u, b)).all()
    # values that are stored exactly are stored exactly again
    g = np.random.default_rng(0)
    c = g.integers(-7, 8, (50, 16))
    c[:, 0] = 7
    x = c * SCALES[g.integers(0, 255, 50)][:, None]
    assert np.array_equal(decode(*encode(x)), x)
