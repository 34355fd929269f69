"""What the calls on a paged cache refuse on the host, before anything is enqueued; no call here gets as far as a CUDA call (every one
has a fault, its pointers are never looked through)."""
import ctypes

import pytest

from paper_2603_14303_b200 import binding, build

P = 0x1000      # an aligned address that nothing reads
OFF = 0x1004    # one that is not
INVALID, UNSUPPORTED = binding.SC_ERR_INVALID_ARG, binding.SC_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def _cache(**kw):
    c = dict(k=P, v=P, page_stride=8 * 16 * 128, head_stride=16 * 128, row_stride=128, num_pages=100, page_size=16, page_heads=8, table=P,
             table_stride=40, table_heads=1, max_pages=40, count=None, k_min=P, k_max=P)
    assert set(kw) <= set(c)
    c.update(kw)
    return binding._PagedCache(**c)


def _rows(**kw):
    r = dict(k=P, v=P, kv_token=1024, kv_head=128, count=None, seq_off=P, seq_len=None, cache_len=P, len_out=0x2000, q=P, q_out=P, q_token=4096,
             q_head=128, qo_token=4096, qo_head=128, inv_freq=P, rot_dim=128, positions=None)
    assert set(kw) <= set(r)
    r.update(kw)
    return binding._PagedRows(**r)


SHAPES = [(dict(Hq=30), INVALID), (dict(Hkv=0), INVALID), (dict(B=-1), INVALID), (dict(Hq=0), INVALID), (dict(d=0), UNSUPPORTED),
          (dict(d=12), UNSUPPORTED), (dict(d=264), UNSUPPORTED), (dict(dt=2), UNSUPPORTED), (dict(dt=-1), UNSUPPORTED),
          (dict(B=2 ** 30), UNSUPPORTED)]
TABLES = [dict(num_pages=-1), dict(page_size=0), dict(page_size=-4), dict(max_pages=-1), dict(max_pages=2 ** 28, table_stride=2 ** 28),
          dict(page_heads=4), dict(page_heads=0), dict(page_heads=1), dict(table_heads=3), dict(table=None), dict(table_stride=39)]
POOLS = [dict(k=None), dict(v=None), dict(k=OFF), dict(v=OFF), dict(page_stride=100), dict(head_stride=-2048), dict(row_stride=132),
         dict(row_stride=120)]
SIZES = dict(dt=0, B=2, Hq=32, Hkv=8, d=128)


def append(lib, cache, rows, flags=0, T=7, **size):
    s = {**SIZES, **size}
    return lib.sc_paged_append(cache, rows, s["dt"], s["B"], s["Hq"], s["Hkv"], T, s["d"], flags, None, None)


def decode(lib, cache, q=P, lens=P, scale=0.0, flags=0, out=P, ws=P, bytes_=1 << 40, **size):
    s = {**SIZES, **size}
    return lib.sc_paged_decode_attn(cache, q, s["dt"], s["B"], s["Hq"], s["Hkv"], s["d"], lens, scale, flags, out, ws, bytes_, None, None)


def select(lib, cache, q=P, lens=P, keep=20, n_first=1, n_last=2, table=P, length=P, **size):
    s = {**SIZES, **size}
    return lib.sc_paged_select(cache, q, s["dt"], s["B"], s["Hq"], s["Hkv"], s["d"], lens, keep, n_first, n_last, table, length, None, None)


@pytest.mark.parametrize("size,code", SHAPES)
def test_shapes(lib, size, code):
    assert append(lib, _cache(), _rows(), **size) == code
    assert decode(lib, _cache(), **size) == code
    assert select(lib, _cache(), **size) == code


@pytest.mark.parametrize("kw", TABLES)
def test_tables(lib, kw):
    assert append(lib, _cache(**kw), _rows()) == INVALID
    assert decode(lib, _cache(**kw)) == INVALID
    assert select(lib, _cache(**kw)) == INVALID


@pytest.mark.parametrize("kw", POOLS)
def test_pools(lib, kw):
    assert append(lib, _cache(**kw), _rows()) == INVALID
    assert decode(lib, _cache(**kw)) == INVALID


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(k=OFF), dict(v=OFF), dict(q=OFF), dict(q_out=OFF), dict(q=None), dict(q_out=None),
                                dict(seq_off=None), dict(cache_len=None), dict(len_out=P), dict(rot_dim=-2), dict(rot_dim=7), dict(rot_dim=130),
                                dict(kv_token=1028), dict(kv_head=-128), dict(q_token=4100), dict(q_head=4), dict(qo_token=-8), dict(qo_head=12),
                                dict(count=P)])
def test_rows(lib, kw):
    assert append(lib, _cache(), _rows(**kw)) == INVALID


@pytest.mark.parametrize("cache,kw", [(dict(table_heads=8), {}), (dict(page_heads=1, table_heads=8), {}), (dict(k_min=None), {}), (dict(k_max=OFF), {}),
                                      ({}, dict(T=-1)), ({}, dict(flags=1)), ({}, dict(flags=64))])
def test_append(lib, cache, kw):
    assert append(lib, _cache(**cache), _rows(), **kw) == INVALID
    assert lib.sc_paged_append(None, _rows(), 0, 2, 32, 8, 7, 128, 0, None, None) == INVALID
    assert lib.sc_paged_append(_cache(), None, 0, 2, 32, 8, 7, 128, 0, None, None) == INVALID


@pytest.mark.parametrize("kw", [dict(q=None), dict(q=OFF), dict(lens=None), dict(out=None), dict(out=OFF), dict(ws=None), dict(ws=OFF), dict(bytes_=100),
                                dict(scale=-1.0), dict(scale=float("nan")), dict(flags=2), dict(flags=16), dict(flags=32)])
def test_decode(lib, kw):
    assert decode(lib, _cache(), **kw) == INVALID


@pytest.mark.parametrize("kw,code", [(dict(q=None), INVALID), (dict(q=OFF), INVALID), (dict(lens=None), INVALID), (dict(table=None), INVALID),
                                     (dict(length=None), INVALID), (dict(keep=0), INVALID), (dict(keep=2), INVALID), (dict(n_first=-1), INVALID),
                                     (dict(n_last=0), INVALID), (dict(keep=2 ** 31 - 1, n_first=2 ** 31 - 1), INVALID),
                                     (dict(keep=2 ** 28), INVALID)])
def test_select(lib, kw, code):
    assert select(lib, _cache(), **kw) == code


def test_select_needs_bounds_and_tables_it_can_hold(lib):
    assert select(lib, _cache(k_min=None)) == INVALID
    assert select(lib, _cache(k_max=OFF)) == INVALID
    many = binding.SC_SELECT_MAX_PAGES + 1
    assert select(lib, _cache(max_pages=many, table_stride=many)) == UNSUPPORTED


def test_more_rows_than_a_launch_can_number(lib):
    wide = dict(max_pages=2 ** 26, table_stride=2 ** 26)
    assert decode(lib, _cache(**wide), B=4, Hq=32, Hkv=8) == UNSUPPORTED      # 4 * 8 heads x 2^26 tiles of 16 rows
    assert decode(lib, _cache(**wide, page_heads=2), B=1, Hq=128, Hkv=2) == UNSUPPORTED   # 2 heads x 16 groups of queries
    tiny = dict(page_heads=32, page_size=1, max_pages=1, table_stride=1)
    assert decode(lib, _cache(**tiny), B=2 ** 25, Hq=32, Hkv=32) == UNSUPPORTED   # 2^30 heads, of four tiles at least


def test_nothing_to_do(lib):
    """No sequences: fine without any pointer but the structures."""
    empty = _cache(k=None, v=None, num_pages=0, table=None, max_pages=0, k_min=None, k_max=None)
    assert append(lib, empty, _rows(k=None, v=None, q=None, q_out=None, seq_off=None, cache_len=None, len_out=None), B=0, T=0) == binding.SC_OK
    assert decode(lib, empty, q=None, lens=None, out=None, ws=None, bytes_=0, B=0) == binding.SC_OK
    assert select(lib, empty, q=None, lens=None, table=None, length=None, B=0) == binding.SC_OK


def test_workspace_sizes(lib):
    """The lengths and the batch do not matter: a workspace for one call serves any other of its head size or below."""
    f = lib.sc_paged_decode_workspace_bytes
    sizes = {f(B, Hkv * G, Hkv, d) for B in (1, 7, 1000) for Hkv, G in ((8, 4), (1, 1), (4, 16)) for d in (8, 64, 128, 256)}
    assert max(sizes) < 64 << 20 and f(0, 8, 8, 128) > 0
    for d, wider in zip((8, 64, 128), (64, 128, 256)):
        assert f(3, 32, 8, d) <= f(1, 8, 8, wider) and f(3, 32, 8, d) == f(1, 1, 1, d)


def test_structures_match_the_header(lib):
    """Field order and sizes of the two structures, as the C side has them (64-bit, natural alignment)."""
    assert ctypes.sizeof(binding._PagedCache) == 104 and binding._PagedCache.table.offset == 56 and binding._PagedCache.k_max.offset == 96
    assert ctypes.sizeof(binding._PagedRows) == 144 and binding._PagedRows.q.offset == 72 and binding._PagedRows.positions.offset == 136
