"""Argument checks of the serving entry points, which need no device, and the sizes of their workspaces."""
import ctypes
import struct

import pytest

import __graft_entry__ as entry
from paper_2602_02071_b200 import binding

P, BAD = 256, 8                                        # an address that is aligned, one that is not


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return binding.load()


def window(lib, q=P, k=P, v=P, out=P, lse=None, lengths=None, strides=None, B=1, H=4, Hkv=2, S=100, D=64, window=10, sinks=0,
           scale=0.0, dtype=binding.DTYPE_BF16):
    return lib.baps_attention_window_fwd(q, k, v, out, lse, lengths, strides, B, H, Hkv, S, D, window, sinks, scale, dtype, None)


def test_window(lib):
    for bad in (dict(q=None), dict(out=None), dict(S=0), dict(B=-1), dict(H=3), dict(window=0), dict(sinks=-1), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(strides=(ctypes.c_int64 * 12)(*[64] * 11, 4)),
                dict(strides=(ctypes.c_int64 * 12)(*[64] * 11, 0)), dict(strides=(ctypes.c_int64 * 12)(*[64] * 11, -64)),
                dict(strides=(ctypes.c_int64 * 12)(1 << 40, *[64] * 11))):
        assert window(lib, **bad) == -1, bad
    for bad in (dict(D=96), dict(dtype=binding.DTYPE_F32), dict(dtype=9), dict(B=70000), dict(H=70000, Hkv=1)):
        assert window(lib, **bad) == -2, bad
    for bad in (dict(q=BAD), dict(v=BAD), dict(out=BAD), dict(lse=2), dict(lengths=3)):
        assert window(lib, **bad) == -3, bad


def cache(k=P, v=P, ks=P, vs=P, n_pages=8, Hkv=2, page=16, D=64):
    return struct.pack("4Q4i", *(x or 0 for x in (k, v, ks, vs)), n_pages, Hkv, page, D)


BAD_CACHES = [(-1, dict(k=None)), (-1, dict(vs=None)), (-1, dict(n_pages=0)), (-1, dict(Hkv=0)), (-2, dict(page=48)), (-2, dict(D=96)),
              (-2, dict(n_pages=1 << 30)), (-3, dict(v=BAD)), (-3, dict(ks=2))]


def append(lib, c=None, k=P, v=P, strides=None, n=4, starts=P, lengths=P, table=P, width=4, B=2, max_new=4, dtype=binding.DTYPE_F16):
    return lib.baps_kv_append(c or cache(), k, v, strides, n, starts, lengths, table, width, B, max_new, dtype, None)


def attention(lib, c=None, q=P, out=P, lse=None, table=P, width=4, lengths=P, strides=None, B=2, H=4, T=1, window=5, sinks=0, scale=0.0,
              dtype=binding.DTYPE_F16, ws=P, ws_bytes=1 << 40):
    return lib.baps_kv_attention(q, out, lse, c or cache(), table, width, lengths, strides, B, H, T, window, sinks, scale, dtype, ws,
                                 ws_bytes, None)


def fork(lib, c=None, table=P, lengths=P, rows=2, refs=P, parents=P, new_rows=2, width=4, reserve=0, window=5, sinks=0, new_table=P,
         new_lengths=P, new_refs=P, ws=P, ws_bytes=1 << 40):
    return lib.baps_kv_fork(c or cache(), table, lengths, rows, refs, parents, new_rows, width, reserve, window, sinks, new_table,
                            new_lengths, new_refs, ws, ws_bytes, None)


def compact(lib, c=None, table=P, rows=2, width=4, refs=P, new_table=P, new_refs=P, page_map=P, n_live=P, ws=P, ws_bytes=1 << 40):
    return lib.baps_kv_compact(c or cache(), table, rows, width, refs, new_table, new_refs, page_map, n_live, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [append, attention, fork, compact])
def test_every_call_checks_the_cache(lib, call):
    for status, bad in BAD_CACHES:
        assert call(lib, c=cache(**bad)) == status, bad


def test_append(lib):
    assert append(lib, n=0) == append(lib, B=0) == append(lib, max_new=0) == 0
    for bad in (dict(n=-1), dict(B=-1), dict(max_new=-1), dict(width=0), dict(k=None), dict(starts=None), dict(table=None),
                dict(strides=(ctypes.c_int64 * 4)(128, 64, 128, 60))):
        assert append(lib, **bad) == -1, bad
    for bad in (dict(dtype=binding.DTYPE_F32), dict(B=70000)):
        assert append(lib, **bad) == -2, bad
    for bad in (dict(k=BAD), dict(lengths=2)):
        assert append(lib, **bad) == -3, bad


def test_attention(lib):
    for bad in (dict(q=None), dict(out=None), dict(table=None), dict(lengths=None), dict(B=0), dict(H=3), dict(T=0),
                dict(width=0), dict(window=0), dict(sinks=-1), dict(scale=-0.5), dict(strides=(ctypes.c_int64 * 6)(64, 64, 64, 64, 64, 12))):
        assert attention(lib, **bad) == -1, bad
    for bad in (dict(T=17), dict(B=4097), dict(dtype=binding.DTYPE_F32), dict(width=1 << 28)):
        assert attention(lib, **bad) == -2, bad
    for bad in (dict(q=BAD), dict(out=BAD), dict(lse=2), dict(ws=BAD)):
        assert attention(lib, **bad) == -3, bad


def test_fork_and_compact(lib):
    for bad in (dict(table=None), dict(new_refs=None), dict(ws=None), dict(rows=0), dict(new_rows=0), dict(width=0), dict(reserve=-1),
                dict(window=0), dict(sinks=-1), dict(ws_bytes=8)):
        assert fork(lib, **bad) == -1, bad
    for bad in (dict(rows=8193), dict(new_rows=1 << 20, width=1 << 12)):
        assert fork(lib, **bad) == -2, bad
    for bad in (dict(refs=4), dict(ws=BAD), dict(parents=2)):
        assert fork(lib, **bad) == -3, bad
    for bad in (dict(rows=-1), dict(table=None), dict(new_table=None), dict(refs=None), dict(n_live=None), dict(ws_bytes=8)):
        assert compact(lib, **bad) == -1, bad
    for bad in (dict(refs=2), dict(ws=BAD), dict(page_map=1)):
        assert compact(lib, **bad) == -3, bad


def test_workspaces(lib):
    def size(B=1, H=8, Hkv=8, T=1, D=64, page=16, width=10000, window=1 << 30, sinks=0):
        return lib.baps_kv_attention_workspace(B, H, Hkv, T, D, page, width, window, sinks)

    assert 0 < size() < size(D=128) <= size(H=64, T=2, D=128)
    assert size(width=20) == size(window=100) == 0                                     # short contexts need none
    for refused in (dict(B=0), dict(B=4097), dict(Hkv=3), dict(T=17), dict(D=96), dict(T=0), dict(page=8), dict(width=0), dict(window=0)):
        assert size(**refused) == 0
    # a call that needs one is refused without it, or with one that is too small
    assert attention(lib, width=10000, window=1 << 30, ws=None) == attention(lib, width=10000, window=1 << 30, ws_bytes=1000) == -1
    pages = lib.baps_kv_pages_workspace
    assert pages(0, 1) > 0 and pages(10, 1000) > pages(0, 1000) and pages(-1, 5) == pages(3, 0) == 0


def test_limits_of_sizes_that_the_header_names(lib):
    """Sizes just beyond each limit; nothing is read or launched for them."""
    for c in (cache(Hkv=32768), cache(n_pages=1 << 26, Hkv=2, page=16), cache(n_pages=1 << 20, Hkv=16, page=128)):
        for call in (append, attention, fork, compact):
            assert call(lib, c=c) == -2
    assert window(lib, S=2 ** 31 - 255) == window(lib, B=65536) == window(lib, H=65536) == -2
    assert append(lib, B=65536) == -2
    for bad in (dict(T=16, H=2 * 4097), dict(B=4097), dict(T=17), dict(width=(2 ** 31 - 64) // 16),
                dict(B=4096, width=1 << 20, window=2 ** 31 - 1)):
        assert attention(lib, **bad) == -2, bad
    assert fork(lib, rows=8193) == fork(lib, new_rows=1 << 20, width=(1 << 11) - 1) == -2
    assert compact(lib, ws=BAD) == fork(lib, ws=BAD) == -3


def test_a_scale_that_is_infinite_in_base_2_is_refused(lib):
    for call in (window, attention):
        assert call(lib, scale=3.4e38) == call(lib, scale=2.4e38) == call(lib, scale=float("inf")) == -1
        assert call(lib, scale=2.0 ** 127, dtype=binding.DTYPE_F32) == -2              # taken: the type is what is refused


def test_sizes_beyond_an_int_need_no_workspace(lib):
    sizes = dict(B=1, H=8, Hkv=8, T=1, D=64, page=16, table_width=10000, window=None, sinks=0)
    assert binding.kv_attention_workspace(**sizes) == binding.kv_attention_workspace(**{**sizes, "window": 2 ** 40}) > 0
    for name in ("B", "H", "Hkv", "T", "D", "page", "table_width", "sinks"):
        for far in (2 ** 32, -2 ** 32):
            assert binding.kv_attention_workspace(**{**sizes, name: sizes[name] + far}) == 0, name
    assert binding.kv_attention_workspace(**{**sizes, "window": -2 ** 32 + 5}) == 0
