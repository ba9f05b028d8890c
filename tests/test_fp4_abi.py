"""What the entry points of the 4-bit cache and of the page bookkeeping refuse, on the host (nothing is launched)."""
import ctypes
import os

import pytest

from paper_2504_15930_amd import sl

FAKE = 0x10000   # a 16-byte aligned address that is never dereferenced by these calls


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sl.LIBRARY):
        from paper_2504_15930_amd import build
        build.build()
    return sl.load()


def _desc(**kw):
    args = dict(batch=4, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, max_blocks=8, num_pages=64,
                num_workers=32)
    args.update(kw)
    return sl.make_desc(**args)


def _fp4_calls(lib, d, **kw):
    """Every entry point of the 4-bit cache and the bookkeeping, with `kw` in place of its pointers."""
    r = ctypes.byref(d) if d is not None else None
    g = lambda name: kw.get(name, FAKE)
    return {
        "attn": lib.sl_decode_attn_fp4(r, g("q"), g("kv"), g("bt"), g("lens"), 0.125, g("out")),
        "prefix": lib.sl_decode_attn_prefix_fp4(r, g("q"), g("kv"), g("bt"), g("lens"), g("gs"), g("sp"), 1, 0.125,
                                                g("out")),
    }


def test_fp4_attention_refusals(lib):
    assert set(_fp4_calls(lib, None).values()) == {-1}
    d = _desc()
    for name in ("q", "kv", "bt", "lens", "out"):
        assert set(_fp4_calls(lib, d, **{name: None}).values()) == {-1}, name
    for name in ("q", "kv", "out"):
        assert set(_fp4_calls(lib, d, **{name: FAKE + 8}).values()) == {-6}, name
    assert set(_fp4_calls(lib, d, bt=FAKE + 2).values()) == {-6}
    assert set(_fp4_calls(lib, d).values()) == {-4}       # no workspace
    for kw, status in [(dict(head_dim=96), -3), (dict(page_size=32), -3), (dict(num_q_heads=7), -2),
                       (dict(num_q_heads=34), -3), (dict(batch=-1), -2), (dict(batch=9000), -3)]:
        assert set(_fp4_calls(lib, _desc(**kw)).values()) == {status}, kw
    assert _fp4_calls(lib, _desc(batch=0), q=None, kv=None)["attn"] == 0


def test_fp4_row_refusals(lib):
    def calls(d, T=3, **kw):
        r = ctypes.byref(d) if d is not None else None
        g = lambda name: kw.get(name, FAKE)
        return {lib.sl_kv_write_fp4(r, g("k"), g("v"), g("slots"), T, g("kv")),
                lib.sl_kv_read_fp4(r, g("kv"), g("slots"), T, g("k"), g("v"))}
    assert calls(None) == {-1}
    d = _desc(batch=0)
    for name in ("k", "v", "slots", "kv"):
        assert calls(d, **{name: None}) == {-1}, name
    for name in ("k", "v", "kv"):
        assert calls(d, **{name: FAKE + 8}) == {-6}, name
    assert calls(d, slots=FAKE + 2) == {-6}
    assert calls(d, T=-1) == {-2}
    assert calls(d, T=1 << 26) == {-3}                     # times 2 KV heads
    assert calls(d, T=0, k=None, kv=None) == {0}
    for kw, status in [(dict(head_dim=96), -3), (dict(page_size=32), -3), (dict(num_kv_heads=0), -2),
                       (dict(num_pages=0), -2), (dict(num_pages=1 << 27), -3)]:
        assert calls(_desc(**kw)) == {status}, kw
    append = lambda d, k=FAKE, kv=FAKE: lib.sl_kv_append_fp4(ctypes.byref(d), k, FAKE, FAKE, FAKE, kv)
    assert append(_desc(), k=None) == -1 and append(_desc(), k=FAKE + 4) == -6 and append(_desc(), kv=FAKE + 4) == -6
    assert append(_desc(head_dim=32)) == -3 and append(_desc(num_pages=1 << 27)) == -3 and append(_desc(batch=0), k=None) == 0


def test_page_refusals(lib):
    def extend(d, cap=4, **kw):
        g = lambda name: kw.get(name, FAKE)
        return lib.sl_pages_extend(ctypes.byref(d) if d is not None else None, g("lens"), g("new"), g("bt"), g("free"),
                                   g("count"), cap, g("lens_out"), g("count_out"), g("start"), g("slots"))

    def release(d, **kw):
        g = lambda name: kw.get(name, FAKE)
        return lib.sl_pages_release(ctypes.byref(d) if d is not None else None, g("new"), g("lens"), g("bt"), g("free"),
                                    g("count"), g("lens_out"), g("count_out"))
    assert extend(None) == -1 and release(None) == -1
    d = _desc()
    for name in ("lens", "new", "bt", "free", "count", "lens_out", "count_out"):
        assert extend(d, **{name: None}) == -1 and release(d, **{name: None}) == -1, name
        assert extend(d, **{name: FAKE + 2}) == -6 and release(d, **{name: FAKE + 2}) == -6, name
    assert extend(d, start=None) == -1 and extend(d, slots=None) == -1 and extend(d, slots=FAKE + 2) == -6
    assert extend(d, cap=-1) == -2
    for kw, status in [(dict(batch=-1), -2), (dict(batch=8193), -3), (dict(page_size=32), -3), (dict(max_blocks=0), -2),
                       (dict(max_blocks=1 << 27), -3), (dict(num_pages=1 << 27), -3),
                       (dict(batch=8192, max_blocks=1 << 15), -3)]:
        assert extend(_desc(**kw)) == status and release(_desc(**kw)) == status, kw
