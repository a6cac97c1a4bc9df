"""Refusals of the paged cache's entry points, without a GPU: every check runs before any HIP call, on fake addresses."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa

FAKE = 0x7F0000001000
INVALID, UNSUPPORTED, WORKSPACE = pa.POT_ERR_INVALID_ARG, pa.POT_ERR_UNSUPPORTED, pa.POT_ERR_WORKSPACE
HEADS = np.arange(32, dtype=np.int32) // 8


def _pages(**over):
    a = dict(codes_se=FAKE, codes_m=None, key_scale=FAKE, values=FAKE, table=FAKE, value_format=0, n_pages=100, Hkv=4,
             page_size=64, table_len=64)
    a.update(over)
    return pa.pot_pages(*a.values())


def _attend(pages=None, **over):
    a = dict(fmt=pa.make_format(), dtype=1, q=FAKE, st=2048, sh=64, pages=_pages() if pages is None else pages, cu=FAKE, lens=FAKE,
             heads=HEADS, B=2, n=40, Hq=32, max_new=32, max_len=4096, window=0, sink=0, otype=1, out=FAKE, ws=FAKE, nws=1 << 30)
    a.update(over)
    heads = a["heads"].ctypes.data if a["heads"] is not None else None
    return pa._lib.pot_paged_attention(
        ctypes.byref(a["fmt"]), a["dtype"], a["q"], a["st"], a["sh"], ctypes.byref(a["pages"]) if a["pages"] else None, a["cu"],
        a["lens"], heads, a["B"], a["n"], a["Hq"], a["max_new"], a["max_len"], a["window"], a["sink"], a["otype"], a["out"],
        a["ws"], a["nws"], None)


def _part(rows=FAKE, st=2560, sh=64, w=None, out=None, sb=0):
    return [rows or 0, sb, st, sh, w or 0, out or 0]


def _append(pages=None, **over):
    a = dict(fmt=pa.make_format(), rope=pa.make_rope(), dtype=1, q=_part(out=FAKE), k=_part(), v=_part(), wtype=1, eps=1e-6,
             pos=FAKE, freq=FAKE, pages=_pages() if pages is None else pages, cu=FAKE, lens=FAKE, B=2, n=40, Hq=32, qtype=1)
    a.update(over)
    parts = np.array(a["q"] + a["k"] + a["v"], np.int64)
    return pa._lib.pot_paged_append(
        ctypes.byref(a["fmt"]), ctypes.byref(a["rope"]), a["dtype"], parts.ctypes.data, a["wtype"], a["eps"], a["pos"], a["freq"],
        ctypes.byref(a["pages"]) if a["pages"] else None, a["cu"], a["lens"], a["B"], a["n"], a["Hq"], a["qtype"], None)


BAD_PAGES = [
    (dict(codes_se=None), INVALID), (dict(key_scale=None), INVALID), (dict(values=None), INVALID), (dict(table=None), INVALID),
    (dict(codes_m=FAKE), INVALID), (dict(codes_se=FAKE + 8), INVALID), (dict(key_scale=FAKE + 8), INVALID),
    (dict(values=FAKE + 8), INVALID), (dict(table=FAKE + 2), INVALID), (dict(value_format=2), INVALID),
    (dict(value_format=-1), INVALID), (dict(n_pages=0), INVALID), (dict(Hkv=0), INVALID), (dict(Hkv=129), UNSUPPORTED),
    (dict(page_size=0), INVALID), (dict(page_size=4), INVALID), (dict(page_size=12), INVALID), (dict(page_size=-8), INVALID),
    (dict(page_size=(1 << 24) + 8), INVALID), (dict(table_len=0), INVALID),
    (dict(n_pages=2 ** 31 - 1, page_size=1024, table_len=1), INVALID),
]


@pytest.mark.parametrize("over,code", BAD_PAGES)
def test_pages_refused(over, code):
    assert _attend(pages=_pages(**over)) == code and pa.pot_last_error() != ""
    assert _append(pages=_pages(**over)) == code and pa.pot_last_error() != ""


BAD_ATTEND = [
    (dict(fmt=pa.make_format(mant_bits=5)), UNSUPPORTED), (dict(fmt=pa.make_format(frac_bits=5)), INVALID),
    (dict(fmt=pa.make_format(mant_bits=2)), INVALID), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(otype=3), INVALID),
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(q=FAKE + 8), INVALID), (dict(out=FAKE + 4), INVALID),
    (dict(st=2044), INVALID), (dict(sh=60), INVALID), (dict(dtype=2, st=2046), INVALID), (dict(cu=None), INVALID),
    (dict(lens=None), INVALID), (dict(cu=FAKE + 2), INVALID), (dict(lens=FAKE + 1), INVALID), (dict(heads=None), INVALID),
    (dict(heads=np.full(32, 4, np.int32)), INVALID), (dict(heads=np.full(32, -1, np.int32)), INVALID),
    (dict(heads=np.zeros(32, np.int32)), UNSUPPORTED), (dict(Hq=30), UNSUPPORTED), (dict(Hq=0), INVALID),
    (dict(Hq=132, heads=np.arange(132, dtype=np.int32) // 33), UNSUPPORTED), (dict(B=-1), INVALID), (dict(n=-1), INVALID),
    (dict(B=65536), UNSUPPORTED), (dict(n=(1 << 23) + 1), UNSUPPORTED), (dict(max_new=0), INVALID), (dict(max_len=0), INVALID),
    (dict(max_len=4097), INVALID), (dict(max_len=1 << 24, pages=_pages(table_len=1 << 20)), UNSUPPORTED),
    (dict(window=-1), INVALID), (dict(sink=-1), INVALID), (dict(ws=None), INVALID), (dict(ws=FAKE + 16), INVALID),
    (dict(nws=1000), WORKSPACE), (dict(pages=None), INVALID),
]


@pytest.mark.parametrize("over,code", BAD_ATTEND)
def test_attention_refuses(over, code):
    if "pages" in over and over["pages"] is None:
        over = dict(over, pages=False)
    assert _attend(**over) == code
    assert pa.pot_last_error() != ""


BAD_APPEND = [
    (dict(fmt=pa.make_format(mant_bits=-1)), UNSUPPORTED), (dict(dtype=3), INVALID), (dict(wtype=3), INVALID), (dict(qtype=-1), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(k=_part(rows=None)), INVALID), (dict(v=_part(rows=None)), INVALID),
    (dict(k=_part(out=FAKE)), INVALID), (dict(v=_part(out=FAKE)), INVALID), (dict(v=_part(w=FAKE)), INVALID), (dict(q=_part()), INVALID),
    (dict(q=_part(rows=None, out=FAKE)), INVALID), (dict(q=_part(rows=FAKE + 8, out=FAKE)), INVALID), (dict(k=_part(st=2556)), INVALID),
    (dict(v=_part(sh=4)), INVALID), (dict(k=_part(w=FAKE + 4)), INVALID), (dict(freq=None), INVALID), (dict(freq=FAKE + 4), INVALID),
    (dict(pos=FAKE + 4), INVALID), (dict(cu=None), INVALID), (dict(lens=None), INVALID), (dict(B=-1), INVALID), (dict(n=-1), INVALID),
    (dict(n=(1 << 23) + 1), UNSUPPORTED), (dict(B=65536), UNSUPPORTED), (dict(Hq=1025), UNSUPPORTED), (dict(Hq=0), INVALID),
    (dict(rope=pa.pot_rope(64, 65, 0, 1)), INVALID), (dict(rope=pa.pot_rope(128, 64, 0, 1)), UNSUPPORTED),
    (dict(rope=pa.pot_rope(64, 64, 2, 1)), INVALID), (dict(rope=pa.pot_rope(64, 64, 0, 5)), INVALID),
]


@pytest.mark.parametrize("over,code", BAD_APPEND)
def test_append_refuses(over, code):
    assert _append(**over) == code
    assert pa.pot_last_error() != ""


def test_nothing_to_do():
    assert _attend(B=0) == 0 and _attend(n=0) == 0 and _append(B=0) == 0 and _append(n=0) == 0


def test_workspace_sizes():
    w = pa.pot_paged_workspace_bytes
    assert w(0, 10, 32, 4, 1, 100) == 0 and w(1, 0, 32, 4, 1, 100) == 0
    for bad in [(1, 1, 30, 4, 1, 100), (1, 1, 32, 4, 0, 100), (1, 1, 32, 4, 1, 0), (1, 1, 256, 4, 1, 1), (-1, 1, 32, 4, 1, 1),
                (1, 1, 32, 4, 1, 1 << 24)]:
        assert w(*bad) == 0
    for B, n, new in [(1, 1, 1), (64, 64, 1), (1, 512, 512), (16, 700, 300), (3, 3000, 2000), (200, 100000, 4096)]:
        last = 0
        for T in (1, 64, 100, 1000, 5000, 40000, 1 << 20, (1 << 24) - 8):  # a longer length never needs less
            got = w(B, n, 32, 4, new, T)
            assert got >= last and got % 256 == 0
            last = got
        # a call with a window is served by the size without one
        for window in (1, 100, 10000):
            assert _attend(B=B, n=n, max_new=new, max_len=1 << 20, pages=_pages(table_len=1 << 14), window=window, sink=4,
                           nws=w(B, n, 32, 4, new, 1 << 20), q=None) == INVALID  # refused for q, not for the size


def test_binding_refuses_host_tensors_and_other_shapes():
    se, cm, sc, v = (t for t in pa.alloc_pages(4, 2, 16, 1, "cpu"))
    table = torch.zeros((3, 2), dtype=torch.int32)
    with pytest.raises(pa.PotError):
        pa.make_pages(se, cm, sc, v, table)  # on the host
    for bad in [(se[:, :, :, :31], cm, sc, v, table), (se, cm[..., :7], sc, v, table), (se, cm, sc.double(), v, table),
                (se, cm, sc, v[:, :, :8], table), (se, cm, sc, v.float(), table), (se, cm, sc, v, table.long()),
                (se, cm, sc, v, table[0]), (se.transpose(0, 1), cm, sc, v, table), (se[0], cm, sc, v, table),
                (se, cm.repeat(1, 1, 1, 5), sc, v, table)]:
        with pytest.raises(pa.PotError):
            pa.make_pages(*bad)
    pages = _pages()
    pages.calls = (3, -1, 0, 2)
    x = torch.zeros((3, 8, 64))
    with pytest.raises(pa.PotError):
        pa.pot_paged_attention(pa.make_format(), x, pages, table[:, 0], table[:, 0], HEADS[:8], 1, 16, x, None)
    with pytest.raises(pa.PotError):
        pa.pot_paged_append(pa.make_format(), pa.make_rope(), x, x, x, None, None, 0.0, None, None, pages, table, table, x)


def test_calls_too_large_for_a_launch():
    w = pa.pot_paged_workspace_bytes
    for B, n, Hq, Hkv in [(65535, 1 << 23, 128, 128), (65535, 65535 * 2, 128, 128), (65535, 1 << 23, 128, 64)]:
        assert w(B, n, Hq, Hkv, 300, 5000) == 0
        assert _attend(B=B, n=n, Hq=Hq, max_new=300, pages=_pages(Hkv=Hkv)) == UNSUPPORTED
    for B, n, Hkv in [(65535, 65535 * 2, 8), (1, 1 << 23, 8), (65535, 1 << 23, 16)]:  # refused for q, not for the sizes
        assert _attend(B=B, n=n, Hq=128, max_new=300, heads=(np.arange(128) // (128 // Hkv)).astype(np.int32),
                       pages=_pages(Hkv=Hkv), q=None) == INVALID
