"""Refusals of the 4-bit cache's entry points, without a GPU: every check runs before any HIP call, on fake addresses."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa

FAKE = 0x7F0000001000
INVALID, UNSUPPORTED, WORKSPACE = pa.POT_ERR_INVALID_ARG, pa.POT_ERR_UNSUPPORTED, pa.POT_ERR_WORKSPACE
HEADS = np.arange(32, dtype=np.int32) // 8


def _decode(append, **over):
    a = dict(fmt=pa.make_format(), engine=0, q=FAKE, k_new=FAKE, v_new=FAKE, se=FAKE, cm=None, sc=FAKE, v4=FAKE, cap=4096,
             lens=FAKE, heads=HEADS, B=1, Hq=32, Hkv=4, T=4096, out=FAKE, ws=FAKE, nws=1 << 30, dbg=None)
    a.update(over)
    heads = a["heads"].ctypes.data if a["heads"] is not None else None
    new = (a["k_new"], a["v_new"]) if append else ()
    fn = pa._lib.pot_append_decode_attention_v4 if append else pa._lib.pot_decode_attention_v4
    return fn(ctypes.byref(a["fmt"]), a["engine"], a["q"], *new, a["se"], a["cm"], a["sc"], a["v4"], a["cap"], a["lens"],
              heads, a["B"], a["Hq"], a["Hkv"], a["T"], a["out"], a["ws"], a["nws"],
              ctypes.byref(a["dbg"]) if a["dbg"] is not None else None, None)


def _tap():
    d = pa.pot_debug()
    d.scores = FAKE
    return d


def _waves(n):
    d = pa.pot_debug()
    d.force_wg_waves = n
    return d


BAD = [
    (dict(fmt=pa.make_format(mant_bits=5)), UNSUPPORTED), (dict(fmt=pa.make_format(frac_bits=5)), INVALID),
    (dict(engine=2), INVALID), (dict(engine=-1), INVALID),
    (dict(engine=1, fmt=pa.make_format(mant_bits=1), cm=FAKE), UNSUPPORTED),
    (dict(q=None), INVALID), (dict(se=None), INVALID), (dict(sc=None), INVALID), (dict(v4=None), INVALID),
    (dict(out=None), INVALID), (dict(ws=None), INVALID), (dict(heads=None), INVALID),
    (dict(cm=FAKE), INVALID), (dict(fmt=pa.make_format(mant_bits=2)), INVALID),
    (dict(v4=FAKE + 8), INVALID), (dict(q=FAKE + 4), INVALID), (dict(lens=FAKE + 2), INVALID), (dict(ws=FAKE + 16), INVALID),
    (dict(T=0), INVALID), (dict(T=-1), INVALID), (dict(T=4097), INVALID), (dict(cap=4097, T=9), INVALID), (dict(B=0), INVALID),
    (dict(T=1 << 24, cap=1 << 24), UNSUPPORTED), (dict(Hq=24, heads=np.arange(24, dtype=np.int32) // 6), UNSUPPORTED),
    (dict(heads=np.full(32, 4, np.int32)), INVALID), (dict(nws=1000), WORKSPACE),
    (dict(dbg=_tap()), UNSUPPORTED), (dict(dbg=_waves(7)), INVALID),
]


@pytest.mark.parametrize("append", [False, True])
@pytest.mark.parametrize("over,code", BAD)
def test_attention_refuses(append, over, code):
    assert _decode(append, **over) == code
    assert pa.pot_last_error() != ""


@pytest.mark.parametrize("over", [dict(k_new=None), dict(v_new=None), dict(k_new=FAKE + 8), dict(v_new=FAKE + 2)])
def test_append_refuses(over):
    assert _decode(True, **over) == INVALID


def _row_calls():
    f = pa.make_format()
    return {
        "store4": lambda n, m, c, t, p=FAKE, o=FAKE: pa._lib.pot_store_values_int4(p, n, m, c, t, o, None),
        "load4": lambda n, m, c, t, p=FAKE, o=FAKE: pa._lib.pot_load_values_int4(p, n, m, c, t, o, None),
        "load8": lambda n, m, c, t, p=FAKE, o=FAKE: pa._lib.pot_load_values_int8(p, FAKE, n, m, c, t, o, None),
        "load16": lambda n, m, c, t, p=FAKE, o=FAKE: pa._lib.pot_load_values(p, n, m, c, t, o, None),
        "keys": lambda n, m, c, t, p=FAKE, o=FAKE: pa._lib.pot_load_keys(ctypes.byref(f), p, None, FAKE, n, m, c, t, o, None),
    }


@pytest.mark.parametrize("name", ["store4", "load4", "load8", "load16", "keys"])
def test_row_calls_refuse(name):
    call = _row_calls()[name]
    big = 1 << 62
    for args in [(-1, 1, 8, 0), (1, -1, 8, 0), (1, 1, 0, 0), (1, 1, 12, 0), (1, 1, -8, 0), (1, 9, 8, 0), (1, 1, 8, 8),
                 (1, 4, 8, 5), (1, 1, 8, -1), (1, big, 8, 0), (1, 1, 8, (1 << 63) - 1), (big, 2, 8, 0),
                 (1 << 31, 2, 8, 0)]:
        assert call(*args) == INVALID, args
        assert pa.pot_last_error() != ""
    assert call(1, 1, 8, 0, p=None) == INVALID
    assert call(1, 1, 8, 0, o=None) == INVALID
    assert call(1, 1, 8, 0, p=FAKE + 8) == INVALID
    assert call(1, 1, 8, 0, o=FAKE + 8) == INVALID
    assert call(0, 1, 8, 0) == pa.POT_OK and call(1, 0, 8, 8) == pa.POT_OK
    assert call(0, 1, 8, 0, p=None, o=None) == pa.POT_OK


def test_key_read_back_refuses_formats():
    L = pa._lib.pot_load_keys
    assert L(ctypes.byref(pa.make_format(5)), FAKE, FAKE, FAKE, 1, 1, 8, 0, FAKE, None) == UNSUPPORTED
    assert L(None, FAKE, None, FAKE, 1, 1, 8, 0, FAKE, None) == INVALID
    assert L(ctypes.byref(pa.make_format(1)), FAKE, None, FAKE, 1, 1, 8, 0, FAKE, None) == INVALID
    assert L(ctypes.byref(pa.make_format(0)), FAKE, FAKE, FAKE, 1, 1, 8, 0, FAKE, None) == INVALID
    assert L(ctypes.byref(pa.make_format(1)), FAKE, FAKE + 4, FAKE, 1, 1, 8, 0, FAKE, None) == INVALID
    assert L(ctypes.byref(pa.make_format(0)), FAKE, None, None, 1, 1, 8, 0, FAKE, None) == INVALID
    assert pa._lib.pot_load_values_int8(FAKE, None, 1, 1, 8, 0, FAKE, None) == INVALID


def _rope(**over):
    rope = dict(rot_dim=64, neighbours=0, n_axes=1, head_dim=64, axis=[0] * 32)
    a = dict(dtype=1, q=FAKE, k=FAKE, v=FAKE, sq=(64, 64, 64), qw=FAKE, kw=FAKE, vw=None, wt=2, eps=1e-6, pos=FAKE, inv=FAKE,
             B=2, S=3, Hq=4, Hkv=2, qt=2, qo=FAKE, ko=FAKE, vo=FAKE)
    for n, x in over.items():
        (rope if n in rope else a)[n] = x
    r = pa.pot_rope(rope["head_dim"], rope["rot_dim"], rope["neighbours"], rope["n_axes"], (ctypes.c_uint8 * 32)(*rope["axis"]))
    parts = (pa.pot_part * 3)(pa.pot_part(a["q"], *a["sq"], a["qw"], a["qo"]), pa.pot_part(a["k"], 64, 64, 64, a["kw"], a["ko"]),
                              pa.pot_part(a["v"], 64, 64, 64, a["vw"], a["vo"]))
    return pa._lib.pot_norm_rope(ctypes.byref(r), a["dtype"], ctypes.byref(parts), a["wt"], a["eps"], a["pos"], a["inv"], a["B"],
                                 a["S"], a["Hq"], a["Hkv"], a["qt"], None)


@pytest.mark.parametrize("over,code", [
    (dict(head_dim=128), UNSUPPORTED), (dict(rot_dim=66), INVALID), (dict(rot_dim=-2), INVALID), (dict(rot_dim=3), INVALID),
    (dict(neighbours=2), INVALID), (dict(n_axes=0), INVALID), (dict(n_axes=5), INVALID), (dict(axis=[1] * 32), INVALID),
    (dict(dtype=3), INVALID), (dict(wt=-1), INVALID), (dict(qt=9), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(B=-1), INVALID), (dict(Hq=0), INVALID),
    (dict(Hkv=0), INVALID), (dict(qo=None), INVALID), (dict(ko=None), INVALID), (dict(vo=None), INVALID), (dict(q=None), INVALID),
    (dict(k=None), INVALID), (dict(vw=FAKE), INVALID), (dict(kw=FAKE + 8), INVALID), (dict(q=FAKE + 2), INVALID), (dict(ko=FAKE + 8), INVALID), (dict(sq=(4, 64, 64)), INVALID),
    (dict(sq=(64, 4, 64)), INVALID), (dict(sq=(64, 64, 4)), INVALID), (dict(pos=None), INVALID), (dict(inv=None), INVALID),
    (dict(pos=FAKE + 4), INVALID), (dict(inv=FAKE + 4), INVALID), (dict(qw=FAKE + 2), INVALID),
    (dict(B=1 << 16, S=1 << 16), INVALID), (dict(Hq=1025), UNSUPPORTED), (dict(Hkv=1 << 30), UNSUPPORTED),
])
def test_norm_rope_refuses(over, code):
    assert _rope(**over) == code
    assert pa.pot_last_error() != ""


def test_norm_rope_refuses_more_tokens_than_a_dispatch_holds():
    assert _rope(B=1 << 14, S=1 << 15) == INVALID
    assert "too large" in pa.pot_last_error()


def test_norm_rope_of_nothing():
    assert _rope(B=0) == pa.POT_OK and _rope(S=0) == pa.POT_OK
    assert _rope(q=None, k=None, v=None, qo=None, ko=None, vo=None) == pa.POT_OK
    assert pa._lib.pot_norm_rope(None, 1, None, 2, 0.0, None, None, 1, 1, 1, 1, 2, None) == INVALID
    assert pa._lib.pot_norm_rope(ctypes.byref(pa.make_rope()), 1, None, 2, 0.0, None, None, 1, 1, 1, 1, 2, None) == INVALID


@pytest.mark.parametrize("lens", [torch.zeros(4, dtype=torch.int64), torch.zeros(8, dtype=torch.int32)[::2]])
def test_binding_refuses_lengths_of_another_type(lens):
    with pytest.raises(pa.PotError) as e:
        pa.pot_decode_attention_v4(pa.make_format(), 0, FAKE, FAKE, None, FAKE, FAKE, 8, lens, HEADS, 4, 32, 4, 8, FAKE, FAKE,
                                   ws_bytes=1 << 30)
    assert e.value.status == INVALID


def test_binding_refuses_too_few_lengths():
    with pytest.raises(pa.PotError) as e:
        pa.pot_decode_attention_v4(pa.make_format(), 0, FAKE, FAKE, None, FAKE, FAKE, 8, torch.zeros(3, dtype=torch.int32), HEADS,
                                   4, 32, 4, 8, FAKE, FAKE, ws_bytes=1 << 30)
    assert e.value.status == INVALID


@pytest.mark.parametrize("rot_dim,axes", [(64, [0] * 31), (64, [0] * 33), (32, [0] * 32), (64, [0] * 31 + [4]), (64, [-1] * 32),
                                          (64, [256] * 32), (8, [])])
def test_binding_refuses_axes_that_are_not_one_a_pair(rot_dim, axes):
    with pytest.raises(pa.PotError) as e:
        pa.make_rope(rot_dim, axis_of_pair=axes)
    assert e.value.status == INVALID


def test_binding_refuses_tensors_that_do_not_go_together():
    x = torch.zeros((2, 3, 4, 64))
    out = torch.zeros((2, 4, 3, 64))
    pos, inv = torch.zeros((1, 2, 3), dtype=torch.int64), torch.zeros(32, dtype=torch.float64)
    w = torch.ones(64)
    good = dict(rope=pa.make_rope(), q=x, k=None, v=None, q_weight=w, k_weight=None, eps=1e-6, positions=pos, inv_freq=inv,
                q_out=out, k_out=None, v_out=None)
    for over in [dict(q_out=None), dict(q_out=out.transpose(1, 2)), dict(q_out=torch.zeros((2, 3, 4, 32))),
                 dict(q=x.transpose(2, 3).contiguous().transpose(2, 3)), dict(q=x[..., :32]), dict(q=x.double()),
                 dict(positions=pos.int()), dict(positions=pos[:, :, :2]), dict(inv_freq=inv.float()),
                 dict(inv_freq=inv[:31]), dict(q_weight=torch.ones(63)), dict(q_weight=torch.ones(128)[::2]),
                 dict(q_out=out.double()), dict(k=x.half(), k_out=out.half()), dict(k=x, k_out=out),
                 dict(rope=pa.make_rope(axis_of_pair=[0, 1] * 16)),
                 dict(k=x, k_out=out.half(), v=x[:, :, :2], v_out=out[:, :2].half().contiguous())]:
        with pytest.raises(pa.PotError) as e:
            pa.pot_norm_rope(**dict(good, **over))
        assert e.value.status == INVALID, over
