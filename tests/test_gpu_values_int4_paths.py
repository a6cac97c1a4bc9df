"""The 4-bit store's other forms: one token of each sequence, inside the append, four records a wave, and launches whose
waves step over more records than the grid holds. Special rows in each."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from cache4_util import GROUP, dequantise4, place4, quantise4, take4
from parity_util import DEV, to_dev
from test_gpu_values_int4 import _expected, _rows, _special_rows, _store

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t0", range(8))
def test_special_rows_as_one_token_of_each_sequence(t0):
    v = np.ascontiguousarray(_special_rows()[0][:, None])  # [24, 1, 64]
    got = _store(v, 16, t0 + 5).cpu().numpy()
    n, s, z = quantise4(v)
    values = take4(got)
    assert np.array_equal(values[:, t0 + 5], dequantise4(n, s, z)[:, 0])
    # the bytes too, but for the sign of a minimum of 0
    want = _expected(v, 16, t0 + 5)
    at = 272 + 2 * ((t0 + 5) % 8)
    for i in range(24):
        g = (t0 + 5) // 8
        if z[i, 0] == 0:
            assert got[i, g, at:at + 2].view(np.float16)[0] == 0
            want[i, g, at:at + 2] = got[i, g, at:at + 2]
    assert np.array_equal(got, want)


@pytest.mark.parametrize("T", [8, 13, 71])
def test_special_rows_in_an_append(T):
    """The appended record holds what a store of many tokens (other code than the store of one) makes of the row."""
    B, Hkv, Hq, cap = 12, 2, 4, 72
    rows = _special_rows()[0]
    fmt = pa.make_format()
    cache = pa.alloc_pot_cache(B, Hkv, cap, 0, DEV)
    rng = np.random.default_rng(0)
    around = rng.standard_normal((B * Hkv, cap, 64)).astype(np.float16)
    around[:, T - 1] = rows
    want = _store(around, cap, 0).view(B * Hkv, cap // 8, GROUP)
    before = around.copy()
    before[:, T - 1] = 3.0
    got = _store(before, cap, 0)
    k = torch.randn((B, Hkv, 64), device=DEV).half()
    q = torch.randn((B, Hq, 64), device=DEV)
    out = torch.empty((B, Hq, 64), device=DEV)
    ws = pa.alloc_workspace(pa.pot_decode_workspace_bytes(B, Hq, Hkv, T), DEV)
    pa.pot_append_decode_attention_v4(fmt, 0, q, k, to_dev(rows.reshape(B, Hkv, 64)), cache["codes_se"], None,
                                      cache["key_scale"], got, cap, None, np.arange(Hq) // (Hq // Hkv), B, Hq, Hkv, T, out, ws)
    torch.cuda.synchronize()
    got, want = got.cpu().numpy(), want.cpu().numpy()
    n, s, z = quantise4(rows)
    zero = z == 0
    at = 272 + 2 * ((T - 1) % 8)
    got[zero, (T - 1) // 8, at:at + 2] &= 0  # a minimum of 0 may have either sign
    want[zero, (T - 1) // 8, at:at + 2] &= 0
    assert np.array_equal(got, want)
    assert np.isfinite(out.cpu().numpy()).all()


@pytest.mark.parametrize("n_seq,n_tok,t_cap,t0", [
    (3000, 77, 88, 5),       # 11 records a sequence: a wave of four, one of four whole ones, one of three
    (4100, 64, 64, 0),       # 8: all whole
    (1, 262143, 262152, 1),  # one long prompt, 32768 records
    (8200, 26, 40, 7),       # 5: four from inside a record, and one
])
def test_store_of_four_records_a_wave(n_seq, n_tok, t_cap, t0):
    period = 1000 if n_seq == 1 else n_tok
    base = _rows(n_tok, 1 if n_seq == 1 else 37, period)
    base[:, :24] = _special_rows()[0][:min(24, period)]
    v = np.tile(base, (1, n_tok // period + 1, 1))[:, :n_tok] if n_seq == 1 else base[np.arange(n_seq) % 37]
    got = _store(np.ascontiguousarray(v), t_cap, t0).cpu().numpy()
    n, s, z = quantise4(base)
    if n_seq == 1:
        n, s, z = (np.tile(a, (1, n_tok // period + 1) + (1,) * (a.ndim - 2))[:, :n_tok] for a in (n, s, z))
        want = np.full((1, t_cap // 8, GROUP), 0xA5, np.uint8)
        t = t0 + np.arange(n_tok)
        c = np.arange(64)
        low = n[0, :, c % 32 < 16].T.reshape(n_tok, 2, 16)
        high = n[0, :, c % 32 >= 16].T.reshape(n_tok, 2, 16)
        where = 16 * np.arange(16)[None, None] + 8 * np.arange(2)[None, :, None] + (t % 8)[:, None, None]
        want[0, (t // 8)[:, None, None], where] = low | (high << 4)
        for at, a in ((256, s), (272, z)):
            b = np.ascontiguousarray(a[0]).view(np.uint8).reshape(n_tok, 2)
            want[0, (t // 8)[:, None], at + 2 * (t % 8)[:, None] + np.arange(2)] = b
    else:
        want = np.full((37, t_cap // 8, GROUP), 0xA5, np.uint8)
        place4(want, n, s, z, t0)
        want = want[np.arange(n_seq) % 37]
    # a minimum of 0 may have either sign
    for a in (got, want):
        minima = a[:, :, 272:].reshape(a.shape[0], -1, 8, 2)
        minima[(minima[..., 0] == 0) & (minima[..., 1] == 0x80)] = 0
        a[:, :, 272:] = minima.reshape(a.shape[0], -1, 16)
    assert np.array_equal(got, want)


MANY = (1 << 22) + 4099  # one record a sequence: more than the 2^22 waves of the largest grid


@pytest.mark.parametrize("n_tok,t0", [(1, 3), (2, 5), (8, 0)])
def test_more_records_than_waves(n_tok, t0):
    base = _rows(3, 1009, n_tok)
    idx = torch.arange(MANY, device=DEV) % 1009
    rows = to_dev(base)[idx]
    cache = torch.full((MANY, 1, GROUP), 0xA5, dtype=torch.uint8, device=DEV)
    pa.pot_store_values_int4(rows, MANY, n_tok, 8, t0, cache)
    small = _store(base, 8, t0)
    assert np.array_equal(small.cpu().numpy(), _expected(base, 8, t0))
    assert torch.equal(cache[-5000:], small[idx[-5000:]]) and torch.equal(cache, small[idx])
    out, want = torch.empty_like(rows), torch.empty_like(to_dev(base))
    pa.pot_load_values_int4(cache, MANY, n_tok, 8, t0, out)
    pa.pot_load_values_int4(small, 1009, n_tok, 8, t0, want)
    assert torch.equal(out, want[idx])


@pytest.mark.parametrize("fmt", ["fp16", "int8"])
def test_more_groups_than_waves_read_back(fmt):
    base = _rows(4, 1009, 3)
    idx = torch.arange(MANY, device=DEV) % 1009
    rows = to_dev(base)
    out, want = torch.empty((MANY, 3, 64), dtype=torch.float16, device=DEV), torch.empty_like(rows)
    if fmt == "fp16":
        small = torch.zeros((1009, 8, 64), dtype=torch.float16, device=DEV)
        pa.pot_store_values(rows, 1009, 3, 8, 5, small)
        pa.pot_load_values(small[idx], MANY, 3, 8, 5, out)
        want = rows
    else:
        small, exps = torch.zeros((1009, 8, 64), dtype=torch.uint8, device=DEV), torch.zeros((1009, 8), dtype=torch.int8, device=DEV)
        pa.pot_store_values_int8(rows, 1009, 3, 8, 5, small, exps)
        pa.pot_load_values_int8(small, exps, 1009, 3, 8, 5, want)
        pa.pot_load_values_int8(small[idx], exps[idx], MANY, 3, 8, 5, out)
    assert torch.equal(out, want[idx])


@pytest.mark.parametrize("k,hadamard", [(0, False), (2, False), (4, True)])
def test_more_key_rows_than_waves_read_back(k, hadamard):
    """Eight (rotated: sixteen) rows a wave."""
    rows = (1 << 22) * (16 if hadamard else 8) + 40
    fmt = pa.make_format(k, hadamard=hadamard)
    base = to_dev(_rows(5, 1, 1000)[0])
    se = torch.empty((1000, 32), dtype=torch.uint8, device=DEV)
    cm = torch.empty((1000, 8 * k), dtype=torch.uint8, device=DEV) if k else None
    sc = torch.empty(1000, dtype=torch.float32, device=DEV)
    pa.pot_encode_keys(fmt, base, 1000, 1, 0, sc, se, cm)
    want = torch.empty((1000, 64), dtype=torch.float16, device=DEV)
    pa.pot_load_keys(fmt, se, cm, sc, 1, 1000, 1000, 0, want)
    idx = torch.arange(rows, device=DEV) % 1000
    out = torch.empty((rows, 64), dtype=torch.float16, device=DEV)
    pa.pot_load_keys(fmt, se[idx], cm[idx] if k else None, sc[idx], 1, rows, rows, 0, out)
    for at in range(0, rows, 1 << 24):
        assert torch.equal(out[at:at + (1 << 24)], want[idx[at:at + (1 << 24)]]), at
