"""The 4-bit value cache: bytes of the store against the definition, read-back of every value format and of the key
codes against 64 bits, at the edges of groups, and rows that hold nothing finite."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_09208_amd as pa
from cache4_util import GROUP, dequantise4, key_values, place4, quantise4, sylvester, take4
from parity_util import DEV, to_dev

pytestmark = pytest.mark.gpu

RANGES = [  # n_seq, n_tok, t_cap, t0
    (1, 1, 8, 0), (1, 1, 8, 7), (3, 1, 40, 13), (5, 2, 16, 7), (1, 8, 8, 0), (2, 9, 24, 8), (3, 17, 64, 3),
    (1, 61, 64, 3), (2, 64, 64, 0), (7, 333, 400, 21), (300, 1, 16, 9), (2, 4100, 4104, 1), (257, 40, 40, 0),
    (1, 4095, 4096, 1),
]


def _rows(seed, n_seq, n_tok):
    rng = np.random.default_rng(seed)
    v = rng.standard_normal((n_seq, n_tok, 64)).astype(np.float16)
    v[:, ::3] *= np.float16(2.0) ** rng.integers(-12, 12, (n_seq, v[:, ::3].shape[1], 1)).astype(np.float16)
    return v


def _special_rows():
    rng = np.random.default_rng(9)
    r = rng.standard_normal((24, 64)).astype(np.float16)
    r[0] = 0
    r[1] = 1.5
    r[2] = -0.0
    r[3] = np.float16(6e-8) * rng.integers(0, 2, 64)          # subnormal: one step
    r[4] = np.float16(2.0 ** -24) * rng.integers(-20, 20, 64)
    r[5, 7] = np.nan
    r[6] = np.nan
    r[7, 3] = np.inf
    r[8, 3], r[8, 9] = -np.inf, np.inf
    r[9] = np.where(np.arange(64) % 2, 65504, -65504)
    r[10] = np.arange(64) % 16                                 # s = 1: exact
    r[11] = (np.arange(64) % 31) / 2                           # s = 1: ties
    r[12] = -(np.arange(64) % 31) / 2
    r[13, :] = np.nan
    r[13, 63] = 3.0
    r[14] = 65504
    r[15] = np.float16(1) + np.float16(2.0 ** -10) * (np.arange(64) % 3)
    return r[None]


def _store(v, t_cap, t0, fill=0xA5):
    n_seq, n_tok = v.shape[:2]
    cache = torch.full((n_seq, t_cap // 8, GROUP), fill, dtype=torch.uint8, device=DEV)
    pa.pot_store_values_int4(to_dev(v), n_seq, n_tok, t_cap, t0, cache)
    torch.cuda.synchronize()
    return cache


def _expected(v, t_cap, t0, fill=0xA5):
    n, s, z = quantise4(v)
    want = np.full((v.shape[0], t_cap // 8, GROUP), fill, np.uint8)
    place4(want, n, s, z, t0)
    return want


@pytest.mark.parametrize("n_seq,n_tok,t_cap,t0", RANGES)
def test_store_writes_the_defined_bytes_and_no_others(n_seq, n_tok, t_cap, t0):
    v = _rows(n_tok + t0, n_seq, n_tok)
    got = _store(v, t_cap, t0).cpu().numpy()
    assert np.array_equal(got, _expected(v, t_cap, t0))


@pytest.mark.parametrize("t0", [0, 5])
@pytest.mark.parametrize("repeat", [1, 200])
def test_store_of_special_rows(t0, repeat):
    v = np.ascontiguousarray(np.tile(_special_rows(), (1, repeat, 1)))
    t_cap = (v.shape[1] + t0 + 7) // 8 * 8
    got = take4(_store(v, t_cap, t0).cpu().numpy())[:, t0:t0 + v.shape[1]]
    n, s, z = quantise4(v)
    want = dequantise4(n, s, z)  # not the bytes: a minimum of 0 may have either sign
    assert np.isfinite(got).all()
    assert np.array_equal(got, want)
    finite = np.isfinite(v.astype(np.float64)).all(-1)
    err = np.abs(want - v.astype(np.float64))[finite]
    assert (err <= s.astype(np.float64)[finite][:, None] * 0.5 * (1 + 2.0 ** -20)).all()


@pytest.mark.parametrize("n_seq,n_tok,t_cap,t0", RANGES)
@pytest.mark.parametrize("fmt", ["fp16", "int8", "int4"])
def test_values_read_back(n_seq, n_tok, t_cap, t0, fmt):
    v = _rows(7 * n_tok + t0, n_seq, n_tok)
    rows = to_dev(v)
    out = torch.full((n_seq * n_tok * 64 + 64,), 7.0, dtype=torch.float16, device=DEV)
    if fmt == "int4":
        cache = _store(v, t_cap, t0, 0xFF)  # NaN steps and minima around the range
        pa.pot_load_values_int4(cache, n_seq, n_tok, t_cap, t0, out)
        want = dequantise4(*quantise4(v)).astype(np.float16)
    elif fmt == "int8":
        vu, ve = torch.full((n_seq, t_cap, 64), 9, dtype=torch.uint8, device=DEV), torch.full(
            (n_seq, t_cap), 3, dtype=torch.int8, device=DEV)
        pa.pot_store_values_int8(rows, n_seq, n_tok, t_cap, t0, vu, ve)
        pa.pot_load_values_int8(vu, ve, n_seq, n_tok, t_cap, t0, out)
        v8, g = oracle.quantize_values(v.view(np.uint16).reshape(-1, 64))
        want = (v8.astype(np.float64).reshape(v.shape) * 2.0 ** -g.astype(np.float64).reshape(n_seq, n_tok, 1)
                ).astype(np.float16)
    else:
        cache = torch.full((n_seq, t_cap, 64), float("nan"), dtype=torch.float16, device=DEV)
        pa.pot_store_values(rows, n_seq, n_tok, t_cap, t0, cache)
        pa.pot_load_values(cache, n_seq, n_tok, t_cap, t0, out)
        want = v
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    assert (got[-64:] == 7.0).all()
    # int4: z + s n is rounded to fp32 and then to fp16: off by a unit where that passes a tie
    got = got[:-64].reshape(v.shape).astype(np.float64)
    if fmt == "int4":
        exact = dequantise4(*quantise4(v))
        ulp = np.maximum(2.0 ** np.floor(np.log2(np.maximum(np.abs(exact), 2.0 ** -14))) * 2.0 ** -10, 2.0 ** -24)
        assert (np.abs(got - exact) <= ulp * (0.5 + 2.0 ** -12)).all()
    else:
        assert np.array_equal(got, want.astype(np.float64))


@pytest.mark.parametrize("k", [0, 1, 2, 3, 4])
@pytest.mark.parametrize("hadamard", [False, True])
@pytest.mark.parametrize("n_seq,n_tok,t_cap,t0", [(1, 1, 8, 3), (3, 17, 64, 3), (2, 333, 400, 21), (300, 1, 16, 9),
                                                  (2, 4100, 4104, 1)])
def test_keys_read_back(k, hadamard, n_seq, n_tok, t_cap, t0):
    rng = np.random.default_rng(k + n_tok)
    x = (rng.standard_normal((n_seq * t_cap, 64)) * rng.uniform(0.5, 4, 64)).astype(np.float16)
    x[:, 5] = 0
    x[::11] = 0
    x[3::11] *= np.float16(2.0 ** -10)
    se, cm, sc = oracle.encode_keys(x.view(np.uint16), mant_bits=k, hadamard=hadamard)
    out = torch.full((n_seq * n_tok * 64 + 64,), 7.0, dtype=torch.float16, device=DEV)
    fmt = pa.make_format(k, hadamard=hadamard)
    pa.pot_load_keys(fmt, to_dev(se), None if cm is None else to_dev(cm), to_dev(sc), n_seq, n_tok, t_cap, t0, out)
    torch.cuda.synchronize()
    got = out.cpu().numpy()
    assert (got[-64:] == 7.0).all()
    want = key_values(se, cm, sc, k)
    if hadamard:
        want = want @ sylvester() / 8
    size = np.sqrt((want ** 2).sum(-1, keepdims=True)).reshape(n_seq, t_cap, 1)[:, t0:t0 + n_tok]
    want = want.reshape(n_seq, t_cap, 64)[:, t0:t0 + n_tok]
    # half an fp16 unit, and the fp32 sums of 64 terms: 6 additions' half units of at most the row's size
    tol = np.maximum(np.abs(want) * 2.0 ** -11, 2.0 ** -25) * (1 + 2.0 ** -12) + (size * 6 * 2.0 ** -24 if hadamard else 0)
    assert (np.abs(got[:-64].reshape(n_seq, n_tok, 64).astype(np.float64) - want) <= tol).all()


def test_keys_read_back_of_caller_scales_and_odd_codes():
    """Zero codes stay 0 whatever the scale or the planes hold; scales of any size."""
    rng = np.random.default_rng(3)
    se = rng.integers(0, 256, (64, 32), dtype=np.uint8)
    cm = rng.integers(0, 256, (64, 16), dtype=np.uint8)
    sc = np.ones(64, np.float32)
    sc[:6] = [np.inf, 0, 1e-30, 65504, 3e38, 1.0 + 2.0 ** -20]
    for k, planes in ((0, None), (2, cm)):
        out = torch.empty((64, 64), dtype=torch.float16, device=DEV)
        pa.pot_load_keys(pa.make_format(k), to_dev(se), None if planes is None else to_dev(planes), to_dev(sc), 1, 64,
                         64, 0, out)
        got = out.cpu().numpy().astype(np.float64)
        want = key_values(se, planes, sc, k)
        zero = np.stack((se & 7, (se >> 4) & 7), -1).reshape(64, 64) == 7
        assert (got[zero] == 0).all()
        big = np.abs(want) >= 65520
        assert np.array_equal(got[big], np.sign(want[big]) * np.inf)
        assert (np.abs(got - want)[~big] <= np.maximum(np.abs(want[~big]) * 2.0 ** -11, 2.0 ** -25) * (1 + 2.0 ** -12)).all()


def test_offsets_past_4_gib():
    """The last sequence of caches whose byte offsets pass 2^32 (store, read-back of values and keys)."""
    n_seq, t_cap, t0, n_tok = 40, 4 << 20, (4 << 20) - 70, 67
    v = _rows(2, 1, n_tok)
    cache = torch.empty((n_seq, t_cap // 8, GROUP), dtype=torch.uint8, device=DEV)
    last = cache[-1:]
    last.fill_(0)
    all_rows = to_dev(np.ascontiguousarray(np.tile(v, (n_seq, 1, 1))))
    pa.pot_store_values_int4(all_rows, n_seq, n_tok, t_cap, t0, cache)
    out = torch.empty((n_seq, n_tok, 64), dtype=torch.float16, device=DEV)
    pa.pot_load_values_int4(cache, n_seq, n_tok, t_cap, t0, out)
    torch.cuda.synchronize()
    got = last[:, -10:].cpu().numpy()
    want = np.zeros_like(got)
    place4(want, *quantise4(v), 10)
    assert np.array_equal(got, want)
    assert torch.equal(out[0], out[-1])
    del cache, last
    se = torch.empty((n_seq * t_cap, 32), dtype=torch.uint8, device=DEV)
    sc = torch.empty(n_seq * t_cap, dtype=torch.float32, device=DEV)
    x = to_dev(_rows(5, 1, 70)[0])
    pa.pot_encode_keys(pa.make_format(), x, 70, 1, 0, sc[-70:], se[-70:])
    pa.pot_encode_keys(pa.make_format(), x, 70, 1, 0, sc[t_cap - 70:], se[t_cap - 70:])
    pa.pot_load_keys(pa.make_format(), se, None, sc, n_seq, n_tok, t_cap, t0, out)
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[-1])
    assert float(out[-1].abs().sum()) > 0
