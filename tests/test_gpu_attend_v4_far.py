"""Decode attention over 4-bit values at the ends of the scores' range, where fp32 holds them in steps of 2 to 256.

Keys whose codes are all +1 (or -1) give the log2-domain score +-s X_PER_S |q| of a caller's row scale s, so the scales
set every score. One key of a sequence stands further above the others than fp32's steps there, so its weight is all there
is and O is its value.
"""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from cache4_util import GROUP, place4, quantise4, take4
from parity_util import DEV, to_dev

pytestmark = pytest.mark.gpu

X_PER_S = 64 / 8 / np.log(2.0)  # log2-domain score of a key with scale 1 and a query of ones
POT_ENGINES = [(0, 0), (0, 1), (2, 0), (4, 0)]  # mantissa bits, engine


def _decode4(scales, negative, v, q, waves, k=0, engine=0, splits=1, lens=None):
    """O [B, 8, 64] and the cache's values [B, T, 64]; scales [B, T], v fp16 [B, T or 1, 64], q [B, 8] (a head's elements)."""
    B, T = scales.shape
    cap = -(-T // 8) * 8
    codes = np.zeros((B, cap, 32), np.uint8)
    codes[:, :T][negative] = 0x88
    planes = None if k == 0 else torch.zeros((B, cap, 8 * k), dtype=torch.uint8, device=DEV)
    sc = np.zeros((B, cap), np.float32)
    sc[:, :T] = scales
    cache = np.zeros((B, cap // 8, GROUP), np.uint8)
    if v.shape[1] == 1:  # every row the same
        place4(cache[:, :1], *quantise4(np.repeat(v, 8, 1)), 0)
        cache[:] = cache[:, :1]
    else:
        place4(cache, *quantise4(v), 0)
    out = torch.full((B, 8, 64), float("nan"), device=DEV)
    ws = pa.alloc_workspace(pa.pot_decode_workspace_bytes_for_splits(B, 8, 1, T, splits), DEV)
    dbg = pa.pot_debug()
    dbg.force_splits, dbg.force_wg_waves = splits, waves
    queries = to_dev(np.repeat(q.astype(np.float32)[..., None], 64, -1))
    pa.pot_decode_attention_v4(pa.make_format(k), engine, queries, to_dev(codes), planes, to_dev(sc), to_dev(cache), cap, lens,
                               np.zeros(8, np.int32), B, 8, 1, T, out, ws, dbg=dbg)
    torch.cuda.synchronize()
    return out.cpu().numpy().astype(np.float64), take4(cache[:, :1] if v.shape[1] == 1 else cache)[:, :T]


def _rows(rng, B, T):
    """Values whose steps go from fp16's smallest to large ones, constant rows among them."""
    v = rng.standard_normal((B, T, 64)) * 2.0 ** rng.integers(-16, 12, (B, T, 1))
    v[:, ::7] = v[:, ::7, :1]
    return v.astype(np.float16)


def _is_the_value(out, values, best):
    """One weight is left, an exact power of two but for exp2 (the score differences are integers there) that numerator
    and denominator share. p s is rounded (2^-24) and cut into two fp16 parts (2^-22) against |n - 8| <= 8; z + 8 s, its
    product, the sum and the quotient are off by 2^-24 each of at most |z| + 16 s."""
    for b, t in enumerate(best):
        want = values[b, t]
        size = np.abs(want).max() + 16 * (want.max() - want.min())
        err = np.abs(out[b] - want).max()
        assert err <= size * 2.0 ** -20, (b, t, err / size)


@pytest.mark.parametrize("e", [22, 24, 26, 27, 28, 29, 30])
@pytest.mark.parametrize("waves", [4, 16])
@pytest.mark.parametrize("splits", [1, 3])
def test_one_key_far_above_the_others(e, waves, splits):
    rng = np.random.default_rng(e)
    B, T = 64, 64 * waves * 2 + 37
    v, q = _rows(rng, B, T), rng.uniform(0.5, 1.0, (B, 8))
    best = rng.integers(0, T, B)
    best[:3] = [0, T - 1, 64 * waves + 5]
    # the best key's score is 2^e .. 2^(e + 1) for a query of ones, the others' at most half of it
    top = 2.0 ** rng.uniform(e, min(e + 1, 30.9), (B, 1)) / X_PER_S
    scales = top * rng.uniform(0.0, 0.5, (B, T))
    scales[np.arange(B), best] = top[:, 0]
    negative = rng.random((B, T)) < 0.3
    negative[np.arange(B), best] = False
    for k, engine in POT_ENGINES if splits == 1 else POT_ENGINES[:1]:
        w = 12 if waves == 16 and k == 4 else waves
        out, values = _decode4(scales, negative, v, q, w, k, engine, splits)
        _is_the_value(out, values, best)


@pytest.mark.parametrize("e", [20, 26, 28, 30])
@pytest.mark.parametrize("waves", [4, 16])
@pytest.mark.parametrize("splits", [1, 3])
def test_every_key_far_below_zero(e, waves, splits):
    rng = np.random.default_rng(e + 1)
    B, T = 32, 64 * waves * 2 + 21
    v, q = _rows(rng, B, T), rng.uniform(0.5, 1.0, (B, 8))
    best = rng.integers(0, T, B)
    top = 2.0 ** e / X_PER_S
    scales = top * rng.uniform(1.5, min(2.0, 2.0 ** (30.9 - e)), (B, T))
    scales[np.arange(B), best] = top
    out, values = _decode4(scales, np.ones((B, T), bool), v, q, waves, splits=splits)
    _is_the_value(out, values, best)


@pytest.mark.parametrize("waves", [4, 16])
def test_scores_at_minus_two_to_the_31(waves):
    """As for fp16 values: -2^31 is its own ceiling and the integer maximum's "none yet"."""
    step = np.float32(1) / np.float32(127)
    c = np.float32(np.float32(step * np.float32(1.44269502162933349609375)) * np.float32(2.0 ** -10))
    acc = np.float32(-64 * 127 * 128)
    s = np.float32(2.0 ** 31 / (64 * 127 * 128 * float(c)))
    near = (s.view(np.int32) + np.arange(-8, 9)).astype(np.int32).view(np.float32)
    x = (acc * near).astype(np.float32) * c
    s = near[x == np.float32(-2.0 ** 31)][0]
    rng = np.random.default_rng(6)
    T = 64 * waves * 2
    scales = np.full((1, T), s, np.float32)
    best = 64 * waves + 7
    scales[0, best] = 3.0 / X_PER_S
    v = rng.standard_normal((1, T, 64)).astype(np.float16)
    out, values = _decode4(scales, np.ones((1, T), bool), v, np.ones((1, 8)), waves)
    _is_the_value(out, values, [best])


@pytest.mark.parametrize("waves", [4, 16])
def test_constant_values_come_back(waves):
    """Each wave meets a large weight in its first tile and then only weights of 2^-18.3 of it. Numerator and denominator
    are fp32 sums of the same shape: a lane's 8 keys, then its tiles (T / 64 / waves), 8 lanes, the waves. Each of the N
    additions of a chain is off by half a unit of a sum, 2^-24, in either: 2 N 2^-24, and 8 units more for the products,
    the merge and the quotient."""
    T = 1 << 18
    scales = np.full((1, T), (40 - 12 - 18.3) / X_PER_S)
    scales[:, :waves * 64:64] = 39.99 / X_PER_S
    for value in (1.37 / 16, 1.37, -11.7):
        out, values = _decode4(scales, np.zeros((1, T), bool), np.full((1, 1, 64), value, np.float16), np.ones((1, 8)), waves)
        rel = np.abs(out / values[0, 0] - 1).max()
        print(f"waves={waves} |O / v - 1| {rel:.2e}")
        assert rel <= (2 * (8 + T / 64 / waves + 8 + waves) + 8) * 2.0 ** -24
