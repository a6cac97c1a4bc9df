"""Maxima of waves and splits whose difference passes 2^31, in every value format: the sums below leave the result instead
of coming back with a factor of 2^(the difference's low 32 bits)."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_09208_amd as pa
from parity_util import DEV, store_values, to_dev
from test_gpu_attend_v4_far import X_PER_S, _decode4, _is_the_value, _rows

pytestmark = pytest.mark.gpu

LOW = 2.0 ** 31 - 2.0 ** 12


def _decode(kind, scales, negative, v, waves, splits):
    """O [8, 64] of one sequence over fp16 values, INT8 values, or those with power-of-two weights; v fp16 [T, 64]."""
    T = scales.size
    codes = np.zeros((T, 32), np.uint8)
    codes[negative] = 0x88
    q = torch.ones((1, 8, 64), device=DEV)
    out = torch.full((1, 8, 64), float("nan"), device=DEV)
    ws = pa.alloc_workspace(pa.pot_decode_workspace_bytes_for_splits(1, 8, 1, T, splits), DEV)
    dbg = pa.pot_debug()
    dbg.force_splits, dbg.force_wg_waves = splits, waves
    head, tail = (to_dev(codes), None, to_dev(scales)), (T, np.zeros(8, np.int32), 1, 8, 1, T, out, ws)
    if kind == "fp16":
        pa.pot_decode_attention(pa.make_format(), q, *head, store_values(v.view(np.uint16), 1, 1, T), *tail, dbg=dbg)
    else:
        vu, ve = pa.alloc_value_cache_int8(1, 1, T, DEV)
        pa.pot_store_values_int8(to_dev(v), 1, T, T, 0, vu, ve)
        call = pa.pot_decode_attention_v8 if kind == "int8" else pa.pot_decode_attention_v8_pow2
        call(pa.make_format(), 0, q, *head, vu, ve, *tail, dbg=dbg)
    torch.cuda.synchronize()
    return out.cpu().numpy()[0].astype(np.float64)


@pytest.mark.parametrize("kind", ["fp16", "int8", "pow2"])
@pytest.mark.parametrize("waves", [4, 16])
@pytest.mark.parametrize("splits", [1, 3, 70])
@pytest.mark.parametrize("best_x", [2.0 ** 13, 2.0 ** 30])
def test_one_key_far_above_the_others(kind, waves, splits, best_x):
    rng = np.random.default_rng(7)
    T = 64 * waves * 2 if splits < 70 else 70 * 256
    v = rng.standard_normal((T, 64)).astype(np.float16)
    vh, g = oracle.quantize_values(v.view(np.uint16))
    for best in (0, 64 * waves + 7, T - 1):
        scales = np.full(T, LOW / X_PER_S, np.float32)
        negative = np.ones(T, bool)
        scales[best], negative[best] = best_x / X_PER_S, False
        out = _decode(kind, scales, negative, v, waves, splits)
        want = v[best].astype(np.float64) if kind == "fp16" else vh[best].astype(np.float64) * 2.0 ** -float(g[best])
        # one weight is left, the same in both sums: its parts are off by 2^-22, sums and quotient by 2^-24 each
        assert np.abs(out - want).max() <= np.abs(want).max() * 2.0 ** -20


@pytest.mark.parametrize("waves", [4, 16])
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("best_x", [3.0, 2.0 ** 13, 2.0 ** 20, 2.0 ** 30])
def test_one_key_far_above_the_others_over_4_bit_values(waves, splits, best_x):
    rng = np.random.default_rng(5)
    B, T = 16, 64 * waves * 2
    v, q = _rows(rng, B, T), np.ones((B, 8))
    scales = np.full((B, T), LOW / X_PER_S)
    best = rng.integers(0, T, B)
    best[:2] = [0, 64 * waves + 7]
    negative = np.ones((B, T), bool)
    scales[np.arange(B), best] = best_x / X_PER_S
    negative[np.arange(B), best] = False
    out, values = _decode4(scales, negative, v, q, waves, splits=splits)
    _is_the_value(out, values, best)
