"""pot_paged_attention's sums over long caches: one key of a large weight, then very many of one small weight, each of which alone
is lost next to the large one in 32 bits."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from paged_util import DEV, DTYPES, HALF_STEP

pytestmark = pytest.mark.gpu

T, PAGE = 1 << 18, 64
# The large key's score in the log2 domain, the others' being 0: next to its weight the others are 0.45 of the fp32 numbers'
# distance there, 2^-23 of the weight.
SCORE = 23 - np.log2(0.45)


def _pool(v):
    key = torch.zeros((T, 64), dtype=torch.float16, device=DEV)
    key[0, 0] = SCORE * 8 * np.log(2)
    se, cm, sc, vals = pa.alloc_pages(T // PAGE, 1, PAGE, 0, DEV)
    fmt = pa.make_format()
    pa.pot_encode_keys(fmt, key, T, 1, 0, sc, se, cm)
    pa.pot_store_values(v, T // PAGE, PAGE, PAGE, 0, vals)
    assert float(sc[0, 0, 0]) == float(key[0, 0]) and float(sc[0, 0, 1]) == 0
    return fmt, se, cm, sc, vals, float(key[0, 0]) / 8  # the large key's score


@pytest.mark.parametrize("B,new,max_new", [(512, 17, 17), (512, 17, 129), (768, 1, 1), (512, 9, 9)])
@pytest.mark.parametrize("out", ["fp32", "fp16"])
def test_small_weights_next_to_a_large_one(B, new, max_new, out):
    """Sequences that share all their pages, as many as leave every row one key range (of the kernels of many rows and of few).
    Element 0 of the values is 1 everywhere, the others 1 except at the large key."""
    v = torch.ones((T // PAGE, PAGE, 64), dtype=torch.float16, device=DEV)
    v[0, 0, 1:] = 0
    fmt, se, cm, sc, vals, x = _pool(v)
    pages = pa.make_pages(se, cm, sc, vals, torch.arange(T // PAGE, dtype=torch.int32, device=DEV).repeat(B, 1))
    n = B * new
    q = torch.zeros((n, 1, 64), device=DEV)
    q[..., 0] = 1
    o = torch.full((n, 1, 64), 7.5, dtype=DTYPES[out], device=DEV)
    cu = torch.arange(B + 1, dtype=torch.int32, device=DEV) * new
    lens = torch.full((B,), T, dtype=torch.int32, device=DEV)
    ws = torch.full((max(256, pa.pot_paged_workspace_bytes(B, n, 1, 1, max_new, T)),), 0xFF, dtype=torch.uint8, device=DEV)
    pa.pot_paged_attention(fmt, q, pages, cu, lens, np.zeros(1, np.int32), max_new, T, o, ws)
    got = o.double().cpu().numpy().reshape(B, new, 64)
    small = np.exp(-x) * (T - new + np.arange(new))  # the others' weights, in parts of the large one's
    want = np.repeat((small / (1 + small))[:, None], 64, 1)
    want[:, 0] = 1
    # Relative: 6 2^-24 |log2 domain score| ln 2 of a weight's exponent; sums of T / 16 products (16 keys an instruction, with up to
    # 4 roundings each) and of T / 64 tiles, each rounded at half a step of the large weight: (T / 4 + T / 64 + 64) 2^-24. Absolute: a
    # small weight, 2^(7 - SCORE), is held in fp16's subnormal numbers, off by 2^-25, T of them against 2^7; and the same again for
    # outputs of 16 bits, whose denominator has the numbers as multiplied (no low part).
    e = 6 * 2.0 ** -24 * SCORE + (T / 4 + T / 64 + 64) * 2.0 ** -24
    e = e * want + 2 * T * 2.0 ** -25 / 2.0 ** 7
    e = e + (want + e) * HALF_STEP[out]
    off = np.abs(got - want[None])
    assert (off <= e).all(), (float((off / e).max()), off.max(), got[0, -1, :2], want[-1, :2])
    # element 0 alone: the same weights in both sums, whatever they are
    assert (np.abs(got[..., 0] - 1) <= (T / 4 + T / 64 + 64) * 2.0 ** -24 + HALF_STEP[out] + T * 2.0 ** -25 / 2.0 ** 7).all()
