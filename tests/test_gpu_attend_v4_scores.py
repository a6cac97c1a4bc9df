"""The scores of decode attention over 4-bit values, every bit of them: O of two keys whose scores are the same but for
half a unit in the log2 domain moves by far more than its tolerance when the integer score of one is off by one step."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_09208_amd as pa
from cache4_util import GROUP, key_values, place4, quantise4, take4
from parity_util import DEV, to_dev

pytestmark = pytest.mark.gpu

B, T, X0 = 24, 2, 2.0 ** 12


@pytest.mark.parametrize("frac_bits", [6, 7, 9, 12])
@pytest.mark.parametrize("k,engine", [(0, 0), (0, 1), (1, 0), (2, 0), (3, 0), (4, 0)])
@pytest.mark.parametrize("G", [1, 8])
def test_a_score_off_by_one_step_would_show(frac_bits, k, engine, G):
    rng = np.random.default_rng(100 * k + frac_bits)
    q = np.repeat(rng.standard_normal((B, 1, 64)), G, 1).astype(np.float32)
    qh, delta, _ = oracle.quantize_query(q)
    # rows of random codes; of 32 the two whose sums are smallest, where a step is the largest part of a sum
    n = B * 32
    se = rng.integers(0, 256, (n, 32), dtype=np.uint8)
    cm = rng.integers(0, 256, (n, 8 * k), dtype=np.uint8) if k else None
    w = key_values(se, cm, np.ones(n, np.float32), k).reshape(B, 32, 64)
    d = np.einsum("bd,btd->bt", qh[:, 0].astype(np.float64), w)
    at = np.argsort(np.where(np.abs(d) < 4, np.inf, np.abs(d)), 1)[:, :T]
    take = (np.arange(B)[:, None] * 32 + at).reshape(-1)
    d, se = d.reshape(-1)[take], se[take]
    cm = cm[take] if k else None
    se[d < 0] ^= 0x88
    d = np.abs(d).reshape(B, T)
    per = delta[:, 0].astype(np.float64)[:, None] / 8 / np.log(2)
    sc = ((X0 + np.array([0.0, 0.5])) / (d * per)).astype(np.float32)
    cap = 8
    codes = np.zeros((B, cap, 32), np.uint8)
    codes[:, :T] = se.reshape(B, T, 32)
    planes = np.zeros((B, cap, 8 * k), np.uint8)
    if k:
        planes[:, :T] = cm.reshape(B, T, 8 * k)
    scales = np.zeros((B, cap), np.float32)
    scales[:, :T] = sc
    v = np.zeros((B, T, 64), np.float16)
    v[:, 0], v[:, 1] = -1, 1
    v[:, :, ::2] += np.float16(0.25)
    cache = np.zeros((B, cap // 8, GROUP), np.uint8)
    place4(cache, *quantise4(v), 0)
    out = torch.full((B, G, 64), float("nan"), device=DEV)
    ws = pa.alloc_workspace(pa.pot_decode_workspace_bytes(B, G, 1, T), DEV)
    pa.pot_decode_attention_v4(pa.make_format(k, frac_bits), engine, to_dev(q), to_dev(codes), to_dev(planes) if k else None,
                               to_dev(scales), to_dev(cache), cap, None, np.zeros(G, np.int32), B, G, 1, T, out, ws)
    torch.cuda.synchronize()
    x = d * sc.astype(np.float64) * per
    p = np.exp2(x - x.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    values = take4(cache)[:, :T]
    want = np.einsum("bt,btd->bd", p, values)
    # x is a product of three roundings (2^-24 of X0 each, less the common one of the score factor: two a key) and the
    # sum in its exponent: X0 2^-24 5 ln 2 of a weight's ratio, of which p (1 - p) <= 1/4 reaches O times the values'
    # distance (2), and 2^-19 for the weights and sums
    tol = X0 * 2.0 ** -24 * 5 * np.log(2) / 4 * 2 + 2.0 ** -19
    err = np.abs(out.cpu().numpy() - want[:, None]).max()
    assert err <= tol, err / tol
    # what one step (2^-(6 + k) of an element's code times one step of q^) of the first key's sum would move
    x1 = x + np.array([2.0 ** -(6 + k), 0]) / d * X0
    p1 = np.exp2(x1 - x1.max(1, keepdims=True))
    p1 /= p1.sum(1, keepdims=True)
    moved = np.abs(np.einsum("bt,btd->bd", p1, values) - want).max(1)
    assert moved.min() > 10 * tol
