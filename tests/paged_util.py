"""Paged caches for the tests, and attention over them in 64 bits from the definitions in include/pot_attn.h."""
from __future__ import annotations

import numpy as np
import torch

import oracle
import paper_2609_09208_amd as pa
from cache4_util import key_values

DEV = "cuda:0"
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "fp32": 0.0}


def pages_needed(lens, page):
    return [max(0, -(-int(n) // page)) for n in lens]


def make_table(rng, lens, page, spare=2, entries=None):
    """Page numbers in any order, -1 past each sequence's last page."""
    need = pages_needed(lens, page)
    n_pages = sum(need) + spare
    entries = entries or max(1, max(need))
    order = rng.permutation(n_pages)
    table = np.full((len(lens), entries), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, n_pages


def half_once(x):
    """fp64 numbers rounded to fp16 (numpy rounds a double to half once)."""
    with np.errstate(over="ignore"):
        return x.astype(np.float16).astype(np.float64)


class Pool:
    """A pool filled by the library's own encoder and stores, with every row of it random; host copies of what it stands for."""

    def __init__(self, rng, n_pages, Hkv, page, k=0, int4=False, hadamard=False, table=None, scale=1.0, v_scale=1.0):
        self.n_pages, self.Hkv, self.page, self.k, self.int4 = n_pages, Hkv, page, k, int4
        self.fmt = pa.make_format(mant_bits=k, hadamard=hadamard)
        self.table = np.asarray(table, np.int32)
        n_seq, rows = n_pages * Hkv, n_pages * Hkv * page
        chan = rng.uniform(0.5, 4, (Hkv, 1, 64)) * scale
        keys = (rng.standard_normal((n_pages, Hkv, page, 64)) * chan).astype(np.float16)
        vals = (rng.standard_normal((n_pages, Hkv, page, 64)) * v_scale).astype(np.float16)
        self.se, self.cm, self.sc, self.vals = pa.alloc_pages(n_pages, Hkv, page, k, DEV, int4)
        pa.pot_encode_keys(self.fmt, torch.from_numpy(keys).to(DEV), rows, 1, 0, self.sc, self.se, self.cm)
        store = pa.pot_store_values_int4 if int4 else pa.pot_store_values
        store(torch.from_numpy(vals).to(DEV), n_seq, page, page, 0, self.vals)
        self.pages = pa.make_pages(self.se, self.cm, self.sc, self.vals, torch.from_numpy(self.table).to(DEV))

    def keys_host(self):
        """fp64 [n_pages, Hkv, page, 64] in the domain that the codes hold."""
        rows = self.n_pages * self.Hkv * self.page
        cm = self.cm.cpu().numpy().reshape(rows, -1) if self.k else None
        x = key_values(self.se.cpu().numpy().reshape(rows, 32), cm, self.sc.cpu().numpy().reshape(rows), self.k)
        return x.reshape(self.n_pages, self.Hkv, self.page, 64)

    def values_host(self):
        v = self.vals.cpu().numpy()
        if not self.int4:
            v = v.reshape(self.n_pages, self.Hkv, self.page // 8, 64, 8)
            return np.swapaxes(v, -1, -2).reshape(self.n_pages, self.Hkv, self.page, 64).astype(np.float64)
        from cache4_util import take4
        with np.errstate(all="ignore"):
            v = take4(v.reshape(self.n_pages * self.Hkv, self.page // 8, 288))
            return half_once(v).reshape(self.n_pages, self.Hkv, self.page, 64)


def bounds_of(news):
    return np.concatenate(([0], np.cumsum(news))).astype(np.int32)


def attend_host(pool, q, news, lens, heads, window=0, n_sink=0, hadamard=False, cu=None):
    """fp64 O [n, Hq, 64] (NaN rows: not computed), and the largest |score| in the log2 domain of any seen key. q float32
    [n, Hq, 64]: as the kernels read it. Keys on pages outside the pool are not seen."""
    n, Hq, _ = q.shape
    kh, vh = pool.keys_host(), pool.values_host()
    qh, delta, _ = oracle.quantize_query(q.reshape(-1, 64), hadamard=hadamard)
    qd = (qh.astype(np.float64) * delta.astype(np.float64).reshape(-1, 1)).reshape(n, Hq, 64)
    out, top = np.full((n, Hq, 64), np.nan), 0.0
    cu = bounds_of(news) if cu is None else cu
    heads = np.asarray(heads)
    for b, L in enumerate(lens):
        first, count = int(cu[b]), int(cu[b + 1] - cu[b])
        t = np.arange(max(int(L), 0))
        entry = pool.table[b][t // pool.page] if len(t) else np.zeros(0, int)
        real = (entry >= 0) & (entry < pool.n_pages)
        p = np.where(real, entry, 0)
        for h in range(pool.Hkv):
            kd, vd = kh[p, h, t % pool.page], vh[p, h, t % pool.page]
            mine = np.nonzero(heads == h)[0]
            for i in range(count):
                at = L - count + i
                see = real & (t <= at)
                if window:
                    see &= (t > at - window) | (t < n_sink)
                if not see.any():
                    out[first + i, mine] = 0.0
                    continue
                with np.errstate(all="ignore"):
                    x = qd[first + i, mine] @ kd[see].T / 8
                    top = max(top, float(np.abs(x).max()) / np.log(2)) if np.isfinite(x).all() else top
                    w = np.exp(x - x.max(-1, keepdims=True))
                    out[first + i, mine] = w @ vd[see] / w.sum(-1, keepdims=True)
    return out, top


def attend_bound(want, top, vmax, T, out):
    """Bound on |O - O64|, T keys seen at most. A score is made with at most 6 roundings of half a unit (query step, log2 e,
    row scale's product, the difference from the reference, the last product and its sum): 6 2^-24 |x| in its exponent, ln 2 of
    that in a weight, twice (sums and denominator): under 2^-20 |x|. A weight's exp2 and its two fp16 parts: 2^-21 each, twice;
    fp32 sums of T terms in chains of at most T / 8 + 64: T 2^-27 + 2^-18. Outputs of 16 bits: the weights' one fp16 part, half a
    step of fp16 (d_i <= 2^-11 w_i) in both sums, so sum d_i (v_i - O) / sum w_i <= 2^-11 2 vmax; and the output's own half step,
    of a number that may be that much larger."""
    e = vmax * (top * 2.0 ** -20 + 2.0 ** -19 + T * 2.0 ** -27 + 2.0 ** -18)
    if out != "fp32":
        e = e + vmax * 2.0 ** -10
        e = e + (np.abs(want) + e) * HALF_STEP[out]
    return e


def run_attend(pool, q, news, lens, heads, out="fp32", window=0, n_sink=0, max_new=None, max_len=None, cu=None, fill=None,
               ws=None, stream=None):
    """pot_paged_attention on q (a device tensor); out starts as `fill`."""
    n, Hq, _ = q.shape
    cu = bounds_of(news) if cu is None else cu
    o = torch.full((n, Hq, 64), 7.5 if fill is None else fill, dtype=DTYPES[out], device=DEV)
    max_new = max_new or max(1, max(news))
    max_len = max_len or max(1, max(lens))
    if ws is None:
        nb = pa.pot_paged_workspace_bytes(len(lens), n, Hq, pool.Hkv, max_new, max_len)
        ws = torch.full((max(nb, 256),), 0xFF, dtype=torch.uint8, device=DEV)  # NaN, as far as it is read unwritten
    pa.pot_paged_attention(pool.fmt, q, pool.pages, torch.from_numpy(np.asarray(cu, np.int32)).to(DEV),
                           torch.from_numpy(np.asarray(lens, np.int32)).to(DEV), np.asarray(heads, np.int32), max_new, max_len,
                           o, ws, window=window, n_sink=n_sink, stream=stream)
    return o


def check_attend(pool, q, news, lens, heads, out="fp32", window=0, n_sink=0, hadamard=False, **over):
    got = run_attend(pool, q, news, lens, heads, out, window, n_sink, **over).double().cpu().numpy()
    want, top = attend_host(pool, q.float().cpu().numpy(), news, lens, heads, window, n_sink, hadamard, over.get("cu"))
    v = pool.values_host()
    vmax = float(np.abs(v[np.isfinite(v)]).max())
    seen = max(1, min(max(lens), window + n_sink if window else max(lens)))
    done = ~np.isnan(want).all((1, 2)) if len(want) else np.zeros(0, bool)
    fill = over.get("fill")
    assert (got[~done] == (7.5 if fill is None else fill)).all()  # rows of no sequence stay
    off = np.abs(got - want)[done]
    bound = attend_bound(want[done], top, vmax, seen, out)
    assert off.size == 0 or (off <= bound).all(), (float((off / bound).max()), np.unravel_index((off / bound).argmax(), off.shape))
    return got, want
