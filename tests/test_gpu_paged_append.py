"""pot_paged_append against the calls it combines (norm and rotation, key encoder) and the value records, bit for bit, with every
byte of the pool compared: rows that no token belongs to stay as they were."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from cache4_util import quantise4
from paged_util import DEV, DTYPES, bounds_of, make_table

pytestmark = pytest.mark.gpu


def _projection(rng, n, Hq, Hkv, dtype, packed, scale=1.0):
    x = rng.standard_normal((n, Hq + 2 * Hkv, 64)).astype(np.float32) * scale
    if packed:
        t = torch.from_numpy(x).to(DEV).to(dtype)
        return t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:]
    parts = np.split(x, [Hq, Hq + Hkv], 1)
    return [torch.from_numpy(np.ascontiguousarray(p.swapaxes(0, 1))).to(DEV).to(dtype).transpose(0, 1) for p in parts]


def _pool(rng, n_pages, Hkv, page, k, int4):
    """A pool of random bytes."""
    se, cm, sc, v = pa.alloc_pages(n_pages, Hkv, page, k, DEV, int4)
    for t in (se, cm, v):
        if t is not None:
            u = t.view(torch.uint8)
            u.copy_(torch.from_numpy(rng.integers(0, 256, tuple(u.shape), dtype=np.uint8)))
    sc.copy_(torch.from_numpy(rng.standard_normal(tuple(sc.shape)).astype(np.float32)))
    return se, cm, sc, v


def _host(pool):
    return [None if t is None else t.cpu().view(torch.uint8).numpy().copy() for t in pool]


def _combined(q, k, v, rope, qw, kw, eps, pos, freq, q_dtype, fmt):
    """The three calls: queries [n, Hq, 64], and per (kv head, row) codes, planes, scale and fp16 values."""
    n, Hkv = k.shape[:2]
    q_out = None if q is None else torch.empty((1, q.shape[1], n, 64), dtype=q_dtype, device=DEV)
    k_out, v_out = (torch.empty((1, Hkv, n, 64), dtype=torch.float16, device=DEV) for _ in range(2))
    pa.pot_norm_rope(rope, None if q is None else q[None], k[None], v[None], qw, kw, eps, pos, freq, q_out, k_out, v_out)
    rows = Hkv * n
    c = pa.alloc_pot_cache(1, Hkv, n, fmt.mant_bits, DEV)
    pa.pot_encode_keys(fmt, k_out, rows, 1, 0, c["key_scale"], c["codes_se"], c["codes_m"])
    return (None if q is None else q_out[0].transpose(0, 1).contiguous(), c["codes_se"][0], c["codes_m"] if c["codes_m"] is None
            else c["codes_m"][0], c["key_scale"][0], v_out[0])


def _expect(before, table, news, lens, cu, page, n_pages, got, int4):
    """The pool's bytes after the call, from those before."""
    se, cm, sc, v = (None if b is None else b.copy() for b in before)
    _, cse, ccm, csc, cv = got
    cse, csc, cv = cse.cpu().numpy(), csc.cpu().numpy(), cv.cpu().numpy()
    ccm = None if ccm is None else ccm.cpu().numpy()
    sc, v = sc.view(np.float32), v if int4 else v.view(np.float16)
    n_, s_, z_ = quantise4(cv) if int4 else (None, None, None)
    for b, L in enumerate(lens):
        count = int(cu[b + 1] - cu[b])
        for i in range(count):
            t, row = int(L) - count + i, int(cu[b]) + i
            if t < 0 or t // page >= table.shape[1]:
                continue
            p, u = table[b, t // page], t % page
            if not 0 <= p < n_pages:
                continue
            se[p, :, u], sc[p, :, u] = cse[:, row], csc[:, row]
            if cm is not None:
                cm[p, :, u] = ccm[:, row]
            for h in range(cv.shape[0]):
                if int4:
                    rec = v[p, h, u // 8]
                    c = np.arange(16)
                    for half in (0, 1):
                        lo, up = n_[h, row, 32 * half:32 * half + 16], n_[h, row, 32 * half + 16:32 * half + 32]
                        rec[16 * c + 8 * half + u % 8] = lo | (up << 4)
                    rec[256 + 2 * (u % 8):258 + 2 * (u % 8)] = np.atleast_1d(s_[h, row]).view(np.uint8)
                    rec[272 + 2 * (u % 8):274 + 2 * (u % 8)] = np.atleast_1d(z_[h, row]).view(np.uint8)
                else:
                    v[p, h].reshape(-1)[(u // 8) * 512 + 8 * np.arange(64) + u % 8] = cv[h, row]
    return se, cm, sc.view(np.uint8), v.view(np.uint8)


def _check(seed, news, lens, Hq, Hkv, page, k=0, int4=False, hadamard=False, dtype="bf16", q_out="fp32", packed=True, norm=True,
           rot_dim=64, neighbours=False, axes=1, positions=True, pad=0, first=0, table=None, n_pages=None, with_q=True, data=None):
    rng = np.random.default_rng(seed)
    cu = bounds_of(news) + first
    n = int(cu[-1]) + pad
    if table is None:
        table, n_pages = make_table(rng, lens, page)
    q, kk, v = _projection(rng, n, Hq, Hkv, DTYPES[dtype], packed) if data is None else data
    pairs = rot_dim // 2
    rope = pa.make_rope(rot_dim, neighbours, [i * axes // max(1, pairs) for i in range(pairs)])
    freq = torch.from_numpy(10000.0 ** (-np.arange(max(pairs, 1)) / max(pairs, 1))).to(DEV)
    place = np.zeros(n, np.int64)
    for b, L in enumerate(lens):
        m = int(cu[b + 1] - cu[b])
        place[cu[b]:cu[b + 1]] = int(L) - m + np.arange(m)
    pos = rng.integers(-5000, 1 << 20, (max(rope.n_axes, 1), n)) if positions else np.broadcast_to(place, (rope.n_axes, n))
    pos_t = torch.from_numpy(np.array(pos)).to(DEV)
    qw = kw = None
    if norm:
        qw, kw = (torch.from_numpy(rng.uniform(0.5, 1.5, 64).astype(np.float32)).to(DEV).to(DTYPES[dtype]) for _ in range(2))
    fmt = pa.make_format(mant_bits=k, hadamard=hadamard)
    pool = _pool(rng, n_pages, Hkv, page, k, int4)
    before = _host(pool)
    pages = pa.make_pages(*pool, torch.from_numpy(table).to(DEV))
    out = torch.full((n, Hq, 64), 3.25, dtype=DTYPES[q_out], device=DEV) if with_q else None
    pa.pot_paged_append(fmt, rope, q if with_q else None, kk, v, qw, kw, 1e-6, pos_t if positions else None, freq, pages,
                        torch.from_numpy(cu.astype(np.int32)).to(DEV), torch.from_numpy(np.asarray(lens, np.int32)).to(DEV), out)
    after = _host(pool)
    got = _combined(q if with_q else None, kk, v, rope, qw, kw, 1e-6, pos_t, freq, DTYPES[q_out], fmt)
    want = _expect(before, table, news, lens, cu, page, n_pages, got, int4)
    for name, a, w in zip(("codes", "planes", "scales", "values"), after, want):
        if w is not None:
            assert np.array_equal(a.reshape(w.shape), w), (name, np.argwhere(a.reshape(w.shape) != w)[:4])
    if with_q:
        inside = np.zeros(n, bool)
        inside[cu[0]:cu[-1]] = True
        o, w = out.cpu(), got[0].cpu()
        assert torch.equal(o[inside].view(torch.uint8), w[inside].view(torch.uint8))
        assert (o[~inside] == 3.25).all()


RAGGED = ([1, 5, 0, 17, 8, 3], [1, 9, 0, 40, 8, 130])


@pytest.mark.parametrize("int4", [False, True])
@pytest.mark.parametrize("k,hadamard", [(0, False), (1, True), (2, False), (3, True), (4, False)])
def test_formats(k, hadamard, int4):
    _check(1 + k, *RAGGED, 8, 2, 16, k=k, hadamard=hadamard, int4=int4)


@pytest.mark.parametrize("dtype,q_out", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp16"), ("fp32", "fp32"), ("fp16", "bf16")])
@pytest.mark.parametrize("rot_dim,neighbours", [(64, False), (64, True), (32, False), (48, True), (0, False), (2, False)])
def test_rotations_and_types(rot_dim, neighbours, dtype, q_out):
    _check(11, *RAGGED, 4, 2, 24, k=1, int4=True, dtype=dtype, q_out=q_out, rot_dim=rot_dim, neighbours=neighbours, axes=2,
           packed=dtype != "fp32", norm=rot_dim != 48)


@pytest.mark.parametrize("page", [8, 16, 40, 64, 1024])
@pytest.mark.parametrize("Hq,Hkv", [(32, 4), (7, 7), (16, 1), (1, 1), (12, 3)])
def test_pages_and_heads(page, Hq, Hkv):
    _check(21, *RAGGED, Hq, Hkv, page, int4=page != 16)


@pytest.mark.parametrize("int4", [False, True])
@pytest.mark.parametrize("case", [
    ([1], [1]), ([1], [100]), ([8], [8]), ([8], [16]), ([7], [1000]), ([1] * 70, list(range(1, 141, 2))), ([0, 0, 3], [5, 0, 3]),
    ([2] * 3, [2, 3, 9])])
def test_few_tokens(case, int4):
    _check(31, *case, 8, 2, 16, int4=int4, k=1)


@pytest.mark.parametrize("int4", [False, True])
@pytest.mark.parametrize("case", [
    ([1024], [1024]), ([1023, 1], [1023, 1]), ([1040], [2000]), ([500, 0, 600, 3], [501, 7, 600, 1003]), ([1] * 1100, [9] * 1100),
    ([37] * 40, [64] * 40), ([2047], [2049])])
@pytest.mark.parametrize("rot_dim,neighbours", [(64, False), (32, False), (64, True)])
def test_many_tokens(case, rot_dim, neighbours, int4):
    _check(41, *case, 4, 2, 32, int4=int4, k=2, hadamard=int4, rot_dim=rot_dim, neighbours=neighbours)


@pytest.mark.parametrize("news,lens", [([700, 400], [700, 555]), ([3, 1], [3, 20])])
def test_places_as_positions(news, lens):
    _check(51, news, lens, 4, 2, 16, positions=False, int4=True)


@pytest.mark.parametrize("news,lens", [([700, 400], [700, 555]), ([3, 0, 1], [3, 8, 20])])
def test_rows_of_no_sequence_stay(news, lens):
    _check(61, news, lens, 4, 2, 16, pad=13, first=5)


@pytest.mark.parametrize("news,lens", [([5, 3], [3, 3]), ([1200], [1000])])
def test_tokens_before_the_sequence_are_stored_nowhere(news, lens):
    _check(71, news, lens, 4, 2, 16, int4=True)


@pytest.mark.parametrize("many", [False, True])
def test_entries_that_are_no_pages(many):
    news, lens = ([1100, 30], [1100, 30]) if many else ([40, 30], [40, 30])
    rng = np.random.default_rng(5)
    table, n_pages = make_table(rng, lens, 16)
    table[0, 1], table[1, 0], table[0, 2] = n_pages, -7, 2 ** 31 - 1
    _check(81, news, lens, 4, 2, 16, table=table, n_pages=n_pages, int4=True, k=1)
    _check(82, news, lens, 4, 2, 16, table=table[:, :2].copy(), n_pages=n_pages)  # a table that is too short


def test_without_queries():
    _check(91, *RAGGED, 4, 2, 16, with_q=False)
    _check(92, [1500], [1600], 4, 2, 16, with_q=False, int4=True)


@pytest.mark.parametrize("n", [6, 1030])
@pytest.mark.parametrize("int4", [False, True])
def test_special_rows(n, int4):
    """Rows of zeros, infinities, NaN and equal elements (no norm, no rotation: they reach the codes)."""
    rng = np.random.default_rng(7)
    x = rng.standard_normal((n, 6, 64)).astype(np.float32)
    x[0, 2:] = 0
    x[1, 2:, 3] = np.inf
    x[2, 2:, 5] = np.nan
    x[3, 2:] = np.nan
    x[4, 2:] = -2.5
    x[5, 2:, 7] = -70000.0
    t = torch.from_numpy(x).to(DEV)
    _check(101, [n], [n], 2, 2, 16, int4=int4, dtype="fp32", norm=False, rot_dim=0, data=(t[:, :2], t[:, 2:4], t[:, 4:]))


def test_another_stream():
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _check(111, *RAGGED, 4, 2, 16, int4=True)
    torch.cuda.current_stream().wait_stream(s)
