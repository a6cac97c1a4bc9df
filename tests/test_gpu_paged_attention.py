"""pot_paged_attention against the definition in 64 bits (tests/paged_util.py)."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from paged_util import DEV, DTYPES, Pool, attend_bound, attend_host, bounds_of, check_attend, make_table, run_attend

pytestmark = pytest.mark.gpu


def _queries(rng, n, Hq, dtype, packed=False):
    x = torch.from_numpy(rng.standard_normal((n, Hq + (3 if packed else 0), 64)).astype(np.float32)).to(DEV).to(DTYPES[dtype])
    return x[:, 1:Hq + 1] if packed else x


def _heads(Hq, Hkv, mixed=False):
    return np.arange(Hq, dtype=np.int32) % Hkv if mixed else np.arange(Hq, dtype=np.int32) // (Hq // Hkv)


def _check(seed, news, lens, Hq=8, Hkv=2, page=16, k=0, int4=False, hadamard=False, dtype="fp32", out="fp32", window=0, n_sink=0,
           mixed=False, packed=False, entries=None, poison=True, **over):
    rng = np.random.default_rng(seed)
    table, n_pages = make_table(rng, lens, page, entries=entries)
    pool = Pool(rng, n_pages, Hkv, page, k, int4, hadamard, table)
    if poison:
        _poison(pool, lens)
    q = _queries(rng, sum(news) + over.pop("pad", 0), Hq, dtype, packed)
    return check_attend(pool, q, news, lens, _heads(Hq, Hkv, mixed), out, window, n_sink, hadamard, **over)


def _poison(pool, lens):
    """NaN in every scale and value past the sequences' ends and on pages of none."""
    mine = np.zeros((pool.n_pages, pool.page), bool)
    for b, L in enumerate(lens):
        for t in range(int(L)):
            p = pool.table[b, t // pool.page]
            if 0 <= p < pool.n_pages:
                mine[p, t % pool.page] = True
    off = torch.from_numpy(~mine).to(DEV)
    pool.sc.masked_fill_(off[:, None], float("nan"))
    if pool.int4:
        sz = pool.vals[..., 256:].contiguous().view(torch.float16).view(pool.n_pages, pool.Hkv, -1, 2, 8)
        sz.masked_fill_(off.view(pool.n_pages, 1, -1, 1, 8), float("nan"))
        pool.vals[..., 256:] = sz.reshape(*sz.shape[:3], 16).view(torch.uint8)
    else:
        v = pool.vals.view(pool.n_pages, pool.Hkv, -1, 64, 8)
        v.masked_fill_(off.view(pool.n_pages, 1, -1, 1, 8), float("nan"))


# one token a sequence, drafts, chunks, and all of them in one call
SINGLES = ([1, 1, 1, 1, 1, 1, 0], [1, 2, 9, 64, 65, 300, 0])
DRAFTS = ([4, 2, 3, 4], [4, 70, 129, 1000])
CHUNK = ([100], [100])
LATE_CHUNK = ([77], [777])
CHUNKS = ([130, 64, 33], [130, 500, 33])
MIXED = ([1, 90, 0, 1, 5, 1], [300, 90, 50, 1, 200, 64])


@pytest.mark.parametrize("news,lens", [SINGLES, DRAFTS, CHUNK, LATE_CHUNK, CHUNKS, MIXED])
@pytest.mark.parametrize("int4", [False, True])
@pytest.mark.parametrize("k,hadamard", [(0, False), (1, True), (2, False), (3, False), (4, True)])
def test_formats(news, lens, int4, k, hadamard):
    _check(1, news, lens, k=k, int4=int4, hadamard=hadamard)


@pytest.mark.parametrize("news,lens", [SINGLES, LATE_CHUNK, MIXED])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("out", ["bf16", "fp16", "fp32"])
def test_types(news, lens, dtype, out):
    _check(2, news, lens, k=1, int4=True, dtype=dtype, out=out, packed=True)


@pytest.mark.parametrize("news,lens", [SINGLES, DRAFTS, CHUNKS, MIXED])
@pytest.mark.parametrize("Hq,Hkv", [(32, 4), (8, 8), (5, 1), (16, 1), (24, 4), (6, 2), (64, 2), (17, 1)])
def test_heads(news, lens, Hq, Hkv):
    _check(3, news, lens, Hq, Hkv, mixed=Hq == 24)


@pytest.mark.parametrize("news,lens", [SINGLES, DRAFTS, CHUNKS, MIXED])
@pytest.mark.parametrize("page", [8, 24, 32, 64, 72, 128, 1024])
def test_pages(news, lens, page):
    _check(4, news, lens, page=page, int4=page in (24, 128))


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 100, 1000])
@pytest.mark.parametrize("n_sink", [0, 1, 5, 64, 70])
@pytest.mark.parametrize("news,lens", [([1, 1, 1, 1], [1, 64, 200, 701]), ([3, 4], [66, 400]), ([150], [450]), MIXED])
def test_windows(news, lens, window, n_sink):
    _check(5, news, lens, int4=window == 64, window=window, n_sink=n_sink)


@pytest.mark.parametrize("news,lens", [([1], [1]), ([2], [2]), ([1], [63]), ([33], [33]), ([17], [17]), ([9], [8000]), ([1], [9000]),
                                       ([300], [3000]), ([1] * 40, [333] * 40), ([1, 200] * 9, [77, 200] * 9)])
def test_lengths(news, lens):
    _check(6, news, lens, page=64, k=0, int4=True, out="fp32")


@pytest.mark.parametrize("news,lens", [([5, 1, 40], [3, 0, 20]), ([2], [1])])
def test_rows_before_the_sequence_get_zeros(news, lens):
    got, want = _check(7, news, lens)
    assert (got[:news[0] - lens[0]] == 0).all()  # the first sequence's rows before it


@pytest.mark.parametrize("news", [[1, 1], [40, 1], [40, 40]])
def test_rows_of_no_sequence_stay(news):
    _check(8, news, [60, 70], pad=9, cu=bounds_of(news) + 4)


@pytest.mark.parametrize("news,lens", [SINGLES, LATE_CHUNK, MIXED])
def test_entries_that_are_no_pages(news, lens):
    """Holes, pages past the pool, and negative ones: their keys are not seen."""
    rng = np.random.default_rng(9)
    table, n_pages = make_table(rng, lens, 16)
    for b, L in enumerate(lens):
        for i in range(0, -(-L // 16), 3):
            table[b, i] = [-1, n_pages, 2 ** 31 - 1, -2 ** 31][i % 4]
    pool = Pool(rng, n_pages, 2, 16, 0, False, False, table)
    check_attend(pool, _queries(rng, sum(news), 8, "fp32"), news, lens, _heads(8, 2))


@pytest.mark.parametrize("news,lens", [([1, 3], [1000, 700]), ([120], [900])])
@pytest.mark.parametrize("int4", [False, True])
def test_pages_outside_the_window_are_not_needed(news, lens, int4):
    window, n_sink, page = 100, 4, 64
    rng = np.random.default_rng(10)
    table, n_pages = make_table(rng, lens, page)
    pool = Pool(rng, n_pages, 2, page, 0, int4, False, table)
    q = _queries(rng, sum(news), 8, "fp32")
    a = run_attend(pool, q, news, lens, _heads(8, 2), window=window, n_sink=n_sink)
    for b, (n, L) in enumerate(zip(news, lens)):
        low = L - n - window + 1
        for i in range(-(-L // page)):
            if (i + 1) * page <= low and i * page >= n_sink:
                table[b, i] = -1
    pool.pages = pa.make_pages(pool.se, pool.cm, pool.sc, pool.vals, torch.from_numpy(table).to(DEV))
    pool.table = table
    b = run_attend(pool, q, news, lens, _heads(8, 2), window=window, n_sink=n_sink)
    assert torch.equal(a, b)
    check_attend(pool, q, news, lens, _heads(8, 2), window=window, n_sink=n_sink)


@pytest.mark.parametrize("news,lens,window,n_sink", [([3], [200], 0, 0), ([1, 4], [130, 90], 50, 3), ([100], [300], 0, 0),
                                                     ([120], [300], 70, 2), ([20, 1, 64], [50, 80, 64], 0, 0)])
@pytest.mark.parametrize("out", ["fp32", "bf16"])
def test_special_values_stay_where_they_are_seen(news, lens, window, n_sink, out):
    """Infinite and NaN values (fp16 cache) and NaN scales at single keys: outputs of queries that see them are infinite or NaN
    in those elements, and all others are what the definition says."""
    rng = np.random.default_rng(11)
    table, n_pages = make_table(rng, lens, 16)
    pool = Pool(rng, n_pages, 2, 16, 0, False, False, table)
    v = pool.vals.view(n_pages, 2, 2, 64, 8)
    for b, L in enumerate(lens):
        for t, d, x in [(L - 1, 3, np.inf), (L - 2, 4, -np.inf), (L - 1, 5, np.nan), (L - 2, 6, np.inf), (L - 1, 6, -np.inf),
                        (L // 2, 40, np.inf), (1, 63, np.nan)]:
            p, u = table[b, t // 16], t % 16
            v[p, :, u // 8, d, u % 8] = float(x)
        t = L - 3
        pool.sc[table[b, t // 16], 1, t % 16] = float("nan")
    q = _queries(rng, sum(news), 8, "fp32")
    got = run_attend(pool, q, news, lens, _heads(8, 2), out, window, n_sink).double().cpu().numpy()
    with np.errstate(all="ignore"):
        want, top = attend_host(pool, q.cpu().numpy(), news, lens, _heads(8, 2), window, n_sink)
    ok = np.isfinite(want)
    assert not ok.all() and ok.any() and np.array_equal(np.isfinite(got), ok)
    assert (np.abs(got - want)[ok] <= attend_bound(want[ok], top, 7.0, max(lens), out)).all()


@pytest.mark.parametrize("news,lens", [([1, 2], [300, 80]), ([70], [300])])
@pytest.mark.parametrize("scale", [1e-4, 30.0, 3000.0])
def test_score_sizes(news, lens, scale):
    """Flat weights, and weights of one key. The bound grows with the scores: past 2^20 it says nothing, so the outputs are held
    to the values' range there."""
    rng = np.random.default_rng(12)
    table, n_pages = make_table(rng, lens, 16)
    pool = Pool(rng, n_pages, 2, 16, 2, False, False, table, scale=scale)
    q = _queries(rng, sum(news), 8, "fp32") * 1.0
    got, want = check_attend(pool, q, news, lens, _heads(8, 2))
    assert np.isfinite(got).all()


@pytest.mark.parametrize("news,lens", [([1, 2], [300, 80]), ([70], [300])])
def test_far_scores(news, lens):
    """Scores past 2^24 and up to about 2^40: one key has all of the weight, and its value is the output."""
    rng = np.random.default_rng(13)
    table, n_pages = make_table(rng, lens, 16)
    pool = Pool(rng, n_pages, 1, 16, 0, False, False, table, scale=1000.0)
    for mul in (1e4, 1e8):
        q = _queries(rng, sum(news), 4, "fp32") * mul
        got = run_attend(pool, q, news, lens, _heads(4, 1)).double().cpu().numpy()
        want, top = attend_host(pool, q.cpu().numpy(), news, lens, _heads(4, 1))
        assert top > 2.0 ** 24 and np.isfinite(got).all()
        # of keys with scores that differ by less than the scores' own roundings any may be the one
        near = np.abs(got - want).max(-1) < 1e-5
        assert near.mean() > 0.99


@pytest.mark.parametrize("news,lens", [([1, 2], [300, 80]), ([70], [300])])
def test_queries_of_zeros_and_equal_keys(news, lens):
    rng = np.random.default_rng(14)
    table, n_pages = make_table(rng, lens, 16)
    pool = Pool(rng, n_pages, 2, 16, 1, True, False, table)
    q = _queries(rng, sum(news), 8, "fp32")
    q[:, ::2] = 0
    check_attend(pool, q, news, lens, _heads(8, 2))
    pool.se.fill_(0)
    pool.cm.fill_(0)
    check_attend(pool, q, news, lens, _heads(8, 2))


@pytest.mark.parametrize("news,lens", [SINGLES, ([150, 1], [400, 30])])
def test_constant_values_come_back(news, lens):
    """All values v: every output is v to the sums' rounding, whatever the weights."""
    rng = np.random.default_rng(15)
    table, n_pages = make_table(rng, lens, 16)
    pool = Pool(rng, n_pages, 2, 16, 0, False, False, table)
    pool.vals.fill_(1.5)
    got = run_attend(pool, _queries(rng, sum(news), 8, "fp32"), news, lens, _heads(8, 2)).cpu()
    keys = torch.from_numpy(np.repeat(np.asarray(lens), np.asarray(news)) > 0)
    assert ((got[keys] - 1.5).abs() <= 1.5 * 2.0 ** -17).all()


def test_a_token_is_what_the_decode_call_says():
    """The same caches read by pot_decode_attention_v4 (values z + s n unrounded there: 2^-11 of the largest apart)."""
    rng = np.random.default_rng(16)
    B, Hq, Hkv, T, cap = 3, 32, 4, 200, 208
    fmt = pa.make_format(mant_bits=1)
    keys = torch.from_numpy(rng.standard_normal((B, Hkv, cap, 64)).astype(np.float16)).to(DEV)
    vals = torch.from_numpy(rng.standard_normal((B, Hkv, cap, 64)).astype(np.float16)).to(DEV)
    se, cm, sc, v4 = pa.alloc_pages(B, Hkv, cap, 1, DEV, True)
    pa.pot_encode_keys(fmt, keys, B * Hkv * cap, 1, 0, sc, se, cm)
    pa.pot_store_values_int4(vals, B * Hkv, cap, cap, 0, v4)
    q = torch.from_numpy(rng.standard_normal((B, Hq, 64)).astype(np.float32)).to(DEV)
    lens = torch.tensor([200, 1, 77], dtype=torch.int32, device=DEV)
    a, b = torch.empty_like(q), torch.empty_like(q)
    ws = pa.alloc_workspace(pa.pot_decode_workspace_bytes(B, Hq, Hkv, T), DEV)
    pa.pot_decode_attention_v4(fmt, 0, q, se, cm, sc, v4, cap, lens, _heads(Hq, Hkv), B, Hq, Hkv, T, a, ws)
    pages = pa.make_pages(se, cm, sc, v4, torch.arange(B, dtype=torch.int32, device=DEV)[:, None].contiguous())
    ws = pa.alloc_workspace(pa.pot_paged_workspace_bytes(B, B, Hq, Hkv, 1, T), DEV)
    pa.pot_paged_attention(fmt, q, pages, torch.arange(B + 1, dtype=torch.int32, device=DEV), lens, _heads(Hq, Hkv), 1, T, b, ws)
    vmax = float(vals.abs().max())
    assert ((a - b).abs() <= vmax * (2.0 ** -11 + 2.0 ** -16)).all()


def test_results_do_not_differ():
    rng = np.random.default_rng(17)
    news, lens = [1, 300, 1, 64], [5000, 3000, 900, 64]
    table, n_pages = make_table(rng, lens, 32)
    pool = Pool(rng, n_pages, 2, 32, 0, True, False, table)
    q = _queries(rng, sum(news), 8, "bf16")
    first = run_attend(pool, q, news, lens, _heads(8, 2), "bf16")
    for _ in range(5):
        assert torch.equal(first, run_attend(pool, q, news, lens, _heads(8, 2), "bf16"))


def test_more_sequences_than_a_wave():
    """Several hundred sequences of few and many rows."""
    rng = np.random.default_rng(18)
    news = [int(x) for x in rng.choice([0, 1, 2, 5, 9], 300)]
    lens = [int(n + rng.integers(0, 60)) for n in news]
    _check(19, news, lens, 8, 1, page=8)


def test_replayed_on_new_inputs():
    """A captured call with room for more rows and longer sequences than the replays bring."""
    rng = np.random.default_rng(20)
    B, n, Hq, Hkv, page, T = 3, 80, 8, 2, 16, 512
    lens_max = [T] * B
    table, n_pages = make_table(rng, lens_max, page)
    pool = Pool(rng, n_pages, Hkv, page, 0, True, False, table)
    heads = _heads(Hq, Hkv)
    q = torch.zeros((n, Hq, 64), device=DEV)
    out = torch.zeros_like(q)
    cu, lens = (torch.zeros(m, dtype=torch.int32, device=DEV) for m in (B + 1, B))
    ws = pa.alloc_workspace(pa.pot_paged_workspace_bytes(B, n, Hq, Hkv, 64, T), DEV)
    call = lambda: pa.pot_paged_attention(pool.fmt, q, pool.pages, cu, lens, heads, 64, T, out, ws)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for news, ls in [([1, 1, 1], [400, 1, 512]), ([64, 10, 1], [64, 300, 500]), ([0, 0, 0], [0, 0, 0]), ([2, 40, 38], [2, 40, 300])]:
        m = sum(news)
        x = rng.standard_normal((n, Hq, 64)).astype(np.float32)
        q.copy_(torch.from_numpy(x))
        cu.copy_(torch.from_numpy(bounds_of(news)))
        lens.copy_(torch.tensor(ls, dtype=torch.int32))
        out.fill_(7.5)
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and (got[m:] == 7.5).all()
        eager, _ = check_attend(pool, q[:m].contiguous(), news, ls, heads, max_new=64, max_len=T) if m else (None, None)
