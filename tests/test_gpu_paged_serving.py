"""pot_paged_append and pot_paged_attention together, as a server calls them: prompts in chunks, then tokens, then graphs of both;
and where the attention's kernels and key ranges meet."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from paged_util import DEV, DTYPES, Pool, attend_bound, attend_host, bounds_of, check_attend, make_table, run_attend

pytestmark = pytest.mark.gpu


def _heads(Hq, Hkv):
    return np.arange(Hq, dtype=np.int32) // (Hq // Hkv)


def _dev(x, dtype=torch.int32):
    return torch.from_numpy(np.asarray(x)).to(DEV).to(dtype)


class Server:
    """Pages, weights and the two calls for steps of (sequence, new tokens); all tokens' projections are drawn once."""

    def __init__(self, seed, totals, Hq=8, Hkv=2, page=16, k=0, int4=False, hadamard=False, dtype="fp32", out="fp32", window=0,
                 n_sink=0):
        rng = np.random.default_rng(seed)
        self.Hq, self.Hkv, self.out, self.window, self.n_sink = Hq, Hkv, out, window, n_sink
        self.totals, self.heads, self.lens = totals, _heads(Hq, Hkv), [0] * len(totals)
        table, n_pages = make_table(rng, totals, page)
        self.pool = Pool(rng, n_pages, Hkv, page, k, int4, hadamard, table)
        self.rope = pa.make_rope(64)
        self.freq = torch.from_numpy(10000.0 ** (-np.arange(32) / 32)).to(DEV)
        self.x = [torch.from_numpy(rng.standard_normal((n, Hq + 2 * Hkv, 64)).astype(np.float32)).to(DEV).to(DTYPES[dtype])
                  for n in totals]
        self.w = [torch.from_numpy(rng.uniform(0.5, 1.5, 64).astype(np.float32)).to(DEV).to(DTYPES[dtype]) for _ in range(2)]

    def calls(self, x, cu, lens, q, o, ws, max_new, max_len, stream=None):
        Hq, Hkv = self.Hq, self.Hkv
        pa.pot_paged_append(self.pool.fmt, self.rope, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], *self.w, 1e-6, None,
                            self.freq, self.pool.pages, cu, lens, q, stream=stream)
        pa.pot_paged_attention(self.pool.fmt, q, self.pool.pages, cu, lens, self.heads, max_new, max_len, o, ws,
                               window=self.window, n_sink=self.n_sink, stream=stream)

    def rows(self, news):
        x = torch.cat([self.x[b][self.lens[b]:self.lens[b] + m] for b, m in enumerate(news)])
        self.lens = [a + m for a, m in zip(self.lens, news)]
        return x

    def step(self, news, stream=None):
        """Outputs [sum(news), Hq, 64] and the queries that the attention read."""
        x, n = self.rows(news), sum(news)
        q, o = (torch.full((n, self.Hq, 64), 7.5, dtype=DTYPES[self.out], device=DEV) for _ in range(2))
        B, T = len(news), max(self.lens)
        ws = torch.full((max(256, pa.pot_paged_workspace_bytes(B, n, self.Hq, self.Hkv, max(news), T)),), 0xFF,
                        dtype=torch.uint8, device=DEV)
        cu, lens = _dev(bounds_of(news)), _dev(self.lens)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.calls(x, cu, lens, q, o, ws, max(news), T, stream)
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
        torch.cuda.synchronize()
        return o, q

    def check(self, news, lens, o, q):
        want, top = attend_host(self.pool, q.float().cpu().numpy(), news, lens, self.heads, self.window, self.n_sink,
                                bool(self.pool.fmt.hadamard))
        v = self.pool.values_host()
        bound = attend_bound(want, top, float(np.abs(v).max()), max(lens), self.out)
        assert (np.abs(o.double().cpu().numpy() - want) <= bound).all()


STEPS = [[40, 0, 7], [1, 130, 1], [64, 1, 1], [1, 1, 1], [1, 1, 1], [3, 2, 4]]
FORMS = [dict(), dict(k=2, int4=True, page=8), dict(k=4, hadamard=True, window=50, n_sink=3), dict(int4=True, page=64, window=17),
         dict(k=1, dtype="bf16", out="bf16"), dict(Hq=12, Hkv=3, int4=True, dtype="fp16", out="fp16")]


@pytest.mark.parametrize("form", FORMS)
def test_prompts_in_chunks_and_tokens(form):
    """Every step against the definition on the pool as it then stands; and the pool in the end as one call fills it."""
    totals = [sum(s[b] for s in STEPS) for b in range(3)]
    a, b = Server(1, totals, **form), Server(1, totals, **form)
    outs = []
    for news in STEPS:
        o, q = a.step(news)
        a.check(news, a.lens, o, q)
        outs.append(o)
    whole, q = b.step(totals)
    b.check(totals, totals, whole, q)
    for got, want in zip((a.pool.se, a.pool.cm, a.pool.sc, a.pool.vals), (b.pool.se, b.pool.cm, b.pool.sc, b.pool.vals)):
        assert got is None or torch.equal(got, want)


def test_on_another_stream():
    totals = [120, 60, 33]
    a, b = Server(2, totals, int4=True), Server(2, totals, int4=True)
    side = torch.cuda.Stream()
    for news in ([100, 50, 1], [19, 9, 31], [1, 1, 1]):
        (x, _), (y, _) = a.step(news), b.step(news, side)
        assert torch.equal(x, y)


def test_two_graphs_share_workspace_and_pages():
    """Graphs of both calls for steps of tokens and for chunks, with padded rows, one workspace; eager calls in between."""
    totals = [400, 400, 400]
    a, b = Server(3, totals, Hq=16, k=1, int4=True), Server(3, totals, Hq=16, k=1, int4=True)
    T, made = 400, []
    ws = pa.alloc_workspace(max(pa.pot_paged_workspace_bytes(3, n, 16, 2, m, T) for n, m in ((4, 1), (256, 130))), DEV)
    for n, most in ((4, 1), (256, 130)):
        x = torch.zeros((n, 20, 64), device=DEV)
        q, o = (torch.zeros((n, 16, 64), device=DEV) for _ in range(2))
        cu, lens = (torch.zeros(m, dtype=torch.int32, device=DEV) for m in (4, 3))
        call = lambda x=x, cu=cu, lens=lens, q=q, o=o, most=most: b.calls(x, cu, lens, q, o, ws, most, T)  # noqa: E731
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        made.append((g, x, cu, lens, q, o))
    for news in ([130, 100, 3], [1, 1, 1], [1, 0, 1], [64, 130, 20], [1, 1, 1], [0, 0, 1]):
        want, read = a.step(news)
        g, x, cu, lens, q, o = made[0 if max(news) == 1 else 1]
        rows = b.rows(news)
        x.fill_(float("nan"))
        x[:len(rows)] = rows
        cu.copy_(_dev(bounds_of(news)))
        lens.copy_(_dev(b.lens))
        o.fill_(7.5)
        q.fill_(7.5)
        g.replay()
        torch.cuda.synchronize()
        m = len(rows)  # room for more rows and keys may take other key ranges: the definition for both
        a.check(news, a.lens, want, read)
        b.check(news, b.lens, o[:m], q[:m])
        assert torch.equal(read, q[:m])
        assert (o[m:] == 7.5).all() and (q[m:] == 7.5).all()
        again = torch.empty_like(o).fill_(7.5)
        pa.pot_paged_attention(b.pool.fmt, q, b.pool.pages, cu, lens, b.heads, 1 if max(news) == 1 else 130, T, again, ws)
        torch.cuda.synchronize()
        assert torch.equal(again, o)
    for x, y in zip((a.pool.se, a.pool.cm, a.pool.sc, a.pool.vals), (b.pool.se, b.pool.cm, b.pool.sc, b.pool.vals)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv", [(8, 1), (8, 2), (9, 3), (5, 1), (16, 1), (32, 4)])
def test_between_the_kernels(Hq, Hkv, out):
    """Sequences of 1 to 20 tokens beside a chunk, and without one: rows up to 8, up to 16 and more in one call."""
    for seed, news in ((4, [1, 2, 3, 1, 40]), (5, [1, 2, 1, 2]), (6, [1, 1, 1]), (7, [1, 4, 0, 3, 20])):
        rng = np.random.default_rng(seed)
        lens = [n + int(x) for n, x in zip(news, rng.integers(0, 400, len(news)))]
        table, n_pages = make_table(rng, lens, 16)
        pool = Pool(rng, n_pages, Hkv, 16, 1, bool(seed % 2), False, table)
        q = torch.from_numpy(rng.standard_normal((sum(news), Hq, 64)).astype(np.float32)).to(DEV)
        check_attend(pool, q, news, lens, _heads(Hq, Hkv), out)


@pytest.mark.parametrize("news,lens", [([200, 40, 17], [6000, 700, 17]), ([300], [5000]), ([257, 256], [3000, 256]),
                                       ([3] * 70 + [60], [40] * 70 + [4000]), ([129, 1], [8000, 8000])])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (700, 5)])
def test_key_ranges_of_chunks(news, lens, window, n_sink):
    """Rows whose keys are shared out among pieces, beside sequences that are not."""
    rng = np.random.default_rng(8)
    table, n_pages = make_table(rng, lens, 32)
    pool = Pool(rng, n_pages, 1, 32, 0, True, False, table)
    q = torch.from_numpy(rng.standard_normal((sum(news), 8, 64)).astype(np.float32)).to(DEV)
    check_attend(pool, q, news, lens, _heads(8, 1), "fp32", window, n_sink)


@pytest.mark.parametrize("news", [[1, 1, 1], [3, 70, 1]])
def test_strided_queries(news):
    rng = np.random.default_rng(9)
    lens = [300, 200, 90]
    table, n_pages = make_table(rng, lens, 8)
    pool = Pool(rng, n_pages, 2, 8, 3, False, True, table)
    wide = torch.from_numpy(rng.standard_normal((sum(news), 20, 64)).astype(np.float32)).to(DEV)
    by_head = torch.from_numpy(rng.standard_normal((8, sum(news), 64)).astype(np.float32)).to(DEV)
    for q in (wide[:, 4:12], wide[:, ::2][:, :8], by_head.transpose(0, 1)):
        assert torch.equal(run_attend(pool, q, news, lens, _heads(8, 2)), run_attend(pool, q.contiguous(), news, lens, _heads(8, 2)))


@pytest.mark.parametrize("int4", [False, True])
def test_pages_past_32_bits(int4):
    """A pool whose values' and codes' bytes pass 2^32: its last pages give what a small pool of the same pages gives."""
    rng = np.random.default_rng(10)
    Hq, Hkv, page, news, lens = 16, 2, 64, [1, 90, 2], [500, 300, 130]
    n_big = (1 << 32) // (Hkv * page * 32) + 40  # 32 bytes of codes a row; 36 or 128 of values
    table, n_pages = make_table(rng, lens, page)
    small = Pool(rng, n_pages, Hkv, page, 0, int4, False, table)
    se, cm, sc, v = (torch.empty((n_big, *t.shape[1:]), dtype=t.dtype, device=DEV) if t is not None else None
                     for t in (small.se, small.cm, small.sc, small.vals))
    for big, t in ((se, small.se), (sc, small.sc), (v, small.vals)):
        big[n_big - n_pages:] = t
    far = np.where(table >= 0, table + n_big - n_pages, -1).astype(np.int32)
    pages = pa.make_pages(se, cm, sc, v, torch.from_numpy(far).to(DEV))
    n, heads = sum(news), _heads(Hq, Hkv)
    x = torch.from_numpy(rng.standard_normal((n, Hq + 2 * Hkv, 64)).astype(np.float32)).to(DEV)
    cu, ls = _dev(bounds_of(news)), _dev(lens)
    freq = torch.from_numpy(10000.0 ** (-np.arange(32) / 32)).to(DEV)
    ws = pa.alloc_workspace(pa.pot_paged_workspace_bytes(3, n, Hq, Hkv, 90, 500), DEV)
    got = []
    for p in (small.pages, pages):
        q, o = (torch.empty((n, Hq, 64), device=DEV) for _ in range(2))
        pa.pot_paged_append(small.fmt, pa.make_rope(64), x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], None, None, 1e-6, None,
                            freq, p, cu, ls, q)
        pa.pot_paged_attention(small.fmt, q, p, cu, ls, heads, 90, 500, o, ws)
        torch.cuda.synchronize()
        got.append(o)
    assert torch.equal(*got) and bool(torch.isfinite(got[0]).all())
    for big, t in ((se, small.se), (sc, small.sc), (v, small.vals)):
        assert torch.equal(big[n_big - n_pages:].view(torch.uint8), t.view(torch.uint8))


@pytest.mark.parametrize("B,n,cu", [(41, 300, [0, 300] * 21), (4, 300, [0, 300, -7, 10 ** 9, 3]), (3, 40, [50, 20, 40, 10])])
def test_bounds_that_do_not_ascend(B, n, cu):
    """Nonsense in the bounds: nothing outside out and the workspace changes, and other calls go on."""
    rng = np.random.default_rng(12)
    lens = [4000] * B
    table, n_pages = make_table(rng, [4000], 64)
    pool = Pool(rng, n_pages, 1, 64, 0, True, False, np.repeat(table, B, 0))
    q = torch.from_numpy(rng.standard_normal((n, 8, 64)).astype(np.float32)).to(DEV)
    size = pa.pot_paged_workspace_bytes(B, n, 8, 1, 300, 4000)
    ws = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    wide = torch.full((n + 64, 8, 64), 7.5, device=DEV)
    pa.pot_paged_attention(pool.fmt, q, pool.pages, _dev(cu), _dev(lens), _heads(8, 1), 300, 4000, wide[32:32 + n], ws[:size])
    torch.cuda.synchronize()
    assert (ws[size:] == 0x5A).all() and (wide[:32] == 7.5).all() and (wide[32 + n:] == 7.5).all()
    check_attend(pool, q[:40].contiguous(), [40] + [0] * (B - 1), lens, _heads(8, 1))


@pytest.mark.parametrize("B", [65, 1000, 5000])
def test_many_sequences(B):
    """Chunks and tokens among thousands of sequences, some without new tokens: rows find their sequences."""
    rng = np.random.default_rng(11)
    news = rng.choice([0, 1, 1, 1, 2], B)
    news[rng.integers(0, B, 3)] = [40, 17, 33]
    news[-1] = 0
    lens = [int(n) + int(x) for n, x in zip(news, rng.integers(0, 30, B))]
    lens[int(np.argmax(news))] += 2000
    Hq, Hkv, page = 4, 1, 8
    table, n_pages = make_table(rng, lens, page)
    pool = Pool(rng, n_pages, Hkv, page, 0, True, False, table)
    n = int(news.sum())
    x = torch.from_numpy(rng.standard_normal((n, Hq + 2 * Hkv, 64)).astype(np.float32)).to(DEV)
    cu, ls = _dev(bounds_of(news)), _dev(lens)
    q = torch.empty((n, Hq, 64), device=DEV)
    for t in (pool.sc, pool.vals, pool.se):
        t.zero_()
    pa.pot_paged_append(pool.fmt, pa.make_rope(0), x[:, :Hq], x[:, Hq:Hq + 1], x[:, Hq + 1:], None, None, 1e-6, None, None,
                        pool.pages, cu, ls, q)
    assert torch.equal(q, x[:, :Hq])
    # the rows' places in the pool, from the definition
    row = []
    for b, (m, L) in enumerate(zip(news, lens)):
        t = np.arange(L - m, L)
        row.append(table[b, t // page] * page + t % page)
    row = np.concatenate(row).astype(np.int64)
    want = torch.zeros(n_pages * page, 64, dtype=torch.float16, device=DEV)
    want[torch.from_numpy(row).to(DEV)] = x[:, Hq].half()
    scales = pool.sc.reshape(-1).clone()
    pa.pot_encode_keys(pool.fmt, want, n_pages * page, 1, 0, pool.sc, pool.se, None)
    mine = torch.zeros_like(scales, dtype=torch.bool)
    mine[torch.from_numpy(row).to(DEV)] = True
    assert torch.equal(scales[mine], pool.sc.reshape(-1)[mine]) and (scales[~mine] == 0).all()
    check_attend(pool, q, [int(m) for m in news], lens, _heads(Hq, Hkv))
