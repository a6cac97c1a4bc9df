"""max_new and max_len below what the sequences have (include/pot_attn.h): further new tokens are not computed, keys past max_len
are not seen."""
import numpy as np
import pytest
import torch

from paged_util import DEV, Pool, attend_bound, attend_host, bounds_of, make_table, run_attend

pytestmark = pytest.mark.gpu


def _heads(Hq, Hkv):
    return np.arange(Hq, dtype=np.int32) // (Hq // Hkv)


class Cut:
    """A pool of which attend_host sees only each sequence's first `most` keys: the others are on no page of its table."""

    def __init__(self, pool, most):
        self.pool, self.Hkv, self.page, self.n_pages = pool, pool.Hkv, 1, pool.n_pages * pool.page
        self.keys, self.vals = ([np.ascontiguousarray(np.moveaxis(x, 1, 2).reshape(self.n_pages, self.Hkv, 1, 64))
                                 for x in (pool.keys_host(), pool.values_host())])
        t = np.arange(pool.table.shape[1] * pool.page)
        rows = pool.table[:, t // pool.page].astype(np.int64) * pool.page + t % pool.page
        self.table = np.where((pool.table[:, t // pool.page] >= 0) & (t < most), rows, -1)

    def keys_host(self):
        return self.keys

    def values_host(self):
        return self.vals


def _check(seed, news, lens, max_new, max_len, Hq=8, Hkv=2, page=32, k=0, int4=False, out="fp32", window=0, n_sink=0):
    rng = np.random.default_rng(seed)
    table, n_pages = make_table(rng, lens, page)
    pool = Pool(rng, n_pages, Hkv, page, k, int4, False, table)
    q = torch.from_numpy(rng.standard_normal((sum(news), Hq, 64)).astype(np.float32)).to(DEV)
    got = run_attend(pool, q, news, lens, _heads(Hq, Hkv), out, window, n_sink, max_new=max_new, max_len=max_len)
    got = got.double().cpu().numpy()
    cut = Cut(pool, max_len)
    want, top = attend_host(cut, q.cpu().numpy(), news, lens, _heads(Hq, Hkv), window, n_sink)
    vmax = float(np.abs(cut.vals).max())
    cu = bounds_of(news)
    for b, n in enumerate(news):
        first, m = int(cu[b]), min(n, max_new)
        off = np.abs(got[first:first + m] - want[first:first + m]) / attend_bound(want[first:first + m], top, vmax, max_len, out)
        assert off.size == 0 or off.max() <= 1, (b, float(off.max()))
        assert (got[first + m:first + n] == 7.5).all()  # as it was


@pytest.mark.parametrize("news,lens", [([1, 2, 1], [1000, 300, 90]), ([4, 3], [5200, 100]), ([70], [400]), ([150, 1, 40], [450, 600, 130])])
@pytest.mark.parametrize("max_len", [64, 100, 128, 333])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (50, 4), (1000, 70), (3, 0), (100, 130)])
def test_keys_past_max_len(news, lens, max_len, window, n_sink):
    _check(1, news, lens, max(news), max_len, window=window, n_sink=n_sink, int4=window == 50)


@pytest.mark.parametrize("page", [8, 64])
@pytest.mark.parametrize("k,int4,out", [(0, True, "bf16"), (2, False, "fp32"), (4, True, "fp16")])
def test_keys_past_max_len_in_key_ranges(page, k, int4, out):
    """Long enough for key ranges of few rows and of many."""
    _check(2, [1, 300, 2], [4000, 3500, 2900], 300, 2950, page=page, k=k, int4=int4, out=out)
    _check(3, [1, 1, 2], [4000, 3500, 2900], 2, 2950, page=page, k=k, int4=int4, out=out)
    _check(4, [1, 300, 2], [4000, 3500, 2900], 300, 2950, page=page, k=k, int4=int4, out=out, window=1500, n_sink=70)


@pytest.mark.parametrize("news,lens,max_new", [([3, 1, 2], [80, 40, 300], 1), ([40, 5, 0, 90], [100, 5, 70, 400], 33),
                                               ([300, 2, 200], [300, 90, 900], 129), ([20, 20], [20, 200], 2)])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (30, 2)])
def test_new_tokens_past_max_new(news, lens, max_new, window, n_sink):
    _check(5, news, lens, max_new, max(lens), window=window, n_sink=n_sink)
