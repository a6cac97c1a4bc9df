"""pot_paged_attention where a call has more row tiles than the key ranges that it may split them into: every row is computed."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from paged_util import DEV, Pool, attend_bound, attend_host, make_table, run_attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,groups,max_new", [
    (8, 8, [(948, 17, 6720)], 192),
    (24, 4, [(1804, 3, 8960)], 85),
    (4, 4, [(1900, 17, 32768), (1, 129, 32768)], 129),
    (16, 4, [(200, 5, 600), (1, 60, 40000)], 60),
])
def test_more_row_tiles_than_ranges(Hq, Hkv, groups, max_new):
    """groups: (sequences, new tokens of each, keys of each). All read the pages of the longest, and a group's sequences have the
    same queries, so one of each group is computed in 64 bits."""
    rng = np.random.default_rng(1)
    page, lens = 64, [g[2] for g in groups]
    table, n_pages = make_table(rng, [max(lens)], page)
    heads = np.arange(Hq, dtype=np.int32) // (Hq // Hkv)
    pool = Pool(rng, n_pages, Hkv, page, 0, True, False, np.repeat(table, len(groups), 0))
    q = [torch.from_numpy(rng.standard_normal((new, Hq, 64)).astype(np.float32)).to(DEV) for _, new, _ in groups]
    want, top = attend_host(pool, torch.cat(q).cpu().numpy(), [g[1] for g in groups], lens, heads)
    vmax = float(np.abs(pool.values_host()).max())
    B = sum(g[0] for g in groups)
    pool.pages = pa.make_pages(pool.se, pool.cm, pool.sc, pool.vals, torch.from_numpy(np.repeat(table, B, 0)).to(DEV))
    news = [new for count, new, _ in groups for _ in range(count)]
    got = run_attend(pool, torch.cat([x.repeat(g[0], 1, 1) for x, g in zip(q, groups)]), news,
                     [L for count, _, L in groups for _ in range(count)], heads, max_new=max_new, max_len=max(lens))
    got, at, first = got.double().cpu().numpy(), 0, 0
    for count, new, L in groups:
        part, ref = got[at:at + count * new].reshape(count, new, Hq, 64), want[first:first + new]
        off = np.abs(part - ref) / attend_bound(ref, top, vmax, L, "fp32")
        assert off.max() <= 1, (count, new, L, float(off.max()))
        at, first = at + count * new, first + new
