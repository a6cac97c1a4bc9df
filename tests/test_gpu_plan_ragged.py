"""The launch plan of a batch with a length per sequence: four-wave workgroups where the lengths' differences can pay for
their prologues, the plan without lengths elsewhere, and the same result on either."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from parity_util import to_dev
from test_gpu_attend_v4 import _case, _check, _dev, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,T,small", [
    (16, 16000, True), (16, 15900, False),   # 64 units, 16 splits
    (40, 6000, True), (40, 5900, False),     # 160 units, 6 splits
    (64, 6000, True), (64, 5900, False), (64, 4096, False),  # 256 units, 4 splits
])
def test_workgroups_of_a_ragged_batch(B, T, small):
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the plan is for 256 CUs")
    c = _case(B + T, B, 4, 4, T, 0)
    dev = _dev(c)
    lens = np.array([T - b * T // B for b in range(B)], np.int32)
    dbg = _run(c, dev, to_dev(lens))
    assert (dbg.wg_waves == 4) == small, (dbg.wg_waves, dbg.n_splits)
    if small:
        assert dbg.n_splits == 4 * 256 // (4 * B)
    else:
        plain = _run(c, _dev(c))
        assert (dbg.wg_waves, dbg.n_splits) == (plain.wg_waves, plain.n_splits)
    out = dev["out"].cpu().numpy()
    for b in (0, B // 2, B - 1):
        rows = slice(b * 4 * c["t_cap"], (b + 1) * 4 * c["t_cap"])
        one = dict(c, B=1, q=c["q"][b:b + 1], se=c["se"][rows], sc=c["sc"][rows], v4=c["v4"][4 * b:4 * b + 4])
        _check(one, out[b:b + 1], lens[b:b + 1])
