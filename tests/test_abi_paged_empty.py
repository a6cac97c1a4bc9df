"""Paged calls without sequences or without rows are no-ops, on the arrays as a program then has them: a table and lengths without
elements have no address. Before any HIP call, so without a GPU."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from test_abi_device_host import OnGpu
from test_abi_paged_host import INVALID, _append, _attend, _pages, _part

HEADS = np.arange(8, dtype=np.int32) // 4


class Real(OnGpu):
    """A tensor on the GPU whose address is NULL where it has no elements."""

    def data_ptr(self):
        return 0 if self.t.numel() == 0 else super().data_ptr()


def test_arrays_without_an_address():
    none = dict(pages=_pages(table=None), B=0, cu=None, lens=None)
    assert _attend(**none) == 0 and _append(**none) == 0
    assert _attend(**none, n=0, q=None, out=None) == 0
    assert _append(**none, n=0, q=_part(None), k=_part(None), v=_part(None)) == 0
    for missing in (dict(pages=_pages(table=None)), dict(cu=None), dict(lens=None)):  # needed where there are sequences
        for n in (0, 40):
            assert _attend(B=1, n=n, **missing) == INVALID and _append(B=1, n=n, **missing) == INVALID


@pytest.mark.parametrize("n", [0, 3])
def test_binding_without_sequences(n):
    se, _, sc, v = pa.alloc_pages(4, 2, 16, 0, "cpu")
    i32 = dict(dtype=torch.int32)
    pages = pa.make_pages(Real(se), None, Real(sc), Real(v), Real(torch.zeros((0, 2), **i32)))
    cu, lens = Real(torch.zeros(1, **i32)), Real(torch.zeros(0, **i32))
    q, k = Real(torch.zeros((n, 8, 64))), Real(torch.zeros((n, 2, 64)))
    fmt, out = pa.make_format(), Real(torch.zeros((n, 8, 64)))
    pa.pot_paged_append(fmt, pa.make_rope(0), q, k, k, None, None, 1e-6, None, None, pages, cu, lens, out, stream=1)
    pa.pot_paged_attention(fmt, q, pages, cu, lens, HEADS, 1, 16, out, None, stream=1)
