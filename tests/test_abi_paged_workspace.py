"""The workspace of pot_paged_attention is a dense tensor on the queries' GPU: anything else is refused in the binding, without a
GPU. A kernel writes it from its address on, as one piece."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from test_abi_device_host import OnGpu

HEADS = np.arange(8, dtype=np.int32) // 4


class Elsewhere(OnGpu):
    def get_device(self):
        return 1


def _call(monkeypatch, workspace, **kw):
    """The status that the library is asked for; it is not called."""
    asked = []
    monkeypatch.setattr(pa, "_lib", type("Lib", (), {"pot_paged_attention": staticmethod(lambda *a: asked.append(a) or 0)}))
    se, _, sc, v = pa.alloc_pages(4, 2, 16, 0, "cpu")
    pages = pa.make_pages(OnGpu(se), None, OnGpu(sc), OnGpu(v), OnGpu(torch.zeros((3, 2), dtype=torch.int32)))
    q = OnGpu(torch.zeros((3, 8, 64)))
    cu, lens = (OnGpu(torch.zeros(n, dtype=torch.int32)) for n in (4, 3))
    pa.pot_paged_attention(pa.make_format(), q, pages, cu, lens, HEADS, 1, 16, q, workspace, stream=1, **kw)
    return asked[0]


BYTES = torch.zeros(4096, dtype=torch.uint8)


@pytest.mark.parametrize("workspace", [Elsewhere(BYTES), OnGpu(BYTES[::2]), OnGpu(BYTES.view(64, 64).t()), OnGpu(BYTES.view(64, 64)[:, :32])])
@pytest.mark.parametrize("kw", [dict(), dict(ws_bytes=1024)])
def test_refused(monkeypatch, workspace, kw):
    with pytest.raises(pa.PotError) as e:
        _call(monkeypatch, workspace, **kw)
    assert e.value.status == pa.POT_ERR_INVALID_ARG and "workspace" in str(e.value)


def test_on_the_host(monkeypatch):
    with pytest.raises(pa.PotError):
        _call(monkeypatch, BYTES)


def test_taken(monkeypatch):
    address = OnGpu(BYTES).data_ptr()
    assert _call(monkeypatch, OnGpu(BYTES))[-3:] == (address, 4096, 1)
    assert _call(monkeypatch, OnGpu(BYTES.view(torch.float32).view(32, 32)))[-3:] == (address, 4096, 1)
    assert _call(monkeypatch, OnGpu(BYTES), ws_bytes=1024)[-3:] == (address, 1024, 1)
    assert _call(monkeypatch, address, ws_bytes=2048)[-3:] == (address, 2048, 1)
    assert _call(monkeypatch, None)[-3:] == (0, 0, 1)
