"""Tensors that are not where the kernels read: refused in the binding, before any HIP call, so without a GPU. A kernel that
is handed a host address reads or writes out of its memory."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa

FAKE = 0x7F0000001000
HEADS = np.arange(32, dtype=np.int32) // 8
FMT = pa.make_format()


class OnGpu:
    """A tensor as the binding sees one on the GPU: everything of a CPU tensor but its place."""

    is_cuda = True

    def __init__(self, t):
        self.t = t

    def data_ptr(self):
        return FAKE

    def get_device(self):
        return 0

    def __getattr__(self, name):
        return getattr(self.t, name)


def _refused(call):
    with pytest.raises(pa.PotError) as e:
        call()
    assert e.value.status == pa.POT_ERR_INVALID_ARG and "GPU" in str(e.value), str(e.value)


def test_lengths_on_the_host():
    lens = torch.full((4,), 8, dtype=torch.int32)
    args = (FAKE, None, FAKE, FAKE, 8, lens, HEADS, 4, 32, 4, 8, FAKE, FAKE)
    _refused(lambda: pa.pot_decode_attention_v4(FMT, 0, FAKE, *args, ws_bytes=1 << 30))
    _refused(lambda: pa.pot_append_decode_attention_v4(FMT, 0, FAKE, FAKE, FAKE, *args, ws_bytes=1 << 30))


@pytest.mark.parametrize("which", ["q", "k", "v", "q_out", "k_out", "v_out", "q_weight", "k_weight", "positions", "inv_freq"])
def test_norm_rope_of_a_tensor_on_the_host(which):
    rows, out = torch.zeros((2, 3, 4, 64)), torch.zeros((2, 4, 3, 64))
    args = dict(q=rows, k=rows, v=rows, q_weight=torch.ones(64), k_weight=torch.ones(64),
                positions=torch.zeros((1, 2, 3), dtype=torch.int64), inv_freq=torch.zeros(32, dtype=torch.float64),
                q_out=out, k_out=out.half(), v_out=out.half())
    args = {n: t if n == which else OnGpu(t) for n, t in args.items()}
    _refused(lambda: pa.pot_norm_rope(pa.make_rope(), eps=1e-6, **args))


HOST = torch.zeros(1 << 12, dtype=torch.uint8)
CALLS = {
    "store_int4": (lambda *a: pa.pot_store_values_int4(a[0], 1, 8, 8, 0, a[1]), 2),
    "store_int8": (lambda *a: pa.pot_store_values_int8(a[0], 1, 8, 8, 0, a[1], a[2]), 3),
    "store": (lambda *a: pa.pot_store_values(a[0], 1, 8, 8, 0, a[1]), 2),
    "load_keys": (lambda *a: pa.pot_load_keys(FMT, a[0], None, a[1], 1, 8, 8, 0, a[2]), 3),
    "load": (lambda *a: pa.pot_load_values(a[0], 1, 8, 8, 0, a[1]), 2),
    "load_int8": (lambda *a: pa.pot_load_values_int8(a[0], a[1], 1, 8, 8, 0, a[2]), 3),
    "load_int4": (lambda *a: pa.pot_load_values_int4(a[0], 1, 8, 8, 0, a[1]), 2),
    "encode": (lambda *a: pa.pot_encode_keys(FMT, a[0], 8, 1, 0, a[1], a[2]), 3),
    "decode": (lambda *a: pa.pot_decode_attention(FMT, a[0], a[1], None, a[2], a[3], 8, HEADS, 1, 32, 4, 8, a[4], a[5],
                                                  ws_bytes=1 << 30), 6),
    "decode_v4": (lambda *a: pa.pot_decode_attention_v4(FMT, 0, a[0], a[1], None, a[2], a[3], 8, None, HEADS, 1, 32, 4, 8, a[4],
                                                        a[5], ws_bytes=1 << 30), 6),
    "append_v4": (lambda *a: pa.pot_append_decode_attention_v4(FMT, 0, a[0], a[1], a[2], a[3], None, a[4], a[5], 8, None, HEADS,
                                                               1, 32, 4, 8, a[6], a[7], ws_bytes=1 << 30), 8),
}


@pytest.mark.parametrize("name", CALLS)
def test_any_buffer_on_the_host(name):
    call, n = CALLS[name]
    for i in range(n):
        _refused(lambda: call(*(HOST if j == i else FAKE for j in range(n))))


@pytest.mark.parametrize("current", [1, 2])
def test_tensors_of_another_device(monkeypatch, current):
    """Without a stream the call goes to the current device's, where a tensor of another one is not mapped."""
    monkeypatch.setattr(pa, "_raw_device", lambda: current)
    monkeypatch.setattr(pa, "_raw_stream", lambda d: 0x1000 + d)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    assert pa._stream(None) == 0x1000 + current and pa._stream(77) == 77
    assert pa._stream(None, current) == 0x1000 + current
    with pytest.raises(pa.PotError) as e:
        pa._stream(None, 0)
    assert e.value.status == pa.POT_ERR_INVALID_ARG and "current device" in str(e.value)
    assert pa._stream(77, 0) == 77 and pa._device(FAKE) is None
    rows = OnGpu(torch.zeros((1, 1, 4, 64)))
    with pytest.raises(pa.PotError) as e:
        pa.pot_norm_rope(pa.make_rope(0), rows, None, None, None, None, 0.0, None, None, OnGpu(torch.zeros((1, 4, 1, 64))), None,
                         None)
    assert "current device" in str(e.value)


@pytest.mark.parametrize("rot_dim", [66, 128, -2, 3, 65])
def test_a_rope_wider_than_a_head(rot_dim):
    with pytest.raises(pa.PotError) as e:
        pa.make_rope(rot_dim)
    assert e.value.status == pa.POT_ERR_INVALID_ARG


@pytest.mark.parametrize("shape", [(6, 64), (2, 3, 64), (1, 2, 3, 4, 64)])
def test_rows_of_other_dimensions(shape):
    rows = OnGpu(torch.zeros(shape))
    with pytest.raises(pa.PotError) as e:
        pa.pot_norm_rope(pa.make_rope(), rows, None, None, None, None, 0.0, None, None, rows, None, None)
    assert e.value.status == pa.POT_ERR_INVALID_ARG
