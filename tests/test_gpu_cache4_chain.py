"""The operators of the 4-bit cache together, as a decoder uses them: a prompt's projection is normed and rotated and
written, then tokens follow one by one, then the cache is read back; eagerly and as a captured step."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_09208_amd as pa
from cache4_util import attend, attend_bound, key_values, take4
from parity_util import DEV

pytestmark = pytest.mark.gpu

B, S, STEPS, HQ, HKV, CAP = 2, 45, 5, 16, 2, 64


def _projection(seed, tokens):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn((B, tokens, HQ + 2 * HKV, 64), generator=g, device=DEV).to(torch.bfloat16)


class Layer:
    def __init__(self, k, hadamard):
        self.fmt, self.k = pa.make_format(k, hadamard=hadamard), k
        self.cache = pa.alloc_pot_cache(B, HKV, CAP, k, DEV)
        self.v4 = pa.alloc_value_cache_int4(B, HKV, CAP, DEV)
        self.rope = pa.make_rope(64, axis_of_pair=[i * 3 // 32 for i in range(32)])
        self.inv_freq = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64, device=DEV) / 64)
        g = torch.Generator(device=DEV)
        g.manual_seed(1)
        self.qw, self.kw = ((1 + 0.2 * torch.randn(64, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2))
        self.heads = np.arange(HQ, dtype=np.int32) // (HQ // HKV)
        self.ws = pa.alloc_workspace(pa.pot_decode_workspace_bytes(B, HQ, HKV, CAP), DEV)
        self.out = torch.empty((B, HQ, 64), device=DEV)
        self.q = torch.empty((B, HQ, 1, 64), device=DEV)
        self.k1, self.v1 = (torch.empty((B, HKV, 1, 64), dtype=torch.float16, device=DEV) for _ in range(2))

    def _rows(self, x, pos, q, k, v):
        pa.pot_norm_rope(self.rope, x[:, :, :HQ], x[:, :, HQ:HQ + HKV], x[:, :, HQ + HKV:], self.qw, self.kw, 1e-6, pos,
                         self.inv_freq, q, k, v)

    def prompt(self, x, pos):
        n = x.shape[1]
        k, v = (torch.empty((B, HKV, n, 64), dtype=torch.float16, device=DEV) for _ in range(2))
        q = torch.empty((B, HQ, n, 64), dtype=torch.bfloat16, device=DEV)
        self._rows(x, pos, q, k, v)
        c = self.cache
        for s in range(B * HKV):
            b, h = divmod(s, HKV)
            pa.pot_encode_keys(self.fmt, k[b, h], n, 1, 0, c["key_scale"][b, h], c["codes_se"][b, h],
                               c["codes_m"][b, h] if self.k else None)
        pa.pot_store_values_int4(v, B * HKV, n, CAP, 0, self.v4)

    def step(self, x, pos, lens, T):
        self._rows(x, pos, self.q, self.k1, self.v1)
        c = self.cache
        pa.pot_append_decode_attention_v4(self.fmt, 0, self.q, self.k1, self.v1, c["codes_se"], c["codes_m"],
                                          c["key_scale"], self.v4, CAP, lens, self.heads, B, HQ, HKV, T, self.out, self.ws)


def _positions(first, n):
    t = torch.arange(first, first + n, device=DEV)
    return torch.stack((t, t // 7, t % 7)).view(3, 1, n).expand(3, B, n).contiguous()


def _check_attention(layer, n):
    c = layer.cache
    host = {name: None if t is None else t.cpu().numpy().reshape(B * HKV * CAP, -1) for name, t in c.items()}
    keys = key_values(host["codes_se"], host["codes_m"], host["key_scale"][:, 0], layer.k).reshape(B, HKV, CAP, 64)
    values = take4(layer.v4.cpu().numpy().reshape(B * HKV, CAP // 8, 288)).reshape(B, HKV, CAP, 64)
    q = layer.q.cpu().numpy()[:, :, 0]
    want, top = attend(q, keys, values, [n] * B, layer.heads, bool(layer.fmt.hadamard))
    err = np.abs(layer.out.cpu().numpy() - want).max()
    assert err <= attend_bound(top, np.abs(values[:, :, :n]).max(), n)


@pytest.mark.parametrize("k,hadamard", [(0, False), (1, True), (4, True)])
def test_prompt_then_tokens_equals_one_long_prompt(k, hadamard):
    x = _projection(3, S + STEPS)
    whole, apart = Layer(k, hadamard), Layer(k, hadamard)
    whole.prompt(x, _positions(0, S + STEPS))
    apart.prompt(x[:, :S], _positions(0, S))
    for i in range(STEPS):
        n = S + i + 1
        lens = torch.full((B,), n, dtype=torch.int32, device=DEV) if i % 2 else None
        apart.step(x[:, S + i:S + i + 1], _positions(S + i, 1), lens, CAP if i % 2 else n)
        _check_attention(apart, n)
    for name, t in whole.cache.items():
        assert t is None or torch.equal(t, apart.cache[name]), name
    assert torch.equal(whole.v4, apart.v4)
    # read back: what the attention saw
    rows = [torch.empty((B * HKV, S + STEPS, 64), dtype=torch.float16, device=DEV) for _ in range(2)]
    c = apart.cache
    pa.pot_load_keys(apart.fmt, c["codes_se"], c["codes_m"], c["key_scale"], B * HKV, S + STEPS, CAP, 0, rows[0])
    pa.pot_load_values_int4(apart.v4, B * HKV, S + STEPS, CAP, 0, rows[1])
    v = x[:, :, HQ + HKV:].transpose(1, 2).reshape(B * HKV, S + STEPS, 64).float()
    step = (v.amax(-1) - v.amin(-1)) / 15
    assert ((rows[1].float() - v).abs().amax(-1) <= 0.502 * step + v.abs().amax(-1) * 2.0 ** -10).all()
    codes = rows[0].cpu().numpy().reshape(-1, 64)
    if not hadamard:  # codes are fixed points of their own encoding
        se, cm, sc = oracle.encode_keys(codes.view(np.uint16), mant_bits=k)
        n = S + STEPS
        assert np.array_equal(se.reshape(B, HKV, n, 32), c["codes_se"][:, :, :n].cpu().numpy())


def test_a_captured_step_follows_its_inputs():
    layer, eager = Layer(0, False), Layer(0, False)
    x = _projection(4, S + STEPS)
    for one in (layer, eager):
        one.prompt(x[:, :S], _positions(0, S))
    tok = x[:, S:S + 1].clone()
    pos, lens = _positions(S, 1), torch.full((B,), S + 1, dtype=torch.int32, device=DEV)
    layer.step(tok, pos, lens, CAP)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        layer.step(tok, pos, lens, CAP)
    for i in range(STEPS):
        tok.copy_(x[:, S + i:S + i + 1])
        pos.copy_(_positions(S + i, 1))
        lens.fill_(S + i + 1)
        g.replay()
        torch.cuda.synchronize()
        eager.step(x[:, S + i:S + i + 1], _positions(S + i, 1), torch.full((B,), S + i + 1, dtype=torch.int32, device=DEV),
                   CAP)
        torch.cuda.synchronize()
        assert torch.equal(layer.out, eager.out), i
        assert torch.equal(layer.v4, eager.v4) and torch.equal(layer.cache["codes_se"], eager.cache["codes_se"])


def test_bulk_calls_on_another_stream_and_captured():
    n, cap = 1029, 1032
    fmt, heads = pa.make_format(1, hadamard=True), B * HKV
    one = Layer(1, True)
    x = torch.empty((B, n, HQ + 2 * HKV, 64), dtype=torch.bfloat16, device=DEV)
    pos = torch.empty((3, B, n), dtype=torch.int64, device=DEV)
    cache, v4 = pa.alloc_pot_cache(B, HKV, cap, 1, DEV), pa.alloc_value_cache_int4(B, HKV, cap, DEV)
    q = torch.empty((B, HQ, n, 64), dtype=torch.bfloat16, device=DEV)
    k, v, k_back, v_back = (torch.empty((B, HKV, n, 64), dtype=torch.float16, device=DEV) for _ in range(4))
    codes = cache["codes_se"], cache["codes_m"], cache["key_scale"]

    def layer():
        one._rows(x, pos, q, k, v)
        for s in range(heads):
            b, h = divmod(s, HKV)
            pa.pot_encode_keys(fmt, k[b, h], n, 1, 0, cache["key_scale"][b, h], cache["codes_se"][b, h], cache["codes_m"][b, h])
        pa.pot_store_values_int4(v, heads, n, cap, 0, v4)
        pa.pot_load_keys(fmt, *codes, heads, n, cap, 0, k_back)
        pa.pot_load_values_int4(v4, heads, n, cap, 0, v_back)

    def fill(seed):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        pos.copy_(_positions(100 * seed, n))

    side = torch.cuda.Stream()
    results = []
    for seed in range(3):  # eager, on a stream of its own
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            fill(seed)
            layer()
        torch.cuda.current_stream().wait_stream(side)
        results.append([t.clone() for t in (q, k, v, k_back, v_back)])
    torch.cuda.synchronize()
    assert not torch.equal(results[0][3], results[1][3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for seed in (1, 0, 2, 2):
        fill(seed)
        for t in (q, k, v, k_back, v_back):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((q, k, v, k_back, v_back), results[seed]):
            assert torch.equal(got, want), seed
