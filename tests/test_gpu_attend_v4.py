"""Decode attention over PoT keys and 4-bit values against 64 bits: lengths from none to long, empty sequences, head
groups, formats, engines, splits, steps of any size, the append, replays and streams."""
import numpy as np
import pytest
import torch

import oracle
import paper_2609_09208_amd as pa
from cache4_util import GROUP, attend, attend_bound, key_values, place4, quantise4, take4
from parity_util import DEV, to_dev
from workloads import make_decode_inputs

pytestmark = pytest.mark.gpu


def _case(seed, B, Hq, Hkv, T, k=0, hadamard=False, t_cap=None, heads=None, v=None):
    """Host inputs, codes and a cache whose rows past T hold NaN steps and minima and huge keys."""
    d = make_decode_inputs(seed, B, Hq, Hkv, T, t_cap=t_cap)
    t_cap = d["t_cap"]
    se, cm, sc = oracle.encode_keys(d["k_bits"].reshape(-1, 64), mant_bits=k, hadamard=hadamard)
    rows = d["v_bits"].view(np.float16).reshape(B * Hkv, t_cap, 64)[:, :T] if v is None else v
    cache = np.full((B * Hkv, t_cap // 8, GROUP), 0xFF, np.uint8)
    place4(cache, *quantise4(rows), 0)
    if heads is None:
        heads = d["kv_head_of_q"]
    return dict(q=d["q"], se=se, cm=cm, sc=sc, v4=cache, B=B, Hq=Hq, Hkv=Hkv, T=T, t_cap=t_cap, k=k, hadamard=hadamard,
                heads=np.asarray(heads, np.int32))


def _dev(c):
    return dict(q=to_dev(c["q"]), se=to_dev(c["se"]), cm=None if c["cm"] is None else to_dev(c["cm"]), sc=to_dev(c["sc"]),
                v4=to_dev(c["v4"]), out=torch.full((c["B"], c["Hq"], 64), float("nan"), device=DEV))


def _run(c, dev, lens=None, engine=0, splits=0, waves=0, ws=None, stream=None, append=None):
    dbg = pa.pot_debug()
    dbg.force_splits, dbg.force_wg_waves = splits, waves
    B, Hq, Hkv, T = c["B"], c["Hq"], c["Hkv"], c["T"]
    if ws is None:
        n = pa.pot_decode_workspace_bytes_for_splits(B, Hq, Hkv, T, splits) if splits else \
            pa.pot_decode_workspace_bytes(B, Hq, Hkv, T)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    fmt = pa.make_format(c["k"], hadamard=c["hadamard"])
    tail = (dev["se"], dev["cm"], dev["sc"], dev["v4"], c["t_cap"], lens, c["heads"], B, Hq, Hkv, T, dev["out"], ws)
    if append is None:
        pa.pot_decode_attention_v4(fmt, engine, dev["q"], *tail, dbg=dbg, stream=stream)
    else:
        pa.pot_append_decode_attention_v4(fmt, engine, dev["q"], *append, *tail, dbg=dbg, stream=stream)
    return dbg


def _check(c, got, lens=None):
    shape = (c["B"], c["Hkv"], c["t_cap"], 64)
    lens = [c["T"]] * c["B"] if lens is None else lens
    keys = key_values(c["se"], c["cm"], c["sc"], c["k"]).reshape(shape)
    values = take4(c["v4"]).reshape(shape)
    want, top = attend(c["q"], keys, values, lens, c["heads"], c["hadamard"])
    vmax = max([np.abs(values[b, :, :n]).max() for b, n in enumerate(lens) if n] or [0.0])
    for b, n in enumerate(lens):
        if n == 0:
            assert (got[b] == 0).all()
    err = float(np.abs(got - want).max())
    assert err <= attend_bound(top, vmax, c["T"]), (err, top, vmax)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 63, 64, 65, 129, 255, 256, 257, 769, 1025, 2000, 4097])
@pytest.mark.parametrize("k", [0, 2])
def test_lengths(T, k):
    c = _case(T, 2, 16, 2, T, k, t_cap=(T + 15) // 8 * 8)
    dev = _dev(c)
    _run(c, dev)
    _check(c, dev["out"].cpu().numpy())


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("k", [0, 1, 2, 3, 4])
@pytest.mark.parametrize("hadamard", [False, True])
def test_groups_and_formats(G, k, hadamard):
    c = _case(10 * G + k, 3, 3 * G, 3, 301, k, hadamard)
    dev = _dev(c)
    lens = [301, 64, 130]
    _run(c, dev, to_dev(np.array(lens, np.int32)))
    _check(c, dev["out"].cpu().numpy(), lens)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("splits,waves", [(1, 4), (1, 16), (3, 4), (3, 16), (40, 16), (70, 4)])
def test_byte_decode_engine_and_splits(G, splits, waves):
    T = 70 * 256 if splits == 70 else 11000 if splits == 40 else 1500
    c = _case(G + splits, 1, G, 1, T, 0, heads=np.zeros(G))
    for engine in (0, 1):
        dev = _dev(c)
        dbg = _run(c, dev, engine=engine, splits=splits, waves=waves)
        assert dbg.wg_waves == waves
        _check(c, dev["out"].cpu().numpy())


@pytest.mark.parametrize("splits,waves", [(0, 0), (1, 4), (2, 16), (5, 4), (9, 16), (40, 16), (66, 4)])
@pytest.mark.parametrize("k", [0, 1, 4])
def test_ragged_batches(splits, waves, k):
    """A length per sequence, empty ones and ones past the range among them, in any split."""
    T = 66 * 256 if splits >= 40 else 2400
    lens = np.array([T, 0, 1, 63, 64, 65, 1000, T + 77, -5, T - 1], np.int32)
    c = _case(splits + k, len(lens), 8, 1, T, k, heads=np.zeros(8))
    dev = _dev(c)
    _run(c, dev, to_dev(lens), splits=splits, waves=12 if waves == 16 and k == 4 else waves)
    _check(c, dev["out"].cpu().numpy(), np.clip(lens, 0, T))


@pytest.mark.parametrize("splits,waves", [(0, 0), (4, 16), (70, 4)])
def test_a_batch_without_any_key(splits, waves):
    c = _case(5, 3, 8, 2, 70 * 256 if splits == 70 else 1100, 0)
    dev = _dev(c)
    _run(c, dev, torch.zeros(3, dtype=torch.int32, device=DEV), splits=splits, waves=waves)
    assert (dev["out"].cpu().numpy() == 0).all()


def test_interleaved_heads_and_repeats():
    c = _case(6, 2, 8, 4, 700, 1, heads=np.array([3, 0, 1, 2, 2, 3, 0, 1]))
    dev = _dev(c)
    _run(c, dev)
    first = dev["out"].cpu().numpy()
    _check(c, first)
    for _ in range(3):
        _run(c, dev)
        assert np.array_equal(dev["out"].cpu().numpy(), first)


@pytest.mark.parametrize("kind", ["constant", "mixed", "tiny", "large", "rising", "falling"])
@pytest.mark.parametrize("waves", [4, 16])
def test_steps_of_any_size(kind, waves):
    rng = np.random.default_rng(1)
    T, n_seq = 1200, 2
    v = rng.standard_normal((n_seq, T, 64))
    if kind == "constant":
        v = np.repeat(rng.standard_normal((n_seq, T, 1)), 64, -1)
    elif kind == "mixed":
        v = v * 2.0 ** rng.integers(-14, 1, (n_seq, T, 1))
    elif kind == "tiny":
        v = v * 2.0 ** -17
    elif kind == "large":
        v = v * 2.0 ** 13
    elif kind == "rising":
        v = v * 2.0 ** (np.arange(T) * 12 // T - 8)[None, :, None]
    else:
        v = v * 2.0 ** (4 - np.arange(T) * 12 // T)[None, :, None]
    c = _case(3, 1, 16, 2, T, 0, v=v.astype(np.float16))
    dev = _dev(c)
    _run(c, dev, waves=waves, splits=2)
    _check(c, dev["out"].cpu().numpy())


@pytest.mark.parametrize("k,hadamard,engine", [(0, False, 0), (0, True, 1), (1, False, 0), (4, True, 0)])
@pytest.mark.parametrize("T,lens", [(1, None), (8, None), (300, None), (2049, None), (2049, [2049, 0, 1, 8, 65, 1000])])
def test_append_equals_the_separate_calls(k, hadamard, engine, T, lens):
    B, Hq, Hkv = 6, 16, 2
    c = _case(T + k, B, Hq, Hkv, T, k, hadamard, t_cap=(T + 15) // 8 * 8)
    n = np.array([T] * B if lens is None else lens)
    ln = None if lens is None else to_dev(n.astype(np.int32))
    rng = np.random.default_rng(8)
    k_new = to_dev(rng.standard_normal((B, Hkv, 64)).astype(np.float16))
    v_new = to_dev(rng.standard_normal((B, Hkv, 64)).astype(np.float16))
    fused, apart = _dev(c), _dev(c)
    _run(c, fused, ln, engine, append=(k_new, v_new))
    fmt = pa.make_format(k, hadamard=hadamard)
    for b in range(B):
        if n[b] == 0:
            continue
        for h in range(Hkv):
            s = b * Hkv + h
            at = s * c["t_cap"] + n[b] - 1
            pa.pot_encode_keys(fmt, k_new[b, h], 1, 1, 0, apart["sc"][at:], apart["se"][at].data_ptr(),
                               apart["cm"][at].data_ptr() if k else None)
            pa.pot_store_values_int4(v_new[b, h], 1, 1, c["t_cap"], int(n[b]) - 1, apart["v4"][s])
    _run(c, apart, ln, engine)
    torch.cuda.synchronize()
    for name in ("se", "cm", "sc", "v4", "out"):
        if fused[name] is not None:
            assert torch.equal(fused[name], apart[name]), name
    c.update(se=apart["se"].cpu().numpy(), cm=None if not k else apart["cm"].cpu().numpy(), sc=apart["sc"].cpu().numpy(),
             v4=apart["v4"].cpu().numpy())
    _check(c, fused["out"].cpu().numpy(), n)


def test_offsets_past_4_gib():
    """The last sequence of a cache whose value and code offsets pass 2^32 bytes."""
    B, t_cap, T = 40, 4 << 20, 900
    c = _case(4, 1, 8, 1, T, 0, heads=np.zeros(8))
    n = c["t_cap"]
    big = dict(se=torch.empty((B * t_cap, 32), dtype=torch.uint8, device=DEV),
               sc=torch.empty(B * t_cap, dtype=torch.float32, device=DEV),
               v4=torch.empty((B, t_cap // 8, GROUP), dtype=torch.uint8, device=DEV), cm=None)
    big["se"].view(B, t_cap, 32)[:, :n] = to_dev(c["se"])
    big["sc"].view(B, t_cap)[:, :n] = to_dev(c["sc"])
    big["v4"][:, :n // 8] = to_dev(c["v4"])
    big["q"] = to_dev(np.repeat(c["q"], B, 0))
    big["out"] = torch.empty((B, 8, 64), device=DEV)
    wide = dict(c, B=B, t_cap=t_cap, q=np.repeat(c["q"], B, 0))
    _run(wide, big)
    out = big["out"].cpu().numpy()
    assert np.array_equal(out, np.broadcast_to(out[:1], out.shape))
    _check(c, out[-1:])


def test_full_chip_claims_tiles():
    """More work than fits the chip at once, tiles claimed in any order: a sample of it against 64 bits."""
    c = _case(11, 70, 32, 4, 8400, 0)
    dev = _dev(c)
    dbg = _run(c, dev)
    assert dbg.wg_waves > 4
    lens = (8400 - 117 * np.arange(70)).astype(np.int32)
    out = dev["out"].cpu().numpy()
    _run(c, dev, to_dev(lens))
    ragged = dev["out"].cpu().numpy()
    for b in (0, 37, 69):
        one = dict(c, B=1, q=c["q"][b:b + 1])
        rows = slice(b * 4 * c["t_cap"], (b + 1) * 4 * c["t_cap"])
        one.update(se=c["se"][rows], sc=c["sc"][rows], v4=c["v4"][4 * b:4 * b + 4])
        _check(one, out[b:b + 1])
        _check(one, ragged[b:b + 1], lens[b:b + 1])


def test_long_ragged_batch_as_planned():
    """From 1000 keys a split on, sequences with lengths of their own are cut into more, smaller workgroups."""
    B, T = 16, 16001
    c = _case(13, B, 4, 4, T, 0)
    dev = _dev(c)
    lens = np.array([T - b * T // B for b in range(B - 1)] + [0], np.int32)
    dbg = _run(c, dev, to_dev(lens))
    assert dbg.wg_waves == 4 and dbg.n_splits > 4
    _check(c, dev["out"].cpu().numpy(), lens)
    dbg = _run(c, dev)
    assert dbg.wg_waves > 4
    _check(c, dev["out"].cpu().numpy())


def test_graph_replays_and_streams():
    """An append with lengths, captured: replays with other lengths and queries equal the eager calls; two streams with
    a workspace each do too."""
    B, T = 4, 1500
    c = _case(12, B, 16, 2, T, 1)
    dev = _dev(c)
    rng = np.random.default_rng(2)
    new = (to_dev(rng.standard_normal((B, 2, 64)).astype(np.float16)), to_dev(rng.standard_normal((B, 2, 64)).astype(np.float16)))
    ln = torch.tensor([T, 700, 0, 33], dtype=torch.int32, device=DEV)
    ws = pa.alloc_workspace(pa.pot_decode_workspace_bytes(B, 16, 2, T), DEV)
    _run(c, dev, ln, ws=ws, append=new)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _run(c, dev, ln, ws=ws, append=new)
    for i, lens in enumerate([[T, 700, 0, 33], [1, 0, T, 800], [0, 0, 0, 0], [T - 1, 64, 65, T]]):
        ln.copy_(torch.tensor(lens, dtype=torch.int32))
        dev["q"].copy_(to_dev(np.roll(c["q"], i, 1)))
        dev["out"].fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        got = dev["out"].clone()
        _run(c, dev, ln, append=new)
        torch.cuda.synchronize()
        assert torch.equal(got, dev["out"]), i
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    want = dev["out"].clone()
    outs = [dict(dev, out=torch.empty_like(want)) for _ in range(2)]
    spaces = [pa.alloc_workspace(ws.numel(), DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o, w in ((one, outs[0], spaces[0]), (two, outs[1], spaces[1])):
            _run(c, o, ln, ws=w, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0]["out"], want) and torch.equal(outs[1]["out"], want)
