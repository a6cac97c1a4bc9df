"""What goes into a key and value cache held in 4 bits, what reads it, and the attention over it, as timed cases.

Four kinds of pass, at the head shapes and key formats of the tests and the benchmark:

- "qkv": the rows of a QKV projection to what the cache and the decode call take: RMS norm of queries and keys per head
  and the position rotation, one to three axes, in one pass (pot_norm_rope).
- "values": values are written to their cache and read back as the rows that the cache stands for
  (pot_store_values_int4 and pot_load_values_int4).
- "keys": the rows that PoT / PoT-Mk key codes stand for, rotated back where they were rotated (pot_load_keys).
- "attend", "append": decode attention over PoT keys and 4-bit values (pot_decode_attention_v4), with a length per
  sequence in "ragged" cases; "append" takes in the new token first (pot_append_decode_attention_v4) and reads it back.

Keys are N(0, 1) times a per-channel scale from U[0.5, 4] (outlier channels), values and queries N(0, 1).

Definitions (fl: rounded to fp32; d = 64):
- norm and rotation: y = x / sqrt(mean x^2 + eps) * w; pair i of a rotated head, on axis a, turns by the angle
  position_a * inv_freq_i.
- a key code stands for s * sign * (1 + j / 2^k) * 2^-e, s the row's absolute maximum, nearest in log2 distance; values
  up to s * 2^-6.5 are zero. With hadamard the row is H K / 8 (H the 64 x 64 Sylvester matrix).
- a value row is held as z = its minimum (fp16), s = the smallest fp16 number >= fl(fl(max - min) / 15) and
  n = min(15, round-half-even(fl(fl(v - z) * fl(1 / s)))), and stands for z + s n.
- a query is rotated like the keys and held in 8 bits: round-half-even(fl(q * fl(127 / max|q|))) steps of max|q| / 127.

The 4-bit value cache holds groups of 8 tokens, 288 bytes each: byte 16 (c % 16) + 8 (c / 32) + t % 8 has dimension c in
its low half where c % 32 < 16 and in its high half elsewhere; at 256 stand the group's 8 fp16 s, at 272 its 8 fp16 z.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
D = 64
GROUP = 288  # bytes of 8 tokens of the 4-bit value cache
EPS = 1e-6
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _qkv(B, S, Hq, Hkv, dtype, q_out, layout="packed", norm=True, rot_dim=64, pairing="halves", axes=1, far=0, name=None):
    c = dict(kind="qkv", B=B, S=S, Hq=Hq, Hkv=Hkv, dtype=dtype, q_out=q_out, layout=layout, norm=norm, rot_dim=rot_dim,
             pairing=pairing, axes=axes, far=far)
    return c if name is None else dict(c, name=name)


def _values(B, Hkv, n_tok, t_cap, t0, name=None):
    c = dict(kind="values", B=B, Hkv=Hkv, n_tok=n_tok, t_cap=t_cap, t0=t0)
    return c if name is None else dict(c, name=name)


def _keys(B, Hkv, n_tok, t_cap, t0, k, hadamard=False, name=None):
    c = dict(kind="keys", B=B, Hkv=Hkv, n_tok=n_tok, t_cap=t_cap, t0=t0, k=k, hadamard=hadamard)
    return c if name is None else dict(c, name=name)


def _attend(kind, B, Hq, Hkv, T, t_cap, k, hadamard=False, ragged=False, engine=0, name=None):
    c = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, T=T, t_cap=t_cap, k=k, hadamard=hadamard, ragged=ragged, engine=engine)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the projection of one new token of one chat: latency
        _qkv(1, 1, 32, 4, "bf16", "fp32", name="qkv_b1_s1_bf16"),
        # one step of a full batch of a model that reads images: three position axes, far positions
        _qkv(64, 1, 32, 4, "fp16", "fp32", axes=3, far=1 << 20, name="qkv_b64_s1_axes3"),
        # four prompts of ordinary length, one packed projection
        _qkv(4, 8192, 32, 4, "bf16", "bf16", name="qkv_b4_s8192_packed"),
        # a short odd prompt in fp32, separate projections, half of each head turned in neighbouring pairs, no norm
        _qkv(1, 777, 16, 8, "fp32", "fp32", layout="heads", norm=False, rot_dim=32, pairing="neighbours", axes=2,
             name="qkv_s777_fp32_half_rotated"),
        # one new token of each sequence of a full batch
        _values(64, 4, 1, 32768, 20001, name="values_b64_one_token"),
        # four prompts behind a cached prefix, whose ends fall inside a group
        _values(4, 4, 8187, 8192, 3, name="values_b4_t8187"),
        # the keys of an ordinary batch, for attention that takes fp16 rows
        _keys(16, 4, 4096, 4096, 0, 0, name="keys_pot4_b16_t4096"),
        # one long document in the most accurate format, rotated
        _keys(1, 4, 32767, 32768, 1, 4, hadamard=True, name="keys_m4_hadamard_t32767"),
        # one short chat: latency of attention
        _attend("attend", 1, 32, 4, 1024, 2048, 0, name="attend_pot4_b1_t1024"),
        # a serving batch of sequences of all lengths, one slot empty, with a mantissa bit
        _attend("attend", 16, 32, 4, 16383, 16384, 1, ragged=True, name="attend_m1_b16_ragged_t16383"),
        # long context in the most accurate format, four query heads a kv head
        _attend("attend", 8, 16, 4, 32768, 32768, 4, hadamard=True, name="attend_m4_hadamard_b8_t32768_g4"),
        # the largest step: 64 sequences of 32768 keys (the benchmark's layer), the new token taken in first
        _attend("append", 64, 32, 4, 32768, 32768, 0, name="append_pot4_b64_t32768"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["qkv", "values", "keys", "attend", "attend", "append"])
    Hq, Hkv = rng.choice([(32, 4), (32, 4), (32, 8), (16, 4), (16, 8), (8, 8), (64, 8)])
    if kind == "qkv":
        tokens = _log_int(rng, 1, 32768 * 40 // (Hq + 2 * Hkv))
        B = _log_int(rng, 1, min(64, tokens))
        return _qkv(B, max(1, tokens // B), Hq, Hkv, rng.choice(["bf16", "fp16", "fp32"]),
                    rng.choice(["fp32", "bf16", "fp16"]), rng.choice(["packed", "heads"]), rng.random() < 0.7,
                    rng.choice([64, 64, 32, 48]), rng.choice(["halves", "halves", "neighbours"]), rng.choice([1, 1, 2, 3]),
                    rng.choice([0, 0, 1 << 20]))
    k = rng.choice([0, 0, 1, 2, 3, 4])
    hadamard = rng.random() < 0.25
    if kind in ("values", "keys"):
        rows = _log_int(rng, 1, 1 << 20)
        n_seq = _log_int(rng, 1, min(256, rows))
        n_tok, B = max(1, min(32768, rows // n_seq)), max(1, n_seq // Hkv)
        t0 = rng.choice([0, 0, rng.randrange(0, 1000)])
        t_cap = (t0 + n_tok + rng.choice([0, 0, 500]) + 7) // 8 * 8
        return _values(B, Hkv, n_tok, t_cap, t0) if kind == "values" else _keys(B, Hkv, n_tok, t_cap, t0, k, hadamard)
    # B and T over their whole range, together at most a quarter of the largest listed step's keys
    T = _log_int(rng, 1, 32768)
    B = _log_int(rng, 1, max(1, min(64, 2 ** 21 // (T * Hkv))))
    t_cap = (T + rng.choice([0, 0, 1000]) + 7) // 8 * 8
    engine = 1 if k == 0 and rng.random() < 0.3 else 0
    return _attend(kind, B, Hq, Hkv, T, t_cap, k, hadamard, rng.random() < 0.5, engine)


def _lengths(case):
    """The keys of each sequence: all T, or in a ragged batch from T down in equal steps, the last of four or more none."""
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return [T] * B
    got = [T - b * T // B for b in range(B)]
    return got[:-1] + [0] if B >= 4 else got


# ---- what prepare() and the plain forms share: codes as the caches hold them ----------------------------------------

def _hadamard():
    i = torch.arange(D, device=DEV)
    bits = ((i[:, None] & i[None, :])[..., None] >> torch.arange(6, device=DEV)) & 1
    return (1 - 2 * (bits.sum(-1) % 2)).double()


def _over(a, b):
    """fl(a / b) of a tensor and a number or the other way round (torch multiplies by a rounded reciprocal there)."""
    return a / torch.full_like(a, b) if torch.is_tensor(a) else torch.full_like(b, a) / b


def _rotated(x, hadamard):
    """Rows as the quantisers see them (fp32)."""
    return ((x.double() @ _hadamard()) / 8).float() if hadamard else x.float()


def _key_codes(x, k):
    """PoT-Mk codes of fp32 rows [..., 64]: nibbles, mantissas (both uint8) and the row scale."""
    n = 2 ** k
    s = x.abs().amax(-1, keepdim=True)
    u = torch.where(s > 0, x.abs() / s, torch.zeros_like(x))
    m, e = torch.frexp(u)  # u = m 2^e, m in [0.5, 1)
    m, e = m.double() * (2 * n), e.int() - 1
    t = m.floor()
    t = t + (m * m > t * (t + 1)).double()  # nearest in log2 distance; the grid of a binade is n .. 2n - 1
    e = torch.where(t >= 2 * n, e + 1, e)
    j = torch.where(t >= 2 * n, torch.zeros_like(t), t - n)
    j = torch.where(e < -6, torch.zeros_like(j), j)
    zero = u.double() * u.double() <= 2.0 ** -13
    field = torch.where(zero, torch.full_like(e, 7), (-e).clamp(0, 6) + 8 * (x < 0).int())
    return field.to(torch.uint8), torch.where(zero, torch.zeros_like(j), j).to(torch.uint8), s[..., 0]


def _pack_keys(field, j, k):
    """codes_se [..., 32] and codes_m [..., 8k] (None at k = 0) of nibbles and mantissas [..., 64]."""
    pairs = field.unflatten(-1, (32, 2))
    se = pairs[..., 0] | (pairs[..., 1] << 4)
    if not k:
        return se, None
    bits = (j.unsqueeze(-2) >> torch.arange(k, dtype=torch.uint8, device=DEV)[:, None]) & 1
    bits = bits.unflatten(-1, (8, 8)) << torch.arange(8, dtype=torch.uint8, device=DEV)
    return se, bits.sum(-1, dtype=torch.uint8).flatten(-2)


def _key_weights(se, cm, k):
    """sign (1 + j / 2^k) 2^-e of every element (fp32, exact), 0 for the zero code."""
    f = torch.stack((se & 15, se >> 4), -1).flatten(-2)
    w = torch.exp2(-(f & 7).float())
    if k:
        bits = (cm.unflatten(-1, (k, 8)).unsqueeze(-1) >> torch.arange(8, dtype=torch.uint8, device=DEV)) & 1
        steps = torch.exp2(torch.arange(k, device=DEV).float() - k)
        w = w * (1 + (bits.flatten(-2).float() * steps[:, None]).sum(-2))
    w = torch.where(f >= 8, -w, w)
    return torch.where((f & 7) == 7, torch.zeros_like(w), w)


def _value_codes(v):
    """(n uint8 [..., 64], s, z fp16 [...]) of fp16 rows."""
    x = v.float()
    z, hi = x.amin(-1), x.amax(-1)
    f = _over(hi - z, 15.0)
    s = f.half()
    s = torch.where(s.float() < f, (s.view(torch.int16) + 1).view(torch.float16), s)
    n = torch.round((x - z[..., None]) * _over(1.0, s.float())[..., None]).clamp(max=15)
    n = torch.where(s[..., None] > 0, n, torch.zeros_like(n))
    return n.to(torch.uint8), s, z.half()


def _pack_values(n, s, z):
    """The bytes of whole groups: n [..., 8 g, 64], s and z [..., 8 g] to [..., g, 288]."""
    n = n.unflatten(-2, (-1, 8)).unflatten(-1, (2, 2, 16))  # [..., g, 8, half, low / high, 16]
    b = (n[..., 0, :] | (n[..., 1, :] << 4)).movedim(-1, -3).transpose(-1, -2)  # [..., g, 16, half, 8]
    sz = torch.stack((s.unflatten(-1, (-1, 8)), z.unflatten(-1, (-1, 8))), -2).contiguous()
    return torch.cat((b.flatten(-3), sz.view(torch.uint8).flatten(-2)), -1)


def _unpack_values(g):
    """The values (fp32 [..., 8 g, 64]) that whole groups [..., g, 288] stand for."""
    b = g[..., :256].unflatten(-1, (16, 2, 8)).movedim(-1, -3)  # [..., g, 8, 16, half]
    n = torch.stack((b & 15, b >> 4), -1).movedim(-3, -1).flatten(-3).float()  # [..., g, 8, half x low / high x 16]
    sz = g[..., 256:].contiguous().view(torch.float16).float().unflatten(-1, (2, 8, 1))
    return (sz[..., 1, :, :] + sz[..., 0, :, :] * n).flatten(-3, -2)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _channel_scale(g, Hkv):
    return torch.rand((Hkv, 1, D), generator=g, device=DEV) * 3.5 + 0.5


def _axis_of_pair(case):
    """Sections of pairs side by side, as even as they go."""
    pairs = case["rot_dim"] // 2
    return [i * case["axes"] // pairs for i in range(pairs)]


def _prepare_qkv(case, g):
    B, S, Hq, Hkv = case["B"], case["S"], case["Hq"], case["Hkv"]
    dtype = DTYPES[case["dtype"]]
    if case["layout"] == "packed":
        x = _randn(g, B, S, Hq + 2 * Hkv, D).to(dtype)
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    else:
        q, k, v = (_randn(g, B, h, S, D).to(dtype).transpose(1, 2) for h in (Hq, Hkv, Hkv))
    starts = torch.randint(0, 4096, (case["axes"], B, 1), generator=g, device=DEV)
    pos = starts + case["far"] + torch.arange(S, device=DEV)
    st = dict(q=q, k=k, v=v, positions=pos.contiguous(),
              inv_freq=10000.0 ** (-torch.arange(0, case["rot_dim"], 2, dtype=torch.float64, device=DEV) / case["rot_dim"]),
              q_weight=None, k_weight=None,
              q_out=torch.empty((B, Hq, S, D), dtype=DTYPES[case["q_out"]], device=DEV),
              k_out=torch.empty((B, Hkv, S, D), dtype=torch.float16, device=DEV),
              v_out=torch.empty((B, Hkv, S, D), dtype=torch.float16, device=DEV))
    if case["norm"]:
        st["q_weight"], st["k_weight"] = (1 + 0.2 * _randn(g, D)).to(dtype), (1 + 0.2 * _randn(g, D)).to(dtype)
    return st


def _prepare_cache(case, g, c, rows):
    """Key codes of `rows` rows a sequence, as a filled cache holds them."""
    B, Hkv, k = case["B"], case["Hkv"], case["k"]
    x = (_randn(g, B, Hkv, rows, D) * c).half()
    field, j, s = _key_codes(_rotated(x, case["hadamard"]), k)
    se, cm = _pack_keys(field, j, k)
    return dict(codes_se=se, codes_m=cm, key_scale=s)


def prepare(case, seed):
    g = _generator(seed)
    if case["kind"] == "qkv":
        return dict(_prepare_qkv(case, g), case=case)
    B, Hkv, t_cap = case["B"], case["Hkv"], case["t_cap"]
    n_seq = B * Hkv
    if case["kind"] == "values":
        rows = _randn(g, n_seq, case["n_tok"], D).half()
        return dict(case=case, v=rows, v_u4=torch.zeros((B, Hkv, t_cap // 8, GROUP), dtype=torch.uint8, device=DEV),
                    v_out=torch.empty_like(rows))
    c = _channel_scale(g, Hkv)
    st = dict(_prepare_cache(case, g, c, t_cap), case=case)
    if case["kind"] == "keys":
        st["k_out"] = torch.empty((n_seq, case["n_tok"], D), dtype=torch.float16, device=DEV)
        return st
    Hq = case["Hq"]
    st["v_u4"] = _pack_values(*_value_codes(_randn(g, B, Hkv, t_cap, D).half()))
    st["q"] = _randn(g, B, Hq, D)
    st["k_new"] = (_randn(g, B, Hkv, D) * c.view(1, Hkv, D)).half()
    st["v_new"] = _randn(g, B, Hkv, D).half()
    st["k_row"], st["v_row"] = torch.empty((n_seq, 1, D), dtype=torch.float16, device=DEV), torch.empty(
        (n_seq, 1, D), dtype=torch.float16, device=DEV)
    st["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV) if case["ragged"] else None
    st["heads"] = np.arange(Hq, dtype=np.int32) // (Hq // Hkv)
    st["out"] = torch.empty((B, Hq, D), dtype=torch.float32, device=DEV)
    st["workspace"] = torch.empty(32 << 20, dtype=torch.uint8, device=DEV)
    return st


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _run_own(st):
    import paper_2609_09208_amd as pa
    case = st["case"]
    kind = case["kind"]
    if kind == "qkv":
        if "rope" not in st:
            st["rope"] = pa.make_rope(rot_dim=case["rot_dim"], neighbours=case["pairing"] == "neighbours",
                                      axis_of_pair=_axis_of_pair(case))
        pa.pot_norm_rope(st["rope"], st["q"], st["k"], st["v"], st["q_weight"], st["k_weight"], EPS, st["positions"],
                         st["inv_freq"], st["q_out"], st["k_out"], st["v_out"])
        return dict(q=st["q_out"], k=st["k_out"], v=st["v_out"])
    n_seq, t_cap = case["B"] * case["Hkv"], case["t_cap"]
    if kind == "values":
        pa.pot_store_values_int4(st["v"], n_seq, case["n_tok"], t_cap, case["t0"], st["v_u4"])
        pa.pot_load_values_int4(st["v_u4"], n_seq, case["n_tok"], t_cap, case["t0"], st["v_out"])
        return dict(values=st["v_out"])
    if "fmt" not in st:
        st["fmt"] = pa.make_format(mant_bits=case["k"], hadamard=case["hadamard"])
    fmt, se, cm, sc = st["fmt"], st["codes_se"], st["codes_m"], st["key_scale"]
    if kind == "keys":
        pa.pot_load_keys(fmt, se, cm, sc, n_seq, case["n_tok"], t_cap, case["t0"], st["k_out"])
        return dict(keys=st["k_out"])
    B, Hq, Hkv, T = case["B"], case["Hq"], case["Hkv"], case["T"]
    if kind == "attend":
        pa.pot_decode_attention_v4(fmt, case["engine"], st["q"], se, cm, sc, st["v_u4"], t_cap, st["lengths"], st["heads"],
                                   B, Hq, Hkv, T, st["out"], st["workspace"])
        return dict(out=st["out"])
    pa.pot_append_decode_attention_v4(fmt, case["engine"], st["q"], st["k_new"], st["v_new"], se, cm, sc, st["v_u4"], t_cap,
                                      st["lengths"], st["heads"], B, Hq, Hkv, T, st["out"], st["workspace"])
    # the row that was taken in, read back where every sequence has it at T - 1
    pa.pot_load_keys(fmt, se, cm, sc, n_seq, 1, t_cap, T - 1, st["k_row"])
    pa.pot_load_values_int4(st["v_u4"], n_seq, 1, t_cap, T - 1, st["v_row"])
    return dict(out=st["out"], k_row=st["k_row"], v_row=st["v_row"])


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _turned(x, w, cos, sin, case):
    """fp32 rows [B, S, H, 64] after norm and rotation; cos and sin [B, S, 1, pairs]."""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    r = case["rot_dim"]
    if case["pairing"] == "halves":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, y[..., r:]), -1)
    a, b = y[..., 0:r:2], y[..., 1:r:2]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), y[..., r:]), -1)


def _plain_qkv(st):
    case = st["case"]
    axis = torch.tensor(_axis_of_pair(case), device=DEV)
    angle = st["positions"][axis].movedim(0, -1).double() * st["inv_freq"]
    cos, sin = angle.cos().float().unsqueeze(2), angle.sin().float().unsqueeze(2)
    q = _turned(st["q"], st["q_weight"], cos, sin, case)
    k = _turned(st["k"], st["k_weight"], cos, sin, case)
    rows = lambda x, dtype: x.transpose(1, 2).to(dtype).contiguous()  # noqa: E731
    return dict(q=rows(q, DTYPES[case["q_out"]]), k=rows(k, torch.float16), v=rows(st["v"], torch.float16))


def _plain_keys(st, first, last):
    """fp16 rows first .. last - 1 of every sequence."""
    case = st["case"]
    cm = st["codes_m"][:, :, first:last] if case["k"] else None
    x = _key_weights(st["codes_se"][:, :, first:last], cm, case["k"]) * st["key_scale"][:, :, first:last, None]
    x = x @ (_hadamard().float() / 8) if case["hadamard"] else x
    return x.half().flatten(0, 1)


def _plain_attend(st):
    case = st["case"]
    B, Hq, Hkv, T = case["B"], case["Hq"], case["Hkv"], case["T"]
    x = _rotated(st["q"], case["hadamard"]).view(B, Hkv, Hq // Hkv, D)
    top = x.abs().amax(-1, keepdim=True)
    qi = torch.round(x * _over(127.0, top)).clamp(-127, 127)
    cm = st["codes_m"][:, :, :T] if case["k"] else None
    w = _key_weights(st["codes_se"][:, :, :T], cm, case["k"])
    scores = (qi @ w.transpose(-1, -2)) * st["key_scale"][:, :, None, :T] * (_over(top, 127.0) / 8)
    if case["ragged"]:
        there = torch.arange(T, device=DEV) < st["lengths"].view(B, 1, 1, 1)
        scores = torch.where(there, scores, torch.full_like(scores, -math.inf))
    most = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(most > -math.inf, most, torch.zeros_like(most)))
    total = p.sum(-1, keepdim=True)
    v = _unpack_values(st["v_u4"][:, :, :(T + 7) // 8])[:, :, :T]
    return ((p @ v) / torch.where(total > 0, total, torch.ones_like(total))).view(B, Hq, D)


def _plain_take_in(st):
    """The new token of every sequence that has one, written at the sequence's last row."""
    case = st["case"]
    B, Hkv, k = case["B"], case["Hkv"], case["k"]
    lengths = torch.tensor(_lengths(case), device=DEV)
    b = torch.nonzero(lengths)[:, 0]
    t = lengths[b] - 1
    field, j, s = _key_codes(_rotated(st["k_new"], case["hadamard"]), k)
    se, cm = _pack_keys(field, j, k)
    st["codes_se"][b, :, t], st["key_scale"][b, :, t] = se[b], s[b]
    if k:
        st["codes_m"][b, :, t] = cm[b]
    n, s, z = _value_codes(st["v_new"])
    # the token's bytes of its group: 16 columns of 2 bytes 8 apart, then its s and z
    new = _pack_values(n.unsqueeze(-2).expand(-1, -1, 8, -1), s.unsqueeze(-1).expand(-1, -1, 8),
                       z.unsqueeze(-1).expand(-1, -1, 8))[:, :, 0]
    byte = torch.arange(GROUP, device=DEV)
    token = torch.where(byte < 256, byte % 8, (byte - 256) // 2 % 8)
    old = st["v_u4"][b, :, t // 8]
    st["v_u4"][b, :, t // 8] = torch.where(token == (t % 8).view(-1, 1, 1), new[b], old)


def _plain(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "qkv":
        return _plain_qkv(st)
    if kind == "values":
        n, s, z = _value_codes(st["v"])
        return dict(values=(z.float()[..., None] + s.float()[..., None] * n.float()).half())
    if kind == "keys":
        return dict(keys=_plain_keys(st, case["t0"], case["t0"] + case["n_tok"]))
    if kind == "attend":
        return dict(out=_plain_attend(st))
    _plain_take_in(st)
    T = case["T"]
    row = _unpack_values(st["v_u4"][:, :, (T - 1) // 8]).half().unflatten(-2, (-1, 8))[..., (T - 1) % 8, :]
    return dict(out=_plain_attend(st), k_row=_plain_keys(st, T - 1, T), v_row=row.reshape(-1, 1, D))


def run(state):
    return _run_own(state) if own else _plain(state)


def work(case):
    B = case["B"]
    if case["kind"] == "qkv":
        size = {"fp16": 2, "bf16": 2, "fp32": 4}
        kv, rows = 2 * case["Hkv"], B * case["S"]
        per = (case["Hq"] + kv) * size[case["dtype"]] + case["Hq"] * size[case["q_out"]] + kv * 2
        per_element = 6 if case["norm"] else 3
        return {"bytes": rows * (D * per + 8 * case["axes"]),
                "flops": rows * (case["Hq"] + case["Hkv"]) * D * per_element}
    if case["kind"] == "values":
        rows = B * case["Hkv"] * case["n_tok"]
        return {"bytes": rows * (128 + 36 + 36 + 128), "flops": rows * D * 8}
    row = 36 + 8 * case["k"]
    if case["kind"] == "keys":
        rows = B * case["Hkv"] * case["n_tok"]
        return {"bytes": rows * (row + 128), "flops": rows * D * (13 if case["hadamard"] else 1)}
    keys = sum(_lengths(case))
    new = B * case["Hkv"] * (256 + 3 * (row + 36) + 256) if case["kind"] == "append" else 0
    return {"bytes": keys * case["Hkv"] * (row + 36) + B * case["Hq"] * D * 8 + new, "flops": keys * case["Hq"] * D * 4}


# ---- the same in 64 bits, from the definitions ----------------------------------------------------------------------

def _exact_value_rows(v):
    """What value rows stand for, and what the codes are made of, with the definition's fp32 roundings."""
    x = v.double()
    z = x.amin(-1, keepdim=True)
    f = ((x.amax(-1, keepdim=True) - z).float().double() / torch.full_like(z, 15.0)).float().double()
    ulp = torch.exp2((torch.floor(torch.log2(f.clamp(min=2.0 ** -24))) - 10).clamp(min=-24))
    s = torch.ceil(f / ulp) * ulp
    inv = torch.where(s > 0, (torch.ones_like(s) / s).float().double(), torch.zeros_like(s))
    return z + s * torch.round(((x - z).float().double() * inv).float().double()).clamp(max=15)


def _exact_unpacked(g):
    """fp64 values of whole groups, by looking every element's byte up."""
    t, c = torch.arange(8, device=DEV)[:, None], torch.arange(D, device=DEV)
    byte = g[..., 16 * (c % 16) + 8 * (c // 32) + t].long()
    n = torch.where(c % 32 < 16, byte % 16, byte // 16).double()
    sz = g[..., 256:].contiguous().view(torch.float16).double()
    return (sz[..., 8:, None] + sz[..., :8, None] * n).flatten(-3, -2)


def _exact_sylvester():
    h = torch.ones((1, 1), dtype=torch.float64, device=DEV)
    for _ in range(6):
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h


def _exact_weights(se, cm, k):
    """fp64 sign (1 + j / 2^k) 2^-e: magnitudes from a table of the 16 fields, mantissa bits one plane at a time."""
    table = torch.tensor([2.0 ** -e for e in range(7)] + [0.0] + [-2.0 ** -e for e in range(7)] + [0.0], dtype=torch.float64,
                         device=DEV)
    m = torch.arange(D, device=DEV)
    w = table[((se.index_select(-1, m // 2) >> (4 * (m % 2)).to(torch.uint8)) & 15).long()]
    j = torch.zeros_like(w)
    for b in range(k):
        j += ((cm.index_select(-1, 8 * b + m // 8) >> (m % 8).to(torch.uint8)) & 1).double() * 2.0 ** (b - k)
    return w * (1 + j)


def _exact_key_rows(x, case):
    """fp64 rows that new keys stand for, in the domain that the codes hold: the nearest grid value in log2 distance."""
    k, n = case["k"], 2 ** case["k"]
    x = (x.double() @ _exact_sylvester() / 8).float().double() if case["hadamard"] else x.double()
    s = x.abs().amax(-1, keepdim=True)
    u = (x.abs() / s).float().double()
    grid = [(1 + j / n) * 2.0 ** -e for e in range(7) for j in range(n) if e or not j]  # the top is the maximum itself
    grid = torch.tensor(sorted(grid), dtype=torch.float64, device=DEV)
    above = (u[..., None] ** 2 > grid[:-1] * grid[1:]).sum(-1)
    val = torch.where(u * u > 2.0 ** -13, grid[above], torch.zeros_like(u))
    return torch.sign(x) * val * s


def _exact_attend(case, st, new=None):
    """fp64 attention, batch row by batch row; new: the decoded last row of every sequence that takes one in."""
    B, Hq, Hkv = case["B"], case["Hq"], case["Hkv"]
    x = st["q"].double()
    x = (x @ _exact_sylvester() / 8).float().double() if case["hadamard"] else x
    top = x.abs().amax(-1, keepdim=True)
    inv = (torch.full_like(top, 127.0) / top).float().double()
    qd = torch.round((x * inv).float().double()).clamp(-127, 127) * (top / torch.full_like(top, 127.0)).float().double()
    qd = qd.view(B, Hkv, Hq // Hkv, D)
    out = torch.zeros((B, Hkv, Hq // Hkv, D), dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        cm = st["codes_m"][b, :, :n] if case["k"] else None
        kd = _exact_weights(st["codes_se"][b, :, :n], cm, case["k"]) * st["key_scale"][b, :, :n, None].double()
        vd = _exact_unpacked(st["v_u4"][b, :, :(n + 7) // 8])[:, :n]
        if new is not None:
            kd[:, n - 1], vd[:, n - 1] = new[0][b], new[1][b]
        p = torch.softmax(qd[b] @ kd.transpose(-1, -2).contiguous() / 8, -1)
        out[b] = p @ vd
    return out.view(B, Hq, D)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "qkv":
        axis = torch.tensor(_axis_of_pair(case), device=DEV)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                           st["positions"].double()[axis].permute(1, 2, 0) * st["inv_freq"])[:, None]
        r = case["rot_dim"]
        i = torch.arange(r, device=DEV)
        order = i.view(2, r // 2) if case["pairing"] == "halves" else i.view(r // 2, 2).t()

        def rows(x, w):
            y = x.transpose(1, 2).double()
            if w is not None:
                y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS) * w.double()
            z = torch.complex(y[..., order[0]], y[..., order[1]]) * turn
            y[..., order[0]], y[..., order[1]] = z.real, z.imag
            return y

        return dict(q=rows(st["q"], st["q_weight"]), k=rows(st["k"], st["k_weight"]), v=st["v"].transpose(1, 2).double())
    if kind == "values":
        return dict(values=_exact_value_rows(st["v"]))
    if kind == "keys":
        at = slice(case["t0"], case["t0"] + case["n_tok"])
        x = _exact_weights(st["codes_se"][:, :, at], st["codes_m"][:, :, at] if case["k"] else None, case["k"])
        x = x * st["key_scale"][:, :, at, None].double()
        return dict(keys=(x @ _exact_sylvester() / 8 if case["hadamard"] else x).flatten(0, 1))
    if kind == "attend":
        return dict(out=_exact_attend(case, st))
    new = _exact_key_rows(st["k_new"], case), _exact_value_rows(st["v_new"])
    row = [None, None]
    if not case["ragged"]:
        k_row = new[0] @ _exact_sylvester() / 8 if case["hadamard"] else new[0]
        row = [k_row.reshape(-1, 1, D), new[1].reshape(-1, 1, D)]
    return dict(out=_exact_attend(case, st, new), k_row=row[0], v_row=row[1])
