"""A paged key and value cache: what takes new tokens in, and the attention of new tokens over it, as timed cases.

Four kinds of pass, at the head shapes and key formats of the tests and the benchmark:

- "append": the rows of a QKV projection, of sequences of any number of new tokens side by side, into the pages of a PoT key
  cache: RMS norm of queries and keys per head and the position rotation, key codes, values in fp16 or 4 bits
  (pot_paged_append); the pages are then read back as the rows that they stand for (pot_load_keys, pot_load_values or
  pot_load_values_int4).
- "attend": attention of each sequence's new tokens over its pages, causal (pot_paged_attention): chunks of a prompt, single
  tokens, and both in one batch.
- "window": the same where a query sees only the last `window` tokens and the first `sinks`. Pages that nobody sees are not
  there any more (their table entries are -1).
- "step": "append", then "attend" or "window" over the same pages, as a layer makes the two calls.

Keys are N(0, 1) times a per-channel scale from U[0.5, 4] (outlier channels), values and queries N(0, 1).

Definitions (fl: rounded to fp32; d = 64):
- token t of sequence b is row t % page_size of page table[b][t // page_size]. The new tokens of sequence b are its last ones.
- norm and rotation: y = x / sqrt(mean x^2 + eps) * w; pair i of a rotated head, on axis a, turns by the angle
  position_a * inv_freq_i. Keys are then rounded to fp16, and so are values.
- a key code stands for s * sign * (1 + j / 2^k) * 2^-e, s the row's absolute maximum, nearest in log2 distance; values
  up to s * 2^-6.5 are zero. With hadamard the row is H K / 8 (H the 64 x 64 Sylvester matrix).
- a value row in 4 bits is held as z = its minimum (fp16), s = the smallest fp16 number >= fl(fl(max - min) / 15) and
  n = min(15, round-half-even(fl(fl(v - z) * fl(1 / s)))), and stands for z + s n rounded to fp16.
- a query is rotated like the keys and held in 8 bits: round-half-even(fl(q * fl(127 / max|q|))) steps of max|q| / 127. The
  query at place t sees the keys at places j <= t with j > t - window or j < sinks.

The fp16 value cache holds groups of 8 tokens, dimension by dimension. The 4-bit one holds groups of 8 tokens in 288 bytes
each: byte 16 (c % 16) + 8 (c / 32) + t % 8 has dimension c in its low half where c % 32 < 16 and in its high half elsewhere;
at 256 stand the group's 8 fp16 s, at 272 its 8 fp16 z.
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


def _case(kind, B, Hq, Hkv, new, T, page, k, values, dtype, out="fp32", chunks=None, ragged=False, window=0, sinks=0,
          hadamard=False, packed=True, norm=True, rot_dim=64, pairing="halves", axes=1, name=None):
    """new: the tokens that each of the first `chunks` sequences brings (all of them, without it); the others bring one. T:
    the tokens of a sequence with them, or of the longest. dtype: of the projection; out: of queries, or of the attention."""
    c = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, new=new, T=T, page=page, k=k, values=values, dtype=dtype, out=out,
             chunks=B if chunks is None else chunks, ragged=ragged, window=window, sinks=sinks, hadamard=hadamard,
             packed=packed, norm=norm, rot_dim=rot_dim, pairing=pairing, axes=axes)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # the new token of one chat: latency
        _case("append", 1, 32, 4, 1, 1001, 16, 0, "int4", "bf16", name="append_b1_one_token_pot4"),
        # one step of a full batch of sequences of all lengths, of a model that reads images (three position axes)
        _case("append", 64, 32, 4, 1, 8000, 64, 0, "int4", "fp16", ragged=True, axes=3, name="append_b64_one_token_axes3"),
        # four prompts of ordinary length, one packed projection, the most accurate keys, values as they are
        _case("append", 4, 32, 4, 2048, 2048, 64, 4, "fp16", "bf16", "bf16", name="append_m4_b4_s2048"),
        # chunks of odd lengths behind cached prefixes: fp32, separate projections, half of each head turned in neighbouring
        # pairs, rotated keys, the smallest pages
        _case("append", 5, 16, 8, 777, 1900, 8, 2, "int4", "fp32", "fp16", ragged=True, hadamard=True, packed=False, norm=False,
              rot_dim=32, pairing="neighbours", axes=2, name="append_m2_hadamard_ragged_s777"),
        # a chunk of a long prompt, taken in piece by piece
        _case("attend", 1, 32, 4, 512, 8192, 64, 0, "int4", "bf16", "bf16", name="attend_pot4_b1_s512_t8192"),
        # a whole prompt at once: the largest case
        _case("attend", 1, 32, 4, 8192, 8192, 64, 1, "fp16", "bf16", "bf16", name="attend_m1_b1_s8192"),
        # a serving batch: two prompts' chunks beside the single tokens of the others, one slot empty
        _case("attend", 16, 32, 4, 300, 8191, 16, 2, "int4", "fp16", "fp16", chunks=2, ragged=True,
              name="attend_m2_b16_mixed_t8191"),
        # drafts of four tokens checked at once, four query heads a kv head
        _case("attend", 32, 16, 4, 4, 4096, 32, 0, "fp16", "fp32", "fp32", name="attend_pot4_b32_s4_t4096_g4"),
        # one step of a serving batch
        _case("attend", 64, 32, 4, 1, 8192, 64, 0, "int4", "fp32", "fp32", name="attend_pot4_b64_t8192"),
        # one step of a model with a window, far into its texts
        _case("window", 64, 32, 4, 1, 32768, 128, 0, "fp16", "fp32", "fp32", ragged=True, window=4096, sinks=4,
              name="window4096_pot4_b64_t32768"),
        # a chunk of two prompts of such a model, odd window
        _case("window", 2, 32, 8, 2048, 4096, 32, 4, "int4", "fp16", "fp16", hadamard=True, window=1000, sinks=5,
              name="window1000_m4_hadamard_b2_s2048"),
        # a layer's step at full batch and long texts: the new tokens taken in, then the attention
        _case("step", 64, 32, 4, 1, 16384, 64, 0, "int4", "bf16", "bf16", name="step_pot4_b64_t16384"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "window", "window", "step"])
    Hq, Hkv = rng.choice([(32, 4), (32, 4), (32, 8), (16, 4), (16, 8), (8, 8), (64, 8), (24, 4), (16, 1)])
    page = rng.choice([8, 16, 16, 32, 64, 64, 128, 48, 256])
    k, values, hadamard = rng.choice([0, 0, 1, 2, 3, 4]), rng.choice(["fp16", "int4"]), rng.random() < 0.25
    dtype, out = rng.choice(["bf16", "fp16", "fp32"]), rng.choice(["bf16", "fp16", "fp32"])
    ragged = rng.random() < 0.5
    turn = dict(packed=rng.random() < 0.7, norm=rng.random() < 0.7, rot_dim=rng.choice([64, 64, 32, 48]),
                pairing=rng.choice(["halves", "halves", "neighbours"]), axes=rng.choice([1, 1, 2, 3]))
    if kind == "append":
        # keys of few bits in small calls only: their steps are as large as what they stand for, and a key that lies between
        # two of them may come out as either
        tokens = _log_int(rng, 1, 8192 if k >= 2 else 256)
        B = _log_int(rng, 1, min(64, tokens))
        new = max(1, tokens // B)
        return _case(kind, B, Hq, Hkv, new, new + rng.choice([0, 0, rng.randrange(0, 1000)]), page, k, values, dtype, out,
                     ragged=ragged, hadamard=hadamard, **turn)
    if kind == "step":
        out = rng.choice(["bf16", "fp16"])
    # T over its whole range; B so that a batch has at most 2^19 tokens in its cache; new ones so that there are at most
    # 2^25 pairs of a query and a key that it sees
    T = _log_int(rng, 1, 32768)
    B = _log_int(rng, 1, max(1, min(64, 2 ** 21 // (T * Hkv))))
    window = _log_int(rng, 1, 8192) if kind == "window" or (kind == "step" and rng.random() < 0.3) else 0
    most = max(1, min(T, 8192, 2 ** 25 * 32 // (Hq * B * min(T, window or T)), 2 ** 27 * 32 // (Hq * B * T)))
    new = rng.choice([1, 1, _log_int(rng, 1, most), _log_int(rng, 1, most)])
    new = min(new, most)
    return _case(kind, B, Hq, Hkv, new, T, page, k, values, dtype, out, chunks=rng.choice([B, B, max(1, B // 4)]),
                 ragged=ragged, window=window, sinks=rng.choice([0, 1, 4, 37]) if window else 0, hadamard=hadamard, **turn)


def _lengths(case):
    """New tokens and all tokens of each sequence: all T, or in a ragged batch from T down in equal steps, the last of four
    or more none."""
    B, T = case["B"], case["T"]
    lens = [T] * B
    if case["ragged"]:
        lens = [T - b * T // B for b in range(B)]
        lens = lens[:-1] + [0] if B >= 4 else lens
    return [min(n, case["new"] if b < case["chunks"] else 1) for b, n in enumerate(lens)], lens


def _first_seen(case, new, length):
    """The first place past the sinks that a new token of the sequence sees."""
    return max(0, length - new + 1 - case["window"]) if case["window"] else 0


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


def _to_half(x):
    """fp64 numbers rounded to fp16 once (a conversion by way of fp32 rounds twice)."""
    ulp = torch.exp2((torch.frexp(x)[1].clamp(min=-13) - 11).double())
    return (torch.round(x / ulp) * ulp).half()


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


def _weights_of(field, j, k):
    """sign (1 + j / 2^k) 2^-e of every element (fp32, exact), 0 for the zero code."""
    e = field & 7
    w = torch.exp2(-e.float()) * (1 + j.float() / 2 ** k)
    return torch.where(e == 7, torch.zeros_like(w), torch.where(field >= 8, -w, w))


def _key_weights(se, cm, k):
    f = torch.stack((se & 15, se >> 4), -1).flatten(-2)
    j = torch.zeros_like(f)
    if k:
        bits = (cm.unflatten(-1, (k, 8)).unsqueeze(-1) >> torch.arange(8, dtype=torch.uint8, device=DEV)) & 1
        j = (bits.flatten(-2) << torch.arange(k, dtype=torch.uint8, device=DEV)[:, None]).sum(-2, dtype=torch.uint8)
    return _weights_of(f, j, k)


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


def _values_of(n, s, z):
    """The fp16 rows that 4-bit rows stand for (as fp32 numbers)."""
    return _to_half(z.double()[..., None] + s.double()[..., None] * n.double()).float()


def _pack_values(n, s, z):
    """The bytes of whole groups: n [..., 8 g, 64], s and z [..., 8 g] to [..., g, 288]."""
    n = n.unflatten(-2, (-1, 8)).unflatten(-1, (2, 2, 16))  # [..., g, 8, half, low / high, 16]
    b = (n[..., 0, :] | (n[..., 1, :] << 4)).movedim(-1, -3).transpose(-1, -2)  # [..., g, 16, half, 8]
    sz = torch.stack((s.unflatten(-1, (-1, 8)), z.unflatten(-1, (-1, 8))), -2).contiguous()
    return torch.cat((b.flatten(-3), sz.view(torch.uint8).flatten(-2)), -1)


def _unpack_values(g):
    """The fp16 rows (fp32 [..., 8 g, 64]) that whole groups [..., g, 288] stand for."""
    b = g[..., :256].unflatten(-1, (16, 2, 8)).movedim(-1, -3)  # [..., g, 8, 16, half]
    n = torch.stack((b & 15, b >> 4), -1).movedim(-3, -1).flatten(-3).flatten(-3, -2)  # [..., 8 g, half x low / high x 16]
    sz = g[..., 256:].contiguous().view(torch.float16).unflatten(-1, (2, 8))
    return _values_of(n, sz[..., 0, :].flatten(-2), sz[..., 1, :].flatten(-2))


def _interleaved(v):
    """fp16 rows [..., 8 g, 64] in the order of the fp16 value cache (same shape)."""
    return v.unflatten(-2, (-1, 8)).transpose(-1, -2).reshape(v.shape)


def _value_rows(st):
    """fp32 rows [pages, Hkv, page, 64] of the value cache."""
    if st["case"]["values"] == "int4":
        return _unpack_values(st["values"])
    v = st["values"]
    return v.reshape(*v.shape[:-2], -1, D, 8).transpose(-1, -2).reshape(v.shape).float()


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _axis_of_pair(case):
    """Sections of pairs side by side, as even as they go."""
    pairs = case["rot_dim"] // 2
    return [i * case["axes"] // pairs for i in range(pairs)]


def _page_table(case, g):
    """Page numbers [B, entries] in any order, -1 where no new token sees or writes the page, and the number of pages."""
    page, (news, lens) = case["page"], _lengths(case)
    entries = max(1, -(-max(lens) // page))
    there = np.zeros((case["B"], entries), dtype=bool)
    for b, (new, n) in enumerate(zip(news, lens)):
        if new:
            first = n - new if case["kind"] == "append" else _first_seen(case, new, n)
            there[b, first // page:(n - 1) // page + 1] = True
            if case["kind"] != "append":
                there[b, :-(-min(n, case["sinks"]) // page)] = True
    there = torch.from_numpy(there).to(DEV)
    used = int(there.sum())
    table = torch.full(there.shape, -1, dtype=torch.int32, device=DEV)
    n_pages = used + 3
    table[there] = torch.randperm(n_pages, generator=g, device=DEV)[:used].int()
    return table, n_pages


def _projection(case, g, n):
    dtype, Hq, Hkv = DTYPES[case["dtype"]], case["Hq"], case["Hkv"]
    if case["packed"]:
        x = _randn(g, n, Hq + 2 * Hkv, D).to(dtype)
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return [_randn(g, h, n, D).to(dtype).transpose(0, 1) for h in (Hq, Hkv, Hkv)]


def prepare(case, seed):
    g = _generator(seed)
    Hkv, Hq, page, k = case["Hkv"], case["Hq"], case["page"], case["k"]
    news, lens = _lengths(case)
    n = sum(news)
    table, n_pages = _page_table(case, g)
    st = dict(case=case, table=table, n_pages=n_pages,
              cu_new=torch.tensor(np.concatenate(([0], np.cumsum(news))), dtype=torch.int32, device=DEV),
              seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
              heads=np.arange(Hq, dtype=np.int32) // (Hq // Hkv))
    c = torch.rand((Hkv, 1, D), generator=g, device=DEV) * 3.5 + 0.5
    if case["kind"] == "append":
        rows = torch.zeros((n_pages, Hkv, page, D), dtype=torch.float16, device=DEV)
        v = rows
    else:
        rows = (_randn(g, n_pages, Hkv, page, D) * c).half()
        v = _randn(g, n_pages, Hkv, page, D).half()
    field, j, s = _key_codes(_rotated(rows, case["hadamard"]), k)
    st["codes_se"], st["codes_m"] = _pack_keys(field, j, k)
    st["key_scale"] = s
    st["values"] = _pack_values(*_value_codes(v)) if case["values"] == "int4" else _interleaved(v)
    q, st["k"], st["v"] = _projection(case, g, n)
    out = DTYPES[case["out"]]
    if case["kind"] in ("attend", "window"):
        st["q"] = q
        st["out"] = torch.empty((n, Hq, D), dtype=out, device=DEV)
        return st
    st["q"] = q
    at = torch.cat([torch.arange(m - w, m) for w, m in zip(news, lens)]).to(DEV)
    st["positions"] = torch.stack([at // (a + 1) for a in range(case["axes"])]).contiguous()
    st["inv_freq"] = 10000.0 ** (-torch.arange(0, case["rot_dim"], 2, dtype=torch.float64, device=DEV) / case["rot_dim"])
    st["q_weight"] = st["k_weight"] = None
    if case["norm"]:
        st["q_weight"], st["k_weight"] = ((1 + 0.2 * _randn(g, D)).to(DTYPES[case["dtype"]]) for _ in range(2))
    st["q_out"] = torch.empty((n, Hq, D), dtype=out if case["kind"] == "append" else torch.float32, device=DEV)
    if case["kind"] == "step":
        st["out"] = torch.empty((n, Hq, D), dtype=out, device=DEV)
    else:
        st["k_rows"] = torch.empty((n_pages * Hkv, page, D), dtype=torch.float16, device=DEV)
        st["v_rows"] = torch.empty_like(st["k_rows"])
    return st


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _run_own(st):
    import paper_2609_09208_amd as pa
    case = st["case"]
    B, Hq, Hkv, page = case["B"], case["Hq"], case["Hkv"], case["page"]
    if "fmt" not in st:  # what a program makes once
        st["fmt"] = pa.make_format(mant_bits=case["k"], hadamard=case["hadamard"])
        st["pages"] = pa.make_pages(st["codes_se"], st["codes_m"], st["key_scale"], st["values"], st["table"])
        if "positions" in st:
            st["rope"] = pa.make_rope(rot_dim=case["rot_dim"], neighbours=case["pairing"] == "neighbours",
                                      axis_of_pair=_axis_of_pair(case))
        if "out" in st:
            n_bytes = pa.pot_paged_workspace_bytes(B, st["q"].shape[0], Hq, Hkv, case["new"], case["T"])
            st["workspace"] = pa.alloc_workspace(n_bytes, DEV)
    q = st["q"]
    if "positions" in st:
        pa.pot_paged_append(st["fmt"], st["rope"], q, st["k"], st["v"], st["q_weight"], st["k_weight"], EPS, st["positions"],
                            st["inv_freq"], st["pages"], st["cu_new"], st["seq_lens"], st["q_out"])
        q = st["q_out"]
    if case["kind"] == "append":
        n_seq = st["n_pages"] * Hkv
        pa.pot_load_keys(st["fmt"], st["codes_se"], st["codes_m"], st["key_scale"], n_seq, page, page, 0, st["k_rows"])
        load = pa.pot_load_values_int4 if case["values"] == "int4" else pa.pot_load_values
        load(st["values"], n_seq, page, page, 0, st["v_rows"])
        return dict(q=q, keys=st["k_rows"], values=st["v_rows"])
    pa.pot_paged_attention(st["fmt"], q, st["pages"], st["cu_new"], st["seq_lens"], st["heads"], case["new"], case["T"],
                           st["out"], st["workspace"], window=case["window"], n_sink=case["sinks"])
    return dict(out=st["out"], q=q) if case["kind"] == "step" else dict(out=st["out"])


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _turned(x, w, cos, sin, case):
    """fp32 rows [n, H, 64] after norm and rotation; cos and sin [n, 1, pairs]."""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    r = case["rot_dim"]
    if case["pairing"] == "halves":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, y[..., r:]), -1)
    a, b = y[..., 0:r:2], y[..., 1:r:2]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), y[..., r:]), -1)


def _places(st):
    """Of every packed row: its sequence, its place there, and the first row of its sequence."""
    cu, n = st["cu_new"].long(), st["q"].shape[0]
    row = torch.arange(n, device=DEV)
    b = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    return b, st["seq_lens"].long()[b] - cu[b + 1] + row, cu[b]


def _plain_append(st):
    """The projection's queries, and the new keys (weights, scale) and values as the caches hold them."""
    case = st["case"]
    axis = torch.tensor(_axis_of_pair(case), device=DEV)
    angle = st["positions"][axis].t().double() * st["inv_freq"]
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    q = _turned(st["q"], st["q_weight"], cos, sin, case).to(st["q_out"].dtype)
    key = _turned(st["k"], st["k_weight"], cos, sin, case).half()
    field, j, s = _key_codes(_rotated(key, case["hadamard"]), case["k"])
    v = st["v"].half()
    v = _values_of(*_value_codes(v)) if case["values"] == "int4" else v.float()
    return q, _weights_of(field, j, case["k"]), s, v


def _plain_attend(st, q, w, s, v):
    """q [n, Hq, 64] over key weights w, scales s and values v [pages, Hkv, page, ...]."""
    case = st["case"]
    B, Hq, Hkv, page, T = case["B"], case["Hq"], case["Hkv"], case["page"], case["T"]
    G, new = Hq // Hkv, case["new"]
    x = _rotated(q, case["hadamard"])
    top = x.abs().amax(-1, keepdim=True)
    inv = torch.where(top > 0, _over(127.0, top), torch.zeros_like(top))
    qi, step = torch.round(x * inv).clamp(-127, 127), _over(top, 127.0) / 8
    # the new tokens by sequence, and every sequence's keys side by side
    row = (st["cu_new"][:-1, None].long() + torch.arange(new, device=DEV)).clamp(max=q.shape[0] - 1)
    by_head = lambda y: y[row].unflatten(2, (Hkv, G)).movedim(2, 1).flatten(2, 3)  # noqa: E731  [B, Hkv, new G, ...]
    qi, step = by_head(qi), by_head(step)
    t = torch.arange(T, device=DEV)
    p = st["table"].long()[:, t // page].clamp(min=0)
    keys, scale, vals = (y[p, :, (t % page).expand(B, T)].transpose(1, 2) for y in (w, s, v))
    scores = qi @ keys.transpose(-1, -2).contiguous()
    scores.mul_(scale.unsqueeze(2)).mul_(step)
    lens = st["seq_lens"].long()[:, None]
    at = lens - (st["cu_new"][1:] - st["cu_new"][:-1]).long()[:, None] + torch.arange(new, device=DEV)  # [B, new]
    sees = (t <= at[..., None]) & (t < lens[..., None])
    if case["window"]:
        sees = sees & ((t > at[..., None] - case["window"]) | (t < case["sinks"]))
    scores.unflatten(2, (new, G)).masked_fill_(~sees[:, None, :, None], -math.inf)
    most = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(most > -math.inf, most, torch.zeros_like(most))).exp_()
    total = scores.sum(-1, keepdim=True)
    o = (scores @ vals.contiguous()) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.unflatten(2, (new, G)).movedim(1, 2).flatten(2, 3)  # [B, new, Hq, 64]
    b, _, first = _places(st)
    return o[b, torch.arange(q.shape[0], device=DEV) - first].to(st["out"].dtype)


def _plain(st):
    case = st["case"]
    page, kind = case["page"], case["kind"]
    if kind in ("attend", "window"):
        w = _key_weights(st["codes_se"], st["codes_m"], case["k"])
        return dict(out=_plain_attend(st, st["q"], w, st["key_scale"], _value_rows(st)))
    q, w, s, v = _plain_append(st)
    b, at, _ = _places(st)
    p, u = st["table"].long()[b, at // page], at % page
    if kind == "append":
        x = w * s[..., None]
        x = (x @ (_hadamard().float() / 8)).half() if case["hadamard"] else x.half()
        keys, values = (torch.zeros((st["n_pages"], case["Hkv"], page, D), dtype=torch.float16, device=DEV) for _ in range(2))
        keys[p, :, u], values[p, :, u] = x, v.half()
        return dict(q=q, keys=keys.flatten(0, 1), values=values.flatten(0, 1))
    w_all, s_all, v_all = _key_weights(st["codes_se"], st["codes_m"], case["k"]), st["key_scale"].clone(), _value_rows(st)
    w_all[p, :, u], s_all[p, :, u], v_all[p, :, u] = w, s, v
    return dict(out=_plain_attend(st, q, w_all, s_all, v_all), q=q)


def run(state):
    return _run_own(state) if own else _plain(state)


def _seen(case):
    """Pairs of a new token and a key that it sees, and the keys of each sequence that some new token sees, in all."""
    pairs = keys = 0
    for new, n in zip(*_lengths(case)):
        if not new:
            continue
        at = np.arange(n - new, n, dtype=np.int64)
        low = np.maximum(0, at + 1 - case["window"]) if case["window"] else np.zeros_like(at)
        pairs += int((at + 1 - low + np.minimum(low, case["sinks"])).sum())
        first = _first_seen(case, new, n)
        keys += n - first + min(first, case["sinks"])
    return pairs, keys


def work(case):
    size = {"fp16": 2, "bf16": 2, "fp32": 4}
    Hq, Hkv, n = case["Hq"], case["Hkv"], sum(_lengths(case)[0])
    row = 36 + 8 * case["k"] + (36 if case["values"] == "int4" else 128)  # a key and its value
    w = {"bytes": 0, "flops": 0}
    if case["kind"] in ("append", "step"):
        out = size[case["out"]] if case["kind"] == "append" else 4
        w["bytes"] += n * (D * (Hq + 2 * Hkv) * size[case["dtype"]] + D * Hq * out + 8 * case["axes"] + Hkv * row)
        w["flops"] += n * (Hq + Hkv) * D * (6 if case["norm"] else 3) + n * Hkv * D * 12
        if case["kind"] == "append":
            w["bytes"] += n * Hkv * (row + 256)
    if case["kind"] != "append":
        pairs, keys = _seen(case)
        q = 4 if case["kind"] == "step" else size[case["dtype"]]
        w["bytes"] += keys * Hkv * row + n * Hq * D * (q + size[case["out"]])
        w["flops"] += pairs * Hq * D * 4
    return w


# ---- the same in 64 bits, from the definitions ----------------------------------------------------------------------

def _exact_half(x):
    """fp64 numbers rounded to fp16, as fp64: to whole steps of 2^(exponent - 10), the exponent at least -14."""
    a = x.abs()
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -14)))
    e = torch.where(torch.exp2(e) > a.clamp(min=2.0 ** -14), e - 1, e)
    step = torch.exp2(e - 10)
    return torch.round(x / step) * step


def _exact_value_rows(v):
    """What value rows in 4 bits stand for, with the definition's roundings."""
    x = v.double()
    z = x.amin(-1, keepdim=True)
    f = ((x.amax(-1, keepdim=True) - z).float().double() / torch.full_like(z, 15.0)).float().double()
    ulp = torch.exp2((torch.floor(torch.log2(f.clamp(min=2.0 ** -24))) - 10).clamp(min=-24))
    s = torch.ceil(f / ulp) * ulp
    inv = torch.where(s > 0, (torch.ones_like(s) / s).float().double(), torch.zeros_like(s))
    return _exact_half(z + s * torch.round(((x - z).float().double() * inv).float().double()).clamp(max=15))


def _exact_values(st, p):
    """fp64 rows [pages, Hkv, page, 64] of pages p, by looking every element's place up."""
    t, c = torch.arange(8, device=DEV)[:, None], torch.arange(D, device=DEV)
    v = st["values"][p]
    if st["case"]["values"] == "fp16":
        return v.flatten(-2).unflatten(-1, (-1, 512))[..., 8 * c + t].flatten(-3, -2).double()
    byte = v[..., 16 * (c % 16) + 8 * (c // 32) + t].long()
    n = torch.where(c % 32 < 16, byte % 16, byte // 16).double()
    sz = v[..., 256:].contiguous().view(torch.float16).double()
    return _exact_half(sz[..., 8:, None] + sz[..., :8, None] * n).flatten(-3, -2)


def _exact_sylvester():
    h = torch.ones((1, 1), dtype=torch.float64, device=DEV)
    for _ in range(6):
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h


def _exact_keys(st, p):
    """fp64 rows [pages, Hkv, page, 64] that pages p stand for, in the domain that the codes hold."""
    k = st["case"]["k"]
    table = torch.tensor([2.0 ** -e for e in range(7)] + [0.0] + [-2.0 ** -e for e in range(7)] + [0.0], dtype=torch.float64,
                         device=DEV)
    m = torch.arange(D, device=DEV)
    se = st["codes_se"][p]
    w = table[((se.index_select(-1, m // 2) >> (4 * (m % 2)).to(torch.uint8)) & 15).long()]
    j = torch.zeros_like(w)
    for b in range(k):
        j += ((st["codes_m"][p].index_select(-1, 8 * b + m // 8) >> (m % 8).to(torch.uint8)) & 1).double() * 2.0 ** (b - k)
    return w * (1 + j) * st["key_scale"][p].double().unsqueeze(-1)


def _exact_encoded(x, case):
    """fp64 rows that new keys stand for, in the domain that the codes hold: the nearest grid value in log2 distance."""
    k, n = case["k"], 2 ** case["k"]
    x = (x @ _exact_sylvester() / 8).float().double() if case["hadamard"] else x
    s = x.abs().amax(-1, keepdim=True)
    u = (x.abs() / s).float().double()
    grid = [(1 + j / n) * 2.0 ** -e for e in range(7) for j in range(n) if e or not j]  # the top is the maximum itself
    grid = torch.tensor(sorted(grid), dtype=torch.float64, device=DEV)
    above = torch.zeros_like(u, dtype=torch.long)
    for a, b in zip(grid[:-1], grid[1:]):
        above += u * u > a * b
    val = torch.where(u * u > 2.0 ** -13, grid[above], torch.zeros_like(u))
    return torch.sign(x) * val * s


def _exact_turned(st, x, w):
    case = st["case"]
    axis = torch.tensor(_axis_of_pair(case), device=DEV)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       st["positions"].double()[axis].t() * st["inv_freq"])[:, None]
    r = case["rot_dim"]
    i = torch.arange(r, device=DEV)
    order = i.view(2, r // 2) if case["pairing"] == "halves" else i.view(r // 2, 2).t()
    y = x.double().clone()
    if w is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS) * w.double()
    z = torch.complex(y[..., order[0]], y[..., order[1]]) * turn
    y[..., order[0]], y[..., order[1]] = z.real, z.imag
    return y


def _exact_attend(st, q, new_keys=None, new_values=None):
    """fp64 attention, sequence by sequence and kv head by kv head, some hundred tokens at a time."""
    case = st["case"]
    Hq, Hkv, page = case["Hq"], case["Hkv"], case["page"]
    G = Hq // Hkv
    x = q.double()
    x = (x @ _exact_sylvester() / 8).float().double() if case["hadamard"] else x
    top = x.abs().amax(-1, keepdim=True)
    inv = (torch.full_like(top, 127.0) / top).float().double()
    qd = torch.round((x * inv).float().double()).clamp(-127, 127) * (top / torch.full_like(top, 127.0)).float().double()
    out = torch.zeros((q.shape[0], Hq, D), dtype=torch.float64, device=DEV)
    first_row = 0
    for b, (new, n) in enumerate(zip(*_lengths(case))):
        if not new:
            continue
        mine = slice(first_row, first_row + new)
        p = st["table"][b, :(n + page - 1) // page].long().clamp(min=0)
        kd, vd = (y.transpose(0, 1).flatten(1, 2)[:, :n].clone() for y in (_exact_keys(st, p), _exact_values(st, p)))
        if new_keys is not None:
            kd[:, n - new:], vd[:, n - new:] = new_keys[mine].transpose(0, 1), new_values[mine].transpose(0, 1)
        j = torch.arange(n, device=DEV)
        for i in range(0, new, 512):
            at = torch.arange(n - new + i, min(n, n - new + i + 512), device=DEV)[:, None]
            off = j > at
            if case["window"]:
                off = off | ((at - j >= case["window"]) & (j >= case["sinks"]))
            rows = slice(first_row + i, first_row + i + at.shape[0])
            for h in range(Hkv):
                sc = qd[rows, h * G:(h + 1) * G] @ kd[h].t().contiguous() / 8  # [tokens, G, n]
                pr = torch.softmax(sc.masked_fill(off[:, None], -math.inf), -1)
                out[rows, h * G:(h + 1) * G] = pr @ vd[h]
        first_row += new
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("attend", "window"):
        return dict(out=_exact_attend(st, st["q"]))
    q = _exact_turned(st, st["q"], st["q_weight"])
    keys = _exact_encoded(_exact_half(_exact_turned(st, st["k"], st["k_weight"])), case)
    v = st["v"].half()
    v = _exact_value_rows(v) if case["values"] == "int4" else v.double()
    if case["kind"] == "step":
        return dict(out=_exact_attend(st, q.float(), keys, v), q=q)
    keys = keys @ _exact_sylvester() / 8 if case["hadamard"] else keys
    rows = [torch.zeros((st["n_pages"], case["Hkv"], case["page"], D), dtype=torch.float64, device=DEV) for _ in range(2)]
    first_row = 0
    for b, (new, n) in enumerate(zip(*_lengths(case))):
        for i in range(new):
            t = n - new + i
            p, u = int(st["table"][b, t // case["page"]]), t % case["page"]
            rows[0][p, :, u], rows[1][p, :, u] = keys[first_row + i], v[first_row + i]
        first_row += new
    return dict(q=q, keys=rows[0].flatten(0, 1), values=rows[1].flatten(0, 1))
