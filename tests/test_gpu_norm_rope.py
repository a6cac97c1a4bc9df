"""Norm and position rotation of a projection against 64 bits: types, layouts, axes, pairings, far positions, parts left
out, and rows that stay what they are."""
import numpy as np
import pytest
import torch

import paper_2609_09208_amd as pa
from parity_util import DEV

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
HALF_UNIT = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
SMALLEST = {"fp16": 2.0 ** -25, "bf16": 0.0, "fp32": 0.0}


def _inv_freq(rot_dim, base=10000.0):
    return base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=DEV) / max(rot_dim, 1))


def _reference(x, w, eps, pos, inv_freq, axis, rot_dim, neighbours, turn=True):
    """fp64 [B, H, S, 64] on the host, and the size of each row's elements after the norm."""
    y = x.cpu().double().transpose(1, 2).clone()
    if w is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * w.cpu().double()
    size = y.abs()
    if turn and rot_dim:
        angle = pos.cpu().double()[axis].permute(1, 2, 0)[:, None] * inv_freq.cpu()
        cos, sin = angle.cos(), angle.sin()
        r = rot_dim
        i = torch.arange(r)
        first, second = (i[0:r:2], i[1:r:2]) if neighbours else (i[:r // 2], i[r // 2:])
        a, b = y[..., first].clone(), y[..., second].clone()
        y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
        m = a.abs() + b.abs()
        size[..., first], size[..., second] = m, m
    return y, size


def _bound(want, size, out, top_angle):
    """Half a unit of the output, and of the fp32 steps before: the norm's sum (6 additions and a square: 7 half units,
    halved by the root), root, quotient and two products (5), the rotation's products and sum (3), cos and sin (4: of an
    angle's rounding, 1e-9, and of their series): 16 half units of the pair's elements; far angles also lose 2^-51 of
    themselves."""
    return (want.abs() * HALF_UNIT[out] + SMALLEST[out]) * (1 + 2.0 ** -8) + size * (16 * 2.0 ** -24 + top_angle * 2.0 ** -51)


def _run(B, S, Hq, Hkv, dtype="bf16", q_out="fp32", layout="packed", norm=True, rot_dim=64, neighbours=False, axes=(0,),
         first=0, eps=1e-6, weight="same", seed=0, parts="qkv"):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 31 * S + Hq)
    t = TYPES[dtype]
    if layout == "packed":
        x = (3 * torch.randn((B, S, Hq + 2 * Hkv, 64), generator=g, device=DEV)).to(t)
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    elif layout == "heads":
        q, k, v = ((3 * torch.randn((B, h, S, 64), generator=g, device=DEV)).to(t).transpose(1, 2) for h in (Hq, Hkv, Hkv))
    else:  # rows further apart than they are long, tokens in reverse order of storage of batch rows
        q, k, v = ((3 * torch.randn((S, h + 1, B, 80), generator=g, device=DEV)).to(t)[:, :h, :, 8:72].permute(2, 0, 1, 3)
                   for h in (Hq, Hkv, Hkv))
    axis = [axes[i % len(axes)] for i in range(rot_dim // 2)] if layout == "packed" else [
        axes[i * len(axes) // (rot_dim // 2)] for i in range(rot_dim // 2)]
    rope = pa.make_rope(rot_dim, neighbours, axis)
    pos = torch.randint(0, 5000, (rope.n_axes, B, S), generator=g, device=DEV) + first
    inv = _inv_freq(rot_dim)
    wt = t if weight == "same" else torch.float32
    qw, kw = ((1 + 0.3 * torch.randn(64, generator=g, device=DEV)).to(wt) for _ in range(2)) if norm else (None, None)
    q, k, v = (p if n in parts else None for n, p in zip("qkv", (q, k, v)))
    guard = 64
    outs = []
    for p, ty in ((q, TYPES[q_out]), (k, torch.float16), (v, torch.float16)):
        n = 0 if p is None else p.shape[2] * B * S * 64
        outs.append(torch.full((n + guard,), 7.0, dtype=ty, device=DEV))
    shaped = [None if p is None else o[:-guard].view(B, p.shape[2], S, 64) for p, o in zip((q, k, v), outs)]
    pa.pot_norm_rope(rope, q, k, v, qw, kw, eps, pos, inv, *shaped)
    torch.cuda.synchronize()
    top = float((pos.double().abs().max() * inv.max()).item()) if rot_dim else 0.0
    for name, p, o, w, ty in (("q", q, outs[0], qw, q_out), ("k", k, outs[1], kw, "fp16"), ("v", v, outs[2], None, "fp16")):
        assert (o[-guard:] == 7.0).all()
        if p is None:
            continue
        got = o[:-guard].view(B, p.shape[2], S, 64).cpu().double()
        want, size = _reference(p, w, eps, pos, inv, axis, rot_dim, neighbours, name != "v")
        over = (got - want).abs() / _bound(want, size, ty, top).clamp(min=1e-300)
        assert float(over.max()) <= 1, (name, float(over.max()))


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("q_out", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("layout", ["packed", "heads", "wide"])
@pytest.mark.parametrize("norm", [True, False])
def test_types_and_layouts(dtype, q_out, layout, norm):
    _run(2, 37, 12, 3, dtype, q_out, layout, norm, weight="same" if layout != "wide" else "fp32")


@pytest.mark.parametrize("rot_dim", [0, 2, 6, 16, 30, 32, 48, 62, 64])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rotated_part_of_a_head(rot_dim, neighbours, dtype):
    _run(3, 5, 8, 2, dtype, "fp32", "packed", True, rot_dim, neighbours)


@pytest.mark.parametrize("axes", [(0, 1), (0, 1, 2), (2, 0, 1), (3, 1, 2, 0)])
@pytest.mark.parametrize("layout", ["packed", "heads"])
def test_position_axes(axes, layout):
    _run(2, 19, 8, 4, "bf16", "fp32", layout, axes=axes)


@pytest.mark.parametrize("first", [1 << 20, (1 << 31) - 5000, -(1 << 31), -2500])
@pytest.mark.parametrize("neighbours", [False, True])
def test_far_and_negative_positions(first, neighbours):
    _run(2, 9, 4, 1, "fp32", "fp32", first=first, neighbours=neighbours)


@pytest.mark.parametrize("B,S,Hq,Hkv", [(1, 1, 1, 1), (1, 1, 32, 4), (64, 1, 32, 4), (1, 2, 3, 1), (7, 1, 5, 5),
                                        (1, 777, 16, 8), (5, 129, 64, 8), (2, 1031, 8, 1), (300, 3, 8, 8), (1, 17, 128, 16)])
def test_shapes(B, S, Hq, Hkv):
    _run(B, S, Hq, Hkv)
    _run(B, S, Hq, Hkv, "fp32", "fp32", "heads", False, 32, True)


@pytest.mark.parametrize("parts", ["q", "k", "v", "qk", "kv", "qv"])
def test_parts_left_out(parts):
    _run(2, 13, 6, 3, parts=parts)


def test_no_rotation_needs_no_positions():
    x = torch.randn((2, 3, 4, 64), device=DEV)
    out = torch.empty((2, 4, 3, 64), device=DEV)
    pa.pot_norm_rope(pa.make_rope(0), x, None, None, None, None, 0.0, None, None, out, None, None)
    assert torch.equal(out, x.transpose(1, 2))


def test_zero_infinite_and_nan_rows_stay_by_themselves():
    x = torch.randn((1, 8, 4, 64), device=DEV)
    x[0, 1] = 0
    x[0, 2, 1, 5] = float("nan")
    x[0, 3, 2, 9] = float("inf")
    w = torch.ones(64, device=DEV)
    out = torch.empty((1, 4, 8, 64), device=DEV)
    pos = torch.arange(8, device=DEV).view(1, 1, 8)
    pa.pot_norm_rope(pa.make_rope(), x, None, None, w, None, 1e-6, pos, _inv_freq(64), out, None, None)
    bad = torch.zeros((4, 8), dtype=torch.bool, device=DEV)
    bad[1, 2] = bad[2, 3] = True
    assert torch.isfinite(out[0][~bad]).all()
    assert (out[0, :, 1] == 0).all()
    assert out[0, 1, 2].isnan().any() and out[0, 2, 3].isnan().any()


def test_values_beyond_fp16_are_infinite():
    x = torch.full((1, 2, 1, 64), 1e6, device=DEV)
    v = torch.empty((1, 1, 2, 64), dtype=torch.float16, device=DEV)
    pa.pot_norm_rope(pa.make_rope(0), None, None, x, None, None, 0.0, None, None, None, None, v)
    assert (v == float("inf")).all()


def test_rows_read_more_than_once():
    """A broadcast batch (stride 0)."""
    x = torch.randn((1, 6, 5, 64), device=DEV).expand(4, 6, 5, 64)
    out = torch.empty((4, 5, 6, 64), device=DEV)
    pa.pot_norm_rope(pa.make_rope(0), x, None, None, None, None, 0.0, None, None, out, None, None)
    assert torch.equal(out, x.transpose(1, 2))


def test_offsets_past_2_to_31_elements():
    """A projection and outputs of over 2^31 elements: the last token."""
    B, S, H = 1, (1 << 20) + 3, 33
    x = torch.empty((B, S, H, 64), dtype=torch.bfloat16, device=DEV)
    x[:, -2:] = torch.randn((B, 2, H, 64), device=DEV)
    out = torch.empty((B, H, S, 64), dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(S, device=DEV).view(1, B, S)
    pa.pot_norm_rope(pa.make_rope(), x, None, None, None, None, 0.0, pos, _inv_freq(64), out, None, None)
    torch.cuda.synchronize()
    want, size = _reference(x[:, -2:], None, 0, pos[:, :, -2:], _inv_freq(64), [0] * 32, 64, False)
    assert ((out[:, :, -2:].cpu().double() - want).abs() <= _bound(want, size, "bf16", float(S))).all()
