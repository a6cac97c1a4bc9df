"""Norm and rotation of many tokens (from 1024 on a wave goes through the heads of eight tokens) against 64 bits: widths and
pairings, types, axes, parts left out, rows of NaN, and rows whose squares pass fp32's range."""
import pytest
import torch

import paper_2609_09208_amd as pa
from parity_util import DEV
from test_gpu_norm_rope import HALF_UNIT, SMALLEST, TYPES, _inv_freq, _reference, _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rot_dim", [2, 6, 16, 30, 32, 48, 62])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_rotated_part_of_a_head(rot_dim, neighbours, dtype):
    _run(3, 347, 8, 2, dtype, "fp32", "packed", True, rot_dim, neighbours)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("q_out", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("layout", ["packed", "heads", "wide"])
@pytest.mark.parametrize("rot_dim,neighbours", [(64, False), (64, True), (32, False)])
def test_types_and_layouts(dtype, q_out, layout, rot_dim, neighbours):
    _run(2, 517, 5, 3, dtype, q_out, layout, True, rot_dim, neighbours, weight="same" if layout != "wide" else "fp32")


@pytest.mark.parametrize("axes", [(0, 1), (2, 0, 1), (3, 1, 2, 0)])
@pytest.mark.parametrize("rot_dim,neighbours", [(64, False), (48, False), (64, True)])
def test_position_axes(axes, rot_dim, neighbours):
    _run(2, 519, 8, 4, "bf16", "fp32", "packed", True, rot_dim, neighbours, axes=axes)


@pytest.mark.parametrize("parts", ["q", "k", "v", "qk", "kv", "qv"])
@pytest.mark.parametrize("rot_dim", [64, 32])
def test_parts_left_out(parts, rot_dim):
    _run(2, 513, 6, 3, rot_dim=rot_dim, parts=parts)


@pytest.mark.parametrize("B,S,Hq,Hkv", [(1, 1024, 1, 1), (1023, 1, 3, 1), (1025, 1, 3, 1), (1, 4097, 64, 8), (7, 1171, 32, 4)])
@pytest.mark.parametrize("first", [0, -(1 << 31)])
def test_shapes(B, S, Hq, Hkv, first):
    _run(B, S, Hq, Hkv, first=first)
    _run(B, S, Hq, Hkv, "fp32", "fp32", "heads", False, 32, first=first)


@pytest.mark.parametrize("tokens", [8, 1032])
@pytest.mark.parametrize("rot_dim", [64, 32])
def test_rows_of_nan_stay_by_themselves(tokens, rot_dim):
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.randn((1, tokens, 3, 64), generator=g, device=DEV)
    bad = torch.zeros((1, 3, tokens), dtype=torch.bool, device=DEV)
    for t, h in ((1, 0), (2, 1), (tokens - 1, 2), (tokens - 8, 1)):
        x[0, t, h] = float("nan")
        bad[0, h, t] = True
    w = torch.ones(64, device=DEV)
    out = torch.empty((1, 3, tokens, 64), device=DEV)
    pos = torch.arange(tokens, device=DEV).view(1, 1, tokens)
    pa.pot_norm_rope(pa.make_rope(rot_dim), x, None, None, w, None, 1e-6, pos, _inv_freq(rot_dim), out, None, None)
    assert out[bad].isnan().all()
    assert torch.isfinite(out[~bad]).all()


@pytest.mark.parametrize("tokens", [24, 1032])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("q_out", ["bf16", "fp32"])
@pytest.mark.parametrize("rot_dim", [64, 32])
def test_rows_whose_squares_pass_fp32(tokens, dtype, q_out, rot_dim):
    """Rows of 2^-130 to 2^127: the norm is that of the definition, though x^2 is infinite or 0 in fp32."""
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    size = torch.tensor([2.0 ** e for e in (-130, -110, -90, -70, -64, -63, -40, 0, 30, 57, 62, 63, 64, 90, 120, 124)],
                        dtype=torch.float64, device=DEV)
    rows = torch.randn((1, tokens, 4, 64), generator=g, device=DEV).double().clamp(-7, 7)
    x = (rows * size[torch.arange(tokens * 4, device=DEV) % len(size)].view(1, tokens, 4, 1)).float().to(TYPES[dtype])
    w = 1 + 0.2 * torch.randn(64, generator=g, device=DEV)
    pos = torch.arange(tokens, device=DEV).view(1, 1, tokens)
    for eps in (0.0, 1e-30, 1e-6):
        out = torch.empty((1, 4, tokens, 64), dtype=TYPES[q_out], device=DEV)
        pa.pot_norm_rope(pa.make_rope(rot_dim), x, None, None, w, None, eps, pos, _inv_freq(rot_dim), out, None, None)
        # eps is a float
        want, size_of = _reference(x, w, torch.tensor(eps).double().item(), pos, _inv_freq(rot_dim), [0] * (rot_dim // 2),
                                   rot_dim, False)
        bound = (want.abs() * HALF_UNIT[q_out] + SMALLEST[q_out]) * (1 + 2.0 ** -8) + size_of * (
            16 * 2.0 ** -24 + tokens * 2.0 ** -51) + 2.0 ** -133  # bf16's and fp32's smallest numbers
        over = ((out.cpu().double() - want).abs() / bound).nan_to_num(nan=float("inf"))
        assert float(over.max()) <= 1, (eps, float(over.max()))


@pytest.mark.parametrize("part", ["q", "k"])
def test_weights_of_a_part_left_out_are_not_looked_at(part):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn((1, 5, 3, 64), generator=g, device=DEV).to(torch.bfloat16)
    w = (1 + 0.2 * torch.randn(64, generator=g, device=DEV)).to(torch.bfloat16)
    out = torch.empty((1, 3, 5, 64), dtype=torch.float16, device=DEV)
    pos = torch.arange(5, device=DEV).view(1, 1, 5)
    for other in (None, w.double(), w.float()):
        got = torch.zeros_like(out)
        mine, theirs = (x, w, got), (None, other, None)
        (q, qw, qo), (k, kw, ko) = (mine, theirs) if part == "q" else (theirs, mine)
        pa.pot_norm_rope(pa.make_rope(), q, k, None, qw, kw, 1e-6, pos, _inv_freq(64), qo, ko, None)
        if other is None:
            out.copy_(got)
        assert torch.equal(got, out)


@pytest.mark.parametrize("tokens", [11, 1033])
@pytest.mark.parametrize("normed", ["q", "k"])
@pytest.mark.parametrize("rot_dim,neighbours", [(64, False), (64, True), (32, False), (0, False)])
def test_one_part_normed_and_the_other_not(tokens, normed, rot_dim, neighbours):
    """Eight heads of a token share a wave where there are few tokens: five of q and three of k here."""
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x = torch.randn((1, tokens, 11, 64), generator=g, device=DEV).to(torch.bfloat16)
    q, k, v = x[:, :, :5], x[:, :, 5:8], x[:, :, 8:]
    w = 1 + 0.2 * torch.randn(64, generator=g, device=DEV)
    weights = (w, None) if normed == "q" else (None, w)
    pos = torch.randint(0, 5000, (1, 1, tokens), generator=g, device=DEV)
    outs = (torch.empty((1, 5, tokens, 64), device=DEV), *(torch.empty((1, 3, tokens, 64), dtype=torch.float16, device=DEV)
                                                         for _ in range(2)))
    pa.pot_norm_rope(pa.make_rope(rot_dim, neighbours), q, k, v, *weights, 1e-6, pos, _inv_freq(rot_dim), *outs)
    for rows, weight, out, ty, turn in ((q, weights[0], outs[0], "fp32", True), (k, weights[1], outs[1], "fp16", True),
                                        (v, None, outs[2], "fp16", False)):
        want, size = _reference(rows, weight, 1e-6, pos, _inv_freq(rot_dim), [0] * (rot_dim // 2), rot_dim, neighbours, turn)
        bound = (want.abs() * HALF_UNIT[ty] + SMALLEST[ty]) * (1 + 2.0 ** -8) + size * (16 * 2.0 ** -24 + 5000 * 2.0 ** -51)
        assert ((out.cpu().double() - want).abs() <= bound).all()
