"""A host model of the decode kernel's loads of a tile's 4-bit values: every byte a lane's operands need arrives from its
place in the record layout, and nothing is read past the sequence's rows (lanes past the buffer's end read zeros)."""
import numpy as np
import pytest

GROUP, STEPS, MINIMA, TILE = 288, 256, 272, 64


def _window(t0, v_end):
    """Byte range of the tile's buffer resource in the sequence, as tile_rsrc makes it."""
    return t0 * (GROUP // 8), v_end * (GROUP // 8)


def _loads(lane):
    """(what, byte offset, bytes) of a lane's loads, as load_values_buf makes them."""
    part, grp, c = (lane & 15) >> 3, lane >> 4, lane & 15
    got = [(("values", kb), (grp + 4 * kb) * GROUP + c * 16, 16) for kb in (0, 1)]
    at = (4 * part + grp) * GROUP
    return got + [("steps", at + STEPS, 16), ("minima", at + MINIMA, 16)]


@pytest.mark.parametrize("t_len", [1, 7, 8, 9, 63, 64, 65, 200, 256])
def test_windows_end_with_the_rows(t_len):
    t_cap = (t_len + 7) // 8 * 8
    for t0 in range(0, t_len, TILE):
        t_end = min(t_len, t0 + 1024)
        v_end = ((t_end - 1) & ~7) + 8
        first, last = _window(t0, v_end)
        assert first % 16 == 0 and last <= t_cap * (GROUP // 8)
        for lane in range(64):
            for _, off, n in _loads(lane):
                # whole loads are inside or outside: records do not straddle the end
                assert first + off + n <= last or first + off >= last


def test_operands_come_from_their_places():
    rng = np.random.default_rng(0)
    n = rng.integers(0, 16, (TILE, 64))
    s, z = rng.integers(0, 1 << 16, (2, TILE))
    tile = np.zeros(8 * GROUP, np.uint8)
    for t in range(TILE):
        g, u = divmod(t, 8)
        for d in range(64):
            at = g * GROUP + 16 * (d % 16) + 8 * (d // 32) + u
            tile[at] |= n[t, d] << (4 if d % 32 >= 16 else 0)
        tile[g * GROUP + STEPS:].view(np.uint16)[u] = s[t]
        tile[g * GROUP + MINIMA:].view(np.uint16)[u] = z[t]
    order = [0, 2, 1, 3, 4, 6, 5, 7]
    for lane in range(64):
        part, grp, c = (lane & 15) >> 3, lane >> 4, lane & 15
        for what, off, size in _loads(lane):
            data = tile[off:off + size]
            if what == "steps" or what == "minima":
                keys = [32 * part + 8 * grp + i for i in range(8)]
                assert list(data.view(np.uint16)) == [(s if what == "steps" else z)[k] for k in keys]
                continue
            kb, w = what[1], data.view(np.uint32)
            for nb in range(4):
                mask = 0x00F000F0 if nb & 1 else 0x000F000F
                words = [w[2 * (nb // 2)] & mask, w[2 * (nb // 2)] >> 8 & mask, w[2 * (nb // 2) + 1] & mask,
                         w[2 * (nb // 2) + 1] >> 8 & mask]
                got = [int(x) >> (16 * h) & 0xFFFF for x in words for h in (0, 1)]
                got = [x >> 4 if nb & 1 else x for x in got]
                assert got == [n[32 * kb + 8 * grp + i, 16 * nb + c] for i in order]
