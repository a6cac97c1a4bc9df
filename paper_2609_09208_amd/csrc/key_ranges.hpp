// Arithmetic of the decode kernels' key ranges and of their loads of 4-bit values, plain
// enough for a host compiler: the tests check it over every length and split there.
#pragma once

#if defined(__HIPCC__)
#define POT_BOTH __host__ __device__
#else
#define POT_BOTH
#endif

namespace potattn {

constexpr int kWTile = 64;  // keys per wave tile

// 4-bit values: groups of 8 tokens, kI4GroupBytes bytes each. Byte 16 (d % 16) +
// 8 (d / 32) + t % 8 of a group has the n of dimension d in its low half where
// d % 32 < 16 and in its high half elsewhere, so 16 consecutive bytes are the
// matrix-core operands of 8 tokens for the dimensions c, 16 + c, 32 + c and 48 + c,
// and a token has its bytes to itself; behind them the tokens' 8 fp16 steps s and 8
// fp16 minima z. A value is z + s n.
constexpr int kI4Steps = 256, kI4Minima = 272, kI4GroupBytes = 288;

// Keys of a split when a sequence of t_all keys is cut into n_splits ranges of whole tiles.
POT_BOTH constexpr int own_split_len(int t_all, int n_splits) {
  return ((t_all + n_splits - 1) / n_splits + kWTile - 1) / kWTile * kWTile;
}

// Keys begin .. end - 1 of a split and its tiles; none (tiles <= 0) past the sequence's end.
struct KeyRange {
  int begin, end, tiles;
};
POT_BOTH constexpr KeyRange split_range(int t_all, int split, int split_len) {
  const int begin = split * split_len;
  const int end = t_all < begin + split_len ? t_all : begin + split_len;
  return {begin, end, (end - begin + kWTile - 1) / kWTile};
}
// The split that holds the sequence's last key, which takes the appended token in.
POT_BOTH constexpr bool holds_last(const KeyRange& r, int t_all) {
  return r.begin < t_all && r.end == t_all;
}
// End of the range's last 8-token group, up to which scales and values are read.
POT_BOTH constexpr int groups_end(const KeyRange& r) { return ((r.end - 1) & ~7) + 8; }

// Bytes from a tile's first record to what a lane loads of its 4-bit values: 16 bytes of
// K-block kb (four groups on per block), the steps of the 8 keys whose weights it forms.
POT_BOTH constexpr int value_offset_i4(int lane, int kb) {
  return (lane >> 4) * kI4GroupBytes + (lane & 15) * 16 + kb * 4 * kI4GroupBytes;
}
POT_BOTH constexpr int step_offset_i4(int lane) {
  return (4 * ((lane & 15) >> 3) + (lane >> 4)) * kI4GroupBytes + kI4Steps;
}

}  // namespace potattn
