// Where the lanes of a copy read when one wave brings a 64-key tile of K or V^T into LDS by itself
// (window_rows_kernel).  Plain arithmetic without a GPU type, so that a host program can go
// through every lane of every copy and compare the bytes with the buffer's.
#pragma once

#include <stdint.h>

namespace track {

// Key of a K tile's LDS row, channel of a V^T tile's: permuted within every 32 (attention_tile.h).
constexpr int att_perm(int row) {
  return (row & ~31) | (((row >> 2) & 3) << 3) | (((row >> 4) & 1) << 2) | (row & 3);
}

// Swizzle of a V^T row's 16-byte units.
constexpr int att_vswz(int row) { return ((row & 7) ^ ((row >> 3) & 1)) & 6; }

// A lane's offset in bytes from the tile's first key on: vec of the lane, scalar of the wave.  A buffer's
// size is compared with the vector offset alone (the scalar one is not part of the documented check).
struct TileOffset {
  uint32_t vec, scalar;
};

// Whether all 64 keys of the tile are there.  If not, the whole offset of a copy has to be in its
// vector part, for the buffer's size to cut off what lies past the last key.
constexpr bool tile_whole(int key0, int keys) { return key0 + 64 <= keys; }
constexpr TileOffset tile_offset(bool whole, uint32_t lane, uint32_t row) {
  return whole ? TileOffset{lane, row} : TileOffset{lane + row, 0};
}

// Copy i of 16 fills LDS rows 4 i .. + 3 of K (16 lanes a row of 256 bytes) or 8 i .. + 7 of V^T
// (8 lanes a row of 128), laid out as in the block kernel.  The key att_perm(4 i + lane / 16) is
// att_perm(4 i) + lane / 16 and the channel att_perm(8 i + lane / 8) likewise, and the
// swizzles' bits of i and of the lane do not meet: one offset a lane for V^T, one for each i % 4 for
// K, the rest (the row's) is wave-uniform.  krow, vrow: bytes from key to key of K, from channel to channel
// of V^T.
constexpr uint32_t tile_k_lane(int i, int lane, uint32_t krow) {
  return (uint32_t)(lane >> 4) * krow + (uint32_t)((((lane & 15) ^ (lane >> 4)) ^ (4 * (i & 3))) << 4);
}
constexpr uint32_t tile_k_row(int i, uint32_t krow) { return (uint32_t)att_perm(4 * i) * krow; }
constexpr uint32_t tile_v_lane(int lane, uint32_t vrow) {
  return (uint32_t)att_perm(lane >> 3) * vrow + (uint32_t)(((lane & 7) ^ ((lane >> 3) & 6)) << 4);
}
constexpr uint32_t tile_v_row(int i, uint32_t vrow) { return (uint32_t)att_perm(8 * i) * vrow; }

}  // namespace track
