// Goes through every lane of every copy of a 64-key tile of K and of V^T, for every number of keys left, and compares
// the bytes read with the buffer's.  The memory system returns zero for a lane whose VECTOR offset is not below the
// buffer's size, and reads at base + vector + scalar offset otherwise.  "planted" makes every tile a whole one, which has
// to be found.
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <set>

#include "tile_copy.h"

using namespace track;

constexpr int D = 128, TK = 64;

static int faults = 0;
static void check(bool ok, const char* what, int left, int i, int lane) {
  if (ok) return;
  if (++faults <= 5) printf("%s: %d keys left, copy %d, lane %d\n", what, left, i, lane);
}

static void tile_k(int left, int64_t ldk, int heads, bool planted) {
  const uint32_t krow = (uint32_t)ldk * 2;
  const int64_t size = (int64_t)(left < TK ? left : TK) * krow;  // of the buffer, from the tile's first key on
  // past the tile's last key the last of `heads` heads may end the memory
  const int64_t end = (int64_t)(left - 1) * krow + D * 2 + (heads > 1 ? krow - D * 2 : 0);
  std::set<int64_t> units;
  for (int i = 0; i < 16; ++i)
    for (int lane = 0; lane < 64; ++lane) {
      const TileOffset o = tile_offset(planted || tile_whole(0, left), tile_k_lane(i, lane, krow), tile_k_row(i, krow));
      const int row = 4 * i + (lane >> 4), key = att_perm(row), unit = (lane & 15) ^ (row & 15);
      const int64_t at = (int64_t)o.vec + o.scalar;
      check(at == (int64_t)key * krow + unit * 16, "K offset", left, i, lane);
      const bool read = o.vec < size;
      check(read == (key < left), "K range check", left, i, lane);
      if (read) check(at + 16 <= end, "K read past the end", left, i, lane);
      if (key < left) check(units.insert(at).second, "K unit twice", left, i, lane);
    }
  check((int)units.size() == (left < TK ? left : TK) * 16, "K units", left, -1, -1);
}

static void tile_v(int left, int64_t ldv, int key0, bool planted) {
  const uint32_t vrow = (uint32_t)ldv * 2;
  const int64_t Lk = key0 + left, vend = (D - 1) * ldv + (Lk + 7) / 8 * 8;  // elements up to the last row's last key
  const int64_t size = (vend - key0) * 2;
  for (int i = 0; i < 16; ++i)
    for (int lane = 0; lane < 64; ++lane) {
      const TileOffset o = tile_offset(planted || tile_whole(key0, (int)Lk), tile_v_lane(lane, vrow), tile_v_row(i, vrow));
      const int row = 8 * i + (lane >> 3), channel = att_perm(row), unit = (lane & 7) ^ att_vswz(row);
      const int64_t at = (int64_t)o.vec + o.scalar;
      check(at == (int64_t)channel * vrow + unit * 16, "V offset", left, i, lane);
      const bool read = o.vec < size;
      if (unit * 8 < left) check(read, "V key not read", left, i, lane);
      if (read) check(at + 16 <= size, "V read past the end", left, i, lane);
    }
}

int main(int argc, char** argv) {
  const bool planted = argc > 1 && !strcmp(argv[1], "planted");
  for (int left = 1; left <= 2 * TK; ++left) {
    for (int64_t ldk : {D, 5 * D, 1 << 22}) tile_k(left, ldk, ldk > D ? 2 : 1, planted);
    for (int64_t ldk : {5 * D, 1 << 22}) tile_k(left, ldk, 1, planted);
    for (int key0 : {0, 64, 4096})
      for (int64_t more : {0, 8, 64, 1 << 20}) tile_v(left, (key0 + left + 7) / 8 * 8 + more, key0, planted);
  }
  if (faults) printf("%d faults\n", faults);
  return faults ? 1 : 0;
}
