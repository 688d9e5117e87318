// Goes through every thread of the kernels of the 4-bit cache and compares the bytes that it takes with those of the layout, and each with
// the 68 D bytes of a head's 64 tokens; then through page ids.  "planted" lets one thread start a byte later, which has to be found.
#include <cstdio>
#include <cstring>
#include <set>

#include "cache4_layout.h"

using namespace track;

static int faults = 0;
static void check(bool ok, const char* what, int a, int b, int c) {
  if (!ok && ++faults <= 5) printf("%s: %d %d %d\n", what, a, b, c);
}

template <int D>
static void layout() {
  std::set<int> seen;
  for (int tok = 0; tok < 64; ++tok) {
    for (int ch = 0; ch < D; ch += 2) {
      const int k = C4<D>::k_code(tok, ch), v = C4<D>::v_code(tok, ch);
      check(k >= 0 && k < C4<D>::V && seen.insert(k).second, "K code", D, tok, ch);
      check(v >= C4<D>::V && v < C4<D>::KE && seen.insert(v).second, "V code", D, tok, ch);
    }
    for (int g = 0; g < D / 32; ++g) {
      const int k = C4<D>::k_exp(tok, g), v = C4<D>::v_exp(tok, g);
      check(k >= C4<D>::KE && k < C4<D>::VE && seen.insert(k).second, "K exponent", D, tok, g);
      check(v >= C4<D>::VE && v < C4<D>::BYTES && seen.insert(v).second, "V exponent", D, tok, g);
    }
  }
  check((int)seen.size() == C4<D>::BYTES && C4<D>::BYTES % 128 == 0, "bytes", D, (int)seen.size(), 0);
  // rows in and out: a wave's 16 slots, 16 bytes of V a lane
  for (int r = 0; r < 4; ++r)
    for (int lane = 0; lane < D / 2; ++lane) {
      const int at = C4<D>::v_code(8 * r, 2 * lane);
      check(at % 16 == 0 && at + 16 <= C4<D>::KE, "row V", D, r, lane);
      for (int s = 0; s < 16; ++s) check(at + s == C4<D>::v_code(c4_token(r, s), 2 * lane), "row V slot", D, lane, s);
    }
  std::set<int> tokens;
  for (int r = 0; r < 4; ++r)
    for (int s = 0; s < 16; ++s) tokens.insert(c4_token(r, s));
  check(tokens.size() == 64 && *tokens.begin() == 0 && *tokens.rbegin() == 63, "tokens", D, 0, 0);
  for (int tok = 0; tok < 64; ++tok)
    for (int u = 0; u < D / 8; ++u)
      check(C4<D>::k_code(tok, 8 * u) % 4 == 0 && C4<D>::k_code(tok, 8 * u) + 3 == C4<D>::k_code(tok, 8 * u + 6), "row K", D, tok, u);
  // float32 attention
  std::set<int> taken;
  for (int t = 0; t < 256; ++t) {
    typedef C4F32<D> A;
    check(A::k_codes(t) % 4 == 0 && A::v_codes(t) % 4 == 0 && A::v_exp(t) % 4 == 0, "f32 alignment", D, t, 0);
    check(A::k_exp(t) == C4<D>::k_exp(t >> 2, A::k_channel(t) / 32), "f32 K exponent", D, t, 0);
    for (int i = 0; i < A::N; ++i) {
      check(A::k_codes(t) + i == C4<D>::k_code(t >> 2, A::k_channel(t) + 2 * i), "f32 K", D, t, i);
      check(A::k_channel(t) / 32 == (A::k_channel(t) + 2 * i) / 32, "f32 K group", D, t, i);
      const int key = A::v_key(t, i / 4) + i % 4;
      check(A::v_key(t, i / 4) % 4 == 0 && key < 64, "f32 V run", D, t, i);
      check(A::v_codes(t) + i == C4<D>::v_code(key, A::v_channel(t)), "f32 V", D, t, i);
      check(A::v_exp(t) + i == C4<D>::v_exp(key, A::v_group(t)) && A::v_channel(t) / 32 == A::v_group(t), "f32 V exponent", D, t, i);
      taken.insert(A::k_codes(t) + i), taken.insert(A::v_codes(t) + i);
    }
  }
  check((int)taken.size() == C4<D>::KE, "f32 codes", D, (int)taken.size(), 0);
}

static void rows(int planted) {
  typedef C4<128> L;
  for (int lane = 0; lane < 64; ++lane) {
    const int j = lane & 15, g = lane >> 4;
    for (int i = 0; i < 4; ++i) {
      const int at = (int)(c4_row_k(lane) + c4_row_k_block(i)) + (lane == 37 ? planted : 0), key = c4_row_key(i, j);
      check(at % 16 == 0 && at + 16 <= L::V, "few rows K", lane, i, at);
      for (int x = 0; x < 16; ++x) check(at + x == L::k_code(key, 32 * g + 2 * x), "few rows K code", lane, i, x);
      check((int)c4_row_ke(lane) + i == L::k_exp(key, g), "few rows K exponent", lane, i, 0);
      const int m = i, v = (int)(c4_row_v(lane, 0) + (c4_row_v(0, m) - c4_row_v(0, 0)));
      const int e = (int)(c4_row_ve(lane, 0) + (c4_row_ve(0, m) - c4_row_ve(0, 0)));
      check(v % 16 == 0 && v + 16 <= L::KE && e % 16 == 0 && e + 16 <= L::BYTES, "few rows V", lane, m, v);
      for (int x = 0; x < 16; ++x) {
        const int tok = 32 * (x >> 3) + 8 * g + (x & 7);
        check(v + x == L::v_code(tok, 32 * m + 2 * j), "few rows V code", lane, m, x);
        check(e + x == L::v_exp(tok, m), "few rows V exponent", lane, m, x);
      }
    }
    check((int)c4_row_ke(lane) % 4 == 0 && (int)c4_row_ke(lane) + 4 <= L::VE, "few rows K exponents", lane, 0, 0);
  }
  for (int t = 0; t < 256; ++t) {
    const int k = (int)c4_tile_codes(false, t), v = (int)c4_tile_codes(true, t), e = (int)c4_tile_exp(true, t);
    check(k % 16 == 0 && k + 16 <= L::V && v % 16 == 0 && v + 16 <= L::KE && e % 16 == 0 && e + 16 <= L::BYTES, "tile", t, k, v);
    check((int)c4_tile_exp(false, t) == L::k_exp(c4_tile_key(t), c4_tile_group(t)), "tile K exponent", t, 0, 0);
    for (int x = 0; x < 16; ++x) {
      const int tok = 32 * (x >> 3) + 8 * c4_tile_r(t) + (x & 7);
      check(k + x == L::k_code(c4_tile_key(t), 32 * c4_tile_group(t) + 2 * x), "tile K code", t, x, 0);
      check(v + x == L::v_code(tok, c4_tile_channel(t)), "tile V code", t, x, 0);
      check(e + x == L::v_exp(tok, c4_tile_channel(t) >> 5), "tile V exponent", t, x, 0);
    }
  }
}

static void pages() {
  const int big = 2147483647;
  for (int n : {1, 2, 1000, big})
    for (int64_t id : {(int64_t)-big - 1, (int64_t)-1, (int64_t)0, (int64_t)n - 1, (int64_t)n, (int64_t)big})
      if (id <= big) check(c4_page((int)id, n) == (id >= 0 && id < n), "page id", (int)id, n, 0);
  // every block of a page inside it, also where the pool passes 32 bits
  for (int blocks : {1, 3, 1024})
    for (int page : {0, 7, 1 << 20}) {
      const int64_t stride = (int64_t)(1 << 19) * C4<128>::BYTES;
      for (int entry : {0, 5})
        for (int in = 0; in < blocks; ++in) {
          const int64_t at = c4_block(page, blocks, entry * blocks + in, entry, stride);
          check(at == ((int64_t)page * blocks + in) * stride && at + stride <= ((int64_t)page + 1) * blocks * stride, "block", blocks, page, in);
        }
    }
}

int main(int argc, char** argv) {
  layout<32>(), layout<64>(), layout<128>();
  rows(argc > 1 && !strcmp(argv[1], "planted"));
  pages();
  if (faults) printf("%d faults\n", faults);
  return faults != 0;
}
