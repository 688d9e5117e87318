// Where the parts of 64 tokens of a head lie in the 4-bit cache, and what the threads of its kernels take of them.
// Plain arithmetic without a GPU type, so that a host program can go through every thread of every kernel and compare
// its bytes with the layout's and with a page's end.
#pragma once

#include <stdint.h>

namespace track {

constexpr int C4_BLOCK = 64;  // tokens that lie together

// Parts of a head's 64 tokens, in bytes: K codes at 0, V codes, exponents of K and of V.
template <int D>
struct C4 {
  static constexpr int G = D / 32, V = 32 * D, KE = 64 * D, VE = 66 * D, BYTES = 68 * D;
  // of token tok (0..63): the byte of channels ch and ch + 1 (ch even), of group grp's exponent
  static constexpr int k_code(int tok, int ch) { return tok * (D / 2) + ch / 2; }
  static constexpr int v_code(int tok, int ch) {
    return V + (ch >> 5) * 1024 + ((tok >> 3) & 3) * 256 + ((ch & 31) >> 1) * 16 + 8 * (tok >> 5) + (tok & 7);
  }
  static constexpr int k_exp(int tok, int grp) {
    return KE + (4 * ((tok >> 3) & 3) + (tok & 3)) * (4 * G) + 4 * grp + 2 * (tok >> 5) + ((tok >> 2) & 1);
  }
  static constexpr int v_exp(int tok, int grp) { return VE + 64 * grp + ((tok >> 3) & 3) * 16 + 8 * (tok >> 5) + (tok & 7); }
};

// Few rows (128 channels): a lane's 16 bytes of K for 16-key block i of 4, the 4 bytes of these keys' exponents, its 16 bytes
// of V group m and the 16 exponents of that group.  Lane 16 g + j has key c4_row_key(i, j) and its channels 32 g .. + 31, and
// of V channels 32 m + 2 j, + 1 of the keys 32 s + 8 g + 0..7.
constexpr int c4_row_key(int i, int j) { return 32 * (i >> 1) + 8 * (j >> 2) + 4 * (i & 1) + (j & 3); }
constexpr uint32_t c4_row_k(int lane) { return (uint32_t)(c4_row_key(0, lane & 15) * 64 + 16 * (lane >> 4)); }
constexpr uint32_t c4_row_k_block(int i) { return (uint32_t)(c4_row_key(i, 0) * 64); }
constexpr uint32_t c4_row_ke(int lane) { return (uint32_t)(C4<128>::KE + ((lane & 15) * 4 + (lane >> 4)) * 4); }
constexpr uint32_t c4_row_v(int lane, int m) { return (uint32_t)(C4<128>::V + lane * 16 + 1024 * m); }
constexpr uint32_t c4_row_ve(int lane, int m) { return (uint32_t)(C4<128>::VE + (lane >> 4) * 16 + 64 * m); }

// Blocks of rows (128 channels): thread t of 256 takes 16 bytes of K and one exponent, another 256 take 16 of V and 16 exponents.
// V's bytes go to threads in an order that lets 16 of them write to all banks of LDS: 8 bytes j of two r beside each other.
constexpr int c4_tile_key(int t) { return t >> 2; }            // K: the key, the group
constexpr int c4_tile_group(int t) { return t & 3; }
constexpr int c4_tile_j(int t) { return (t & 7) | ((t >> 1) & 8); }            // V: byte j of a group's 16
constexpr int c4_tile_r(int t) { return ((t >> 3) & 1) | ((t >> 4) & 2); }     // r of the keys 32 s + 8 r
constexpr int c4_tile_channel(int t) { return 32 * (t >> 6) + 2 * c4_tile_j(t); }  // the two channels' first
constexpr uint32_t c4_tile_codes(bool v, int t) {
  return (uint32_t)(v ? C4<128>::V + (t >> 6) * 1024 + c4_tile_r(t) * 256 + c4_tile_j(t) * 16 : t * 16);
}
constexpr uint32_t c4_tile_exp(bool v, int t) {
  return (uint32_t)(v ? C4<128>::VE + (t >> 6) * 64 + c4_tile_r(t) * 16 : C4<128>::k_exp(c4_tile_key(t), c4_tile_group(t)));
}

// Float32: thread t of 256 takes D / 8 bytes (D / 4 channels) of key t / 4, and D / 8 bytes of V: runs of 4 keys of two channels.
template <int D>
struct C4F32 {
  static constexpr int N = D / 8;
  static constexpr int k_channel(int t) { return (t & 3) * (D / 4); }
  static constexpr int k_codes(int t) { return C4<D>::k_code(t >> 2, k_channel(t)); }
  static constexpr int k_exp(int t) { return C4<D>::k_exp(t >> 2, k_channel(t) >> 5); }
  static constexpr int v_group(int t) { return t * N >> 10; }
  static constexpr int v_r(int t) { return (t * N >> 8) & 3; }
  static constexpr int v_channel(int t) { return 32 * v_group(t) + 2 * ((t * N >> 4) & 15); }
  static constexpr int v_first(int t) { return t * N & 15; }  // 8 s + c of its first byte
  static constexpr int v_codes(int t) { return C4<D>::V + t * N; }
  static constexpr int v_exp(int t) { return C4<D>::VE + v_group(t) * 64 + v_r(t) * 16 + v_first(t); }
  // the first key of run i (4 bytes)
  static constexpr int v_key(int t, int i) { return 32 * ((v_first(t) + 4 * i) >> 3) + 8 * v_r(t) + ((v_first(t) + 4 * i) & 7); }
};

// Rows in and out: slot 8 s + c of wave r of a block is token 32 s + 8 r + c.
constexpr int c4_token(int r, int slot) { return 32 * (slot >> 3) + 8 * r + (slot & 7); }

// Page ids from the table are taken as they are: whether one is a page of the pool, and where block t of a
// sequence lies in it (entry: t / blocks of a page, which the caller has found to be in the table).
constexpr bool c4_page(int id, int n_pages) { return id >= 0 && id < n_pages; }
constexpr int64_t c4_block(int page, int blocks, int t, int entry, int64_t stride) {
  return ((int64_t)page * blocks + (t - entry * blocks)) * stride;
}

}  // namespace track
