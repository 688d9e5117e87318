// A paged cache that holds keys and values in 4 bits: rows into it with the rotation on the way, rows back out of it,
// and window attention that reads it as it lies.
//
// 32 channels of a token's head share a power of two 2^e, kept as the byte e + 127; a value is a sign and a magnitude
// code 0..7 for 0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e (the 4-bit floats with one exponent a group that the matrix and
// conversion units know): v_cvt_scalef32_pk_bf16_fp4 turns a byte of two codes into two bfloat16 values, exactly, one instruction
// at the full rate (35.7 T lanes a second).  e is the smallest of -124..125 at which the largest magnitude of the group does not
// pass 6 when it is rounded, so no value moves by more than half a step.
//
// 64 tokens of a head lie together (68 D bytes, whole 128-byte lines), K, V, exponents of K, of V, each in the order
// in which a lane of v_mfma_f32_16x16x32_bf16 takes it:
//   K codes      [64 tokens][D / 2]                       16 bytes: a key's group of 32 channels, 4 steps' operands
//   V codes      [D / 32 groups][4 r][16 j][2 s][8 c]     a byte: channels 32 group + 2 j, + 1 of token 32 s + 8 r + c;
//                                                         16 bytes: two channels of the 16 keys whose weights a lane holds
//   K exponents  [4 r][4 c][D / 32][2 s][2 h]             of token 32 s + 8 r + 4 h + c; 4 bytes: those of a lane's 4 keys
//   V exponents  [D / 32][4 r][2 s][8 c]
// A page is its blocks of 64 tokens one after another, a block its heads.
#include "cache4_layout.h"
#include "window.h"

namespace track {

constexpr int C4_MIN = -124, C4_MAX = 125;  // exponents: half of 2^-124 and six of 2^125 are normal bfloat16 values
constexpr int64_t C4_HEADS = 1 << 19;

// The cache as the kernels take it.
struct CacheArgs {
  uint8_t* pages;
  const int32_t* table;
  int64_t ld_table, stride;  // entries between sequences; bytes of 64 tokens of all heads
  int table_pages, n_pages, blocks, cap;  // pages of a sequence, of the pool; 64-token blocks a page; places of a sequence
  WinDiv by_blocks;
};

// The 64 places from 64 t on of sequence b and head h, or null where no page holds them.  All wave-uniform.
template <int D>
__device__ __forceinline__ uint8_t* c4_at(const CacheArgs& c, int b, int h, int t) {
  const int slot = (int)c.by_blocks((uint32_t)t);
  if (slot >= c.table_pages) return nullptr;
  const int page = __builtin_amdgcn_readfirstlane(c.table[b * c.ld_table + slot]);
  if (!c4_page(page, c.n_pages)) return nullptr;
  return c.pages + c4_block(page, c.blocks, t, slot, c.stride) + (int64_t)h * C4<D>::BYTES;
}

// Tiles in their order, the block of 64 places and the table's entry of each from the last one's: tiles seen whole lie one
// after another but for the step from the first tokens to the window (by division 60 scalar instructions a tile, a fifth of a
// tile's time).
struct C4Walk {
  int idx, t, slot, in;  // the tile's place in the order, its block, the entry, the block in the page
  template <class Tiles>
  __device__ __forceinline__ void set(const CacheArgs& c, const Tiles& tiles, int i) {
    idx = i;
    t = tiles.template key<C4_BLOCK>(i) >> 6;
    slot = (int)c.by_blocks((uint32_t)t);
    in = t - slot * c.blocks;
  }
  // the next one, of `end` (the last one again)
  template <class Tiles>
  __device__ __forceinline__ void step(const CacheArgs& c, const Tiles& tiles, int end) {
    if (idx + 1 >= end) return;
    if (idx < tiles.edge || idx + 1 == tiles.edge + tiles.fs) {
      set(c, tiles, idx + 1);
    } else {
      ++idx, ++t, ++in;
      if (in == c.blocks) in = 0, ++slot;
    }
  }
  __device__ __forceinline__ int entry(const CacheArgs& c, int b) const {
    int zero;  // a vector load: a scalar one would be waited for with every read of LDS
    asm("v_mov_b32 %0, 0" : "=v"(zero));
    return c.table[b * c.ld_table + slot + zero];
  }
};

// The places of block `in` of the page that an entry names; the pool's first where it names none.
template <int D>
__device__ __forceinline__ const uint8_t* c4_of_entry(const CacheArgs& c, int entry, int h, int in, bool& there) {
  const int page = __builtin_amdgcn_readfirstlane(entry);
  there = c4_page(page, c.n_pages);
  return there ? c.pages + c4_block(page, c.blocks, in, 0, c.stride) + (int64_t)h * C4<D>::BYTES : c.pages;
}

// ---------------------------------------------------------------- rounding to 4 bits
// The exponent byte of a group whose largest magnitude is m (255: an infinity or a NaN in it).
__device__ __forceinline__ int c4_exponent(float m) {
  const uint32_t w = __float_as_uint(m);
  const int x = (int)(w >> 23) - 127;                      // m = f 2^x, f in [1, 2)
  const int e = x - 2 + ((w & 0x7fffff) >= 0x600000);      // 7 2^(x - 2) = 1.75 2^x
  return x == 128 ? 255 : 127 + min(max(e, C4_MIN), C4_MAX);
}

// Eight channels' codes at scale 2^e, given as its float (exact for float32 values: the conversion rounds once, ties to the
// even code).
__device__ __forceinline__ uint32_t c4_codes(const float (&x)[8], float s) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
}

// The largest of four lanes beside each other.
__device__ __forceinline__ uint32_t c4_quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));  // quad_perm [1, 0, 3, 2]
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));  // quad_perm [2, 3, 0, 1]
}

// The largest magnitude of a lane's 8 values, as bits (an infinity or a NaN is above all numbers).
__device__ __forceinline__ uint32_t c4_top(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  return m;
}

// Four bytes of codes of the lane's 8 channels, and the exponent byte of the group that they and those of the 3 lanes beside
// it make.
__device__ __forceinline__ uint32_t c4_round8(const float (&x)[8], int& byte) {
  byte = c4_exponent(__uint_as_float(c4_quad_max(c4_top(x))));
  const uint32_t w = c4_codes(x, __uint_as_float((uint32_t)byte << 23));
  return byte == 255 ? 0 : w;
}

// ---------------------------------------------------------------- rows in and out
struct RowsArgs {
  CacheArgs c;
  void *k, *v;
  int64_t ldk, sk, ldv, sv;
  const int32_t *start, *n;
  int B, L, heads, nblk;  // 64-token blocks that a sequence's rows can touch
  int hsplit;             // workgroups that share 16 tokens' heads
  bool vec;               // 16-byte aligned rows
  // rotation
  const int32_t* pos;
  const double* freqs;
  double amp;
  int pairs, sec0, sec1;
};

// The 16 tokens of a workgroup in a block of 64: slot 8 s + c is token 32 s + 8 r + c, r the quarter.  All wave-uniform.
struct RowsPart {
  int b, r, first;       // place of the block's first token, less the sequence's start
  int n;                 // rows of the sequence
  uint32_t there;        // slots that hold a row of the call, in a place that the cache has
  template <int D>
  __device__ __forceinline__ uint8_t* init(const RowsArgs& a, int item) {
    r = item & 3;
    const int blk = item >> 2;
    b = blk / a.nblk;
    n = a.n ? __builtin_amdgcn_readfirstlane(max(0, min(a.n[b], a.L))) : a.L;
    const int start = __builtin_amdgcn_readfirstlane(max(-(int)WIN_MAX, min(a.start[b], (int)WIN_MAX)));
    const int t = (start >> 6) + (blk - b * a.nblk);
    first = t * C4_BLOCK - start;
    there = 0;
    if (t < 0 || t * (int64_t)C4_BLOCK >= a.c.cap) return nullptr;
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      const int i = row(s);
      there |= (uint32_t)(i >= 0 && i < n) << s;
    }
    return there ? c4_at<D>(a.c, b, 0, t) : nullptr;
  }
  __device__ __forceinline__ int token(int slot) const { return c4_token(r, slot); }
  __device__ __forceinline__ int row(int slot) const { return first + token(slot); }
};

// A lane's 8 channels as they lie in memory.
template <typename T>
struct C4Unit {
  u32x4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p, bool vec) {
    if (vec) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = ((const u32x4*)p)[i];
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[0][i] = (uint32_t)p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i >> 2][i & 3] = __float_as_uint(p[i]);
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 2) x[i] = __uint_as_float(i & 1 ? w[0][i >> 1] & 0xffff0000u : w[0][i >> 1] << 16);
      else x[i] = __uint_as_float(w[i >> 2][i & 3]);
    }
  }
};

// The wave's own LDS writes, before its reads.
__device__ __forceinline__ void c4_settle() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Appends.  A workgroup takes 16 tokens of a block, forms their angles once while its first rows are under way, and its waves
// walk the heads; a lane has 8 channels of a token, D / 8 lanes a token.  Codes and exponents change places through LDS into
// the order of the cache, and leave in 16-byte units.  A key is what its rotation in float64 rounds to: float32 would fall to
// either side of a border of two codes (one value in some 10^6, a whole step off).  Sines, cosines, products and sum are
// float64, which the vector units multiply and add at float32's rate; the float32 value that the conversion to 4 bits takes is
// off the sum by its own rounding, which matters only where it meets a border, a number of at most three bits.  There it moves
// on to the next one on the sum's side.  (In float32 with a margin and float64 again where that held a border: 132 us for the
// three axes below, 184 for halves.) What bounds it: memory, and the conversions, whose time shows beside it.  2 x 32760
// tokens of 12 heads: bfloat16 as they are 107 us (4.8 TB/s), turned on three axes 115, as halves 124, float32 on three axes
// 191 (4.8).  Angles in the order of the pairs instead of the lanes': halves 145; rows only after the angles: 117, one head 28
// instead of 26.  A token for each of 16 sequences takes 6.2 us, a chain of
// loads and one of sines (8.3 where absent tokens were turned too).
template <typename T, int D, int ROT>
__global__ __launch_bounds__(256) void cache_append_kernel(RowsArgs a) {
  constexpr int LPT = D / 8, TPS = 64 / LPT, STEPS = 16 / TPS, G = D / 32;
  __shared__ double2 cs[ROT ? 16 * (D / 2) : 1];
  __shared__ __attribute__((aligned(16))) uint32_t kcodes[4][16 * LPT], vcodes[4][16 * LPT];
  __shared__ __attribute__((aligned(16))) uint8_t kexp[4][16 * G], vexp[4][16 * G];  // in the cache's order
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int item = (int)blockIdx.x / a.hsplit, part = (int)blockIdx.x - item * a.hsplit;
  RowsPart w;
  uint8_t* const block = w.init<D>(a, item);
  if (!block) return;  // the whole workgroup
  const int u = lane % LPT, sub = lane / LPT;
  // the lane that has the other channels of this one's pairs (half layout), if they are a unit
  const bool whole = ROT == 2 && (a.pairs & 7) == 0;
  const int other = (8 * u < a.pairs ? a.pairs : (8 * u < 2 * a.pairs ? -a.pairs : 0)) / 8;
  // a head's rows; the first ones are under way while the angles are formed
  const T* kp[STEPS];
  C4Unit<T> rk[STEPS], rv[STEPS];
  auto fetch = [&](int h) {
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int slot = st * TPS + sub;
      const int64_t row = w.there >> slot & 1 ? w.row(slot) : 0;  // (any row of the sequence in a slot without one)
      kp[st] = (const T*)a.k + w.b * a.sk + row * a.ldk + (int64_t)h * D;
      rk[st].load(kp[st] + 8 * u, a.vec);
      rv[st].load((const T*)a.v + w.b * a.sv + row * a.ldv + (int64_t)h * D + 8 * u, a.vec);
    }
  };
  const int h0 = part * 4 + wave;
  if (h0 < a.heads) fetch(h0);
  // a pair's place among those of a token: the first ones of all lanes beside each other, so that a read meets no bank twice
  constexpr int PER = ROT == 1 ? 4 : 8;
  auto angle_at = [](int p) { return (p & (PER - 1)) * (D / 2 / PER) + p / PER; };
  if constexpr (ROT != 0) {
    // thread: pair p of every (512 / D)-th slot
    constexpr int N = D / 32;
    const int p = threadIdx.x % (D / 2), s0 = threadIdx.x / (D / 2);
    const bool rotated = p < a.pairs;
    const int axis = (p >= a.sec0) + (p >= a.sec1);
    const double f = a.freqs[rotated ? p : 0] * 0.15915494309189533577;
    const int32_t* const pp = a.pos + ((int64_t)(rotated ? axis : 0) * a.B + w.b) * a.L;
    int at[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int slot = s0 + i * (512 / D);
      at[i] = pp[w.there >> slot & 1 ? w.row(slot) : 0];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      double sn = 0.0, cn = 1.0;  // copied channels
      if (rotated && (w.there >> (s0 + i * (512 / D)) & 1)) {
        const double t = (double)at[i] * f;
        sincospi(2.0 * (t - rint(t)), &sn, &cn);
        sn *= a.amp, cn *= a.amp;
      }
      cs[(s0 + i * (512 / D)) * (D / 2) + angle_at(p)] = double2{cn, sn};
    }
    __syncthreads();
  }
  // the pair of channel i of unit un, and whether the channel is the pair's first
  auto pair_of = [&](int un, int i, bool& low) {
    if constexpr (ROT == 1) {
      low = !(i & 1);
      return 4 * un + (i >> 1);
    } else {
      const int ch = 8 * un + i;
      low = ch < a.pairs;
      return low ? ch : ch - a.pairs;
    }
  };
  // the lane's pairs where its unit is all first channels, all second ones or all copied
  const bool low0 = 8 * u < a.pairs;
  const int first = min(low0 ? u : u - a.pairs / 8, D / 16 - 1);
  // the exponent's place in the cache's order: K [4 c][G][2 s][2 h], V [G][2 s][8 c]
  auto kexp_at = [&](int un, int slot) {
    const int c = slot & 7;
    return (c & 3) * (4 * G) + 4 * (un >> 2) + 2 * (slot >> 3) + (c >> 2);
  };
  const bool all = w.there == 0xffff;
  for (int h = h0; h < a.heads; h += 4 * a.hsplit) {
    uint8_t* const to = block + (int64_t)h * C4<D>::BYTES;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      if (!(w.there >> (st * TPS) & ((1u << TPS) - 1u))) continue;  // (a single token's wave has one such step)
      const int slot = st * TPS + sub;
      float x[8];
      uint32_t word;
      int byte;
      rk[st].get(x);
      if constexpr (ROT == 0) {
        word = c4_round8(x, byte);
      } else {
        float z[8];  // the other channel of each one's pair
        if constexpr (ROT == 1) {
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = x[i ^ 1];
        } else if (whole) {
          C4Unit<T> o;  // another lane's
#pragma unroll
          for (int j = 0; j < (int)sizeof(T) / 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) o.w[j][e] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane + other), (int)rk[st].w[j][e]);
          o.get(z);
        } else {
          const int un = att_lane() % LPT;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int ch = 8 * un + i;
            z[i] = ldf(kp[st] + (ch < a.pairs ? ch + a.pairs : (ch < 2 * a.pairs ? ch - a.pairs : ch)));
          }
        }
        double r[8];
        float y[8];
        const double2* const at = cs + slot * (D / 2);
        auto turn = [&](int i, const double2& t, bool low, bool rotated) {
          r[i] = (double)x[i] * t.x + (double)(low ? -z[i] : z[i]) * t.y;
          y[i] = rotated ? (float)r[i] : x[i];
          r[i] = rotated ? r[i] : (double)x[i];
        };
        if (ROT == 2 && whole) {
#pragma unroll
          for (int i = 0; i < 8; ++i) turn(i, at[first + i * (D / 16)], low0, 8 * u < 2 * a.pairs);
        } else {
          const int un = ROT == 2 ? att_lane() % LPT : u;  // (formed here: eight pairs' places would stay in registers)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            bool low;
            const int p = pair_of(un, i, low);
            turn(i, at[ROT == 1 ? (i >> 1) * (D / 8) + u : angle_at(min(p, D / 2 - 1))], low, p < a.pairs);
          }
        }
        uint32_t few = ~0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) few = min(few, __float_as_uint(y[i]) << 12);
        if (__ballot(few == 0)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const double d = fabs((double)y[i]), m = fabs(r[i]);
            const uint32_t bits = __float_as_uint(y[i]), to = m < d ? ~0u : (m > d ? 1u : 0u);  // (a NaN stays)
            y[i] = __uint_as_float(bits + (bits << 12 ? 0u : to));  // (others could meet one)
          }
        }
        word = c4_round8(y, byte);
      }
      kcodes[wave][slot * LPT + u] = word;
      if ((u & 3) == 0) kexp[wave][kexp_at(u, slot)] = (uint8_t)byte;
      rv[st].get(x);
      vcodes[wave][slot * LPT + u] = c4_round8(x, byte);
      if ((u & 3) == 0) vexp[wave][16 * (u >> 2) + slot] = (uint8_t)byte;
      if (ROT == 2) __builtin_amdgcn_sched_barrier(0);
    }
    c4_settle();
    if (lane < D / 2) {
      // K: 16 bytes of one token; V: group lane / 16, byte lane % 16 of a group's 16, of the 16 tokens
      const int slot = lane / G;
      if (w.there >> slot & 1)
        *(u32x4*)(to + C4<D>::k_code(w.token(slot), 32 * (lane % G))) = *(const u32x4*)&kcodes[wave][4 * lane];
      const uint8_t* const from = (const uint8_t*)vcodes[wave] + lane;
      uint8_t* const vt = to + C4<D>::v_code(8 * w.r, 2 * lane);
      if (all) {
        u32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[i] = (uint32_t)from[(4 * i) * (D / 2)] | (uint32_t)from[(4 * i + 1) * (D / 2)] << 8 |
                 (uint32_t)from[(4 * i + 2) * (D / 2)] << 16 | (uint32_t)from[(4 * i + 3) * (D / 2)] << 24;
        *(u32x4*)vt = o;
      } else {
        for (int s = 0; s < 16; ++s)
          if (w.there >> s & 1) vt[s] = from[s * (D / 2)];
      }
    }
    if (all) {
      const int i = lane & (4 * G - 1);  // G words of 4 exponents for each of 4 c, or of 4 runs of 4 tokens for each group
      if (lane < 4 * G) *(uint32_t*)(to + C4<D>::k_exp(8 * w.r, 0) + 4 * i) = ((const uint32_t*)kexp[wave])[i];
      else if (lane < 8 * G) *(uint32_t*)(to + C4<D>::v_exp(8 * w.r, i >> 2) + 4 * (i & 3)) = ((const uint32_t*)vexp[wave])[i];
    } else if (lane < 16 * G) {
      const int slot = lane & 15, grp = lane >> 4, c = slot & 7;
      if (w.there >> slot & 1) {
        to[C4<D>::k_exp(w.token(slot), grp)] = kexp[wave][(c & 3) * (4 * G) + 4 * grp + 2 * (slot >> 3) + (c >> 2)];
        to[C4<D>::v_exp(w.token(slot), grp)] = vexp[wave][lane];
      }
    }
    c4_settle();
    if (h + 4 * a.hsplit < a.heads) fetch(h + 4 * a.hsplit);
  }
}

// ---------------------------------------------------------------- 4 bits back to values
// Byte SEL of w as the two values that it stands for at scale s.
template <int SEL>
__device__ __forceinline__ uint32_t c4_pair(uint32_t w, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL));
}
template <int SEL>
__device__ __forceinline__ f32x2 c4_pair_f32(uint32_t w, float s) {
  return __builtin_bit_cast(f32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, SEL));
}
// Byte I of w as a float whose exponent it is (255 gives NaN in the conversions).  They look at the exponent alone (checked for all
// 256 with signs and mantissas of every kind), so the other bytes' bits stay in those: one instruction instead of two.
template <int I>
__device__ __forceinline__ float c4_scale(uint32_t w) {
  return __uint_as_float(I < 3 ? w << (23 - 8 * I) : w >> 1);
}
// Four bytes of codes, 8 channels of one group, as bfloat16.
__device__ __forceinline__ u32x4 c4_eight(uint32_t w, float s) {
  return u32x4{c4_pair<0>(w, s), c4_pair<1>(w, s), c4_pair<2>(w, s), c4_pair<3>(w, s)};
}
// Two channels (a byte each key) of four keys with exponents e: the channels' four keys, two words each (the first channel's
// in lo, or what the selectors of v_perm take).
__device__ __forceinline__ void c4_four(uint32_t w, uint32_t e, uint32_t (&lo)[2], uint32_t (&hi)[2], uint32_t first = 0x05040100, uint32_t second = 0x07060302) {
  const uint32_t a = c4_pair<0>(w, c4_scale<0>(e)), b = c4_pair<1>(w, c4_scale<1>(e));
  const uint32_t c = c4_pair<2>(w, c4_scale<2>(e)), d = c4_pair<3>(w, c4_scale<3>(e));
  lo[0] = __builtin_amdgcn_perm(b, a, first), hi[0] = __builtin_amdgcn_perm(b, a, second);
  lo[1] = __builtin_amdgcn_perm(d, c, first), hi[1] = __builtin_amdgcn_perm(d, c, second);
}

// Channels of a row at p: a lane's 8 in bfloat16, 4 and 4 that lie `half` further in float32, so that the lanes of a store
// cover whole lines (65520 tokens of 12 heads: with 8 beside each other 239 us, 211 so).  Codes are 2 bytes each of lo and
// hi.  Past the caches: 2 x 32760 tokens of 12 heads 114 -> 110 us.
template <typename T>
__device__ __forceinline__ void c4_store8(T* p, int half, bool vec, uint32_t lo, uint32_t hi, float s, float s2) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 x = c4_eight(lo | hi << 16, s);
    if (vec) {
      __builtin_nontemporal_store(x, (u32x4*)p);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = (bf16_t)(i & 1 ? x[i >> 1] >> 16 : x[i >> 1]);
    }
  } else {
    const f32x2 a = c4_pair_f32<0>(lo, s), b = c4_pair_f32<1>(lo, s), c = c4_pair_f32<0>(hi, s2), d = c4_pair_f32<1>(hi, s2);
    if (vec) {
      __builtin_nontemporal_store(f32x4{a[0], a[1], b[0], b[1]}, (f32x4*)p);
      __builtin_nontemporal_store(f32x4{c[0], c[1], d[0], d[1]}, (f32x4*)(p + half));
    } else {
      p[0] = a[0], p[1] = a[1], p[2] = b[0], p[3] = b[1];
      p[half] = c[0], p[half + 1] = c[1], p[half + 2] = d[0], p[half + 3] = d[1];
    }
  }
}

// Rows out of the cache: the append's shape the other way round.  Places without a page read as zero.  What bounds it: memory,
// four bytes written (bfloat16) for each one read: 2 x 32760 tokens of 12 heads 110 us among other work, 4.6 TB/s, 80 (6.4)
// replayed on one cache, whose 107 MB then come out of the Infinity Cache; float32 211 (4.3).
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_read_kernel(RowsArgs a) {
  constexpr int LPT = D / 8, TPS = 64 / LPT, STEPS = 16 / TPS, G = D / 32;
  __shared__ u32x4 codes[4][D / 2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int item = (int)blockIdx.x / a.hsplit, part = (int)blockIdx.x - item * a.hsplit;
  RowsPart w;
  const uint8_t* const block = w.init<D>(a, item);
  const int u = lane % LPT, sub = lane / LPT;
  // the lane's channels: c0 .. + 3 and c1 .. + 3
  constexpr bool WIDE = sizeof(T) == 2;
  const int c0 = WIDE ? 8 * u : 4 * u, c1 = WIDE ? c0 + 4 : c0 + D / 2;
  if (!block) {  // rows in places that the cache does not have
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int row = w.row(st * TPS + sub);
      if (row < 0 || row >= w.n) continue;
      for (int h = part * 4 + wave; h < a.heads; h += 4 * a.hsplit) {
        c4_store8((T*)a.k + w.b * a.sk + (int64_t)row * a.ldk + (int64_t)h * D + c0, c1 - c0, a.vec, 0, 0, 1.0f, 1.0f);
        c4_store8((T*)a.v + w.b * a.sv + (int64_t)row * a.ldv + (int64_t)h * D + c0, c1 - c0, a.vec, 0, 0, 1.0f, 1.0f);
      }
    }
    return;
  }
  for (int h = part * 4 + wave; h < a.heads; h += 4 * a.hsplit) {
    const uint8_t* const from = block + (int64_t)h * C4<D>::BYTES;
    if (lane < D / 2) codes[wave][lane] = *(const u32x4*)(from + C4<D>::v_code(8 * w.r, 2 * lane));
    c4_settle();
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int slot = st * TPS + sub, tok = w.token(slot);
      if (!(w.there >> slot & 1)) continue;
      const int64_t row = w.row(slot);
      uint32_t lo, hi;
      if constexpr (WIDE) {
        const uint32_t k = *(const uint32_t*)(from + C4<D>::k_code(tok, c0));
        lo = k & 0xffff, hi = k >> 16;
      } else {
        lo = *(const uint16_t*)(from + C4<D>::k_code(tok, c0)), hi = *(const uint16_t*)(from + C4<D>::k_code(tok, c1));
      }
      auto scale = [&](int at) { return __uint_as_float((uint32_t)from[at] << 23); };
      const float ks = scale(C4<D>::k_exp(tok, c0 >> 5)), ks2 = WIDE ? ks : scale(C4<D>::k_exp(tok, c1 >> 5));
      c4_store8((T*)a.k + w.b * a.sk + row * a.ldk + (int64_t)h * D + c0, c1 - c0, a.vec, lo, hi, ks, ks2);
      const uint8_t* const p = (const uint8_t*)codes[wave] + slot;  // 16 bytes for each byte of a token
      lo = (uint32_t)p[8 * c0] | (uint32_t)p[8 * c0 + 16] << 8;
      hi = (uint32_t)p[8 * c1] | (uint32_t)p[8 * c1 + 16] << 8;
      const float vs = scale(C4<D>::v_exp(tok, c0 >> 5)), vs2 = WIDE ? vs : scale(C4<D>::v_exp(tok, c1 >> 5));
      c4_store8((T*)a.v + w.b * a.sv + row * a.ldv + (int64_t)h * D + c0, c1 - c0, a.vec, lo, hi, vs, vs2);
    }
    c4_settle();
  }
}

// ---------------------------------------------------------------- few rows, bfloat16
// A byte of 0x80 for each byte of x that is 253 or more: 255, and the exponents that no append writes and at which 6 is an
// infinity in bfloat16.
__device__ __forceinline__ uint32_t c4_nan_bytes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x03030303u) & x & 0x80808080u; }
// Bytes of four keys of which `left` are to keep (any number).
__device__ __forceinline__ uint32_t c4_keep(int left) { return (uint32_t)((1ull << (8 * min(max(left, 0), 4))) - 1ull); }

// What a lane takes of a 64-key tile: 4 keys' groups of K with their exponents, two channels of each V group for its 16 keys,
// and these keys' exponents of every group.
struct C4Raw {
  u32x4 k[4], v[4], e[4];
  uint32_t ke;
};

// At most 16 rows a key head (a token of 16 query heads, four tokens of 4).  The four waves of a workgroup take every fourth
// tile of its share.  The layout makes every operand a lane's own bytes, so a tile goes from memory to registers, 16 bytes a
// lane and whole lines a load, and there to bfloat16; nothing passes through LDS until the waves' sums meet. The next tile's K
// takes the place of this one's as soon as its logits are formed, V that of V. What bounds it: memory (8 sequences of 8 key
// heads, 100003 to 56000 keys, 680 MB: 112 us and the join 4, 6.1 TB/s; 160 with the table read and the places divided tile by
// tile), and for short windows the chain of loads (1024 of 8192 keys: 7.3 and 4.4).  Loads go past the caches also where
// sequences share their pages: 32 sequences of 8 key heads on 32760 shared keys take 134 us so and 126 through the caches, after 1
// GiB written elsewhere 137 and 131, 16 on 8192 27.1 and 27.0, 30.8 and 31.3; on pages of their own 189 and 210, 192 and 275,
// 33 and 32, 36 and 65.  What the host could know of it, one table row for all, is a part of it only.  K's codes and exponents are also what
// v_mfma_scale_f32_16x16x128_f8f6f4 takes as they lie, with queries split into two 8-bit halves. Its sums are not float32:
// checked on this chip, they drop what lies some 15 bits below the largest product.  So K is turned into bfloat16.
template <bool SPLIT>
__global__ __launch_bounds__(256, 3) void cache_rows_kernel(WinArgs a, CacheArgs ca) {
  constexpr int BKV = C4_BLOCK, D = ATT_D, F = D / 16;
  __shared__ f32x4 so[4][F][64];
  __shared__ float sm[4][16], sl[4][16];
  __shared__ u32x4 qs[D / 32][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int jq = lane & 15, g = lane >> 4;
  int rb, sp, h, b;
  win_place<false>(a, rb, sp, h, b);
  const WinSeq seq = win_seq(a, b);
  const int rows = seq.qlen * a.n;  // at most 16
  if (rows == 0) return;            // the whole workgroup

  int lo0, hi0, lo1, hi1;
  win_range(a, seq, 0, lo0, hi0);
  win_range(a, seq, seq.qlen - 1, lo1, hi1);
  WinTiles tiles;
  tiles.init<BKV>(seq, __builtin_amdgcn_readfirstlane(lo0), __builtin_amdgcn_readfirstlane(hi0),
                  __builtin_amdgcn_readfirstlane(lo1), __builtin_amdgcn_readfirstlane(hi1));
  int i0 = 0, i1 = tiles.n;
  if (SPLIT) win_share(tiles.n, sp, a.nsplit, i0, i1);

  // the lane's row (the last one again past the end)
  int e;
  const int qi = win_query(a, min(jq, rows - 1), e), head = h * a.n + e;
  WinMask<1> mask;
  mask.sink = tiles.sink;
  win_range(a, seq, qi, mask.lo[0], mask.hi[0]);
  if (tiles.sink == 0 && seq.sink >= lo1) mask.lo[0] = 0;
  // a lane's channels 32 g + 8 step .. + 7, as its bytes of K hold them
  const bf16_t* qp = (const bf16_t*)a.q + b * a.sq + (int64_t)qi * a.ldq + (int64_t)head * D + 32 * g;
  // (the waves have the same rows; from LDS a tile, and in an order that takes V group by group, 168 registers are enough:
  // three waves a SIMD)
  if (wave == 0) {
#pragma unroll
    for (int kc = 0; kc < D / 32; ++kc) qs[kc][lane] = *(const u32x4*)(qp + kc * 8);
  }
  __syncthreads();
  const uint32_t koff = c4_row_k(lane), keoff = c4_row_ke(lane), voff = c4_row_v(lane, 0), veoff = c4_row_ve(lane, 0);
  // Loads that are not needed (no page, past the share) read the pool's first block: as many for every
  // tile, so that the wait for the older ones can count.
  C4Raw r;
  auto fetch_k = [&](const uint8_t* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.k[i] = __builtin_nontemporal_load((const u32x4*)(p + (koff + c4_row_k_block(i))));
    r.ke = __builtin_nontemporal_load((const uint32_t*)(p + keoff));
  };
  auto fetch_v = [&](const uint8_t* p) {
#pragma unroll
    for (int m = 0; m < 4; ++m) r.v[m] = __builtin_nontemporal_load((const u32x4*)(p + (voff + (c4_row_v(0, m) - c4_row_v(0, 0)))));
#pragma unroll
    for (int m = 0; m < 4; ++m) r.e[m] = __builtin_nontemporal_load((const u32x4*)(p + (veoff + (c4_row_ve(0, m) - c4_row_ve(0, 0)))));
  };

  f32x4 o[F];
  float m = -INFINITY, l = 0.0f;  // reference (log2 units), the lane's part of the denominator
#pragma unroll
  for (int f = 0; f < F; ++f) o[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // the tile's page, and the entries of the next ones, two tiles ahead
  bool there = false;
  const uint8_t* at = nullptr;
  C4Walk next;
  int entry = 0;
  if (i0 + wave < i1) {
    next.set(ca, tiles, i0 + wave);
    at = c4_of_entry<D>(ca, next.entry(ca, b), h, next.in, there);
    fetch_k(at);
    next.set(ca, tiles, min(i0 + wave + 4, i1 - 1));
    entry = next.entry(ca, b);
    fetch_v(at);
  }
  for (int idx = i0 + wave; idx < i1; idx += 4) {
    bool next_there;
    at = c4_of_entry<D>(ca, entry, h, next.in, next_there);
    const int key0 = tiles.key<BKV>(idx);
    const bool edge = idx < tiles.edge || !there;
    const float ks[4] = {c4_scale<0>(r.ke), c4_scale<1>(r.ke), c4_scale<2>(r.ke), c4_scale<3>(r.ke)};
    f32x4 s[BKV / 16];
    bf16x8 qf[D / 32];
#pragma unroll
    for (int kc = 0; kc < D / 32; ++kc) qf[kc] = __builtin_bit_cast(bf16x8, qs[kc][lane]);
#pragma unroll
    for (int kc = 0; kc < D / 32; ++kc)
#pragma unroll
      for (int i = 0; i < BKV / 16; ++i)
        s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, c4_eight(r.k[i][kc], ks[i])), qf[kc],
                                                       kc ? s[i] : f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    fetch_k(at);
    next.set(ca, tiles, min(idx + 8, i1 - 1));
    entry = next.entry(ca, b);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t lost = 0;  // groups of V in which a key that the row sees holds no number
    if (edge) {
      WinMask<1> mk = mask;
      mk.key0 = key0;
      mk.begin();
      if (!there) mk.bits[0] = 0xffff;
#pragma unroll
      for (int i = 0; i < BKV / 16; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[i][x] = mk.apply(0, 32 * (i >> 1) + 4 * (i & 1) + x, s[i][x]);
      // V past the last key, which may be anything, takes exponent 0 (a weight of zero would not remove a NaN or an infinity),
      // and so do groups that may hold one, whose keys some rows may not see: they are put into the rows that do
      const int last = there ? seq.klen - key0 - 8 * g : 0;
      uint32_t any = 0;
#pragma unroll
      for (int mm = 0; mm < 4; ++mm)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          r.e[mm][w] &= c4_keep(last - 32 * (w >> 1) - 4 * (w & 1));
          any |= c4_nan_bytes(r.e[mm][w]);
        }
      if (__ballot(any != 0)) {
#pragma unroll
        for (int mm = 0; mm < 4; ++mm)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t bad = c4_nan_bytes(r.e[mm][w]) >> 7;
            const uint32_t seen = ~(mk.bits[0] >> (4 * w));
            const uint32_t hit = (bad & seen & 1u) | ((bad >> 8) & (seen >> 1) & 1u) | ((bad >> 16) & (seen >> 2) & 1u) |
                                 ((bad >> 24) & (seen >> 3) & 1u);
            lost |= hit << mm;
            r.e[mm][w] &= ~(bad * 255u);
          }
        lost |= (uint32_t)__shfl_xor((int)lost, 16);
        lost |= (uint32_t)__shfl_xor((int)lost, 32);
      }
    }
    float t = -INFINITY;
#pragma unroll
    for (int i = 0; i < BKV / 16; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) t = fmaxf(t, s[i][x]);
    const float mn = fmaxf(m, group_max2(t, t) * a.scale_log2);
    if (__ballot(mn > m)) {
      const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      l *= alpha;
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[f][x] *= alpha;
      m = mn;
    }
    const float nm = m == -INFINITY ? 0.0f : -m;
    u32x4 pw[BKV / 32];
#pragma unroll
    for (int c = 0; c < BKV / 32; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 x = s[2 * c + (q >> 1)];
        const float p0 = __builtin_amdgcn_exp2f(fmaf(x[2 * (q & 1)], a.scale_log2, nm));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(x[2 * (q & 1) + 1], a.scale_log2, nm));
        pw[c][q] = pack_bf2(p0, p1);
        // the denominator adds the weights as rounded for the product with V
        l += __uint_as_float(pw[c][q] << 16) + __uint_as_float(pw[c][q] & 0xffff0000u);
      }
#pragma unroll
    for (int c = 0; c < BKV / 32; ++c)
#pragma unroll
      for (int mm = 0; mm < D / 32; ++mm) {
        uint32_t lo[2][2], hi[2][2];
#pragma unroll
        for (int w = 0; w < 2; ++w) c4_four(r.v[mm][2 * c + w], r.e[mm][2 * c + w], lo[w], hi[w]);
        const bf16x8 p = __builtin_bit_cast(bf16x8, pw[c]);
        o[2 * mm] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{lo[0][0], lo[0][1], lo[1][0], lo[1][1]}), p, o[2 * mm], 0, 0, 0);
        o[2 * mm + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u32x4{hi[0][0], hi[0][1], hi[1][0], hi[1][1]}), p, o[2 * mm + 1], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    if (edge && __ballot(lost != 0)) {
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[f][x] = lost >> (f >> 1) & 1 ? NAN : o[f][x];
    }
    __builtin_amdgcn_sched_barrier(0);
    fetch_v(at);
    __builtin_amdgcn_sched_barrier(0);
    there = next_there;
  }

  // join the four waves: each takes one of the four groups of 32 channels; a lane's are 32 wave + 8 g .. + 7
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int f = 0; f < F; ++f) so[wave][f][lane] = o[f];
  if (g == 0) {
    sm[wave][jq] = m;
    sl[wave][jq] = l;
  }
  __syncthreads();
  float mx = -INFINITY, sum = 0.0f, wt[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sm[w][jq]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mi = sm[w][jq];
    wt[w] = mi == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mi - mx);  // a wave without keys
    sum = fmaf(wt[w], sl[w][jq], sum);
  }
  if (jq >= rows) return;
  const int64_t pr = ((((int64_t)sp * a.B + b) * a.Hk + h) * a.Lq) * a.n + jq;
  const float inv = SPLIT ? 1.0f : win_inverse(sum);
  f32x4 v0 = {0.0f, 0.0f, 0.0f, 0.0f}, v1 = v0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const f32x4 x = so[w][2 * wave][lane], y = so[w][2 * wave + 1][lane];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v0[i] = fmaf(wt[w], x[i], v0[i]);
      v1[i] = fmaf(wt[w], y[i], v1[i]);
    }
  }
  const int ch = 32 * wave + 8 * g;
  if constexpr (SPLIT) {
    *(f32x4*)(a.po + pr * D + ch) = f32x4{v0[0], v1[0], v0[1], v1[1]};
    *(f32x4*)(a.po + pr * D + ch + 4) = f32x4{v0[2], v1[2], v0[3], v1[3]};
  } else {
    *(u32x4*)((bf16_t*)a.out + b * a.so + (int64_t)qi * a.ldo + (int64_t)head * D + ch) =
        u32x4{pack_bf2(v0[0] * inv, v1[0] * inv), pack_bf2(v0[1] * inv, v1[1] * inv), pack_bf2(v0[2] * inv, v1[2] * inv),
              pack_bf2(v0[3] * inv, v1[3] * inv)};
  }
  if (wave == 0 && g == 0) {
    if constexpr (SPLIT) a.pml[pr] = float2{mx, sum};
    else if (a.lse) a.lse[((int64_t)b * a.Hk * a.n + head) * a.Lq + qi] = win_lse(mx, sum);
  }
}

// ---------------------------------------------------------------- many rows, bfloat16
// 256 rows a workgroup, 32 a wave, and the tile body of the plain attention on tiles that the workgroup turns into bfloat16 in
// LDS (attention_tile.h's layout): half of the threads take K's 16 bytes each, half V's.  The next tile's bytes are under way
// while one is computed on. What bounds it: the matrix cores and the conversions in turn.  12 heads, 4680 queries on thirteen
// frames of 1560 keys, 583 GFLOP: 637 us (549 on bfloat16 keys in window.hip, 26 instructions a thread and 32 KB into LDS a
// tile fewer); matrix cores busy 50% of the cycles in which a CU has work, 78% of all: 228 workgroups on 256 CUs.  On the way:
// 864 with scalar table reads and divisions a tile, 676 with V written in the bytes' order.
template <bool QLOG2, bool SPLIT>
__global__ __launch_bounds__(512) void cache_blocks_kernel(WinArgs a, CacheArgs ca) {
  constexpr int BKV = ATT_BKV, D = ATT_D, SLOT = ATT_SLOT;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * SLOT + 2 * 256];  // two tiles, and where V holds no number
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int jq = lane & 15, g = lane >> 4;
  int rb, sp, h, b;
  win_place<true>(a, rb, sp, h, b);
  const WinSeq seq = win_seq(a, b);
  const int rows = seq.qlen * a.n;
  const int r0 = rb * ATT_BQ;
  if (r0 >= rows) return;  // the whole workgroup

  // windows of the block's first and last row, and of the wave's
  auto range_of = [&](int r, int& lo, int& hi) {
    win_range(a, seq, (int)a.by_n((uint32_t)min(r, rows - 1)), lo, hi);
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
  };
  int lo0, hi0, lo1, hi1;
  range_of(r0, lo0, hi0);
  range_of(r0 + ATT_BQ - 1, lo1, hi1);
  WinTiles tiles;
  tiles.init<BKV>(seq, lo0, hi0, lo1, hi1);
  const int wr0 = r0 + 32 * wave;
  int wlo, whi, unused;
  range_of(wr0, wlo, unused);
  range_of(wr0 + 31, unused, whi);
  if (tiles.sink == 0 && seq.sink >= lo1) wlo = 0;
  const bool live = wr0 < rows;

  bf16x8 qf[D / 32][ATT_QB];
  WinMask<ATT_QB> mask;
  mask.sink = tiles.sink;
#pragma unroll
  for (int i = 0; i < ATT_QB; ++i) {
    int e;
    const int qi = win_query(a, min(wr0 + 16 * i + jq, rows - 1), e);
    win_range(a, seq, qi, mask.lo[i], mask.hi[i]);
    if (tiles.sink == 0 && seq.sink >= lo1) mask.lo[i] = 0;
    const bf16_t* qp = (const bf16_t*)a.q + b * a.sq + (int64_t)qi * a.ldq + (int64_t)(h * a.n + e) * D + g * 8;
#pragma unroll
    for (int kc = 0; kc < D / 32; ++kc) qf[kc][i] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qp + kc * 32));
  }

  // What this thread brings in: 16 bytes of K, group kg of key kt, or 16 of V, channels vc and vc + 1 of the keys 32 s + 8 vr
  // + 0..7.  The LDS row of key (channel) 8 q + 4 x + j of 32 is 16 x + 4 q + j; K's four units and V's two differ from the
  // first in an XOR, and the rows of two channels beside each other have one swizzle.  Where j has bit 1 the second channel
  // goes first: the 16 threads that write together then meet every bank once (in the bytes' own order four times: 676 us, 644
  // so).
  const bool isv = wave >= 4;
  uint32_t put;
  {
    auto row_of = [](int x) { return (x & 96) | (((x >> 2) & 1) << 4) | (((x >> 3) & 3) << 2) | (x & 3); };
    const int t8 = tid & 255, r = row_of(isv ? c4_tile_channel(t8) : c4_tile_key(t8));
    put = (uint32_t)(isv ? ATT_K_BYTES + (r ^ ((t8 >> 1) & 1)) * ATT_VROW + ((c4_tile_r(t8) ^ att_vswz(r)) << 4)
                         : r * 256 + (((4 * c4_tile_group(t8)) ^ (r & 15)) << 4));
  }
  struct Raw {
    u32x4 w, e;
  };
  const uint32_t from = c4_tile_codes(isv, tid & 255), efrom = c4_tile_exp(isv, tid & 255);
  auto fetch = [&](const uint8_t* p, Raw& r) {
    r.w = *(const u32x4*)(p + from);
    if (isv) r.e = *(const u32x4*)(p + efrom);
    else r.e[0] = p[efrom];
  };
  auto spread = [&](Raw& r, int key0, bool edge) {  // into the slot that put points at
    if (!isv) {
      const float s = __uint_as_float(r.e[0] << 23);
#pragma unroll
      for (int i = 0; i < 4; ++i) *(u32x4*)(smem + (put ^ (uint32_t)(i << 4))) = c4_eight(r.w[i], s);
      return;
    }
    if (edge) {
      // V past the last key takes exponent 0, and so do groups that hold no number (below)
      const int t8 = (wave & 3) * 64 + att_lane(), vr = c4_tile_r(t8);
      u32x4 bad;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        r.e[w] &= c4_keep(seq.klen - key0 - 8 * vr - 32 * (w >> 1) - 4 * (w & 1));
        bad[w] = c4_nan_bytes(r.e[w]) >> 7;
        r.e[w] &= ~(bad[w] * 255u);
      }
      if (c4_tile_j(t8) == 0) *(u32x4*)(smem + 2 * SLOT + (put & SLOT ? 256 : 0) + ((t8 >> 6) * 4 + vr) * 16) = bad;
    }
    const uint32_t sel = tid & 2 ? 0x07060302u : 0x05040100u;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      uint32_t lo[2][2], hi[2][2];
#pragma unroll
      for (int w = 0; w < 2; ++w) c4_four(r.w[2 * s + w], r.e[2 * s + w], lo[w], hi[w], sel, sel ^ 0x02020202u);
      *(u32x4*)(smem + (put ^ (uint32_t)(s << 6))) = u32x4{lo[0][0], lo[0][1], lo[1][0], lo[1][1]};
      *(u32x4*)(smem + (put ^ (uint32_t)(s << 6) ^ ATT_VROW)) = u32x4{hi[0][0], hi[0][1], hi[1][0], hi[1][1]};
    }
  };
  auto barrier = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((15 << 0) | (3 << 14) | (7 << 4) | (0 << 8));  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  uint32_t ko = jq * 256 + ((g ^ jq) << 4), vo = jq * ATT_VROW + ((g ^ att_vswz(jq)) << 4);
  int slot = 0;  // byte offset of the slot computed on
  AttState st;
  st.reset();
  int i0 = 0, i1 = tiles.n;
  if (SPLIT) win_share(tiles.n, sp, a.nsplit, i0, i1);
  // Tile idx is in LDS, the next one's bytes are under way, and the table's entry of the one after it.  Tiles without a page
  // are passed over.
  Raw raw;
  int idx = i0, entry = 0, in1 = 0;  // in1: of the next one, the block in its page
  bool there = false;
  C4Walk walk = {};                  // the one whose entry is under way
  if (idx < i1) {
    walk.set(ca, tiles, idx);
    fetch(c4_of_entry<D>(ca, walk.entry(ca, b), h, walk.in, there), raw);
    walk.step(ca, tiles, i1);
    entry = walk.entry(ca, b);
    in1 = walk.in;
    spread(raw, tiles.key<BKV>(idx), idx < tiles.edge);
  }
  put ^= SLOT;
  barrier();
  // edge tiles in a loop of their own: with both kinds in one the accumulators are copied tile by tile (250 registers, 1.3
  // times as slow)
  auto step = [&](auto edge) {
    bool next_there;
    fetch(c4_of_entry<D>(ca, entry, h, in1, next_there), raw);  // (past the share: this tile again)
    const int key1 = walk.t * BKV;
    walk.step(ca, tiles, i1);
    entry = walk.entry(ca, b);
    in1 = walk.in;
    if constexpr (decltype(edge)::value) {
      const int key0 = tiles.key<BKV>(idx);
      if (live && there && key0 <= whi && (key0 + BKV > wlo || key0 < tiles.sink)) {
        mask.key0 = key0;
        att_tile_masked<WinMask<ATT_QB>, QLOG2, 4, true, false>(smem, qf, ko, vo, st, mask, a.scale_log2);
        // rows that see a key whose V holds no number in a group of channels have none there
        u32x4 bad[4];
        uint32_t any = 0;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          bad[m] = *(const u32x4*)(smem + 2 * SLOT + (slot ? 256 : 0) + (m * 4 + g) * 16);
          any |= bad[m][0] | bad[m][1] | bad[m][2] | bad[m][3];
        }
        if (__ballot(any != 0)) {
          WinMask<ATT_QB> mk = mask;
          mk.begin();
#pragma unroll
          for (int i = 0; i < ATT_QB; ++i) {
            uint32_t lost = 0;
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
              for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                  lost |= ((bad[m][w] >> (8 * x)) & ~(mk.bits[i] >> (4 * w + x)) & 1u) << m;
            lost |= (uint32_t)__shfl_xor((int)lost, 16);
            lost |= (uint32_t)__shfl_xor((int)lost, 32);
#pragma unroll
            for (int f = 0; f < D / 16; ++f) {
              const float add = lost >> (f >> 1) & 1 ? NAN : 0.0f;  // (onto the sums in place)
#pragma unroll
              for (int r = 0; r < 4; ++r) st.o[f][i][r] += add;
            }
          }
        }
      }
    } else {
      if (live && there) att_tile_masked<AttAll, QLOG2, 4, true, false>(smem, qf, ko, vo, st, AttAll{}, a.scale_log2);
    }
    spread(raw, key1, idx + 1 < tiles.edge);
    ko ^= SLOT;
    vo ^= SLOT;
    slot ^= SLOT;
    put ^= SLOT;
    ++idx;
    there = next_there;
    barrier();
  };
  const int ie = min(i1, tiles.edge);
  while (idx < ie) step(std::true_type{});
  while (idx < i1) step(std::false_type{});

  // lane: query jq of each block, channels 32 p + 8 g .. + 7
#pragma unroll
  for (int i = 0; i < ATT_QB; ++i) {
    const int r = wr0 + 16 * i + jq;
    const float m = att_of_block(st.ms, i, lane), l = st.lsum[i][0];
    if (r >= rows) continue;
    if constexpr (SPLIT) {
      const int64_t pr = ((((int64_t)sp * a.B + b) * a.Hk + h) * a.Lq) * a.n + r;
      float* o = a.po + pr * D + 8 * g;
#pragma unroll
      for (int p = 0; p < D / 32; ++p) {
        *(f32x4*)(o + 32 * p) = st.o[2 * p][i];
        *(f32x4*)(o + 32 * p + 4) = st.o[2 * p + 1][i];
      }
      if (g == 0) a.pml[pr] = float2{m, l};
    } else {
      int e;
      const int qi = win_query(a, r, e), head = h * a.n + e;
      const float inv = win_inverse(l);
      bf16_t* o = (bf16_t*)a.out + b * a.so + (int64_t)qi * a.ldo + (int64_t)head * D + 8 * g;
#pragma unroll
      for (int p = 0; p < D / 32; ++p) {
        const f32x4 &x = st.o[2 * p][i], &y = st.o[2 * p + 1][i];
        *(u32x4*)(o + 32 * p) = u32x4{pack_bf2(x[0] * inv, x[1] * inv), pack_bf2(x[2] * inv, x[3] * inv),
                                      pack_bf2(y[0] * inv, y[1] * inv), pack_bf2(y[2] * inv, y[3] * inv)};
      }
      if (a.lse && g == 0) a.lse[((int64_t)b * a.Hk * a.n + head) * a.Lq + qi] = win_lse(m, l);
    }
  }
}

// ---------------------------------------------------------------- float32
// 16 rows a workgroup; a tile of 64 keys is turned into float32 in LDS (rows of K, rows of V^T, 16-byte units at unit ^ (row &
// 7)), each of the four waves takes 16 of its keys, and the next two tiles' bytes are under way meanwhile. What bounds it: a
// tile's conversion, two barriers, products and softmax in turn, with as many workgroups a CU as the registers allow (five at 32
// channels, four at 64, two at 128): 2 x 8 heads of 64, 301 queries on 1801 keys 38.0 us and the join 4.3, a call among others
// 38.4, 43 TFLOP/s (47 with one tile ahead); 12 heads of 64, 1500 on 4000 keys 74 TFLOP/s, of 128, 2000 on 6000 69, 16 of 32,
// 1800 on 1800 63.  Single tokens take the same form with most of its 16 rows empty: 8 heads of 128, 8000 keys 21 us, 8 x 40 heads
// over 8, 32760 keys 248 (1.2 TB/s).
template <int D, bool VEC, bool SPLIT>
__global__ __launch_bounds__(256, D == 128 ? 2 : 3) void cache_f32_kernel(WinArgs a, CacheArgs ca) {
  constexpr int C = D / 16, TK = C4_BLOCK, W = 4, ROWS = 16;
  constexpr int HALF = TK * D * 4, NW = D / 32;  // words of codes a thread brings, of K and of V
  constexpr int SO = W * C * 1024, LDS = 2 * HALF > SO + W * 128 ? 2 * HALF : SO + W * 128;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[LDS];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int jq = lane & 15, g = lane >> 4;
  int rb, sp, h, b;
  win_place<true>(a, rb, sp, h, b);
  const WinSeq seq = win_seq(a, b);
  const int rows = seq.qlen * a.n;
  const int r0 = rb * ROWS;
  if (r0 >= rows) return;  // the whole workgroup
  int lo0, hi0, lo1, hi1;
  win_range(a, seq, (int)a.by_n((uint32_t)r0), lo0, hi0);
  win_range(a, seq, (int)a.by_n((uint32_t)min(r0 + ROWS - 1, rows - 1)), lo1, hi1);
  lo0 = __builtin_amdgcn_readfirstlane(lo0), hi0 = __builtin_amdgcn_readfirstlane(hi0);
  lo1 = __builtin_amdgcn_readfirstlane(lo1), hi1 = __builtin_amdgcn_readfirstlane(hi1);
  WinTiles tiles;
  tiles.init<TK>(seq, lo0, hi0, lo1, hi1);
  int i0 = 0, i1 = tiles.n;
  if (SPLIT) win_share(tiles.n, sp, a.nsplit, i0, i1);
  int wlo = lo0;
  if (tiles.sink == 0 && seq.sink >= lo1) wlo = 0;
  const int mine = 16 * wave;

  typedef C4F32<D> At;
  const int kt = tid >> 2, kc = At::k_channel(tid), vc = At::v_channel(tid);
  struct Raw {
    uint32_t k[NW], v[NW], e[NW], ke;
  };
  auto fetch = [&](const uint8_t* p, Raw& r) {
    const uint32_t* kp = (const uint32_t*)(p + At::k_codes(tid));
    const uint32_t* vp = (const uint32_t*)(p + At::v_codes(tid));
    const uint32_t* ep = (const uint32_t*)(p + At::v_exp(tid));
#pragma unroll
    for (int i = 0; i < NW; ++i) r.k[i] = kp[i], r.v[i] = vp[i], r.e[i] = ep[i];
    r.ke = p[At::k_exp(tid)];
  };
  auto spread = [&](const Raw& r) {
    const float s = __uint_as_float(r.ke << 23);
    uint8_t* const kto = smem + kt * (D * 4);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const int unit = kc / 4 + 2 * i;
      const f32x2 x0 = c4_pair_f32<0>(r.k[i], s), x1 = c4_pair_f32<1>(r.k[i], s), x2 = c4_pair_f32<2>(r.k[i], s), x3 = c4_pair_f32<3>(r.k[i], s);
      *(f32x4*)(kto + ((unit ^ (kt & 7)) << 4)) = f32x4{x0[0], x0[1], x1[0], x1[1]};
      *(f32x4*)(kto + (((unit + 1) ^ (kt & 7)) << 4)) = f32x4{x2[0], x2[1], x3[0], x3[1]};
    }
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const int unit = At::v_key(tid, i) >> 2;
      const f32x2 x0 = c4_pair_f32<0>(r.v[i], c4_scale<0>(r.e[i])), x1 = c4_pair_f32<1>(r.v[i], c4_scale<1>(r.e[i]));
      const f32x2 x2 = c4_pair_f32<2>(r.v[i], c4_scale<2>(r.e[i])), x3 = c4_pair_f32<3>(r.v[i], c4_scale<3>(r.e[i]));
#pragma unroll
      for (int y = 0; y < 2; ++y)
        *(f32x4*)(smem + HALF + (vc + y) * (TK * 4) + ((unit ^ ((vc + y) & 7)) << 4)) = f32x4{x0[y], x1[y], x2[y], x3[y]};
    }
  };
  // (a barrier that leaves the loads under way)
  auto lds_barrier = [&]() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((15 << 0) | (3 << 14) | (7 << 4) | (0 << 8));  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  WinF32<D, false, true> st;
  st.template begin<VEC>(a, seq, tiles, lo1, h, r0 + jq, rows);
  // two tiles' bytes are under way, and the table's entry of the one after them; tiles without a page are passed over
  Raw raw, raw1;
  bool there = false, there1 = false;
  C4Walk walk = {};
  int entry = 0;
  auto next = [&](Raw& r, bool& got) {
    fetch(c4_of_entry<D>(ca, entry, h, walk.in, got), r);
    walk.step(ca, tiles, i1);
    entry = walk.entry(ca, b);
  };
  if (i0 < i1) {
    walk.set(ca, tiles, i0);
    entry = walk.entry(ca, b);
    next(raw, there);
    next(raw1, there1);
  }
  auto tile = [&](int idx, Raw& r, bool& got) {
    const bool now = got;
    spread(r);
    next(r, got);
    lds_barrier();
    const int key0 = tiles.key<TK>(idx), k0 = key0 + mine;
    const bool edge = idx < tiles.edge;
    if (now && (!edge || (k0 <= hi1 && (k0 + 16 > wlo || k0 < tiles.sink)))) {
      const uint8_t* const kb = smem + (mine + jq) * (D * 4);
      const uint8_t* const vb = smem + HALF + jq * (TK * 4) + ((((mine >> 2) + g) ^ (jq & 7)) << 4);
      st.step([&](int c) { return *(const f32x4*)(kb + (((4 * c + g) ^ (jq & 7)) << 4)); },
              [&](int c) { return *(const f32x4*)(vb + 16 * c * (TK * 4)); }, edge, k0, seq.klen, a.scale_log2);
    }
    lds_barrier();
  };
  for (int idx = i0; idx < i1; idx += 2) {
    tile(idx, raw, there);
    if (idx + 1 < i1) tile(idx + 1, raw1, there1);
  }
  __syncthreads();
  st.template end<VEC, SPLIT>(a, b, h, sp, r0 + jq, rows, (f32x4*)smem, (float*)(smem + SO));
}

// ---------------------------------------------------------------- host
int64_t cache4_page_bytes(int heads, int head_dim, int page_tokens) {
  if (heads < 1 || heads > C4_HEADS || (head_dim != 32 && head_dim != 64 && head_dim != 128) || page_tokens < C4_BLOCK ||
      page_tokens > 65536 || page_tokens % C4_BLOCK)
    return 0;
  return (int64_t)(page_tokens / C4_BLOCK) * heads * 68 * head_dim;
}

// empty: a call that does nothing, perhaps of no sequences, whose table has no address.
static track_status cache_check(const char* what, const track_cache4* c, bool empty, CacheArgs* a) {
  if (!c) return fail(TRACK_E_INVALID, "%s: null cache", what);
  if (!cache4_page_bytes(c->heads, c->head_dim, c->page_tokens))
    return fail(TRACK_E_UNSUPPORTED, "%s: pages of %d tokens (multiples of 64 up to 65536), %d heads of %d channels (32, 64, 128)", what,
                c->page_tokens, c->heads, c->head_dim);
  if (c->n_pages < 1 || c->n_pages > INT32_MAX || c->table_pages < 0 || c->table_pages > WIN_MAX / c->page_tokens ||
      c->ld_table < 0)
    return fail(TRACK_E_SHAPE, "%s: %lld pages, %d of a sequence (2^28 tokens at most), %lld between sequences", what, (long long)c->n_pages,
                c->table_pages, (long long)c->ld_table);
  if (!c->pages || (c->table_pages && !c->table && !empty)) return fail(TRACK_E_INVALID, "%s: null pointer in the cache", what);
  if (((uintptr_t)c->pages & 127) || ((uintptr_t)c->table & 3))
    return fail(TRACK_E_INVALID, "%s: pages need 128-byte alignment, the table 4", what);
  a->pages = (uint8_t*)c->pages;
  a->table = c->table;
  a->ld_table = c->ld_table;
  a->blocks = c->page_tokens / C4_BLOCK;
  a->stride = (int64_t)c->heads * 68 * c->head_dim;
  a->table_pages = c->table_pages;
  a->n_pages = (int)c->n_pages;
  a->cap = c->table_pages * c->page_tokens;
  a->by_blocks = win_div(a->blocks);
  return TRACK_OK;
}

// Workgroups that share 16 tokens' heads, four a turn: one while the tokens alone fill the chip twice.
static int rows_heads(int64_t items, int heads) {
  return (int)std::max<int64_t>(1, std::min<int64_t>((heads + 3) / 4, (2 * (int64_t)device_cus() + items - 1) / items));
}

template <typename T, int D>
static void append_launch(const RowsArgs& a, int rot, unsigned grid, hipStream_t s) {
  if (rot == 0) cache_append_kernel<T, D, 0><<<grid, 256, 0, s>>>(a);
  else if (rot == 1) cache_append_kernel<T, D, 1><<<grid, 256, 0, s>>>(a);
  else cache_append_kernel<T, D, 2><<<grid, 256, 0, s>>>(a);
}

static track_status cache_rows(const char* what, bool read, int dtype, const track_cache4* cache, const track_rope_config* rope,
                               int64_t B, int64_t L, void* k, int64_t ldk, int64_t sk, void* v, int64_t ldv, int64_t sv,
                               const int32_t* start, const int32_t* n, const int32_t* pos, const double* freqs, float amplitude,
                               hipStream_t s) {
  if (dtype != TRACK_DTYPE_F32 && dtype != TRACK_DTYPE_BF16) return fail(TRACK_E_INVALID, "%s: bad dtype %d", what, dtype);
  RowsArgs a = {};
  const track_status st = cache_check(what, cache, B == 0 || L == 0, &a.c);
  if (st != TRACK_OK) return st;
  const int D = cache->head_dim;
  const int64_t width = (int64_t)cache->heads * D;
  if (B < 0 || L < 0 || L > WIN_MAX) return fail(TRACK_E_SHAPE, "%s: %lld x %lld tokens", what, (long long)B, (long long)L);
  if (rope && rope->head_dim != D) return fail(TRACK_E_SHAPE, "%s: rotation of %d channels, %d in the cache", what, rope->head_dim, D);
  if (ldk < width || ldv < width || sk < 0 || sv < 0)
    return fail(TRACK_E_SHAPE, "%s: rows of %lld and %lld elements for %d heads of %d", what, (long long)ldk, (long long)ldv, cache->heads, D);
  if (read && (sequences_overlap(B, L, ldk, sk, width) || sequences_overlap(B, L, ldv, sv, width)))
    return fail(TRACK_E_SHAPE, "%s: sequences overlap in the output", what);
  if (B == 0 || L == 0) return TRACK_OK;
  const uintptr_t es = dtype == TRACK_DTYPE_BF16 ? 2 : 4;
  if (!k || !v || !start || (rope && (!pos || !freqs))) return fail(TRACK_E_INVALID, "%s: null pointer", what);
  if (((uintptr_t)k | (uintptr_t)v) & (es - 1) || ((uintptr_t)start | (uintptr_t)n | (uintptr_t)pos) & 3 || (uintptr_t)freqs & 7)
    return fail(TRACK_E_INVALID, "%s: rows, lengths, positions or frequencies are not aligned to their elements", what);
  if (!std::isfinite(amplitude)) return fail(TRACK_E_INVALID, "%s: scale is not finite", what);
  a.k = k, a.v = v, a.ldk = ldk, a.sk = sk, a.ldv = ldv, a.sv = sv;
  a.start = start, a.n = n;
  a.B = (int)B, a.L = (int)L, a.heads = cache->heads;
  a.nblk = (int)((L + C4_BLOCK - 2) / C4_BLOCK + 1);
  a.vec = !((((uintptr_t)k | (uintptr_t)v) & 15) || ((ldk | ldv | (B > 1 ? sk | sv : 0)) * (int64_t)es & 15));
  if (B > INT32_MAX || B * a.nblk >= (int64_t)1 << 22) return fail(TRACK_E_SHAPE, "%s: %lld x %lld tokens are too many", what, (long long)B, (long long)L);
  a.hsplit = rows_heads(4 * B * a.nblk, a.heads);
  int rot = 0;
  if (rope) {
    rot = rope->layout == TRACK_ROPE_HALF ? 2 : 1;
    a.pos = pos, a.freqs = freqs, a.amp = amplitude;
    a.pairs = rope->rot_dim / 2;
    a.sec0 = rope->axes > 1 ? rope->section[0] : a.pairs;
    a.sec1 = rope->axes > 2 ? rope->section[0] + rope->section[1] : a.pairs;
  }
  ProfScope prof(TRACK_PROF_OTHER, s);
  const unsigned grid = (unsigned)(4 * B * a.nblk * a.hsplit);
#define TRACK_C4_ROWS(T, DH)                                              \
  do {                                                                    \
    if (read) cache_read_kernel<T, DH><<<grid, 256, 0, s>>>(a);           \
    else append_launch<T, DH>(a, rot, grid, s);                           \
  } while (0)
  if (es == 2) {
    if (D == 32) TRACK_C4_ROWS(bf16_t, 32);
    else if (D == 64) TRACK_C4_ROWS(bf16_t, 64);
    else TRACK_C4_ROWS(bf16_t, 128);
  } else {
    if (D == 32) TRACK_C4_ROWS(float, 32);
    else if (D == 64) TRACK_C4_ROWS(float, 64);
    else TRACK_C4_ROWS(float, 128);
  }
#undef TRACK_C4_ROWS
  TRACK_LAUNCH_CHECK();
  return TRACK_OK;
}

track_status cache4_append(int dtype, const track_cache4* cache, const track_rope_config* rope, int64_t B, int64_t L, const void* k,
                           int64_t ldk, int64_t sk, const void* v, int64_t ldv, int64_t sv, const int32_t* start, const int32_t* n,
                           const int32_t* pos, const double* freqs, float amplitude, hipStream_t s) {
  return cache_rows("cache4_append", false, dtype, cache, rope, B, L, (void*)k, ldk, sk, (void*)v, ldv, sv, start, n, pos, freqs,
                    amplitude, s);
}

track_status cache4_read(int dtype, const track_cache4* cache, int64_t B, int64_t L, void* k, int64_t ldk, int64_t sk, void* v,
                         int64_t ldv, int64_t sv, const int32_t* start, const int32_t* n, hipStream_t s) {
  return cache_rows("cache4_read", true, dtype, cache, nullptr, B, L, k, ldk, sk, v, ldv, sv, start, n, nullptr, nullptr, 1.0f, s);
}

// How a call is taken: at most 16 rows a key head, blocks of 256, or 16 float32 rows a workgroup; shares of the keys.
struct CachePlan {
  enum Form { BLOCKS, ROWS, F32 } form;
  int64_t nrb;
  int nsplit;
};

// Shares of the keys for few rows.  None up to 12 tiles, three a wave: the join is a launch more (32 heads of 960 keys 10.6 us
// with one, 8.9 with 4, of 576 8.7 and 8.7, 128 of 576 9.7 and 10.8).  Then as many as make the three workgroups a CU that are
// resident, of four tiles or fewer, and twice as many for what takes some 100 us, which evens
// out lengths. Join included, replayed on three caches in turn: 64 key heads of 100003 to 56000 keys 124 us with 8, 122 with
// 12, 126 with 16, 118 with 24, 117 with 32, 127 with 64; 48 of 32760 51 with 8, 44 with 16, 48 with 24, 45 with 32; 8 of
// 100003 36 with 32, 29 with 64 and 96; 64 of 16384 32 with 8, 34 with 12, 37 with 24; 512 of 2000 29 with one, 35 with 2; 8
// of 16384 17 with 16, 14 with 32, 13 with 64.
static int64_t cache_rows_split(int64_t tiles, int64_t blocks, int64_t cus) {
  if (tiles <= 12) return 1;
  return std::min((blocks * tiles >= 192 * cus ? 6 : 3) * cus / blocks, (tiles + 3) / 4);
}

// Shares for float32 rows: as many workgroups as the registers allow at once (four a CU at 64 channels, two at 128; at 32, where
// they allow five, four too); and where the row blocks do not fill the last of their rounds, what fills it better by a tenth, of
// eight tiles at least (12 heads of 128, 1000 causal rows on 2000 keys, 756 blocks over 512 places: 199 us with one share, 153
// with two).  Grows with the tiles.
static int64_t cache_f32_split(int64_t tiles, int64_t blocks, int D, int64_t cus) {
  const int64_t places = (D == 128 ? 2 : 4) * cus;
  auto waste = [&](int64_t s) {  // rounds over those that full ones would take, and the join
    return (double)((blocks * s + places - 1) / places * places) / (double)(blocks * s) * (1.0 + 0.03 * (double)(s - 1));
  };
  const int64_t base = std::max<int64_t>(1, places / blocks);
  int64_t best = base;
  for (int64_t s = base + 1; s <= std::min<int64_t>(8, tiles / 8); ++s)
    if (waste(s) < waste(best)) best = s;
  return waste(best) < 0.9 * waste(base) ? best : std::min(base, tiles / 4);
}

static CachePlan cache_plan(int dtype, const track_window& w, int64_t B, int Hk, int n, int D, int64_t Lq, int64_t Lk) {
  const int64_t rows = Lq * n, cus = device_cus();
  CachePlan p;
  p.form = dtype == TRACK_DTYPE_F32 ? CachePlan::F32 : (rows <= 16 ? CachePlan::ROWS : CachePlan::BLOCKS);
  const int64_t block = p.form == CachePlan::BLOCKS ? ATT_BQ : 16;
  p.nrb = (rows + block - 1) / block;
  const int64_t tiles = (win_span(w, std::min(rows, block), n, Lk) + C4_BLOCK - 1) / C4_BLOCK;
  const int64_t blocks = p.nrb * Hk * B;
  int64_t s;
  if (p.form == CachePlan::ROWS) s = cache_rows_split(tiles, blocks, cus);
  else if (p.form == CachePlan::F32) s = cache_f32_split(tiles, blocks, D, cus);
  else s = win_blocks_split(tiles, blocks, rows * Hk * B, cus);
  p.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>(s, 1024));
  return p;
}

static size_t cache_plan_bytes(const CachePlan& p, int64_t B, int Hk, int n, int D, int64_t Lq) {
  return p.nsplit == 1 ? 0 : (size_t)(p.nsplit * B * Hk * Lq * n) * (size_t)(4 * D + 8);
}

static bool cache_fits(const CachePlan& p, int64_t B, int Hk, int n, int64_t Lq) {
  return p.nrb * p.nsplit * Hk * B < (int64_t)1 << 23 && (p.nsplit == 1 || B * Hk * n * Lq < (int64_t)1 << 25);
}

int64_t attention_cache4_bytes(int dtype, const track_window* w, int B, int H, int Hk, int D, int64_t Lq, int64_t Lk) {
  if (win_check("attention_cache4", dtype, w, B, H, Hk, D, Lq, Lk) != TRACK_OK) return -1;
  if (B == 0 || Lq == 0) return 0;
  const CachePlan p = cache_plan(dtype, *w, B, Hk, H / Hk, D, Lq, Lk);
  if (!cache_fits(p, B, Hk, H / Hk, Lq)) {
    fail(TRACK_E_SHAPE, "attention_cache4: too many row blocks");
    return -1;
  }
  return (int64_t)cache_plan_bytes(p, B, Hk, H / Hk, D, Lq);
}

track_status attention_cache4(int dtype, const track_window* w, const track_cache4* cache, int B, int H, int64_t Lq, int64_t Lk,
                              const void* q, int64_t ldq, int64_t sq, void* out, int64_t ldo, int64_t so, float* lse,
                              const int32_t* q_len, const int32_t* k_len, const int32_t* q_start, void* ws, size_t ws_bytes,
                              hipStream_t s) {
  CacheArgs ca = {};
  track_status st = cache_check("attention_cache4", cache, B == 0 || Lq == 0, &ca);
  if (st != TRACK_OK) return st;
  const int Hk = cache->heads, D = cache->head_dim;
  st = win_check("attention_cache4", dtype, w, B, H, Hk, D, Lq, Lk);
  if (st != TRACK_OK) return st;
  if (Lk > ca.cap) return fail(TRACK_E_SHAPE, "attention_cache4: %lld keys, the table has places for %d", (long long)Lk, ca.cap);
  if (B == 0 || Lq == 0) return TRACK_OK;
  if (!q || !out) return fail(TRACK_E_INVALID, "attention_cache4: null pointer");
  const int n = H / Hk;
  if (ldq < (int64_t)H * D || ldo < (int64_t)H * D) return fail(TRACK_E_SHAPE, "attention_cache4: leading dimension too small");
  if (sq < 0 || so < 0 || sequences_overlap(B, Lq, ldo, so, (int64_t)H * D))
    return fail(TRACK_E_SHAPE, "attention_cache4: sequences overlap in out, or a negative stride");
  if (((uintptr_t)lse | (uintptr_t)q_len | (uintptr_t)k_len | (uintptr_t)q_start) & 3)
    return fail(TRACK_E_INVALID, "attention_cache4: lse and lengths need 4-byte alignment");
  const uintptr_t ptrs = (uintptr_t)q | (uintptr_t)out;
  const int64_t strides = ldq | ldo | (B > 1 ? sq | so : 0);
  const bool vec = !(ptrs & 15) && !(strides & (dtype == TRACK_DTYPE_BF16 ? 7 : 3));
  if (dtype == TRACK_DTYPE_BF16 && !vec) return fail(TRACK_E_INVALID, "attention_cache4: bf16 path needs 16-byte aligned rows");
  if (ptrs & 3) return fail(TRACK_E_INVALID, "attention_cache4: float32 path needs 4-byte aligned rows");
  CachePlan p = cache_plan(dtype, *w, B, Hk, n, D, Lq, Lk);
  if (!cache_fits(p, B, Hk, n, Lq)) return fail(TRACK_E_SHAPE, "attention_cache4: too many row blocks");
  if (p.form == CachePlan::BLOCKS) p.nsplit = win_held(p.nsplit, B, Hk, n, D, Lq, ws, ws_bytes);
  const size_t need = cache_plan_bytes(p, B, Hk, n, D, Lq);
  if (need && (!ws || ws_bytes < need)) return fail(TRACK_E_NOMEM, "attention_cache4: workspace of %zu bytes needed", need);
  if (need && ((uintptr_t)ws & 255)) return fail(TRACK_E_INVALID, "attention_cache4: workspace must be 256-byte aligned");
  const int64_t joined = (int64_t)B * H * Lq;
  WinArgs a = {};
  a.q = q, a.out = out, a.ldq = ldq, a.sq = sq, a.ldo = ldo, a.so = so;
  a.lse = lse, a.q_len = q_len, a.k_len = k_len, a.q_start = q_start;
  win_visible(a, *w, B, Hk, n, D, Lq, Lk);
  a.nrb = (int)p.nrb, a.nsplit = p.nsplit;
  a.by_nrb = win_div(a.nrb), a.by_nsplit = win_div(a.nsplit);
  a.by_inner = win_div(p.form == CachePlan::ROWS ? Hk : B);
  a.po = (float*)ws;
  a.pml = need ? (float2*)(a.po + (int64_t)p.nsplit * joined * D) : nullptr;
  const bool split = p.nsplit > 1, log2q = a.scale_log2 == 1.0f;
  ProfScope prof(TRACK_PROF_ATTN_SELF, s);
  const unsigned gr = (unsigned)(p.nrb * p.nsplit * Hk * B);
#define TRACK_C4_F32(DH)                                                            \
  do {                                                                              \
    if (vec && split) cache_f32_kernel<DH, true, true><<<gr, 256, 0, s>>>(a, ca);   \
    else if (vec) cache_f32_kernel<DH, true, false><<<gr, 256, 0, s>>>(a, ca);      \
    else if (split) cache_f32_kernel<DH, false, true><<<gr, 256, 0, s>>>(a, ca);    \
    else cache_f32_kernel<DH, false, false><<<gr, 256, 0, s>>>(a, ca);              \
  } while (0)
  switch (p.form) {
    case CachePlan::ROWS:
      if (split) cache_rows_kernel<true><<<gr, 256, 0, s>>>(a, ca);
      else cache_rows_kernel<false><<<gr, 256, 0, s>>>(a, ca);
      break;
    case CachePlan::BLOCKS:
      if (log2q && split) cache_blocks_kernel<true, true><<<gr, 512, 0, s>>>(a, ca);
      else if (log2q) cache_blocks_kernel<true, false><<<gr, 512, 0, s>>>(a, ca);
      else if (split) cache_blocks_kernel<false, true><<<gr, 512, 0, s>>>(a, ca);
      else cache_blocks_kernel<false, false><<<gr, 512, 0, s>>>(a, ca);
      break;
    default:
      if (D == 32) TRACK_C4_F32(32);
      else if (D == 64) TRACK_C4_F32(64);
      else TRACK_C4_F32(128);
  }
#undef TRACK_C4_F32
  TRACK_LAUNCH_CHECK();
  if (split) {
    window_join(dtype, a, D, s);
    TRACK_LAUNCH_CHECK();
  }
  return TRACK_OK;
}

}  // namespace track
