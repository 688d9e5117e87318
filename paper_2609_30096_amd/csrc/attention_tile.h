// The 64-key tile of the bfloat16 attention kernels: LDS layout, copies' row order, online
// softmax and both products for one wave's 32 queries.
#pragma once

#include <math.h>

#include <type_traits>

#include "common.h"
#include "tile_copy.h"

namespace track {

constexpr int ATT_D = 128;
// log2 headroom before the reference max is moved (lazy rescale): probabilities
// stay below 2^64, which bf16 P and the float32 sums of up to 2^31 keys carry
constexpr float ATT_TAU = 64.0f;
constexpr float ATT_MLO = -64.0f;  // below this row max the reference leaves 0

// Maxima over the four 16-lane groups (lanes l, l + 16, l + 32, l + 48) of a and
// of b: lanes 0..31 return that of a, lanes 32..63 that of b.
__device__ __forceinline__ float group_max2(float a, float b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  const float x = __uint_as_float(r[0]), y = __uint_as_float(r[1]);
  const float m = fmaxf(x, y);
  const auto t = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
  const float u = __uint_as_float(t[0]), v = __uint_as_float(t[1]);
  return fmaxf(u, v);
}

// K and V^T tiles travel from global memory straight into LDS
// (buffer_load ... lds, 16 bytes per lane) through a ring of two slots, with
// no register staging and no LDS store instructions.  Per tile the K source
// is a buffer resource starting at the tile's first key, so keys past Lk read
// as zero; V^T columns are addressed through the vector offset (row and
// column together), so the resource's range check covers every V^T read.
// A DMA copy lands lane-contiguously, so every layout choice is made on the
// source side: each lane picks the 16-byte chunk that belongs at its LDS
// position.  The XOR swizzles keep the 16-row fragment reads conflict free:
// K rows are 256 bytes (unit u of row r at u ^ (r & 15)); V^T rows are 128
// bytes (unit u at u ^ att_vswz(r)).  Each lane's fragment offsets are computed
// once and switch slots with an XOR.  Rows are permuted within every 32: LDS row
// 16 h + 4 q + j holds key (or channel) 8 q + 4 h + j.  A lane's logits of a pair of
// 16-key blocks are
// then 8 consecutive keys, the P operand's k-block, which meets one contiguous
// 16-byte V^T chunk, and its outputs of a pair of 16-channel blocks are 8
// consecutive channels, one 16-byte store (att_perm and att_vswz: tile_copy.h).
typedef __attribute__((address_space(3))) void* att_lds_ptr_t;

// The lane index, computed where it is used (opaque to the compiler, which would
// otherwise keep values derived from it live across long loops).
__device__ __forceinline__ int att_lane() {
  int ln;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(ln));
  return ln;
}

template <int N>
__device__ __forceinline__ void att_wait_vmcnt() {
  // s_waitcnt vmcnt(N) (gfx9 encoding), expcnt and lgkmcnt not waited on
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

constexpr int ATT_NW = 8, ATT_BKV = 64;
constexpr int ATT_BQ = 32 * ATT_NW;                 // queries per workgroup
constexpr int ATT_K_BYTES = ATT_BKV * ATT_D * 2;    // K tile, 16 KB
constexpr int ATT_VROW = ATT_BKV * 2;               // V^T tile row, 128 bytes
constexpr int ATT_V_BYTES = ATT_D * ATT_VROW;       // V^T tile, 16 KB
constexpr int ATT_SLOT = ATT_K_BYTES + ATT_V_BYTES;  // one ring slot, 32 KB
// key sequences of at most this many 64-key tiles (an even number) take the item-loop kernel
constexpr int ATT_ITEMS_MAX_TILES = 32;

constexpr int ATT_LA = 3;  // fragments read ahead of their MFMAs
constexpr int ATT_QB = 2;  // 16-query blocks per wave

// What a lane keeps of its wave's 32 queries (lane l holds query 16 b + l % 16 of
// block b) across the tiles.
struct AttState {
  f32x4 o[ATT_D / 16][ATT_QB];  // O^T: channels att_perm of 16 f + 4 (l / 16) + 0..3, of query block b
  f32x4 lsum[ATT_QB];           // row sums (every element the sum of the lane's query)
  float ms;                     // reference max: block 0's in lanes 0..31, block 1's in lanes 32..63
  bool zref;                    // every row of the wave has reference 0
  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int b = 0; b < ATT_QB; ++b) {
#pragma unroll
      for (int f = 0; f < ATT_D / 16; ++f) o[f][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      lsum[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    ms = -INFINITY;
    zref = false;
  }
};

// The value of the lane's query of block b, of one kept as ms is.
__device__ __forceinline__ float att_of_block(float v, int b, int lane) {
  const int src = (32 * b + (lane & 15)) << 2;
  return __int_as_float(__builtin_amdgcn_ds_bpermute(src, __float_as_int(v)));
}

// What a tile leaves out.  hidden(b, c): whether the lane's query of block b does not see the
// lane's key c (after begin()), c = 0..3, 4..7, 32..35, 36..39 counted from 8 (lane / 16) on in
// the tile; BITS masks have apply(b, c, s) instead, the logit s or -inf.
// WEIGHED: keys of weight zero are left out of O one by one, so that what their V holds
// (an infinity, a NaN) stays out of it; a matrix product would make 0 x inf of it.
struct AttAll {
  static constexpr bool ACTIVE = false, BITS = false, WEIGHED = false;
  __device__ __forceinline__ void begin() {}
};
struct AttBelow {  // keys at or past the end
  static constexpr bool ACTIVE = true, BITS = false, WEIGHED = false;
  int Lk, key0;
  int lim;         // valid keys from this lane's first on
  __device__ __forceinline__ void begin() { lim = Lk - key0 - 8 * (att_lane() >> 4); }
  __device__ __forceinline__ bool hidden(int, int c) const { return c >= lim; }
};

// One 64-key tile for one wave's 32 queries: S^T = K Q^T from the slot's K
// tile, the online-softmax update (lazy rescale), and O^T += V^T P^T from the
// slot's V^T tile.  ko / vo are the lane's fragment offsets (depth step 0, key chunk
// 0; the others differ in one XOR); keys that the mask hides get
// probability zero.  The probabilities are rounded to bfloat16, the type that the matrix cores multiply at
// full rate (float32 runs at a thirteenth of it), and the row sums add the rounded ones: the weights
// that meet V then add up to one, and a V of equal rows comes out as it is.  KB 16-key blocks of the tile
// (2: the half that ko and vo point at).  With SAFE a row whose logits so far are all -inf (a wave of a split sequence can begin with
// such a tile) takes reference 0 instead.
// FIRST: the sequence's first tile, which starts O and the sums (no rescale, nothing to
// zero) and the references: 212.7 -> 207.3 us at 2 x 12 heads, 32760 x 512, 12 times a CU.
template <class Mask, bool QLOG2, int KB, bool SAFE, bool FIRST>
__device__ __forceinline__ void att_tile_masked(const uint8_t* kb, const bf16x8 (&qf)[ATT_D / 32][ATT_QB], uint32_t ko,
                                                uint32_t vo, AttState& st, Mask mask, float scale_log2) {
  constexpr int QB = ATT_QB;
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const uint8_t* vb = kb + ATT_K_BYTES;
  f32x4 s[KB][QB];
#pragma unroll
  for (int i = 0; i < KB; ++i)
#pragma unroll
    for (int b = 0; b < QB; ++b) s[i][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  // fragment j: 16-key block j % KB of depth step j / KB
  auto kfrag = [&](int j) {
    return __builtin_bit_cast(bf16x8, *(const u32x4*)(kb + (j % KB) * 4096 + (ko ^ (uint32_t)(j / KB * 64))));
  };
  constexpr int KF = ATT_D / 32 * KB;
  bf16x8 kf[ATT_LA + 1];
#pragma unroll
  for (int j = 0; j < ATT_LA; ++j) kf[j] = kfrag(j);
#pragma unroll
  for (int j = 0; j < KF; ++j) {
    if (j + ATT_LA < KF) kf[(j + ATT_LA) % (ATT_LA + 1)] = kfrag(j + ATT_LA);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < QB; ++b)
      s[j % KB][b] =
          __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[j % (ATT_LA + 1)], qf[j / KB][b], s[j % KB][b], 0, 0, 0);
  }
  float mx[QB];
#pragma unroll
  for (int b = 0; b < QB; ++b) mx[b] = -INFINITY;
  mask.begin();
#pragma unroll
  for (int i = 0; i < KB; ++i)
#pragma unroll
    for (int b = 0; b < QB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (Mask::ACTIVE) {
          if constexpr (Mask::BITS) s[i][b][r] = mask.apply(b, 32 * (i >> 1) + 4 * (i & 1) + r, s[i][b][r]);
          else if (mask.hidden(b, 32 * (i >> 1) + 4 * (i & 1) + r)) s[i][b][r] = -INFINITY;
        }
        mx[b] = fmaxf(mx[b], s[i][b][r]);
      }
  const float mt = QLOG2 ? group_max2(mx[0], mx[1]) : group_max2(mx[0], mx[1]) * scale_log2;
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (FIRST) {
    st.ms = mt >= ATT_MLO && mt <= ATT_TAU ? 0.0f : fmaxf(-INFINITY, mt);
    st.zref = !__ballot(st.ms != 0.0f);
  } else if (__ballot(mt > st.ms + ATT_TAU)) {
    float mn = fmaxf(st.ms, mt);
    if (mn >= ATT_MLO && mn <= ATT_TAU) mn = 0.0f;
    const float alpha = SAFE && mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.ms - mn);
    st.ms = mn;
    st.zref = !__ballot(mn != 0.0f);
    const int lane = att_lane();
#pragma unroll
    for (int b = 0; b < QB; ++b) {
      const float al = att_of_block(alpha, b, lane);
#pragma unroll
      for (int r = 0; r < 4; ++r) st.lsum[b][r] *= al;
#pragma unroll
      for (int f = 0; f < ATT_D / 16; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) st.o[f][b][r] *= al;
    }
  }
  // probabilities exp2(s c - m) (c = 1 with QLOG2); without the shift while every row
  // of the wave has reference 0, a wave-uniform branch
  bf16x8 pf[KB / 2][QB];
  auto probs = [&](auto shift_tag) {
    constexpr bool SHIFT = decltype(shift_tag)::value;
    float nm[QB];
    if constexpr (SHIFT) {
      const int lane = att_lane();
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        nm[b] = -att_of_block(st.ms, b, lane);
        if (SAFE && nm[b] == INFINITY) nm[b] = 0.0f;
      }
    }
#pragma unroll
    for (int c = 0; c < KB / 2; ++c)
#pragma unroll
      for (int b = 0; b < QB; ++b) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            x[k] = s[2 * c + (e >> 1)][b][2 * (e & 1) + k];
            if constexpr (SHIFT) x[k] = QLOG2 ? x[k] + nm[b] : fmaf(x[k], scale_log2, nm[b]);
            else if constexpr (!QLOG2) x[k] *= scale_log2;
          }
          const bf16x2 pb =
              __builtin_convertvector(f32x2{__builtin_amdgcn_exp2f(x[0]), __builtin_amdgcn_exp2f(x[1])}, bf16x2);
          w[e] = __builtin_bit_cast(uint32_t, pb);
        }
        pf[c][b] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
      }
  };
  if (st.zref) probs(std::false_type{});
  else probs(std::true_type{});
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  // fragment j: 16-channel block j / (KB / 2), key chunk j % (KB / 2)
  auto vfrag = [&](int j) {
    return __builtin_bit_cast(
        bf16x8, *(const u32x4*)(vb + j / (KB / 2) * 16 * ATT_VROW + (vo ^ (uint32_t)(j % (KB / 2) * 64))));
  };
  constexpr int VF = ATT_D / 16 * (KB / 2);
  bf16x8 vf[ATT_LA + 1];
#pragma unroll
  for (int j = 0; j < ATT_LA; ++j) vf[j] = vfrag(j);
#pragma unroll
  for (int c = 0; c < KB / 2; ++c)
#pragma unroll
    for (int b = 0; b < QB; ++b)
      st.lsum[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[c][b], FIRST && c == 0 ? zero : st.lsum[b], 0, 0, 0);
  if constexpr (Mask::WEIGHED) {
    static_assert(KB == 4 && !FIRST, "whole tiles");
    const uint8_t* const vt = vb + (vo & ATT_SLOT);
    const int lane = att_lane();
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll 1
      for (int k = 0; k < 32; ++k) {  // key 32 c + k
        float p[QB];
        uint32_t on[QB];  // V times 0 where the weight is 0
#pragma unroll
        for (int b = 0; b < QB; ++b) {
          const u32x4 own = __builtin_bit_cast(u32x4, pf[c][b]);
          const int e = (k >> 1) & 3;
          const uint32_t w = e == 0 ? own[0] : (e == 1 ? own[1] : (e == 2 ? own[2] : own[3]));
          const uint32_t got = __builtin_amdgcn_ds_bpermute(((lane & 15) + 16 * (k >> 3)) << 2, (int)w);
          p[b] = __uint_as_float(k & 1 ? got & 0xffff0000u : got << 16);
          on[b] = p[b] != 0.0f ? 0xffffffffu : 0u;
        }
#pragma unroll
        for (int f = 0; f < ATT_D / 16; ++f)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int row = 16 * f + 4 * (lane >> 4) + r;
            const uint32_t v =
                *(const bf16_t*)(vt + row * ATT_VROW + (((4 * c + (k >> 3)) ^ att_vswz(row)) << 4) + 2 * (k & 7));
#pragma unroll
            for (int b = 0; b < QB; ++b)
              st.o[f][b][r] = fmaf(p[b], __uint_as_float((v << 16) & on[b]), st.o[f][b][r]);
          }
      }
    return;
  }
#pragma unroll
  for (int j = 0; j < VF; ++j) {
    if (j + ATT_LA < VF) vf[(j + ATT_LA) % (ATT_LA + 1)] = vfrag(j + ATT_LA);
    __builtin_amdgcn_sched_barrier(0);
    const int f = j / (KB / 2), c = j % (KB / 2);
#pragma unroll
    for (int b = 0; b < QB; ++b)
      st.o[f][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j % (ATT_LA + 1)], pf[c][b],
                                                           FIRST && c == 0 ? zero : st.o[f][b], 0, 0, 0);
  }
}

// The same with the keys at or past Lk (MASK) left out.
template <bool MASK, bool QLOG2, int KB = ATT_BKV / 16, bool SAFE = false, bool FIRST = false>
__device__ __forceinline__ void att_tile(const uint8_t* kb, const bf16x8 (&qf)[ATT_D / 32][ATT_QB], uint32_t ko,
                                         uint32_t vo, AttState& st, int key0, int Lk, float scale_log2) {
  if constexpr (MASK)
    att_tile_masked<AttBelow, QLOG2, KB, SAFE, FIRST>(kb, qf, ko, vo, st, AttBelow{Lk, key0, 0}, scale_log2);
  else
    att_tile_masked<AttAll, QLOG2, KB, SAFE, FIRST>(kb, qf, ko, vo, st, AttAll{}, scale_log2);
}

// The wave's 32 rows from q0 on of one (batch, head): op points at row 0, channel 0.
__device__ __forceinline__ void att_store(const AttState& st, bf16_t* __restrict__ op, int64_t ldo, int q0, int Lq,
                                          int lane) {
  const bool wide = (((uintptr_t)op | (uintptr_t)(ldo * 2)) & 15) == 0;  // rows may be 8-byte aligned only
#pragma unroll
  for (int b = 0; b < ATT_QB; ++b) {
    const float inv = 1.0f / st.lsum[b][0];
    const int qi = q0 + 16 * b + (lane & 15);
    if (qi < Lq) {
      bf16_t* orow = op + (int64_t)qi * ldo + 8 * (lane >> 4);
#pragma unroll
      for (int p = 0; p < ATT_D / 32; ++p) {
        const f32x4 &x = st.o[2 * p][b], &y = st.o[2 * p + 1][b];
        const u32x4 pk = {pack_bf2(x[0] * inv, x[1] * inv), pack_bf2(x[2] * inv, x[3] * inv),
                          pack_bf2(y[0] * inv, y[1] * inv), pack_bf2(y[2] * inv, y[3] * inv)};
        if (wide) {
          *(u32x4*)(orow + 32 * p) = pk;
        } else {
          *(u32x2*)(orow + 32 * p) = u32x2{pk[0], pk[1]};
          *(u32x2*)(orow + 32 * p + 4) = u32x2{pk[2], pk[3]};
        }
      }
    }
  }
}

}  // namespace track
