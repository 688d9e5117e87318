// Rotary positions of queries and keys, with or without the RMSNorm of each head in the
// same pass: y = m A R(pos f) n(x), n(x) = x / sqrt(mean(x^2) + eps) g over a head (or x).
//
// Each element is read once and written once, so HBM bounds it (65520 tokens: 24 heads of 128
// 133 us, 6.1 TB/s; 80 heads with the norm, out of fused rows, 494 us, 5.4 TB/s); what is left to
// decide is how little else a wave does.  A wave takes one token and walks its heads (of q, then of
// k).  It forms the token's angles itself, one pair a lane: the position times the float64
// frequency in turns, reduced to half a turn in float64 (a float32 product is off by 0.06
// radian at position 10^6), one sincospi.  LDS hands every lane the angles of its own
// pairs, which stay in registers over all heads: a few instructions a token where a table
// of [tokens, pairs] would be as many bytes again as a head, and no scratch memory.
//
// A head is D / (2 V) units of two V-element loads (16 bytes each in the wide form) that
// hold whole pairs, so no lane needs another's elements, and that lie V elements apart from
// lane to lane, so that a load covers whole lines: channels V u .. and rot / 2 + V u .. of the
// half layout (copied ones likewise, by halves), V u .. and D / 2 + V u .. of the interleaved one
// (as 2 V u .. and 2 V u + V .. a load took every other 16 bytes).  A head takes the next power of two
// of lanes (8 for 128 bfloat16 channels, 8 heads a step); the sum of squares meets by DPP
// moves and lane swaps.
//
// Channels past rot_dim go out as they came (behind the norm as it leaves them): turned by cos 1 and
// sin 0 an infinity or a NaN in one would reach the channel beside it, and -0 would become 0.
#include <math.h>

#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace track {

// Pairs of the widest head: one wave's angles in LDS.
constexpr int ROPE_MAX_PAIRS = ROPE_MAX_DIM / 2;
constexpr int ROPE_STEPS = 2;  // head groups whose loads a wave has under way together (4: up to 13% slower, 2% faster at most)

struct RopeArgs {
  const void* x[2];  // q, k
  void* y[2];
  int64_t ldx[2], sx[2], ldy[2], sy[2];
  int heads[2];
  const void* g[2];
  float mul[2];
  const int32_t* pos;
  const double* freqs;
  float amp, eps;
  double dir;      // turns a radian, negative for the inverse
  int D, pairs;    // channels of a head, rotated pairs
  int sec0, sec1;  // first pair of axis 1 and of axis 2
  uint32_t tokens, L, wpt;
  int lph_log2;    // lanes a head
};

template <typename T, int V>
struct RopeVec;
template <>
struct RopeVec<bf16_t, 8> { typedef u32x4 type; };
template <>
struct RopeVec<bf16_t, 4> { typedef u32x2 type; };
template <>
struct RopeVec<bf16_t, 1> { typedef bf16_t type; };
template <>
struct RopeVec<float, 4> { typedef f32x4 type; };
template <>
struct RopeVec<float, 1> { typedef float type; };

template <typename T, int V>
__device__ __forceinline__ void rope_unpack(const typename RopeVec<T, V>::type& r, float (&f)[V]) {
  if constexpr (V == 1) {
    f[0] = ldf(&r);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = r[j];
  } else {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      f[2 * j] = __uint_as_float(r[j] << 16);
      f[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
    }
  }
}

template <typename T, int V>
__device__ __forceinline__ typename RopeVec<T, V>::type rope_pack(const float (&f)[V]) {
  typename RopeVec<T, V>::type r;
  if constexpr (V == 1) {
    stf(&r, f[0]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = f[j];
  } else {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) r[j] = pack_bf2(f[2 * j], f[2 * j + 1]);
  }
  return r;
}

// Sum over aligned groups of 2^n lanes, in every lane of the group (the whole wave takes part).
__device__ __forceinline__ float group_sum(float v, int n) {
  if (n > 0) v = dpp_add<0xb1>(v);   // quad_perm [1, 0, 3, 2]
  if (n > 1) v = dpp_add<0x4e>(v);   // quad_perm [2, 3, 0, 1]
  if (n > 2) v = dpp_add<0x141>(v);  // row_half_mirror: the other quad of eight
  if (n > 3) v = dpp_add<0x140>(v);  // row_mirror: the other eight of sixteen
  if (n > 4) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if (n > 5) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  return v;
}

// NU units a lane: 2 only where a head of more than 128 channels moves element by element.
// PAST: 0 through the caches, 1 stores past them, 2 loads too (rope_heads).
template <typename T, int V, int NU, bool NORM, bool HALF, int PAST>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  typedef typename RopeVec<T, V>::type Raw;
  constexpr int ST = NU == 1 ? ROPE_STEPS : 1;
  __shared__ float cs[4][2][ROPE_MAX_PAIRS];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const uint32_t gw = blockIdx.x * 4 + wv;
  const uint32_t tok = __builtin_amdgcn_readfirstlane(gw / a.wpt);
  if (tok >= a.tokens) return;  // wave-uniform
  const int part = (int)(gw - tok * a.wpt);
  const uint32_t b = __builtin_amdgcn_readfirstlane(tok / a.L), l = tok - b * a.L;

  const int units = a.D / (2 * V), rot_units = a.pairs / V;
  const int lph = 1 << a.lph_log2, hp = 64 >> a.lph_log2;
  const int u0 = lane & (lph - 1), hslot = lane >> a.lph_log2;
  int e0[NU], e1[NU];  // the units' channels
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = u0 + 64 * i;
    if (!HALF && V > 1) {
      e0[i] = V * u;
      e1[i] = V * (units + u);
    } else if (u < rot_units) {
      e0[i] = HALF ? V * u : 2 * u;
      e1[i] = HALF ? a.pairs + V * u : 2 * u + 1;
    } else {  // copied channels, from 2 pairs = 2 V rot_units on
      e0[i] = V * (rot_units + u);
      e1[i] = V * (units + u);
    }
  }
  const int total = a.heads[0] + a.heads[1];
  const T* const xr[2] = {(const T*)a.x[0] + b * a.sx[0] + l * a.ldx[0], (const T*)a.x[1] + b * a.sx[1] + l * a.ldx[1]};
  T* const yr[2] = {(T*)a.y[0] + b * a.sy[0] + l * a.ldy[0], (T*)a.y[1] + b * a.sy[1] + l * a.ldy[1]};

  Raw lo[ST][NU], hi[ST][NU];
  auto load = [&](int h0) {
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      const int h = h0 + s * (int)a.wpt * hp + hslot;
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        lo[s][i] = Raw{};
        hi[s][i] = Raw{};
        if (h < total && u0 + 64 * i < units) {
          const T* p = h < a.heads[0] ? xr[0] + (int64_t)h * a.D : xr[1] + (int64_t)(h - a.heads[0]) * a.D;
          if constexpr (PAST > 1) {
            lo[s][i] = __builtin_nontemporal_load((const Raw*)(p + e0[i]));
            hi[s][i] = __builtin_nontemporal_load((const Raw*)(p + e1[i]));
          } else {
            lo[s][i] = *(const Raw*)(p + e0[i]);
            hi[s][i] = *(const Raw*)(p + e1[i]);
          }
        }
      }
    }
  };
  load(part * hp);  // under way while the angles are formed

  // gains of the lane's channels
  Raw gl[2][NU], gh[2][NU];
  if constexpr (NORM) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        gl[t][i] = Raw{};
        gh[t][i] = Raw{};
        if (a.heads[t] && u0 + 64 * i < units) {
          gl[t][i] = *(const Raw*)((const T*)a.g[t] + e0[i]);
          gh[t][i] = *(const Raw*)((const T*)a.g[t] + e1[i]);
        }
      }
  }

  // angles, a pair a lane
  for (int p = lane; p < a.pairs; p += 64) {
    const int axis = (p >= a.sec0) + (p >= a.sec1);
    const double turns = (double)a.pos[(int64_t)axis * a.tokens + tok] * (a.freqs[p] * a.dir);
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[wv][0][p] = c * a.amp;
    cs[wv][1][p] = s * a.amp;
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  float c[NU][V], s[NU][V];
  bool turn0[NU], turn1[NU];  // whether the first load's channels are rotated, the second's (whole units are)
#pragma unroll
  for (int i = 0; i < NU; ++i) {
    const int u = u0 + 64 * i;
    turn0[i] = HALF || V == 1 ? u < rot_units : e0[i] < 2 * a.pairs;
    turn1[i] = HALF || V == 1 ? u < rot_units : e1[i] < 2 * a.pairs;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      // pair j of the lane: of the unit, or of its first load's V / 2 pairs and its second's
      const int p = HALF || V == 1 ? V * u + j : (j < V / 2 ? e0[i] / 2 + j : e1[i] / 2 + j - V / 2);
      c[i][j] = p < a.pairs ? cs[wv][0][p] : 1.0f;
      s[i][j] = p < a.pairs ? cs[wv][1][p] : 0.0f;
    }
  }

  for (int h0 = part * hp; h0 < total; h0 += ST * (int)a.wpt * hp) {
    if (h0 != part * hp) load(h0);
#pragma unroll
    for (int st = 0; st < ST; ++st) {
      const int h = h0 + st * (int)a.wpt * hp + hslot;
      const bool isk = h >= a.heads[0];
      float xl[NU][V], xh[NU][V];
#pragma unroll
      for (int i = 0; i < NU; ++i) {
        rope_unpack<T, V>(lo[st][i], xl[i]);
        rope_unpack<T, V>(hi[st][i], xh[i]);
      }
      if constexpr (NORM) {
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NU; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) sq = fmaf(xl[i][j], xl[i][j], fmaf(xh[i][j], xh[i][j], sq));
        sq = group_sum(sq, a.lph_log2);
        const float rstd = (1.0f / sqrtf(sq / (float)a.D + a.eps)) * (isk ? a.mul[1] : a.mul[0]);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
          float f[V], g[V];
          rope_unpack<T, V>(isk ? gl[1][i] : gl[0][i], f);
          rope_unpack<T, V>(isk ? gh[1][i] : gh[0][i], g);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            xl[i][j] *= rstd * f[j];
            xh[i][j] *= rstd * g[j];
          }
        }
      }
      if (h < total) {
        T* p = isk ? yr[1] + (int64_t)(h - a.heads[0]) * a.D : yr[0] + (int64_t)h * a.D;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
          if (u0 + 64 * i >= units) continue;
          Raw rl = lo[st][i], rh = hi[st][i];
          if constexpr (HALF || V == 1) {
            if (turn0[i]) {
#pragma unroll
              for (int j = 0; j < V; ++j) {
                const float x0 = xl[i][j], x1 = xh[i][j];
                xl[i][j] = x0 * c[i][j] - x1 * s[i][j];
                xh[i][j] = x0 * s[i][j] + x1 * c[i][j];
              }
            }
          } else {
            if (turn0[i]) {
#pragma unroll
              for (int j = 0; j < V / 2; ++j) {
                const float x0 = xl[i][2 * j], x1 = xl[i][2 * j + 1];
                xl[i][2 * j] = x0 * c[i][j] - x1 * s[i][j];
                xl[i][2 * j + 1] = x0 * s[i][j] + x1 * c[i][j];
              }
            }
            if (turn1[i]) {
#pragma unroll
              for (int j = 0; j < V / 2; ++j) {
                const float x0 = xh[i][2 * j], x1 = xh[i][2 * j + 1];
                xh[i][2 * j] = x0 * c[i][V / 2 + j] - x1 * s[i][V / 2 + j];
                xh[i][2 * j + 1] = x0 * s[i][V / 2 + j] + x1 * c[i][V / 2 + j];
              }
            }
          }
          if (NORM || turn0[i]) rl = rope_pack<T, V>(xl[i]);
          if (NORM || turn1[i]) rh = rope_pack<T, V>(xh[i]);
          if constexpr (PAST > 0) {
            __builtin_nontemporal_store(rl, (Raw*)(p + e0[i]));
            __builtin_nontemporal_store(rh, (Raw*)(p + e1[i]));
          } else {
            *(Raw*)(p + e0[i]) = rl;
            *(Raw*)(p + e1[i]) = rh;
          }
        }
      }
    }
  }
}

// Waves a token: one while the tokens alone give every SIMD of the chip a few waves; below
// that as many as a token has head groups, so that the heads go side by side.
static uint32_t rope_waves_per_token(int64_t tokens, int groups) {
  const int64_t simds = 4 * (int64_t)device_cus();
  const int64_t want = (4 * simds + tokens - 1) / tokens;
  return (uint32_t)std::max<int64_t>(1, std::min<int64_t>(want, groups));
}

template <typename T, int V, int NU, int PAST>
static void rope_launch(const RopeArgs& a, bool norm, bool half, unsigned grid, hipStream_t s) {
  if (norm && half) rope_kernel<T, V, NU, true, true, PAST><<<grid, 256, 0, s>>>(a);
  else if (norm) rope_kernel<T, V, NU, true, false, PAST><<<grid, 256, 0, s>>>(a);
  else if (half) rope_kernel<T, V, NU, false, true, PAST><<<grid, 256, 0, s>>>(a);
  else rope_kernel<T, V, NU, false, false, PAST><<<grid, 256, 0, s>>>(a);
}

track_status rope_heads(int dtype, const track_rope_config& c, int64_t B, int64_t L, const track_head_rows& q,
                        const track_head_rows* k, const void* g_q, const void* g_k, float eps, float q_scale,
                        const int32_t* pos, const double* freqs, float amplitude, bool inverse, hipStream_t s) {
  const int64_t tokens = B * L;
  RopeArgs a = {};
  const track_head_rows* rows[2] = {&q, k};
  const void* g[2] = {g_q, g_k};
  const size_t es = dtype == TRACK_DTYPE_BF16 ? 2 : 4;
  uintptr_t bits = 0;  // of all addresses a lane forms, in elements' bytes
  for (int t = 0; t < 2; ++t) {
    if (!rows[t]) continue;
    const track_head_rows& r = *rows[t];
    a.x[t] = r.x;
    a.y[t] = r.y;
    a.ldx[t] = r.ldx;
    a.sx[t] = r.sx;
    a.ldy[t] = r.ldy;
    a.sy[t] = r.sy;
    a.heads[t] = r.heads;
    a.g[t] = g[t];
    bits |= (uintptr_t)r.x | (uintptr_t)r.y | (uintptr_t)g[t] | (uintptr_t)(r.ldx * es) | (uintptr_t)(r.ldy * es);
    if (B > 1) bits |= (uintptr_t)(r.sx * es) | (uintptr_t)(r.sy * es);
  }
  a.mul[0] = q_scale;
  a.mul[1] = 1.0f;
  a.pos = pos;
  a.freqs = freqs;
  a.amp = amplitude;
  a.eps = eps;
  a.dir = (inverse ? -1.0 : 1.0) / (2.0 * M_PI);
  a.D = c.head_dim;
  a.pairs = c.rot_dim / 2;
  a.sec0 = c.axes > 1 ? c.section[0] : a.pairs;
  a.sec1 = c.axes > 2 ? c.section[0] + c.section[1] : a.pairs;
  a.tokens = (uint32_t)tokens;
  a.L = (uint32_t)L;
  // the widest units that hold whole pairs, all rotated or all copied, and that every address allows
  const bool norm = g_q != nullptr, half = c.layout == TRACK_ROPE_HALF;
  auto fits = [&](int v) {
    const bool whole = half ? a.pairs % v == 0 && (a.D - 2 * a.pairs) % (2 * v) == 0 : 2 * a.pairs % v == 0 && a.D % (2 * v) == 0;
    return whole && (bits | (uintptr_t)(a.D * es)) % (v * es) == 0;
  };
  const int V = es == 2 && fits(8) ? 8 : (fits(4) ? 4 : 1);
  const int units = a.D / (2 * V);
  while ((1 << a.lph_log2) < std::min(units, 64)) ++a.lph_log2;
  // Stores past the caches where a store covers whole 128-byte lines.  With shorter runs a line
  // is left half written between two stores: 16 heads of 64 channels 42 us, 46 past the caches;
  // with whole ones 2 x 4099 x 16 heads of 64 float32 channels 12.5 -> 10.1 us, 65520 x 24 heads
  // of 128 148 -> 142, 8192 x 48 heads 35.5 -> 35, float32 64-channel norms 91 -> 76.
  const bool lines = V > 1 && (half ? a.pairs : a.D / 2) * es >= 128;
  const int hp = 64 >> a.lph_log2, total = a.heads[0] + a.heads[1];
  // Loads too where the heads are more than the 256 MB that the Infinity Cache holds, so that the
  // call would push out its own.  Kept and past the caches, one buffer again and again, after 1 GiB
  // written elsewhere, and with heads just written: 65520 x 24 heads of 128 (403 MB) 140 and 133 us,
  // 192 and 138, 152 and 135; 80 heads with the norm 509 and 494, 559 and 499, 558 and 499.  Smaller ones
  // may still be there: 20000 x 48 (246 MB) 73 and 88, 138 and 92, 75 and 75; 4680 x 24 (29 MB) 10.0 and 9.7,
  // 19.4 and 15.0, 13.0 and 14.8.
  const int past = !lines ? 0 : (tokens * total * a.D * es > ((int64_t)256 << 20) ? 2 : 1);
  a.wpt = rope_waves_per_token(tokens, (total + hp - 1) / hp);
  const int64_t grid = (tokens * a.wpt + 3) / 4;
  if (grid >= (int64_t)1 << 24)
    return fail(TRACK_E_SHAPE, "rope: %lld tokens are too many", (long long)tokens);
  ProfScope prof(TRACK_PROF_NORM, s);
  const unsigned g1 = (unsigned)grid;
  if (es == 2) {
    if (past == 2 && V == 8) rope_launch<bf16_t, 8, 1, 2>(a, norm, half, g1, s);
    else if (past && V == 8) rope_launch<bf16_t, 8, 1, 1>(a, norm, half, g1, s);
    else if (V == 8) rope_launch<bf16_t, 8, 1, 0>(a, norm, half, g1, s);
    else if (V == 4) rope_launch<bf16_t, 4, 1, 0>(a, norm, half, g1, s);
    else if (units <= 64) rope_launch<bf16_t, 1, 1, 0>(a, norm, half, g1, s);
    else rope_launch<bf16_t, 1, 2, 0>(a, norm, half, g1, s);
  } else {
    if (past == 2 && V == 4) rope_launch<float, 4, 1, 2>(a, norm, half, g1, s);
    else if (past && V == 4) rope_launch<float, 4, 1, 1>(a, norm, half, g1, s);
    else if (V == 4) rope_launch<float, 4, 1, 0>(a, norm, half, g1, s);
    else if (units <= 64) rope_launch<float, 1, 1, 0>(a, norm, half, g1, s);
    else rope_launch<float, 1, 2, 0>(a, norm, half, g1, s);
  }
  TRACK_LAUNCH_CHECK();
  return TRACK_OK;
}

}  // namespace track
