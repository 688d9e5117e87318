// What the window attention kernels and those on a 4-bit cache share: arguments, the keys that a row sees,
// the tiles that a block of rows takes, masks, and the float32 step of 16 rows against 16 keys.
#pragma once

#include <math.h>

#include <algorithm>

#include "attention_tile.h"
#include "common.h"
#include "kernels.h"

namespace track {

// Division by a number that the host knows, for dividends below 2^31: with s = ceil(log2 d) and
// m = ceil(2^(31 + s) / d) < 2^32, floor(x m / 2^(31 + s)) = floor(x / d), since m d exceeds
// 2^(31 + s) by less than d <= 2^s (a hardware division is some 30 instructions, and the limits
// of a block's, a wave's and a lane's rows take a dozen: 1 - 2 us of a single token's call).
struct WinDiv {
  uint32_t d, m, s;
  __device__ __forceinline__ uint32_t operator()(uint32_t x) const { return d == 1 ? x : __umulhi(x, m) >> s; }
};

inline WinDiv win_div(int64_t d) {
  if (d == 1) return WinDiv{1, 0, 0};
  const uint32_t s = 32 - (uint32_t)__builtin_clz((uint32_t)d - 1);  // ceil(log2 d)
  return WinDiv{(uint32_t)d, (uint32_t)((((uint64_t)1 << (31 + s)) + (uint64_t)d - 1) / (uint64_t)d), s - 1};
}

// One call's arguments as the kernels take them.
struct WinArgs {
  const void *q, *k, *vt;
  void* out;
  int64_t ldq, sq, ldk, sk, ldv, sv, ldo, so;
  float* lse;
  const int32_t *q_len, *k_len, *q_start;
  // limits in tokens: from a group's first key back, and on to the first key past them (2^31 - 1:
  // no limit, or one that no key is as far away as: lengths are at most 2^28, positions within +- 2^29)
  int before, past;
  int lift;           // multiple of the group that makes every position positive
  int sink;
  int B, Hk, n;       // sequences, key heads, query heads of each
  int Lq, Lk;
  int nrb, nsplit;    // row blocks, shares of the keys
  WinDiv by_group, by_n, by_nrb, by_nsplit, by_Hk;
  WinDiv by_inner;    // sequences of a head, or heads of a sequence (win_place)
  int64_t vend;       // elements of a head's V^T up to its last row's last key, rounded up to 16 bytes
  float scale_log2;
  // attention with changed logits (win_score_range, WinScore)
  const float* slopes;                // [query heads], or null
  const int32_t *doc_end, *prefix;    // [B][docs], [B][docs + 1], or null
  int docs;
  bool order;                         // win_place_docs
  float cap_log2, cap_in;             // cap log2(e) (0: none), 2 scale log2(e) / cap
  float* po;          // [nsplit][B][Hk][Lq n][D]: a share's sums
  float2* pml;        // [nsplit][B][Hk][Lq n]: its reference (log2 units) and its denominator
};

// One sequence of the batch, in wave-uniform registers.
struct WinSeq {
  int b, qlen, klen, sink;
  int start;  // position of its first query
};

__device__ __forceinline__ WinSeq win_seq(const WinArgs& a, int b) {
  WinSeq s;
  s.b = b;
  // lengths from device memory are cut to the buffers
  s.qlen = a.q_len ? __builtin_amdgcn_readfirstlane(max(0, min(a.q_len[b], a.Lq))) : a.Lq;
  s.klen = a.k_len ? __builtin_amdgcn_readfirstlane(max(0, min(a.k_len[b], a.Lk))) : a.Lk;
  s.start = a.q_start ? __builtin_amdgcn_readfirstlane(max(-(int)WIN_MAX, min(a.q_start[b], (int)WIN_MAX))) : s.klen - s.qlen;
  s.sink = min(a.sink, s.klen);
  return s;
}

// The window [lo, hi] of query i, cut to [0, klen) (lo = klen or hi = -1: nothing left).
__device__ __forceinline__ void win_range(const WinArgs& a, const WinSeq& s, int i, int& lo, int& hi) {
  const uint32_t p = (uint32_t)(s.start + i + a.lift);  // in [0, 2^30 + 2^28)
  const int first = (int)(a.by_group(p) * a.by_group.d) - a.lift;  // of the query's group
  lo = first > a.before ? min(first - a.before, s.klen) : 0;
  hi = a.past - 1 < s.klen - 1 - first ? max(first + a.past - 1, -1) : s.klen - 1;
}

// The keys [lo, hi] of query i inside its document, those of the document's prefix among them whatever the window's
// end is; they grow with the position, like the window.  Ends of documents ascend: the last one at or before the
// position and the first behind it, all in the wave's lanes at once for 64 at most, by halves beyond (a dependent load each) and
// where the lanes have sequences of their own (ONE false).
template <bool ONE = true>
__device__ __forceinline__ void win_score_range(const WinArgs& a, const WinSeq& s, int i, int& lo, int& hi) {
  win_range(a, s, i, lo, hi);
  if (!a.docs && !a.prefix) return;
  const int p = s.start + i;
  int first = 0, end = INT32_MAX, d = 0;
  const int32_t* const ends = a.doc_end + (int64_t)s.b * a.docs;
  if (!ONE || a.docs > 64) {
    int n = a.docs;  // ends at or before p: d .. d + n
    while (n > 0) {
      const int half = n >> 1;
      const bool before = ends[d + half] <= p;
      d = before ? d + half + 1 : d;
      n = before ? n - half - 1 : half;
    }
    if (d > 0) first = ends[d - 1];
    if (d < a.docs) end = ends[d];
  } else if (a.docs > 0) {
    const int all = ends[min(att_lane(), a.docs - 1)];
    for (int k = 0; k < a.docs; ++k) {
      const int e = __builtin_amdgcn_readlane(all, k);
      const bool before = e <= p;
      d += before;
      first = before ? e : first;
      end = before ? end : min(end, e);
    }
  }
  if (a.prefix && a.past != INT32_MAX) {
    const int n = max(0, min(a.prefix[(int64_t)s.b * (a.docs + 1) + d], (int)WIN_MAX));
    hi = max(hi, min(max(-(int)WIN_MAX, min(first, (int)WIN_MAX)) + n, s.klen) - 1);
  }
  lo = max(lo, min(first, s.klen));
  hi = min(hi, max(end, 0) - 1);
}

// Query of row r, and the row's head among those of its key head.
__device__ __forceinline__ int win_query(const WinArgs& a, int r, int& e) {
  const int i = (int)a.by_n((uint32_t)r);
  e = r - i * a.n;
  return i;
}

// The tiles of TK keys that rows with windows from [lo0, hi0] (the first row's) to [lo1, hi1]
// (the last's) see between them, in the order they are taken: those seen in part by some
// row, then those seen whole by all.
struct WinTiles {
  int sink;          // first tokens, 0 where the window covers them
  int ns, w0;        // tiles of first tokens, first tile of the window
  int n, fs, fa, fb;  // all tiles; seen whole: [0, fs) and [fa, fb)
  int edge;          // tiles seen in part
  template <int TK>
  __device__ __forceinline__ void init(const WinSeq& s, int lo0, int hi0, int lo1, int hi1) {
    sink = s.sink;
    if (sink >= lo1) sink = lo0 = lo1 = 0;  // every row sees all from key 0 to its hi
    ns = (min(sink, hi1 + 1) + TK - 1) / TK;
    w0 = max(lo0 / TK, ns);
    n = ns + max(0, hi1 / TK + (hi1 >= 0) - w0);
    fs = min(sink, hi0 + 1) / TK;
    const int t0 = max((lo1 + TK - 1) / TK, w0), t1 = min((hi0 + 1) / TK, w0 + n - ns);
    fa = ns + t0 - w0;
    fb = ns + t1 - w0;
    if (t1 <= t0) fa = fb = n;
    edge = n - fs - (fb - fa);
  }
  // first key of the tile at place idx of the order
  template <int TK>
  __device__ __forceinline__ int key(int idx) const {
    int m;
    if (idx < edge) {
      m = fs + idx;
      if (m >= fa) m += fb - fa;
    } else {
      m = idx - edge;
      if (m >= fs) m += fa - fs;
    }
    return (m < ns ? m : m - ns + w0) * TK;
  }
};

// Share s of S of n tiles: [i0, i1).
__device__ __forceinline__ void win_share(int n, int s, int S, int& i0, int& i1) {
  const int q = (int)((uint32_t)n / (uint32_t)S), more = n - q * S;
  i0 = __builtin_amdgcn_readfirstlane(q * s + min(s, more));
  i1 = __builtin_amdgcn_readfirstlane(i0 + q + (s < more));
}

__device__ __forceinline__ float win_inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }  // nothing seen: zeros
__device__ __forceinline__ float win_lse(float m, float l) {
  return l == 0.0f ? -INFINITY : 0.69314718056f * (m + log2f(l));
}

// The keys of a tile that a lane's queries do not see.  A lane holds two runs of 8 keys of a
// tile, 32 apart; a bit for each that is hidden, and a hidden logit's bits replaced by those of
// -inf: two instructions an element and no branch (as comparisons with && and || the same
// was compiled to branches around single accumulator elements, and with two query blocks to
// moves that lost one of them).
template <int NB, bool WEIGHED_ = false>
struct WinMask {
  static constexpr bool ACTIVE = true, BITS = true, WEIGHED = WEIGHED_;
  int lo[NB], hi[NB];
  int sink, key0;
  uint32_t bits[NB];
  static __device__ __forceinline__ uint32_t below(int n) { return (1u << min(max(n, 0), 8)) - 1u; }
  __device__ __forceinline__ void begin() {
    key0 += 8 * (att_lane() >> 4);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      bits[b] = 0;
#pragma unroll
      for (int run = 0; run < 2; ++run) {
        const int k = key0 + 32 * run;
        bits[b] |= ((below(lo[b] - k) & ~below(sink - k)) | (below(hi[b] + 1 - k) ^ 0xffu)) << (8 * run);
      }
    }
  }
  __device__ __forceinline__ float apply(int b, int c, float s) const {
    const int at = (c & 7) + (c >> 5) * 8;
    const uint32_t t = (uint32_t)((int32_t)(bits[b] << (31 - at)) >> 31);
    return __uint_as_float((t & 0xff800000u) | (~t & __float_as_uint(s)));
  }
};

// What becomes of a logit s = q k before the softmax, in log2 units: cap tanh(scale s / cap) or scale s, less
// slope |p - j| for a query at place p and a key at j.  Both are template values: an element takes 2 instructions without either.
template <bool CAP_, bool BIAS_>
struct WinScore {
  static constexpr bool ON = true, CAP = CAP_, BIAS = BIAS_;
  // x: the logit, far: p - j, slope: in log2 units
  // tanh(y) = 1 - 2 / (exp(2 y) + 1): off by some 5 units of 2^-24 of the cap, also where it is near 0, a hundredth of
  // what the weights' rounding to bfloat16 takes at a cap of 50
  static __device__ __forceinline__ float apply(const WinArgs& a, float x, float far, float slope) {
    if constexpr (CAP)
      x = fmaf(-2.0f * a.cap_log2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * a.cap_in) + 1.0f), a.cap_log2);
    else
      x *= a.scale_log2;
    if constexpr (BIAS) x = fmaf(-fabsf(far), slope, x);
    return x;
  }
};
struct WinPlain {
  static constexpr bool ON = false, CAP = false, BIAS = false;
};

template <class S>
__device__ __forceinline__ void win_seen(const WinArgs& a, const WinSeq& s, int i, int& lo, int& hi) {
  if constexpr (S::ON) win_score_range(a, s, i, lo, hi);
  else win_range(a, s, i, lo, hi);
}

// The head's slope in log2 units.
template <class S>
__device__ __forceinline__ float win_slope(const WinArgs& a, int head) {
  if constexpr (S::BIAS) return a.slopes[head] * 1.4426950408889634f;
  else return 0.0f;
}

// A mask that changes the logits too; EDGE: it hides keys.
template <int NB, class S, bool EDGE, bool WEIGHED_ = false>
struct WinScoreMask : WinMask<NB, WEIGHED_> {
  const WinArgs* a;
  int p[NB];          // the lane's queries' places
  float slope[NB], far[NB];
  __device__ __forceinline__ void begin() {
    const int k = this->key0 + 8 * (att_lane() >> 4);
    if constexpr (EDGE) WinMask<NB, WEIGHED_>::begin();
    if constexpr (S::BIAS) {
#pragma unroll
      for (int b = 0; b < NB; ++b) far[b] = (float)(p[b] - k);
    }
  }
  __device__ __forceinline__ float apply(int b, int c, float s) const {
    s = S::apply(*a, s, S::BIAS ? far[b] - (float)c : 0.0f, S::BIAS ? slope[b] : 0.0f);
    if constexpr (EDGE) return WinMask<NB, WEIGHED_>::apply(b, c, s);
    else return s;
  }
};

// 16 bytes a lane from the buffer at `off` (and the wave's `scalar` more) to LDS, lanes side by side.
// (Functions of their own: in a template, with arguments that depend on it, the host's pass rejects
// the builtin.)
__device__ __forceinline__ void win_copy(__amdgpu_buffer_rsrc_t rs, uint8_t* lds, uint32_t off, uint32_t scalar = 0) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (att_lds_ptr_t)lds, 16, off, scalar, 0, 0);
}
// The same past the caches (the `nt` bit).
__device__ __forceinline__ void win_copy_past(__amdgpu_buffer_rsrc_t rs, uint8_t* lds, uint32_t off, uint32_t scalar) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (att_lds_ptr_t)lds, 16, off, scalar, 0, 2);
}

template <bool VEC>
__device__ __forceinline__ f32x4 win_load4(const float* p) {
  if constexpr (VEC) return *(const f32x4*)p;
  else return f32x4{p[0], p[1], p[2], p[3]};
}

// Bits of a pair of keys of which `left` are to keep (any number).
__device__ __forceinline__ uint32_t win_keep(int left) { return (uint32_t)((1ull << (16 * min(max(left, 0), 2))) - 1ull); }

// Row block, share, key head and sequence of a workgroup.  LOCAL: neighbouring row blocks go to one XCD, whose L2 then serves
// their common keys (over the XCDs in turn, 12 heads 16384 x 16384 under a causal mask took 955 us instead of 824, 2 x 12
// heads over a 21-frame video 5.2 ms instead of 4.8), and the sequences follow each other inside a head, so that short ones do
// not leave one XCD idle (4 sequences of 5000 to 3100 queries: 439 -> 385 us).  Single tokens use a key once and go over the
// XCDs in turn (8 sequences of 8 key heads, 100003 keys 491 us, 500 the other way; 48 x 32760 131 and 132, 8 of 100003 to
// 56000 keys 395 and 397, one of 100003 70 and 68).  The last rows of a sequence, which see most keys under a causal mask,
// start first.
template <bool LOCAL>
__device__ __forceinline__ void win_place_of(const WinArgs& a, uint32_t id, int& rb, int& sp, int& h, int& b) {
  const uint32_t t = a.by_nrb(id), u = a.by_nsplit(t), v = a.by_inner(u);
  rb = a.nrb - 1 - (int)(id - t * a.nrb);
  sp = (int)(t - u * a.nsplit);
  const int w = (int)(u - v * a.by_inner.d);
  h = LOCAL ? (int)v : w;
  b = LOCAL ? w : (int)v;
}
template <bool LOCAL>
__device__ __forceinline__ void win_place(const WinArgs& a, int& rb, int& sp, int& h, int& b) {
  win_place_of<LOCAL>(a, LOCAL ? (uint32_t)xcd_remap((int)blockIdx.x, (int)gridDim.x) : blockIdx.x, rb, sp, h, b);
}

// The same for row blocks of 256 rows inside documents: the workgroups of an XCD take the blocks of their range (up to 256 of
// them) with the most keys first, by eighths of the most that one has, so that a long one does not start when the others end.
// 12 heads of 15600 tokens in documents of 3391, 7460 and 4749: 643 us in the rows' order, 544 so (with a cap and a bias 914
// and 770).  Each wave counts for itself, four blocks a lane; all get the same numbers, so each block is taken once.
__device__ __forceinline__ void win_place_docs(const WinArgs& a, int& rb, int& sp, int& h, int& b) {
  const int q = (int)gridDim.x >> 3, rem = (int)gridDim.x & 7, x = (int)blockIdx.x & 7;
  const int start = x * q + min(x, rem), n = q + (x < rem);
  int j = (int)blockIdx.x >> 3, place = j;
  if (n <= 256) {
    const int lane = att_lane();
    int len[4], most = 0;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      len[c] = -1;
      if (64 * c + lane < n) {
        int r, share, hh, bb, lo, hi, unused;
        win_place_of<true>(a, (uint32_t)(start + 64 * c + lane), r, share, hh, bb);
        WinSeq s;
        s.b = bb;
        s.qlen = a.q_len ? max(0, min(a.q_len[bb], a.Lq)) : a.Lq;
        s.klen = a.k_len ? max(0, min(a.k_len[bb], a.Lk)) : a.Lk;
        s.start = a.q_start ? max(-(int)WIN_MAX, min(a.q_start[bb], (int)WIN_MAX)) : s.klen - s.qlen;
        s.sink = 0;
        const int rows = s.qlen * a.n;
        len[c] = 0;
        if (r * ATT_BQ < rows) {
          win_score_range<false>(a, s, (int)a.by_n((uint32_t)(r * ATT_BQ)), lo, unused);
          win_score_range<false>(a, s, (int)a.by_n((uint32_t)min(r * ATT_BQ + ATT_BQ - 1, rows - 1)), unused, hi);
          len[c] = max(0, hi - lo + 1);
        }
      }
      most = max(most, len[c]);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) most = max(most, __shfl_xor(most, o));
    const float eighth = 8.0f / (float)(most + 1);
    int part[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) part[c] = len[c] < 0 ? -1 : (int)((float)len[c] * eighth);
    bool done = false;
    for (int k = 8; k >= 0 && !done; --k) {  // (8: what rounding may leave at the top)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint64_t in = __ballot(part[c] == k);
        const int count = __builtin_popcountll(in);
        if (!done && j < count) {
          // the j-th lane of those
          const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0));
          place = 64 * c + __builtin_ctzll(__ballot(part[c] == k && before == j));
          done = true;
        }
        if (!done) j -= count;
      }
    }
  }
  win_place_of<true>(a, (uint32_t)(start + __builtin_amdgcn_readfirstlane(place)), rb, sp, h, b);
}

// One wave's 16 rows.  step() takes them against 16 keys with v_mfma_f32_16x16x4_f32 (float32
// products and sums): lane (jq, g) has row jq, kfrag(c) is channels 16 c + 4 g .. + 3 of key jq,
// vfrag(c) keys 4 g .. + 3 of channel 16 c + jq, and the logits that a lane holds (keys 4 g .. + 3
// of its row) are the "B" operand of O^T += V^T P^T as they are.
// REACH: a V without a number reaches the rows that see its key whatever the weight, also one that fell to zero.
template <int D, bool SCORED = false, bool REACH = false>
struct WinF32 {
  static constexpr int C = D / 16;
  f32x4 qf[C], o[C];
  float m, l;  // reference (log2 units), the lane's part of the denominator
  int lo, hi, sink;
  int p;       // SCORED: the row's place and slope
  float slope;
  template <class KF, class VF>
  __device__ __forceinline__ void step(KF kfrag, VF vfrag, bool edge, int key0, int klen, float scale_log2, const WinArgs* a = nullptr) {
    const int lane = att_lane(), jq = lane & 15, g = lane >> 4;
    f32x4 s0 = {0.0f, 0.0f, 0.0f, 0.0f}, s1 = s0;
    // fragments are read ahead of their products
    constexpr int LA = C < 3 ? C : 3;
    f32x4 kf[LA + 1];
#pragma unroll
    for (int c = 0; c < LA; ++c) kf[c] = kfrag(c);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (c + LA < C) kf[(c + LA) % (LA + 1)] = kfrag(c + LA);
      __builtin_amdgcn_sched_barrier(0);
      const f32x4 k = kf[c % (LA + 1)];
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[0], qf[c][0], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[1], qf[c][1], s1, 0, 0, 0);
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[2], qf[c][2], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[3], qf[c][3], s1, 0, 0, 0);
    }
    f32x4 vf[C];
#pragma unroll
    for (int c = 0; c < C; ++c) vf[c] = vfrag(c);
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = s0[e] + s1[e];
    if constexpr (SCORED) {  // in log2 units from here on
      if (a->cap_log2 > 0.0f) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = a->cap_log2 * tanhf(x[e] * a->cap_in);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] *= scale_log2;
      }
      if (a->slopes) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(-fabsf((float)(p - (key0 + 4 * g + e))), slope, x[e]);
      }
      scale_log2 = 1.0f;
    }
    if (edge) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = key0 + 4 * g + e;
        x[e] = (key > hi) | ((key < lo) & (key >= sink)) ? -INFINITY : x[e];
      }
    }
    const float t = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    const float mn = fmaxf(m, group_max2(t, t) * scale_log2);
    if (__ballot(mn > m)) {
      const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      l *= alpha;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[c][e] *= alpha;
      m = mn;
    }
    const float nm = m == -INFINITY ? 0.0f : -m;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], scale_log2, nm));
    l += (x[0] + x[1]) + (x[2] + x[3]);
    if (edge) {
      // V past the last key is cleared, and what else is not finite and may be hidden from some
      // row is weighed key by key
      float z = 0.0f;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          vf[c][e] = key0 + 4 * g + e < klen ? vf[c][e] : 0.0f;
          z = fmaf(vf[c][e], 0.0f, z);
        }
      if (__ballot(z != 0.0f)) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll 1
          for (int gg = 0; gg < 4; ++gg) {
            const float p = __shfl(x[e], jq + 16 * gg);
            const int key = key0 + 4 * gg + e;
            const bool weighed = REACH ? !((key > hi) | ((key < lo) & (key >= sink))) : p != 0.0f;
            const uint32_t on = weighed ? 0xffffffffu : 0u;  // V times 0 where the weight is 0
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t v = __float_as_uint(__shfl(vf[c][e], 4 * g + i + 16 * gg));
                o[c][i] = fmaf(p, __uint_as_float(v & on), o[c][i]);
              }
          }
        return;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < C; ++c) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[c][e], x[e], o[c], 0, 0, 0);
  }
  // the lane's row of `rows`: window, query, nothing summed yet
  template <bool VEC>
  __device__ __forceinline__ void begin(const WinArgs& a, const WinSeq& seq, const WinTiles& tiles, int lo1, int h, int r,
                                        int rows) {
    const int g = (int)(threadIdx.x & 63) >> 4;
    int e;
    const int qi = win_query(a, min(r, rows - 1), e);
    if constexpr (SCORED) {
      win_score_range(a, seq, qi, lo, hi);
      p = seq.start + qi;
      slope = a.slopes ? a.slopes[h * a.n + e] * 1.4426950408889634f : 0.0f;
    } else {
      win_range(a, seq, qi, lo, hi);
      if (tiles.sink == 0 && seq.sink >= lo1) lo = 0;
    }
    sink = tiles.sink;
    const float* qp = (const float*)a.q + seq.b * a.sq + (int64_t)qi * a.ldq + (int64_t)(h * a.n + e) * D + 4 * g;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      qf[c] = win_load4<VEC>(qp + 16 * c);
      o[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    m = -INFINITY;
    l = 0.0f;
  }
  // The sums of each four waves, which have the same rows, joined and stored, through LDS of
  // so[waves][C][64] and sml[waves][2][16].
  template <bool VEC, bool SPLIT>
  __device__ __forceinline__ void end(const WinArgs& a, int b, int h, int sp, int r, int rows, f32x4* so, float* sml) {
    const int lane = (int)(threadIdx.x & 63), jq = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), w0 = wave & ~3;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
#pragma unroll
    for (int c = 0; c < C; ++c) so[(wave * C + c) * 64 + lane] = o[c];
    if (g == 0) {
      sml[wave * 32 + jq] = m;
      sml[wave * 32 + 16 + jq] = l;
    }
    __syncthreads();
    float mx = -INFINITY, sum = 0.0f, wt[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) mx = fmaxf(mx, sml[(w0 + w) * 32 + jq]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mi = sml[(w0 + w) * 32 + jq];
      wt[w] = mi == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mi - mx);  // a wave without keys
      sum = fmaf(wt[w], sml[(w0 + w) * 32 + 16 + jq], sum);
    }
    if (r >= rows) return;
    int e;
    const int qi = win_query(a, r, e), head = h * a.n + e;
    const int64_t pr = ((((int64_t)sp * a.B + b) * a.Hk + h) * a.Lq) * a.n + r;
    const float inv = SPLIT ? 1.0f : win_inverse(sum);
    float* const op = SPLIT ? a.po + pr * D + 4 * g
                            : (float*)a.out + b * a.so + (int64_t)qi * a.ldo + (int64_t)head * D + 4 * g;
    for (int c = wave - w0; c < C; c += 4) {
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const f32x4 u = so[((w0 + w) * C + c) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(wt[w], u[e], v[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= inv;
      if constexpr (VEC || SPLIT) {
        *(f32x4*)(op + 16 * c) = v;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) op[16 * c + e] = v[e];
      }
    }
    if (wave == w0 && g == 0) {
      if constexpr (SPLIT) a.pml[pr] = float2{mx, sum};
      else if (a.lse) a.lse[((int64_t)b * a.Hk * a.n + head) * a.Lq + qi] = win_lse(mx, sum);
    }
  }
};

// Keys that a block of `rows` rows sees at most.
inline int64_t win_span(const track_window& w, int64_t rows, int n, int64_t Lk) {
  if (w.left < 0 || w.right < 0) return Lk;
  const int64_t groups = w.left + w.right + 2 + (rows + n - 1) / n / w.group;
  return std::min(Lk, groups * w.group + w.sink);
}
// Shares of the keys for blocks of rows, by an estimate of the time: rounds of workgroups over
// the CUs, a tile 1.6 us and 5 us beside the tiles, and with shares the join, 3 us and the
// sums' way out and back at 4 TB/s.  Fits measured times within 10% where the matrix cores
// are the bound (1 - 42 shares of 2000, 4096 and 32760 keys, 17 - 400 rows of 8, 12 and 40
// heads): 256 rows of 12 heads, 32760 keys 732 us with one share, 106 with 10, 69 with 21, 83
// with 42; 400 rows of 40 heads, 2000 keys 53 with one, 38 with 3, 52 with 4.
inline int win_blocks_split(int64_t tiles, int64_t blocks, int64_t rows, int64_t cus) {
  const uint32_t n = (uint32_t)tiles, most = std::max<uint32_t>(1, std::min<uint32_t>(n / 2, 64));
  const double join = (double)(2 * rows * (4 * ATT_D + 8)) / 4e6;
  int best = 1;
  double best_t = 0.0;
  for (uint32_t s = 1; s <= most && blocks * s <= 16 * cus; ++s) {  // (32-bit divisions: a call's own time)
    const uint32_t rounds = ((uint32_t)blocks * s + (uint32_t)cus - 1) / (uint32_t)cus;
    double t = rounds * ((n + s - 1) / s * 1.6 + 5.0);
    if (s > 1) t += 3.0 + s * join;
    if (s == 1 || t < best_t) {
      best = (int)s;
      best_t = t;
    }
  }
  return best;
}

// Blocks' shares do not always grow with the keys (12 heads of 200 rows: four for 512, three for 576), so a
// workspace that was made for more keys may hold fewer than these would take: as many as it
// holds.  The other forms' grow.
inline int win_held(int nsplit, int64_t B, int Hk, int n, int D, int64_t Lq, const void* ws, size_t ws_bytes) {
  if (nsplit == 1) return 1;
  const int64_t share = B * (int64_t)Hk * Lq * n * (4 * D + 8), held = ws ? (int64_t)(std::min<size_t>(ws_bytes, INT64_MAX) / share) : 0;
  return (int)std::max<int64_t>(1, std::min<int64_t>(nsplit, held));
}

// Whether a call's window and sizes can be taken (window.hip); `what` begins the message.
track_status win_check(const char* what, int dtype, const track_window* w, int B, int H, int Hk, int D, int64_t Lq, int64_t Lk);

// Sizes, window and scale of a call.
inline void win_visible(WinArgs& a, const track_window& w, int B, int Hk, int n, int D, int64_t Lq, int64_t Lk) {
  a.before = w.left < 0 ? INT32_MAX : (int)std::min<int64_t>(w.left * w.group, INT32_MAX);
  a.past = w.right < 0 ? INT32_MAX : (int)std::min<int64_t>((w.right + 1) * w.group, INT32_MAX);
  a.lift = (int)((2 * WIN_MAX + w.group - 1) / w.group * w.group);
  a.sink = (int)w.sink;
  a.B = B, a.Hk = Hk, a.n = n, a.Lq = (int)Lq, a.Lk = (int)Lk;
  a.by_group = win_div(w.group), a.by_n = win_div(n), a.by_Hk = win_div(Hk);
  a.scale_log2 = w.scale > 0.0 ? (float)(w.scale * 1.4426950408889634) : attn_log2_scale(D);
}

// The shares of each row joined into out and lse (window.hip).
void window_join(int dtype, const WinArgs& a, int D, hipStream_t s);

}  // namespace track
