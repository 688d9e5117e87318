// Attention with a sliding window of groups (tokens or whole frames) and first tokens that
// stay visible: o = softmax(scale q k^T over the keys a row sees) v.  The query at position
// p, of group g = floor(p / G), sees the keys [lo, hi] and those below `sink` up to hi, with
// lo = (g - left) G and hi = (g + right + 1) G - 1, both cut to the sequence's keys.
//
// The query heads that share a key head are rows of one problem: row r = i n + e is query i
// of head e of n, so a K or V^T tile is read once for all of them.  Both limits grow with
// the position, so a block of rows sees two ranges of 64-key tiles (the first tokens and the
// window), and all but the tiles at the ranges' edges are seen whole by every row.  Those
// take the tile body without a mask; the edge tiles come first, in a loop of their own.
//
// Masked places: a hidden key's logit is replaced, whatever K holds there, and its weight is
// zero.  V^T is cleared in LDS behind a sequence's last key.  An infinity or NaN in a V row
// that some rows of the block see and others do not would still reach the others through
// 0 x inf in the matrix product; the edge tiles are the only place where that can happen, so
// their sums are looked at once, and only where one is not finite the edge tiles are taken
// again with the keys weighed one by one.
//
// Attention with changed logits (capped, less a bias by distance, inside documents with prefixes) is the same kernels with
// another range a row, which still grows with the position, and a function of the logit in each tile (window.h).  What
// bounds it: reading K and V^T for single tokens (16 sequences of 16384 keys, capped and biased, 126 us and the join 4,
// 6.5 TB/s), and in blocks of rows the vector unit beside the matrix cores: 12 heads of 15600 tokens in three documents 544 us
// without either, 678 capped, 747 capped and biased (551 GFLOP, 31% of the matrix cores' time; the cap is an exponential
// and a reciprocal more a logit, the bias two instructions).
#include "window.h"

namespace track {

// ---------------------------------------------------------------- many rows, bfloat16
// 256 rows a workgroup, 32 a wave; K and V^T tiles by DMA into a ring of two slots, and the
// tile body of the plain attention.
template <bool QLOG2, bool SPLIT, class S>
__global__ __launch_bounds__(512) void window_blocks_kernel(WinArgs a) {
  static_assert(QLOG2 || !S::ON, "changed logits are in log2 units");
  typedef std::conditional_t<S::ON, WinScoreMask<ATT_QB, S, true>, WinMask<ATT_QB>> Mask;
  typedef std::conditional_t<S::ON, WinScoreMask<ATT_QB, S, true, true>, WinMask<ATT_QB, true>> Weighed;
  typedef std::conditional_t<S::ON, WinScoreMask<ATT_QB, S, false>, AttAll> Whole;
  constexpr int BKV = ATT_BKV, D = ATT_D, SLOT = ATT_SLOT;
  // one object: with a second one the compiler waits for every copy under way before a tile's
  // first fragment read (20% slower)
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * SLOT + 16];
  int* const not_finite = (int*)(smem + 2 * SLOT);
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int jq = lane & 15, g = lane >> 4;
  int rb, sp, h, b;
  if (S::ON && a.order) win_place_docs(a, rb, sp, h, b);
  else win_place<true>(a, rb, sp, h, b);
  const WinSeq seq = win_seq(a, b);
  const int rows = seq.qlen * a.n;
  const int r0 = rb * ATT_BQ;
  if (r0 >= rows) return;  // the whole workgroup
  if (tid == 0) *not_finite = 0;

  // windows of the block's first and last row, and of the wave's
  auto range_of = [&](int r, int& lo, int& hi) {
    win_seen<S>(a, seq, (int)a.by_n((uint32_t)min(r, rows - 1)), lo, hi);
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
  if (!S::ON && tiles.sink == 0 && seq.sink >= lo1) wlo = 0;
  const bool live = wr0 < rows;

  const bf16_t* const kbase = (const bf16_t*)a.k + b * a.sk + (int64_t)h * D;
  const bf16_t* const vbase = (const bf16_t*)a.vt + b * a.sv + (int64_t)h * D * a.ldv;
  bf16x8 qf[D / 32][ATT_QB];
  Mask mask;
  Whole whole;
  mask.sink = tiles.sink;
  if constexpr (S::ON) mask.a = whole.a = &a;
#pragma unroll
  for (int i = 0; i < ATT_QB; ++i) {
    int e;
    const int qi = win_query(a, min(wr0 + 16 * i + jq, rows - 1), e);
    win_seen<S>(a, seq, qi, mask.lo[i], mask.hi[i]);
    if (!S::ON && tiles.sink == 0 && seq.sink >= lo1) mask.lo[i] = 0;
    if constexpr (S::ON) {
      mask.p[i] = whole.p[i] = seq.start + qi;
      mask.slope[i] = whole.slope[i] = win_slope<S>(a, h * a.n + e);
    }
    const bf16_t* qp = (const bf16_t*)a.q + b * a.sq + (int64_t)qi * a.ldq + (int64_t)(h * a.n + e) * D + g * 8;
#pragma unroll
    for (int kc = 0; kc < D / 32; ++kc) qf[kc][i] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qp + kc * 32));
  }
  uint32_t koffg[2], voffg[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 8 * wave + 4 * i + (lane >> 4);
    koffg[i] = (uint32_t)((att_perm(row) * a.ldk + ((lane & 15) ^ (row & 15)) * 8) * 2);
    const int vr = 16 * wave + 8 * i + (lane >> 3);
    voffg[i] = (uint32_t)((att_perm(vr) * a.ldv + ((lane & 7) ^ att_vswz(vr)) * 8) * 2);
  }
  // the tile at key0 into the slot at byte `slot`: K rows past the last key read as zero,
  // V^T columns past the row's end as the next row's (cleared below) or zero
  auto issue = [&](int key0, int slot) {
    const __amdgpu_buffer_rsrc_t rsK = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(kbase + key0 * a.ldk), (short)0, (int)(uint32_t)(min(BKV, seq.klen - key0) * a.ldk * 2), 0x00020000);
    const __amdgpu_buffer_rsrc_t rsV = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(vbase + key0), (short)0, (int)(uint32_t)((a.vend - key0) * 2), 0x00020000);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsK, (att_lds_ptr_t)(smem + slot + wave * 2048 + i * 1024), 16, koffg[i], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsV, (att_lds_ptr_t)(smem + slot + ATT_K_BYTES + wave * 2048 + i * 1024), 16,
                                               voffg[i], 0, 0, 0);
  };
  auto barrier = [&]() {
    att_wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt((15 << 0) | (3 << 14) | (7 << 4) | (0 << 8));  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
  };
  // V^T of keys at or past the last one cleared in the tile just copied (it may be anything
  // there, and a weight of zero does not remove it): 16-byte units of 8 keys, two a thread
  auto clear_past_end = [&](int key0, int slot) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int unit = tid + 512 * i, row = unit >> 3, c = (unit & 7) ^ att_vswz(row);
      u32x4* p = (u32x4*)(smem + slot + ATT_K_BYTES + unit * 16);
      u32x4 v = *p;
#pragma unroll
      for (int w = 0; w < 4; ++w) v[w] &= win_keep(seq.klen - key0 - 8 * c - 2 * w);
      *p = v;
    }
    __syncthreads();
  };

  uint32_t ko = jq * 256 + ((g ^ jq) << 4), vo = jq * ATT_VROW + ((g ^ att_vswz(jq)) << 4);
  int slot = 0;  // byte offset of the slot computed on
  AttState st;
  st.reset();

  int i0 = 0, i1 = tiles.n;
  if (SPLIT) win_share(tiles.n, sp, a.nsplit, i0, i1);
  const int ie = max(i0, min(i1, tiles.edge));  // edge tiles of the share: [i0, ie)
  auto next = [&]() {
    ko ^= SLOT;
    vo ^= SLOT;
    slot ^= SLOT;
    barrier();
  };
  if (i0 < i1) {
    issue(tiles.key<BKV>(i0), 0);
    barrier();
    if (i0 < ie) {
      for (int idx = i0; idx < ie; ++idx) {
        const int key0 = tiles.key<BKV>(idx);
        issue(tiles.key<BKV>(min(idx + 1, i1 - 1)), slot ^ SLOT);
        if (key0 + BKV > seq.klen) clear_past_end(key0, slot);
        if (live && key0 <= whi && (key0 + BKV > wlo || key0 < tiles.sink)) {
          mask.key0 = key0;
          att_tile_masked<Mask, QLOG2, 4, true, false>(smem, qf, ko, vo, st, mask, a.scale_log2);
        }
        next();
      }
      float z = 0.0f;
#pragma unroll
      for (int f = 0; f < D / 16; ++f)
#pragma unroll
        for (int i = 0; i < ATT_QB; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) z = fmaf(st.o[f][i][r], 0.0f, z);
      if (__ballot(z != 0.0f) && lane == 0) *not_finite = 1;
      __syncthreads();
      if (*not_finite) {  // the whole workgroup
        st.reset();
        Weighed weigh;
#pragma unroll
        for (int i = 0; i < ATT_QB; ++i) weigh.lo[i] = mask.lo[i], weigh.hi[i] = mask.hi[i];
        weigh.sink = mask.sink;
        if constexpr (S::ON) {
          weigh.a = &a;
#pragma unroll
          for (int i = 0; i < ATT_QB; ++i) weigh.p[i] = mask.p[i], weigh.slope[i] = mask.slope[i];
        }
        for (int idx = i0; idx < ie; ++idx) {
          const int key0 = tiles.key<BKV>(idx);
          issue(key0, slot);
          barrier();
          if (key0 + BKV > seq.klen) clear_past_end(key0, slot);
          weigh.key0 = key0;
          att_tile_masked<Weighed, QLOG2, 4, true, false>(smem, qf, ko, vo, st, weigh, a.scale_log2);
          __syncthreads();
        }
        issue(tiles.key<BKV>(min(ie, i1 - 1)), slot);
        barrier();
      }
    }
    // the tiles seen whole, the next one's address formed from this one's: they lie one after
    // another but for the step from the first tokens to the window
    const int jump = tiles.edge + tiles.fs;
    const bf16_t* kp = kbase + tiles.key<BKV>(ie) * a.ldk;
    uint32_t vp = 2 * (uint32_t)tiles.key<BKV>(ie);
    const bf16_t* const kj = kbase + tiles.key<BKV>(jump) * a.ldk;
    const uint32_t vj = 2 * (uint32_t)tiles.key<BKV>(jump);
    const int64_t kstep = BKV * a.ldk;
    const __amdgpu_buffer_rsrc_t rsV =
        __builtin_amdgcn_make_buffer_rsrc((void*)vbase, (short)0, (int)(uint32_t)(a.vend * 2), 0x00020000);
    for (int idx = ie; idx < i1; ++idx) {
      const uint32_t vp0 = vp;
      if (idx + 1 < i1) {  // (past the share: this tile again)
        kp = idx + 1 == jump ? kj : kp + kstep;
        vp = idx + 1 == jump ? vj : vp + 2 * BKV;
      }
      const __amdgpu_buffer_rsrc_t rsK =
          __builtin_amdgcn_make_buffer_rsrc((void*)kp, (short)0, (int)(uint32_t)(kstep * 2), 0x00020000);
      uint8_t* const to = smem + (slot ^ SLOT) + wave * 2048;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsK, (att_lds_ptr_t)(to + i * 1024), 16, koffg[i], 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsV, (att_lds_ptr_t)(to + ATT_K_BYTES + i * 1024), 16, voffg[i], vp, 0, 0);
      if (live) {
        if constexpr (S::ON) whole.key0 = (int)(vp0 >> 1);
        att_tile_masked<Whole, QLOG2, 4, true, false>(smem, qf, ko, vo, st, whole, a.scale_log2);
      }
      next();
    }
  }

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
        const u32x4 pk = {pack_bf2(x[0] * inv, x[1] * inv), pack_bf2(x[2] * inv, x[3] * inv),
                          pack_bf2(y[0] * inv, y[1] * inv), pack_bf2(y[2] * inv, y[3] * inv)};
        *(u32x4*)(o + 32 * p) = pk;
      }
      if (a.lse && g == 0) a.lse[((int64_t)b * a.Hk * a.n + head) * a.Lq + qi] = win_lse(m, l);
    }
  }
}

// ---------------------------------------------------------------- few rows, bfloat16
// Cache policy of the copies below.  Past the caches where each key is read once a call, so that
// keeping it would only put out what others left there.  Replays of one buffer, kept and past the
// caches: 8 sequences of 100003 keys 548 and 490 us, 8 of 16384 101 and 89, 48 x 32760 143 and 128, 8
// x 32760 27.0 and 26.9; after 1 GiB written elsewhere 609 and 496, 153 and 93, 201 and 132, 55 and 31;
// with keys just written, 67 MB of them, 27.8 and 28.5 (the worst of nine sizes).
// Through the caches from WIN_SHARED sequences on that share their keys, each of which reads them: 8 key
// heads of 8192 keys, 32 sequences replayed 71 us and past the caches 100, after 1 GiB written elsewhere
// 80 and 97; 32 of 32760 keys 200 and 457, 403 and 450; 16 of 8192 40 and 51, 49 and 50; 16 of 32760 181 and
// 270, 293 and 265; but 8 of 32760 137 and 150, 178 and 152, 2 of 32760 27 and 35, 63 and 38.
constexpr int WIN_SHARED = 16;

// At most 16 rows a key head (a token of 16 query heads, four tokens of 4).  The four waves of
// a workgroup take every fourth 64-key tile of its share, each through 32 KB of LDS of its own:
// copies go by DMA in whole 128-byte lines (operands straight from memory, where adjacent lanes
// read different rows, would pass through the CU's cache 16 bytes a cycle, 1 us a tile: they took
// 582 us where the copies took 538), and no wave waits for another before the sums meet at the end.  K's half is
// filled again as soon as its tile's logits are formed, V^T's once its product is, so copies are
// under way all the time.  The weights are rounded to bfloat16 for the product with V, and the
// denominator adds the rounded ones, as in the block kernel (attention_tile.h).  What bounds it: reading K and V^T (8 sequences of 100003 keys 490 us,
// 6.7 TB/s; 6.2 - 6.5 is what a plain read stream through the caches reaches), and for short windows the
// latency of a tile and of the join (8 heads of 4096 keys 8.2 us).
template <bool SPLIT, bool PAST, class S>
__global__ __launch_bounds__(256) void window_rows_kernel(WinArgs a) {
  constexpr int BKV = ATT_BKV, D = ATT_D, F = D / 16;
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  // one object (see above): four tiles; the sums at the end
  __shared__ __attribute__((aligned(1024))) uint8_t smem[4 * ATT_SLOT];
  typedef f32x4 (*Sums)[F][64];
  typedef float (*Stats)[16];
  const Sums so = (Sums)smem;                                    // [4][F][64]
  const Stats sm = (Stats)(smem + 4 * F * 1024), sl = sm + 4;    // [4][16] each
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int jq = lane & 15, g = lane >> 4;
  int rb, sp, h, b;
  win_place<false>(a, rb, sp, h, b);
  const WinSeq seq = win_seq(a, b);
  const int rows = seq.qlen * a.n;  // at most 16
  if (rows == 0) return;            // the whole workgroup

  int lo0, hi0, lo1, hi1;
  win_seen<S>(a, seq, 0, lo0, hi0);
  win_seen<S>(a, seq, seq.qlen - 1, lo1, hi1);
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
  win_seen<S>(a, seq, qi, mask.lo[0], mask.hi[0]);
  if (!S::ON && tiles.sink == 0 && seq.sink >= lo1) mask.lo[0] = 0;
  const float slope = win_slope<S>(a, head), scale_log2 = S::ON ? 1.0f : a.scale_log2;  // (changed logits are in log2 units)
  const bf16_t* qp = (const bf16_t*)a.q + b * a.sq + (int64_t)qi * a.ldq + (int64_t)head * D + g * 8;
  bf16x8 qf[D / 32];
#pragma unroll
  for (int kc = 0; kc < D / 32; ++kc) qf[kc] = __builtin_bit_cast(bf16x8, *(const u32x4*)(qp + kc * 32));
  const uint8_t* const kbase = (const uint8_t*)((const bf16_t*)a.k + b * a.sk + (int64_t)h * D);
  const uint8_t* const vbase = (const uint8_t*)((const bf16_t*)a.vt + b * a.sv + (int64_t)h * D * a.ldv);
  const uint32_t krow = (uint32_t)a.ldk * 2, vrow = (uint32_t)a.ldv * 2;
  uint8_t* const tile = smem + wave * ATT_SLOT;
  uint32_t kl[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) kl[i] = tile_k_lane(i, lane, krow);
  const uint32_t vl = tile_v_lane(lane, vrow);
  const uint32_t ko = jq * 256 + ((g ^ jq) << 4), vo = jq * ATT_VROW + ((g ^ att_vswz(jq)) << 4);
  // K rows past the last key read as zero, V^T columns as whatever is there (cleared below) or,
  // past the head's last row, as zero.  Whole tiles take the row's offset as a scalar: no
  // instruction of the vector unit a copy.
  auto copy = [&](__amdgpu_buffer_rsrc_t rs, uint8_t* to, TileOffset at) {
    if constexpr (PAST) win_copy_past(rs, to, at.vec, at.scalar);
    else win_copy(rs, to, at.vec, at.scalar);
  };
  auto copy_k = [&](int key0) {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(kbase + (int64_t)key0 * krow), (short)0, (int)(min(BKV, seq.klen - key0) * krow), 0x00020000);
    if (tile_whole(key0, seq.klen)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) copy(rs, tile + i * 1024, tile_offset(true, kl[i & 3], tile_k_row(i, krow)));
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) copy(rs, tile + i * 1024, tile_offset(false, kl[i & 3], tile_k_row(i, krow)));
    }
  };
  auto copy_v = [&](int key0) {
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(vbase + (int64_t)key0 * 2), (short)0, (int)(uint32_t)((a.vend - key0) * 2), 0x00020000);
    if (tile_whole(key0, seq.klen)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) copy(rs, tile + ATT_K_BYTES + i * 1024, tile_offset(true, vl, tile_v_row(i, vrow)));
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) copy(rs, tile + ATT_K_BYTES + i * 1024, tile_offset(false, vl, tile_v_row(i, vrow)));
    }
  };
  // the oldest 16 copies have landed (`more`: 16 younger ones are under way)
  auto landed = [&](bool more) {
    if (more) att_wait_vmcnt<16>();
    else att_wait_vmcnt<0>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // the wave's own LDS reads are done: what they read may be filled again
  auto read = [&]() {
    __builtin_amdgcn_s_waitcnt((15 << 0) | (3 << 14) | (7 << 4) | (0 << 8));  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  f32x4 o[F];
  float m = -INFINITY, l = 0.0f;  // reference (log2 units), the lane's part of the denominator
#pragma unroll
  for (int f = 0; f < F; ++f) o[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  if (i0 + wave < i1) {
    copy_k(tiles.key<BKV>(i0 + wave));
    copy_v(tiles.key<BKV>(i0 + wave));
  }
  for (int idx = i0 + wave; idx < i1; idx += 4) {
    const int key0 = tiles.key<BKV>(idx);
    const bool edge = idx < tiles.edge, more = idx + 4 < i1;
    const int next = more ? tiles.key<BKV>(idx + 4) : 0;
    const int last = seq.klen - 1 - key0;  // the last key's place in the tile (or past it)
    landed(true);                          // K; V^T is under way
    // all fragments, then the products: read one by one each would wait for LDS
    u32x4 kf[BKV / 16][D / 32];
#pragma unroll
    for (int kc = 0; kc < D / 32; ++kc)
#pragma unroll
      for (int i = 0; i < BKV / 16; ++i) kf[i][kc] = *(const u32x4*)(tile + 4096 * i + (ko ^ (uint32_t)(64 * kc)));
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s[BKV / 16];
#pragma unroll
    for (int kc = 0; kc < D / 32; ++kc)
#pragma unroll
      for (int i = 0; i < BKV / 16; ++i)
        s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[i][kc]), qf[kc],
                                                       kc ? s[i] : f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
    read();
    if (more) copy_k(next);
    if constexpr (S::ON) {
      const float far = S::BIAS ? (float)(seq.start + qi - (key0 + 8 * g)) : 0.0f;
#pragma unroll
      for (int i = 0; i < BKV / 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          s[i][r] = S::apply(a, s[i][r], S::BIAS ? far - (float)(32 * (i >> 1) + 4 * (i & 1) + r) : 0.0f, slope);
    }
    if (edge) {
      WinMask<1> mk = mask;
      mk.key0 = key0;
      mk.begin();
#pragma unroll
      for (int i = 0; i < BKV / 16; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[i][r] = mk.apply(0, 32 * (i >> 1) + 4 * (i & 1) + r, s[i][r]);
    }
    float t = -INFINITY;
#pragma unroll
    for (int i = 0; i < BKV / 16; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) t = fmaxf(t, s[i][r]);
    const float mn = fmaxf(m, group_max2(t, t) * scale_log2);
    if (__ballot(mn > m)) {
      const float alpha = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      l *= alpha;
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[f][r] *= alpha;
      m = mn;
    }
    const float nm = m == -INFINITY ? 0.0f : -m;
    u32x4 pw[BKV / 32];
#pragma unroll
    for (int c = 0; c < BKV / 32; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 x = s[2 * c + (e >> 1)];
        const float p0 = __builtin_amdgcn_exp2f(fmaf(x[2 * (e & 1)], scale_log2, nm));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(x[2 * (e & 1) + 1], scale_log2, nm));
        pw[c][e] = pack_bf2(p0, p1);
        // the denominator adds the weights as rounded for the product with V
        l += __uint_as_float(pw[c][e] << 16) + __uint_as_float(pw[c][e] & 0xffff0000u);
      }
    landed(more);  // V^T
    const uint8_t* const vt = tile + ATT_K_BYTES;
    u32x4 vf[F][BKV / 32];
#pragma unroll
    for (int c = 0; c < BKV / 32; ++c)
#pragma unroll
      for (int f = 0; f < F; ++f) vf[f][c] = *(const u32x4*)(vt + f * 16 * ATT_VROW + (vo ^ (uint32_t)(64 * c)));
    bool weigh = false;
    if (edge) {
      // V^T past the last key is cleared, and what else is not finite and may be hidden from
      // some row is weighed key by key
      u16x2 top = {0, 0};
#pragma unroll
      for (int c = 0; c < BKV / 32; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t keep = win_keep(last + 1 - (32 * c + 8 * g + 2 * e));
#pragma unroll
          for (int f = 0; f < F; ++f) {
            vf[f][c][e] &= keep;
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[f][c][e] & 0x7f807f80u));
          }
        }
      weigh = __ballot(top[0] == 0x7f80 || top[1] == 0x7f80) != 0;
    }
    if (weigh) {
      const int ln = att_lane();
#pragma unroll 1
      for (int key = 0; key < BKV; ++key) {
        const u32x4 own = key < 32 ? pw[0] : pw[1];
        const int e = (key >> 1) & 3;
        const uint32_t w = e == 0 ? own[0] : (e == 1 ? own[1] : (e == 2 ? own[2] : own[3]));
        const uint32_t got = __builtin_amdgcn_ds_bpermute(((ln & 15) + 16 * ((key >> 3) & 3)) << 2, (int)w);
        const float p = __uint_as_float(key & 1 ? got & 0xffff0000u : got << 16);
        const uint32_t on = p != 0.0f ? 0xffffffffu : 0u;  // V times 0 where the weight is 0
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int vr = 16 * f + 4 * (ln >> 4) + r;
            const uint32_t v = *(const bf16_t*)(vt + vr * ATT_VROW + (((key >> 3) ^ att_vswz(vr)) << 4) + 2 * (key & 7));
            o[f][r] = fmaf(p, __uint_as_float((v << 16) & on), o[f][r]);
          }
      }
    } else {
#pragma unroll
      for (int c = 0; c < BKV / 32; ++c)
#pragma unroll
        for (int f = 0; f < F; ++f)
          o[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf[f][c]),
                                                         __builtin_bit_cast(bf16x8, pw[c]), o[f], 0, 0, 0);
    }
    read();
    if (more) copy_v(next);
  }
  __syncthreads();  // the tiles' space takes the sums

  // join the four waves: each takes two of the eight 16-channel blocks
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
  const float inv = win_inverse(sum);
#pragma unroll
  for (int fi = 0; fi < 2; ++fi) {
    const int f = 2 * wave + fi, ch = att_perm(16 * f + 4 * g);
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const f32x4 u = so[w][f][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(wt[w], u[e], v[e]);
    }
    if constexpr (SPLIT)
      *(f32x4*)(a.po + pr * D + ch) = v;
    else
      *(u32x2*)((bf16_t*)a.out + b * a.so + (int64_t)qi * a.ldo + (int64_t)head * D + ch) =
          u32x2{pack_bf2(v[0] * inv, v[1] * inv), pack_bf2(v[2] * inv, v[3] * inv)};
  }
  if (wave == 0 && g == 0) {
    if constexpr (SPLIT) a.pml[pr] = float2{mx, sum};
    else if (a.lse) a.lse[((int64_t)b * a.Hk * a.n + head) * a.Lq + qi] = win_lse(mx, sum);
  }
}

// ---------------------------------------------------------------- float32
// Many rows: tiles of 64 keys of K and V^T by DMA into LDS, 16 rows to each four of a workgroup's
// W waves, which take 16 keys of a tile each.  LDS rows keep 16-byte units at unit ^ (row & 7), so
// that the 16 rows of a fragment meet no bank twice in a phase.  8 waves share a ring of two
// slots, the next tile on its way while this one is computed on; 4 waves have one slot and rely
// on the other workgroups of their CU meanwhile, which are twice as many and half as large:
// where the former do not fill the chip twice that counts more (win_plan).  What bounds
// it: the matrix cores (135 - 149 TFLOP/s sustained on this instruction) at 87 - 92 TFLOP/s, the
// rest a tile's softmax and barrier.  2 x 8 heads, 1500 x 1500: 103 us at 64 channels with 8 waves,
// 117 with 4 (140 straight from memory), 213 and 213 at 128 (303); 8 heads of 64, 1501 queries on
// 304 keys each 25.2 and 22.2 us (32.5); 8 of 128, 100 x 8000 63.9 and 56.4 (72).
template <int D, int W, bool SPLIT, bool SCORED>
__global__ __launch_bounds__(64 * W) void window_f32_tiles_kernel(WinArgs a) {
  static_assert(W == 4 || W == 8, "waves");
  constexpr int C = D / 16, TK = 64, SLOTS = W / 4, ROWS = 4 * W;
  constexpr int KU = D / 4, VU = TK / 4;                   // 16-byte units of a K row, of a V^T row
  constexpr int HALF = TK * D * 4, SLOT = 2 * HALF;
  constexpr int NI = HALF / 1024 / W;                      // copies of 1 KB a wave, of K and of V^T
  constexpr int SO = W * C * 1024, LDS = SLOTS * SLOT > SO + W * 128 ? SLOTS * SLOT : SO + W * 128;
  // one object: with a second one the compiler waits for every copy under way before a tile's
  // first fragment read
  __shared__ __attribute__((aligned(1024))) uint8_t smem[LDS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int jq = lane & 15, g = lane >> 4;
  int rb, sp, h, b;
  win_place<true>(a, rb, sp, h, b);
  const WinSeq seq = win_seq(a, b);
  const int rows = seq.qlen * a.n;
  const int r0 = rb * ROWS;
  if (r0 >= rows) return;  // the whole workgroup
  auto range_of = [&](int r, int& lo, int& hi) {
    win_seen<std::conditional_t<SCORED, WinScore<false, false>, WinPlain>>(a, seq, (int)a.by_n((uint32_t)min(r, rows - 1)), lo, hi);
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
  };
  int lo0, hi0, lo1, hi1;
  range_of(r0, lo0, hi0);
  range_of(r0 + ROWS - 1, lo1, hi1);
  WinTiles tiles;
  tiles.init<TK>(seq, lo0, hi0, lo1, hi1);
  int i0 = 0, i1 = tiles.n;
  if (SPLIT) win_share(tiles.n, sp, a.nsplit, i0, i1);
  const int wr0 = r0 + 16 * (wave >> 2), mine = 16 * (wave & 3);  // first row, first key of a tile
  int wlo, whi, unused;
  range_of(wr0, wlo, unused);
  range_of(wr0 + 15, unused, whi);
  if (!SCORED && tiles.sink == 0 && seq.sink >= lo1) wlo = 0;
  const bool live = wr0 < rows;

  const float* const kbase = (const float*)a.k + b * a.sk + (int64_t)h * D;
  const float* const vbase = (const float*)a.vt + b * a.sv + (int64_t)h * D * a.ldv;
  uint32_t koff[NI], voff[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int at = (wave * NI + i) * 64 + lane;
    const int kr = at / KU, vr = at / VU;
    koff[i] = (uint32_t)(kr * a.ldk * 4 + ((at % KU) ^ (kr & 7)) * 16);
    voff[i] = (uint32_t)(vr * a.ldv * 4 + ((at % VU) ^ (vr & 7)) * 16);
  }
  // the tile at key0 into the slot at byte `slot`: K rows past the last key read as zero, V^T
  // columns past the row's end as the next row's (step() clears them) or zero
  auto issue = [&](int key0, int slot) {
    const __amdgpu_buffer_rsrc_t rsK = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(kbase + key0 * a.ldk), (short)0, (int)(uint32_t)(min(TK, seq.klen - key0) * a.ldk * 4), 0x00020000);
    const __amdgpu_buffer_rsrc_t rsV = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(vbase + key0), (short)0, (int)(uint32_t)((a.vend - key0) * 4), 0x00020000);
#pragma unroll
    for (int i = 0; i < NI; ++i)
      win_copy(rsK, smem + slot + (wave * NI + i) * 1024, koff[i]);
#pragma unroll
    for (int i = 0; i < NI; ++i)
      win_copy(rsV, smem + slot + HALF + (wave * NI + i) * 1024, voff[i]);
  };
  auto barrier = [&]() {
    att_wait_vmcnt<0>();
    __builtin_amdgcn_s_waitcnt((15 << 0) | (3 << 14) | (7 << 4) | (0 << 8));  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
  };

  WinF32<D, SCORED> st;
  st.template begin<true>(a, seq, tiles, lo1, h, wr0 + jq, rows);
  if (i0 < i1) {
    issue(tiles.key<TK>(i0), 0);
    barrier();
    int slot = 0;
    for (int idx = i0; idx < i1; ++idx) {
      const int key0 = tiles.key<TK>(idx);
      if (SLOTS == 2 && idx + 1 < i1) issue(tiles.key<TK>(idx + 1), slot ^ SLOT);
      const bool edge = idx < tiles.edge;
      const int k0 = key0 + mine;
      if (live && (!edge || (k0 <= whi && (k0 + 16 > wlo || k0 < tiles.sink)))) {
        const uint8_t* const kt = smem + slot + (mine + jq) * (D * 4);
        const uint8_t* const vt = smem + slot + HALF + jq * (TK * 4) + ((((mine >> 2) + g) ^ (jq & 7)) << 4);
        st.step([&](int c) { return *(const f32x4*)(kt + (((4 * c + g) ^ (jq & 7)) << 4)); },
                [&](int c) { return *(const f32x4*)(vt + 16 * c * (TK * 4)); }, edge, k0, seq.klen, a.scale_log2, &a);
      }
      barrier();
      if constexpr (SLOTS == 2) {
        slot ^= SLOT;
      } else if (idx + 1 < i1) {
        issue(tiles.key<TK>(idx + 1), 0);
        barrier();
      }
    }
  }
  st.template end<true, SPLIT>(a, b, h, sp, wr0 + jq, rows, (f32x4*)smem, (float*)(smem + SO));
}

// Straight from memory: few rows or keys, and rows that are not 16-byte aligned (VEC false:
// loads of single elements).  The four waves share a row block and take a fourth of its keys
// each, 16 a step, the next step's under way.
template <int D, bool VEC, bool SPLIT, bool SCORED>
__global__ __launch_bounds__(256) void window_f32_kernel(WinArgs a) {
  constexpr int C = D / 16, BKV = 16;
  __shared__ f32x4 so[4 * C * 64];
  __shared__ float sml[4 * 32];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int jq = lane & 15, g = lane >> 4;
  int rb, sp, h, b;
  win_place<true>(a, rb, sp, h, b);
  const WinSeq seq = win_seq(a, b);
  const int rows = seq.qlen * a.n;
  const int r0 = rb * 16;
  if (r0 >= rows) return;  // the whole workgroup

  int lo0, hi0, lo1, hi1;
  typedef std::conditional_t<SCORED, WinScore<false, false>, WinPlain> S;
  win_seen<S>(a, seq, (int)a.by_n((uint32_t)r0), lo0, hi0);
  win_seen<S>(a, seq, (int)a.by_n((uint32_t)min(r0 + 15, rows - 1)), lo1, hi1);
  WinTiles tiles;
  tiles.init<BKV>(seq, __builtin_amdgcn_readfirstlane(lo0), __builtin_amdgcn_readfirstlane(hi0),
                  __builtin_amdgcn_readfirstlane(lo1), __builtin_amdgcn_readfirstlane(hi1));
  int i0, i1;
  win_share(tiles.n, (SPLIT ? sp * 4 : 0) + wave, SPLIT ? 4 * a.nsplit : 4, i0, i1);
  WinF32<D, SCORED> st;
  st.template begin<VEC>(a, seq, tiles, lo1, h, r0 + jq, rows);

  const float* kb = (const float*)a.k + b * a.sk + (int64_t)h * D + 4 * g;
  const float* vb = (const float*)a.vt + b * a.sv + ((int64_t)h * D + jq) * a.ldv + 4 * g;
  f32x4 kf[C], vf[C];
  // K row key0 + jq (the last key again past the end) and the V^T columns key0 + 4 g + 0..3,
  // zero past the end
  auto load_k = [&](int key0, f32x4 (&d)[C]) {
    const float* p = kb + min(key0 + jq, seq.klen - 1) * a.ldk;
#pragma unroll
    for (int c = 0; c < C; ++c) d[c] = win_load4<VEC>(p + 16 * c);
  };
  auto load_v = [&](int key0, f32x4 (&d)[C]) {
    if (key0 + BKV <= seq.klen) {
#pragma unroll
      for (int c = 0; c < C; ++c) d[c] = win_load4<VEC>(vb + 16 * c * a.ldv + key0);
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) d[c][j] = key0 + 4 * g + j < seq.klen ? vb[16 * c * a.ldv + key0 + j] : 0.0f;
    }
  };
  if (i0 < i1) {
    load_k(tiles.key<BKV>(i0), kf);
    load_v(tiles.key<BKV>(i0), vf);
  }
  for (int idx = i0; idx < i1; ++idx) {
    f32x4 kn[C], vn[C];
    const bool more = idx + 1 < i1;
    if (more) {
      const int k1 = tiles.key<BKV>(idx + 1);
      load_k(k1, kn);
      load_v(k1, vn);
    }
    st.step([&](int c) { return kf[c]; }, [&](int c) { return vf[c]; }, idx < tiles.edge, tiles.key<BKV>(idx), seq.klen,
            a.scale_log2, &a);
    if (more) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        kf[c] = kn[c];
        vf[c] = vn[c];
      }
    }
  }
  st.template end<VEC, SPLIT>(a, b, h, sp, r0 + jq, rows, so, sml);
}

// The shares of each row joined: D / 4 threads a row and G groups of them, each with every
// G-th share, so that few rows do not wait for one share after another.  Whole calls with one
// group and with eight: 8 heads of 4096 keys, a token 10.6 and 8.2 us, 64 rows 17.3 and 15.5, 128 rows
// 19.2 and 18.7; 160 rows 22.2 and 22.5, 256 rows 24.5 and 25.3, 12 heads of 200 rows on 32760 keys 59.1
// and 60.8: eight below 128 threads a CU (1024 rows of 128 channels).
template <typename T, int G>
__global__ __launch_bounds__(256) void window_join_kernel(WinArgs a, int D) {
  __shared__ f32x4 so[G > 1 ? 256 : 1];
  __shared__ float2 sml[G > 1 ? 256 : 1];
  const int per = D / 4, t = (int)threadIdx.x;
  const int c = t % per * 4, grp = t / per % G;
  const int64_t all = (int64_t)a.B * a.Hk * a.Lq * a.n;
  const int64_t pr = (int64_t)blockIdx.x * (256 / per / G) + t / (per * G);
  float m = -INFINITY, l = 0.0f;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t row = pr < all ? pr : all - 1;  // below 2^25
  const uint32_t per_head = (uint32_t)(a.Lq * a.n), bh = (uint32_t)row / per_head;
  const int b = (int)a.by_Hk(bh), h = (int)bh - b * a.Hk;
  int e;
  const int qi = win_query(a, (int)((uint32_t)row - bh * per_head), e), head = h * a.n + e;
  const bool there = pr < all && !(a.q_len && qi >= min(a.q_len[b], a.Lq));
  auto add = [&](float m1, float l1, const f32x4& u) {
    const float mx = fmaxf(m, m1);
    const float w0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - mx);  // nothing yet, or a share without keys
    const float w1 = m1 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m1 - mx);
    l = w0 * l + w1 * l1;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = w0 * v[e] + w1 * u[e];
    m = mx;
  };
  if (there) {
#pragma unroll 4
    for (int s = grp; s < a.nsplit; s += G) {
      const float2 ml = a.pml[s * all + row];
      add(ml.x, ml.y, *(const f32x4*)(a.po + (s * all + row) * D + c));
    }
  }
  if constexpr (G > 1) {
    so[t] = v;
    sml[t] = float2{m, l};
    __syncthreads();
    if (grp) return;
#pragma unroll
    for (int i = 1; i < G; ++i) add(sml[t + i * per].x, sml[t + i * per].y, so[t + i * per]);
  }
  if (!there) return;
  const float inv = win_inverse(l);
  T* o = (T*)a.out + b * a.so + (int64_t)qi * a.ldo + (int64_t)head * D + c;
  if constexpr (sizeof(T) == 2) {
    *(u32x2*)o = u32x2{pack_bf2(v[0] * inv, v[1] * inv), pack_bf2(v[2] * inv, v[3] * inv)};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = v[e] * inv;
  }
  if (a.lse && c == 0) a.lse[((int64_t)b * a.Hk * a.n + head) * a.Lq + qi] = win_lse(m, l);
}

void window_join(int dtype, const WinArgs& a, int D, hipStream_t s) {
  // groups of shares for few rows (window_join_kernel)
  const int64_t joined = (int64_t)a.B * a.Hk * a.n * a.Lq;
  const int per = D / 4, G = joined * D / 4 < 128 * (int64_t)device_cus() && a.nsplit > 2 ? 8 : 1;
  const int rows_wg = 256 / per / G;
  const unsigned jg = (unsigned)((joined + rows_wg - 1) / rows_wg);
#define TRACK_WIN_JOIN(T)                                               \
  do {                                                                  \
    if (G == 1) window_join_kernel<T, 1><<<jg, 256, 0, s>>>(a, D);      \
    else window_join_kernel<T, 8><<<jg, 256, 0, s>>>(a, D);             \
  } while (0)
  if (dtype == TRACK_DTYPE_BF16) TRACK_WIN_JOIN(bf16_t);
  else TRACK_WIN_JOIN(float);
#undef TRACK_WIN_JOIN
}

// ---------------------------------------------------------------- host
struct WinPlan {
  enum Form { BLOCKS, ROWS, F32_ROWS, F32_TILES4, F32_TILES8 } form;
  int64_t nrb;
  int nsplit;
};

// Shares of the keys for few rows, `blocks` row blocks of `tiles` tiles each.  None up to 16
// tiles, four a wave: the join is a launch more (calls one after another, 8 heads of 1024 keys: 9.7
// us with one share, 11.4 with 2, 11.3 with 4; 2048: 22.3, 15.2 with 2, 12.7 with 4).  Then up to 8
// tiles a wave on a full chip a workgroup on every CU, but two tiles a share; beyond, six
// workgroups a CU with 16 tiles at least, which evens out lengths.  Replayed, join included, 8 key heads of
// 4096 keys: 43.9 us with one share, 12.6 with 8, 10.4 with 16, 9.2 with 32, 13.0 with 48; 32 of
// 1027: 15.7 with 1, 9.8 with 6 and 8, 13.3 with 12; 8 of 16384: 28.9 with 8, 19.4 with 16, 15.7 with 32,
// 20.1 with 48; 48 of 32760: 133 with 4, 137 with 16, 128 with 32, 130 with 48; 64 of 100003: 519 with 6,
// 485 with 16, 492 with 24, 488 with 32; 8 of 100003: 69 with 32, 75 with 48, 80 with 192.
static int rows_split(int64_t tiles, int64_t blocks, int64_t cus) {
  if (tiles <= 16) return 1;
  const bool large = blocks * tiles >= 64 * cus;
  const int64_t s = large ? std::min((6 * cus + blocks - 1) / blocks, tiles / 16) : std::min(cus / blocks, (tiles + 1) / 2);
  return (int)std::max<int64_t>(1, s);
}

static WinPlan win_plan(int dtype, const track_window& w, int64_t B, int Hk, int n, int D, int64_t Lq, int64_t Lk, bool vec) {
  const int64_t rows = Lq * n, cus = device_cus();
  WinPlan p;
  if (dtype == TRACK_DTYPE_F32) {
    // the tiles kernel from 180000 steps of 16 rows, 16 keys and a channel on (8 heads, 300 x 300,
    // 2900 steps: 32 channels 7.8 us straight and 8.4 by tiles, 64 11.4 and 11.1, 128 20.0 and 16.0; 64,
    // 1501 x 304, 15000 steps, 32.5 and 22.2), with 8 waves where those make two workgroups a CU
    // (above), shares of the keys up to that number
    p.nrb = (rows + 15) / 16;
    const int64_t steps = (win_span(w, std::min<int64_t>(rows, 16), n, Lk) + 15) / 16;
    const bool tiles = vec && p.nrb * Hk * B * steps * D >= 180000 && rows > 16;
    const int64_t nrb8 = (rows + 31) / 32;
    p.form = !tiles ? WinPlan::F32_ROWS : (nrb8 * Hk * B >= 2 * cus ? WinPlan::F32_TILES8 : WinPlan::F32_TILES4);
    if (p.form == WinPlan::F32_TILES8) p.nrb = nrb8;
    p.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>(2 * cus / (p.nrb * Hk * B), tiles ? steps / 16 : steps / 32));
    return p;
  }
  if (rows <= 16) {
    p.form = WinPlan::ROWS;
    p.nrb = 1;
    p.nsplit = rows_split((win_span(w, rows, n, Lk) + 63) / 64, Hk * B, cus);
    return p;
  }
  p.form = WinPlan::BLOCKS;
  p.nrb = (rows + ATT_BQ - 1) / ATT_BQ;
  p.nsplit = win_blocks_split((win_span(w, std::min<int64_t>(rows, ATT_BQ), n, Lk) + 63) / 64, p.nrb * Hk * B, rows * Hk * B, cus);
  return p;
}

static size_t win_bytes(const WinPlan& p, int64_t B, int Hk, int n, int D, int64_t Lq) {
  if (p.nsplit == 1) return 0;
  return (size_t)(p.nsplit * B * Hk * Lq * n) * (size_t)(4 * D + 8);
}

// Whether a launch and the join hold the plan.
static bool win_fits(const WinPlan& p, int64_t B, int Hk, int n, int64_t Lq) {
  return p.nrb * p.nsplit * Hk * B < (int64_t)1 << 23 && (p.nsplit == 1 || B * Hk * n * Lq < (int64_t)1 << 25);
}

track_status win_check(const char* what, int dtype, const track_window* w, int B, int H, int Hk, int D, int64_t Lq, int64_t Lk) {
  if (!w) return fail(TRACK_E_INVALID, "%s: null window", what);
  if (dtype != TRACK_DTYPE_F32 && dtype != TRACK_DTYPE_BF16)
    return fail(TRACK_E_INVALID, "%s: bad dtype %d", what, dtype);
  if (w->group < 1 || w->sink < 0 || w->left < -1 || w->right < -1 || !(w->scale == 0.0 || (w->scale >= 1e-30 && w->scale <= 1e30)))
    return fail(TRACK_E_INVALID, "%s: window of %lld / %lld groups of %lld, %lld first tokens, scale %g", what,
                (long long)w->left, (long long)w->right, (long long)w->group, (long long)w->sink, w->scale);
  if (w->left > WIN_MAX || w->right > WIN_MAX || w->group > WIN_MAX || w->sink > WIN_MAX)
    return fail(TRACK_E_SHAPE, "%s: window limits are at most 2^28", what);
  if (B < 0 || H < 1 || Hk < 1 || Lq < 0 || Lk < 0)
    return fail(TRACK_E_SHAPE, "%s: bad sizes B=%d H=%d Hk=%d Lq=%lld Lk=%lld", what, B, H, Hk, (long long)Lq, (long long)Lk);
  if (H % Hk) return fail(TRACK_E_SHAPE, "%s: %d query heads over %d key heads", what, H, Hk);
  if (dtype == TRACK_DTYPE_BF16 ? D != ATT_D : (D != 32 && D != 64 && D != 128))
    return fail(TRACK_E_UNSUPPORTED, "%s: head_dim %d (bfloat16: 128; float32: 32, 64, 128)", what, D);
  if (Lk > WIN_MAX || Lq > WIN_MAX / (H / Hk)) return fail(TRACK_E_SHAPE, "%s: sequence too long", what);
  // each has a workgroup at least, and the launch holds fewer than 2^23 (products below stay in 64 bits)
  if ((int64_t)B * Hk >= (int64_t)1 << 23)
    return fail(TRACK_E_SHAPE, "%s: %d sequences of %d key heads are too many", what, B, Hk);
  return TRACK_OK;
}

static int64_t rows_bytes(const char* what, int dtype, const track_window* w, int B, int H, int Hk, int D, int64_t Lq, int64_t Lk) {
  if (win_check(what, dtype, w, B, H, Hk, D, Lq, Lk) != TRACK_OK) return -1;
  if (B == 0 || Lq == 0) return 0;
  int64_t bytes = -1;
  for (bool vec : {true, false}) {  // whatever the rows' alignment turns out to be
    const WinPlan p = win_plan(dtype, *w, B, Hk, H / Hk, D, Lq, Lk, vec);
    if (win_fits(p, B, Hk, H / Hk, Lq)) bytes = std::max(bytes, (int64_t)win_bytes(p, B, Hk, H / Hk, D, Lq));
  }
  if (bytes < 0) fail(TRACK_E_SHAPE, "%s: too many row blocks", what);
  return bytes;
}

int64_t attention_window_bytes(int dtype, const track_window* w, int B, int H, int Hk, int D, int64_t Lq, int64_t Lk) {
  return rows_bytes("attention_window", dtype, w, B, H, Hk, D, Lq, Lk);
}

// What attention_scores adds to a window.
struct ScoreArgs {
  double cap;
  const float* slopes;
  const int32_t *doc_end, *prefix;
  int docs;
};

// One call of either kind (`c` null: a window's).
static track_status attention_rows(const char* what, int dtype, const track_window* w, const ScoreArgs* c, int B, int H, int Hk,
                                   int D, int64_t Lq, int64_t Lk, const void* q, int64_t ldq, int64_t sq, const void* k,
                                   int64_t ldk, int64_t sk, const void* vt, int64_t ldv, int64_t sv, void* out, int64_t ldo,
                                   int64_t so, float* lse, const int32_t* q_len, const int32_t* k_len, const int32_t* q_start,
                                   void* ws, size_t ws_bytes, hipStream_t s) {
  const track_status st = win_check(what, dtype, w, B, H, Hk, D, Lq, Lk);
  if (st != TRACK_OK) return st;
  if (B == 0 || Lq == 0) return TRACK_OK;
  if (!q || !out || (Lk > 0 && (!k || !vt))) return fail(TRACK_E_INVALID, "%s: null pointer", what);
  const int n = H / Hk;
  if (ldq < (int64_t)H * D || ldo < (int64_t)H * D || ldk < (int64_t)Hk * D || ldv < Lk)
    return fail(TRACK_E_SHAPE, "%s: leading dimension too small", what);
  if (sq < 0 || sk < 0 || sv < 0 || so < 0 || sequences_overlap(B, Lq, ldo, so, (int64_t)H * D))
    return fail(TRACK_E_SHAPE, "%s: sequences overlap in out, or a negative stride", what);
  if (((uintptr_t)lse | (uintptr_t)q_len | (uintptr_t)k_len | (uintptr_t)q_start) & 3)
    return fail(TRACK_E_INVALID, "%s: lse and lengths need 4-byte alignment", what);
  // (offsets inside a tile and a head's V^T are 32 bits)
  if (ldk > ((int64_t)1 << 22) || ldv > ((int64_t)1 << 22))
    return fail(TRACK_E_SHAPE, "%s: ldk and ldv are at most 2^22", what);
  const uintptr_t ptrs = (uintptr_t)q | (uintptr_t)k | (uintptr_t)vt | (uintptr_t)out;
  const int64_t strides = ldq | ldk | ldv | ldo | (B > 1 ? sq | sk | sv | so : 0);
  bool vec = true;
  if (dtype == TRACK_DTYPE_BF16) {
    if (ptrs & 15 || strides & 7) return fail(TRACK_E_INVALID, "%s: bf16 path needs 16-byte aligned rows", what);
  } else {
    if (ptrs & 3) return fail(TRACK_E_INVALID, "%s: float32 path needs 4-byte aligned rows", what);
    vec = !(ptrs & 15) && !(strides & 3);
  }
  WinPlan p = win_plan(dtype, *w, B, Hk, n, D, Lq, Lk, vec);
  if (!win_fits(p, B, Hk, n, Lq)) return fail(TRACK_E_SHAPE, "%s: too many row blocks", what);
  if (p.form == WinPlan::BLOCKS) p.nsplit = win_held(p.nsplit, B, Hk, n, D, Lq, ws, ws_bytes);
  const size_t need = win_bytes(p, B, Hk, n, D, Lq);
  if (need && (!ws || ws_bytes < need)) return fail(TRACK_E_NOMEM, "%s: workspace of %zu bytes needed", what, need);
  if (need && ((uintptr_t)ws & 255)) return fail(TRACK_E_INVALID, "%s: workspace must be 256-byte aligned", what);
  const int64_t grid = p.nrb * p.nsplit * Hk * B, joined = (int64_t)B * H * Lq;
  WinArgs a = {};
  a.q = q, a.k = k, a.vt = vt, a.out = out;
  a.ldq = ldq, a.sq = sq, a.ldk = ldk, a.sk = sk, a.ldv = ldv, a.sv = sv, a.ldo = ldo, a.so = so;
  a.lse = lse, a.q_len = q_len, a.k_len = k_len, a.q_start = q_start;
  win_visible(a, *w, B, Hk, n, D, Lq, Lk);
  const int64_t piece = dtype == TRACK_DTYPE_BF16 ? 8 : (vec ? 4 : 1);
  a.vend = (D - 1) * ldv + (Lk + piece - 1) / piece * piece;
  a.nrb = (int)p.nrb, a.nsplit = p.nsplit;
  a.by_nrb = win_div(a.nrb), a.by_nsplit = win_div(a.nsplit);
  a.by_inner = win_div(p.form == WinPlan::ROWS ? Hk : B);
  a.po = (float*)ws;
  a.pml = need ? (float2*)(a.po + (int64_t)p.nsplit * joined * D) : nullptr;
  const bool split = p.nsplit > 1, log2q = a.scale_log2 == 1.0f;
  if (c) {
    a.slopes = c->slopes, a.doc_end = c->doc_end, a.prefix = c->prefix, a.docs = c->docs;
    const double scale = w->scale > 0.0 ? w->scale : 1.0 / sqrt((double)D), log2e = 1.4426950408889634;
    a.cap_log2 = (float)(c->cap * log2e);
    // the argument of exp2 in bfloat16 (exp(2 y)), of tanh in float32
    a.cap_in = c->cap > 0.0 ? (float)(dtype == TRACK_DTYPE_BF16 ? 2.0 * log2e * scale / c->cap : scale / c->cap) : 0.0f;
  }
  a.order = c && c->docs > 0 && p.form == WinPlan::BLOCKS && grid > device_cus() && Lk >= 4096;  // (some 3 us a workgroup)
  ProfScope prof(TRACK_PROF_ATTN_SELF, s);
  const unsigned gr = (unsigned)grid;
#define TRACK_WIN_F32_OF(DH, C)                                                                             \
  do {                                                                                                      \
    if (p.form == WinPlan::F32_TILES8) window_f32_tiles_kernel<DH, 8, false, C><<<gr, 512, 0, s>>>(a);      \
    else if (p.form == WinPlan::F32_TILES4 && split) window_f32_tiles_kernel<DH, 4, true, C><<<gr, 256, 0, s>>>(a); \
    else if (p.form == WinPlan::F32_TILES4) window_f32_tiles_kernel<DH, 4, false, C><<<gr, 256, 0, s>>>(a); \
    else if (vec && split) window_f32_kernel<DH, true, true, C><<<gr, 256, 0, s>>>(a);                      \
    else if (vec) window_f32_kernel<DH, true, false, C><<<gr, 256, 0, s>>>(a);                              \
    else if (split) window_f32_kernel<DH, false, true, C><<<gr, 256, 0, s>>>(a);                            \
    else window_f32_kernel<DH, false, false, C><<<gr, 256, 0, s>>>(a);                                      \
  } while (0)
#define TRACK_WIN_F32(DH)              \
  do {                                 \
    if (c) TRACK_WIN_F32_OF(DH, true); \
    else TRACK_WIN_F32_OF(DH, false);  \
  } while (0)
  auto blocks = [&](auto qlog2, auto score) {
    typedef decltype(score) S;
    if (split) window_blocks_kernel<decltype(qlog2)::value, true, S><<<gr, 512, 0, s>>>(a);
    else window_blocks_kernel<decltype(qlog2)::value, false, S><<<gr, 512, 0, s>>>(a);
  };
  auto few = [&](auto score) {
    typedef decltype(score) S;
    if (B >= WIN_SHARED && sk == 0 && sv == 0) {
      if (split) window_rows_kernel<true, false, S><<<gr, 256, 0, s>>>(a);
      else window_rows_kernel<false, false, S><<<gr, 256, 0, s>>>(a);
    } else {
      if (split) window_rows_kernel<true, true, S><<<gr, 256, 0, s>>>(a);
      else window_rows_kernel<false, true, S><<<gr, 256, 0, s>>>(a);
    }
  };
  auto scored = [&](auto&& launch) {
    if (a.cap_log2 > 0.0f && a.slopes) launch(WinScore<true, true>{});
    else if (a.cap_log2 > 0.0f) launch(WinScore<true, false>{});
    else if (a.slopes) launch(WinScore<false, true>{});
    else launch(WinScore<false, false>{});
  };
  switch (p.form) {
    case WinPlan::BLOCKS:
      if (c) scored([&](auto score) { blocks(std::true_type{}, score); });
      else if (log2q) blocks(std::true_type{}, WinPlain{});
      else blocks(std::false_type{}, WinPlain{});
      break;
    case WinPlan::ROWS:
      if (c) scored(few);
      else few(WinPlain{});
      break;
    default:
      if (D == 32) TRACK_WIN_F32(32);
      else if (D == 64) TRACK_WIN_F32(64);
      else TRACK_WIN_F32(128);
  }
#undef TRACK_WIN_F32
#undef TRACK_WIN_F32_OF
  TRACK_LAUNCH_CHECK();
  if (split) {
    window_join(dtype, a, D, s);
    TRACK_LAUNCH_CHECK();
  }
  return TRACK_OK;
}

track_status attention_window(int dtype, const track_window* w, int B, int H, int Hk, int D, int64_t Lq, int64_t Lk,
                              const void* q, int64_t ldq, int64_t sq, const void* k, int64_t ldk, int64_t sk,
                              const void* vt, int64_t ldv, int64_t sv, void* out, int64_t ldo, int64_t so, float* lse,
                              const int32_t* q_len, const int32_t* k_len, const int32_t* q_start, void* ws,
                              size_t ws_bytes, hipStream_t s) {
  return attention_rows("attention_window", dtype, w, nullptr, B, H, Hk, D, Lq, Lk, q, ldq, sq, k, ldk, sk, vt, ldv, sv, out,
                        ldo, so, lse, q_len, k_len, q_start, ws, ws_bytes, s);
}

static track_status scores_window(const track_scores* c, track_window* w) {
  if (!c) return fail(TRACK_E_INVALID, "attention_scores: null scores");
  if (!(c->cap == 0.0 || (c->cap >= 1e-3 && c->cap <= 1e3))) return fail(TRACK_E_INVALID, "attention_scores: cap %g", c->cap);
  *w = track_window{c->left, c->right, 0, c->group, c->scale};
  return TRACK_OK;
}

int64_t attention_scores_bytes(int dtype, const track_scores* c, int B, int H, int Hk, int D, int64_t Lq, int64_t Lk) {
  track_window w;
  return scores_window(c, &w) == TRACK_OK ? rows_bytes("attention_scores", dtype, &w, B, H, Hk, D, Lq, Lk) : -1;
}

track_status attention_scores(int dtype, const track_scores* c, int B, int H, int Hk, int D, int64_t Lq, int64_t Lk,
                              const void* q, int64_t ldq, int64_t sq, const void* k, int64_t ldk, int64_t sk,
                              const void* vt, int64_t ldv, int64_t sv, void* out, int64_t ldo, int64_t so, float* lse,
                              const float* slopes, const int32_t* doc_end, int docs, const int32_t* prefix,
                              const int32_t* q_len, const int32_t* k_len, const int32_t* q_start, void* ws,
                              size_t ws_bytes, hipStream_t s) {
  track_window w;
  const track_status st = scores_window(c, &w);
  if (st != TRACK_OK) return st;
  if (docs < 0 || docs > SCORES_DOCS) return fail(TRACK_E_SHAPE, "attention_scores: %d documents (2^20 at most)", docs);
  if (docs > 0 && !doc_end && B > 0) return fail(TRACK_E_INVALID, "attention_scores: null pointer");
  if (((uintptr_t)slopes | (uintptr_t)doc_end | (uintptr_t)prefix) & 3)
    return fail(TRACK_E_INVALID, "attention_scores: slopes, documents and prefixes need 4-byte alignment");
  const ScoreArgs args = {c->cap, slopes, doc_end, prefix, docs};
  return attention_rows("attention_scores", dtype, &w, &args, B, H, Hk, D, Lq, Lk, q, ldq, sq, k, ldk, sk, vt, ldv, sv, out, ldo,
                        so, lse, q_len, k_len, q_start, ws, ws_bytes, s);
}

}  // namespace track
