#pragma once
// Forward attention over one rank's share (gfx950).
//
// One workgroup (4 waves) takes one work item -- a tile of query tokens
// with a received key range (no mask inside it but a window's, FlashCP Sec. 3.2:
// every query of a piece sees the same received prefix) and a local key range
// (intra-document causal, Sec. 2.1) -- for `heads_per_tile` query heads of
// one KV head. Each wave owns 32/heads_per_tile query rows of every one of
// those heads (a query per lane). Key tiles of 64 keys are double-buffered
// in LDS and shared by the waves (and so by the heads of the group); later
// tiles are copied from HBM straight into LDS (asynchronous loads, no
// staging registers) while the current one is computed, and the loop is
// software-pipelined across tiles (the scores of the next tile are computed
// beside the softmax of the current one):
//   S^T = K Q^T        MFMA 32x32x16, Q held in registers (B operand), so a
//                      query is a lane and its row statistics are per lane;
//   online softmax     base 2, scale folded into one FMA per score; a row's
//                      output is rescaled only when its maximum grows by
//                      more than 2^8 (the result is the same: numerator and
//                      denominator share the stale maximum). The decision is
//                      per row, so a row's arithmetic does not depend on the
//                      other rows of its tile (any query tiling gives the
//                      same bits, unless the view is split: the chunk length
//                      follows from the number of workgroups, and P is rounded
//                      to bf16 against its chunk's maximum);
//   O^T += V^T P^T     V^T read from LDS with transpose reads, P^T straight
//                      from the S^T accumulator registers.
// Output (template OUT): the final O (bf16, optionally fp32) and LSE; or an
// fp32 partial O/LSE for the log-sum-exp merge; or, for items that carry a
// received and a local range, both partials: the received range is run
// first and its partial written when the local range starts, so the query
// tile is loaded once and the tile pipeline runs on across the switch; or
// (merged) the same two passes followed by their log-sum-exp merge in the
// epilogue: the received partial's O is written to a workspace at the
// switch and read back at the end, its LSE kept in a register, and the
// final O and LSE are written as the merge kernel would write them.
//
// Split views. With few workgroups, or one much longer than the rest, the
// launch lasts as long as its longest key range. The host then gives the
// view a chunk length: each source's keys are taken in chunks of that many
// key tiles, each chunk an online softmax of its own, and a source's partial
// is the chunks' partials merged in key order. The chunks are work items of
// their own (OUT = unit: partial O to a slot, in register order, with its
// LSE), and fwd_combine_kernel merges them, in slots of the caller's workspace
// or, for the partial passes, of the view's bound buffer. Where neither is to
// be had (a partial pass under stream capture, or a view bound without its
// slots), or one source alone is too short to gain by them, one workgroup runs
// its chunks one after the other and merges as it goes (OUT = chunks), keeping
// the merged chunks in its own rows of the output. All of them give the same
// bits. What the merging costs, against the unsplit kernel on the same ranges:
// 8/1 heads over 64K tokens (local and received passes captured together) 324
// -> 333 us, 4/1 heads over 50K 317 -> 330, 16/8 heads of 64 over 44K 226 -> 230
// (in slots, uncaptured: 217, 76 and 123). Reading the kept chunks a block ahead
// made it slower (349, 359, 239), doing it before the tile's copies are issued
// no faster.
//
// Scored views (SC, see score.hpp): a tile's products become scores beside the
// PV products of the tile before, two to eight per slot, and only then are
// masked and take part in the row maximum; from there on scores are in log2
// units and the scale is gone. A cap alone needs no maximum (FIXED): its third of a
// score, the exponential, keeps its place beside the next tile's QK products, the
// other two are beside PV. Per MFMA there are 3.0 transcendental instructions (1.0 without
// a cap) and 5.4 others (4.0): the vector unit is busy 62% of the cycles (42) and the
// matrix unit 44% (55), both at once 25% (23), so that a fifth is left to neither: waits
// within two waves per SIMD. 32/8 heads of 128 over 64K tokens and 8 ranks, two
// passes merged / one: no score function 381 / 355 us, capped 445 / 421; with queries
// scaled by 6, 400 / 373 and 454 / 427.
//
// Windowed views (WIN, see score.hpp): the same walk over the key tiles that some row of
// the query tile sees, sinks first; tiles that a window begins or ends in are masked, the
// received ones too. A row may see nothing of a range: its partial has no weight then,
// as one of an empty range. 32/8 heads of 128, 8193 rows of 64K tokens over 8 ranks,
// window 1024: one pass 171-183 us, where 54 us would move its 290 MB and 95 us multiply
// what the rows see (118 GFLOP at 1240 TFLOP/s). The tiles hold 1.25 times that, at 1.6 us
// for one in each of the 512 resident workgroups, as without windows; the rest is where
// 2208 workgroups of 15.9 tiles (18 at most) begin and end. Window 4096: 500 us, 80% of that rate (1.03
// times the pairs). Matrix unit busy 41% of the cycles (55), vector unit 48% (43), both
// 18% (23). 16 single tokens that see 4100 of their documents' 16K keys each, split:
// 46 us, 5.8 TB/s, and 7 to combine.
#include "common.hpp"
#include "launch.hpp"
#include "score.hpp"

#include <type_traits>

namespace fck {

enum {
  kOutPartial = 0,
  kOutFinal = 1,
  kOutPaired = 2,
  kOutMerged = 3,
  kOutUnit = 4,
  kOutChunks = 5
};

template <int D, int KIND>
struct FwdLds {
  // two K and two V tiles; with a bias the positions of two tiles' keys; windowed, those
  // of the rows
  static constexpr uint32_t bytes =
      4 * 64 * D * 2 + ((KIND & kScoreBias) ? 2 * 256 : 0) + ((KIND & kWindow) ? kWindowLds : 0);
};

template <int D, int HPW, int OUT, int KIND>
__device__ __forceinline__ void fwd_tile(const FwdParams& p, char* smem) {
  constexpr int SC = KIND & kScores;
  constexpr bool WIN = KIND & kWindow;
  constexpr bool LEAN = KIND != 0;  // registers are short: lane's values counted where needed
  constexpr bool CAP = SC & kScoreCap, BIAS = SC & kScoreBias;
  // capped scores alone lie within the cap: the exponentials of a row keep the reference
  // that its first tile gives (set_top), and neither maxima nor rescaling are needed
  // (not windowed: a row may see nothing of the first tile)
  constexpr bool FIXED = SC == kScoreCap && !WIN;
  constexpr bool FINAL = OUT == kOutFinal, MERGED = OUT == kOutMerged, UNIT = OUT == kOutUnit;
  constexpr bool CHUNKS = OUT == kOutChunks;
  constexpr bool PAIRED = OUT == kOutPaired || MERGED;
  constexpr int BN = 64;        // keys per tile
  constexpr int RPW = 32 / HPW;  // query rows per wave and head
  constexpr int KS = D / 16;    // MFMA k-steps over the head dim
  constexpr int DB = D / 32;    // 32-wide output blocks of the head dim
  constexpr float kLazy = 8.0f; // log2 headroom before rescaling
  constexpr uint32_t TILE = BN * D * 2;  // bytes of one K or V tile
  // LDS: K0 | K1 | V0 | V1; key tile j uses K buffer j % 2 and V buffer
  // j % 2. K runs one tile ahead of V: iteration j reads K of tile j+1 and V
  // of tile j while the copies of K of tile j+2 and V of tile j+1 fill the
  // other two buffers. The loop is unrolled by two, so every read names its
  // buffer with a compile-time offset.
  // Ordering rule: a buffer is refilled only after a barrier that follows
  // every wave's last read of it. Iteration j refills K buffer j % 2, last
  // read in iteration j-1 (before its closing barrier) -- or, for j = 0, in
  // the prologue, which therefore ends with a barrier of its own.
  // (a bias: then the positions of the keys of K0 and of K1)
  constexpr uint32_t OP = 4 * TILE;
  constexpr uint32_t OW = OP + (BIAS ? 512 : 0);  // WIN: the rows' windows
  static_assert(OW + (WIN ? kWindowLds : 0) == FwdLds<D, KIND>::bytes, "LDS layout");

  const int lane = threadIdx.x & 63, wave = wave_id();
  const int half = lane >> 5;
  const int b = blockIdx.x;
  int rest;
  const int kvh = kv_head<BIAS>(p, b, (UNIT ? p.n_units : p.n_items) * p.head_chunks, rest);
  const int hc = rest % p.head_chunks;
  const int32_t* it = (UNIT ? p.units : p.items) + 8 * (rest / p.head_chunks);
  const int q0 = it[0], q1 = it[1], r1 = it[3], l1 = it[5];
  int r0 = it[2], l0 = it[4];
  const int ldiag = it[6];
  // a chunk of the source that this partial pass does not compute
  if (UNIT && !p.o_bf16 && !(r1 > r0 ? p.o_f32_recv : p.o_f32)) return;

  // lane -> (query row, head): a wave takes RPW consecutive rows of each of
  // the HPW heads, so a short query range leaves whole waves without rows
  // (they skip the products and only help with the copies and barriers)
  // instead of padding every head's rows to 32
  const int l31 = lane & 31;
  const int h = kvh * p.group + hc * HPW + l31 / RPW;
  const int qrow = q0 + wave * RPW + l31 % RPW;
  const bool qvalid = qrow < q1;
  const bool active = q0 + wave * RPW < q1;  // wave-uniform
  const float c = CAP ? p.cap_in : p.scale_log2;
  // SC: cap2, and the row's share of its scores (what rounding left out: row_lse)
  const float cap2 = p.cap2;
  float slope2 = 0.f, off2 = CAP ? cap2 : 0.f;
  if constexpr (BIAS) {
    float rest;
    slope2 = p.slopes[h];
    off2 = row_offset(off2, slope2, p.q_pos[min(qrow, q1 - 1)], rest);
  }

  bf16x8 qreg[KS];
  auto read_q = [&]() {
    const u16* qp = p.q + ((size_t)qrow * p.hq + h) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      qreg[ks] = qvalid ? *reinterpret_cast<const bf16x8*>(qp + 16 * ks) : zero8();
  };
  // BIAS, final output: the ranges start, whole tiles on, at the first key within
  // reach of a row of the workgroup (the rows' norms from their registers)
  const bool cut = BIAS && (FINAL || MERGED || (UNIT && p.o_bf16)) && p.norms;
  if (cut) {
    read_q();
    float n2 = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int j = 0; j < 8; ++j) n2 = __builtin_fmaf((float)qreg[ks][j], (float)qreg[ks][j], n2);
    n2 = sum_halves(n2);
    const float qn = __builtin_sqrtf(n2 == n2 ? n2 : INFINITY);
    const float bl = score_bound<SC>(p.scale_log2, qn, head_norm(p.norms, p.hq + kvh), cap2);
    const float br = score_bound<SC>(p.scale_log2, qn, head_norm(p.norms, p.hq + p.hkv + kvh), cap2);
    const float at = p.q_pos[min(qrow, q1 - 1)];
    skip_far<BN>(smem + OP, p.recv_pos, p.q_pos, qvalid ? at - reach(br + bl, slope2) : INFINITY,
                 qvalid ? at - reach(bl + bl, slope2) : INFINITY, r0, r1, l0, l1);
  }

  // WIN: what the tile's rows see
  WindowTiles wt{};
  if constexpr (WIN) {
    wt = window_tiles(p.win, q0, q1, r0, r1, l0, l1);
    put_window(smem + OW, 32 * wave + l31, p.win, min(qrow, q1 - 1));
  }
  // key tiles: first the received range, then the local range
  const int n_r = WIN ? wt.recv.n : (r1 - r0 + BN - 1) / BN;
  const int n_t = n_r + (WIN ? wt.local.n : (l1 - l0 + BN - 1) / BN);

  // async copy of the K (or V) rows of key tile j into the buffer at byte
  // offset `ofs`; rows past the range repeat the last row (finite data;
  // those keys are masked)
  const TileLoader<D, BN, 256, BN, LEAN> ld(p.hkv * D);
  // first key of the j-th tile taken (BIAS: each source from its last tile on, or each
  // of its chunks, the nearest keys first, so that maxima seldom grow)
  auto tile_at = [&](int j) {
    const bool rs = j < n_r;
    int t = rs ? j : j - n_r;
    if constexpr (BIAS) {
      const int n = rs ? n_r : n_t - n_r;
      if constexpr (WIN) {
        const KeyTiles k = rs ? wt.recv : wt.local;
        const int g = CHUNKS ? k.at(t) & -p.chunk : 0;  // (a power of 2)
        const int c0 = CHUNKS ? k.before(g) : 0, c1 = CHUNKS ? k.before(g + p.chunk) : n;
        t = c0 + c1 - 1 - t;
      } else {
        const int c0 = CHUNKS ? t & -p.chunk : 0;  // (a power of 2)
        t = c0 + (CHUNKS ? min(p.chunk, n - c0) : n) - 1 - (t - c0);
      }
    }
    if constexpr (WIN) t = rs ? wt.recv.at(t) : wt.local.at(t);
    return (rs ? r0 : l0) + t * BN;
  };
  auto fetch = [&](int j, uint32_t ofs, bool v) {
    const bool rs = j < n_r;
    const int k0 = tile_at(j);
    const int hi = rs ? r1 : l1;
    const size_t base = (size_t(k0) * p.hkv + kvh) * D;
    const u16* src = v ? (rs ? p.v_recv : p.v_loc) : (rs ? p.k_recv : p.k_loc);
    ld.load_at(lds_addr(smem) + ofs, src + base, hi - k0);
    if (BIAS && !v && wave == 0) {  // and the keys' positions, a key per lane
      const float* pos = rs ? p.recv_pos : p.q_pos;
      lds_copy4(pos + k0, 4u * uint32_t(min(int(fresh_lane()), hi - k0 - 1)),
                lds_addr(smem) + OP + ofs / (TILE / 256));
    }
  };

  if (n_t > 0) {
    fetch(0, 0, false);
    fetch(0, 2 * TILE, true);
  }
  if (n_t > 1) fetch(1, TILE, false);

  if (!cut) read_q();

  // per-lane LDS byte offsets of the MFMA operand reads (swizzled tiles):
  // K rows for k-step ks, and the two transpose reads of V^T block db
  uint32_t pk[KS], pv[DB][2];
  {
    const int kb = row_base<D>(0, lane), vb = tr_base<D>(lane);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) pk[ks] = 2u * uint32_t(kb ^ (ks << 4));
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      pv[db][0] = 2u * uint32_t(vb ^ (db << 5));
      pv[db][1] = 2u * uint32_t((vb ^ ((db << 5) | 16)) + 8 * D);
    }
  }

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = zero16();
  float m = -INFINITY;  // reference row maximum (scaled, log2 units)
  float top = 0.f;      // FIXED: exponent of a score at the cap
  float lsum = 0.f;     // this lane's share of the row sum

  // LSE of a row with sum `tot`, natural log (BIAS: and what rounding left out of the
  // row's share, from values read again rather than held across the loop)
  auto row_lse = [&](float tot) {
    float l = (FIXED ? cap2 - top : m) + __log2f(tot);
    if constexpr (BIAS) {
      const int ln = int(fresh_lane()) & 31, r = min(q0 + wave * RPW + ln % RPW, q1 - 1);
      float rest;
      row_offset(CAP ? cap2 : 0.f, p.slopes[kvh * p.group + hc * HPW + ln / RPW], p.q_pos[r], rest);
      l += rest;
    }
    return l * kLn2;
  };

  // this wave's slot of the merged mode's workspace: 32 x D floats, held in
  // register order (instruction k of lane l at 256k + 4l), so that the
  // received partial goes out and comes back with 1 KiB stores and loads
  // (the lane's address is formed where it is used, from an opaque copy of
  // the lane index, not held across the loop)
  auto slot = [&]() {
    return p.o_f32_recv + (size_t(blockIdx.x) * 4 + wave) * (32 * D) + 4 * opaque(uint32_t(lane));
  };
  // paired items: the received partial is complete when the local range
  // starts; write it (merged: to the slot, with its LSE kept in a register)
  // and start the local one from empty
  float lse_recv = -INFINITY;  // merged: the received partial's LSE
  auto switch_source = [&]() {
    const float tot = sum_halves(lsum);
    const float inv = tot > 0.f ? 1.f / tot : 0.f;
    const float lse = tot > 0.f ? row_lse(tot) : -INFINITY;
    if (MERGED) {
      lse_recv = lse;
      if (active) {
        float* const sl = slot();
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            f32x4 v;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) v[jj] = oacc[db][4 * g + jj] * inv;
            *reinterpret_cast<f32x4*>(sl + 256 * (4 * db + g)) = v;
          }
      }
    } else if (qvalid) {
      // (paired partial passes: the caller's [T_q, Hq, D] tensor, stored
      // from the registers; this is not the benchmarked path)
      const size_t ob = ((size_t)qrow * p.hq + h) * D;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 v;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) v[jj] = oacc[db][4 * g + jj] * inv;
          *reinterpret_cast<f32x4*>(p.o_f32_recv + ob + 32 * db + 8 * g + 4 * half) = v;
        }
      if (half == 0) p.lse_recv[(size_t)h * p.t_q + qrow] = lse;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = zero16();
    m = -INFINITY;
    lsum = 0.f;
  };

  // CHUNKS: the end of a chunk of `recv` keys. Its partial (with the source's
  // chunks before it merged in, unless it is the first) becomes oacc and
  // lse_acc; then it is kept for the next chunk, or (`done`, the source's
  // last chunk, the local keys still to come) stored, and the next chunk
  // starts from empty. At the end of the workgroup's keys (`end`) it stays in
  // oacc for the epilogue.
  float lse_acc = -INFINITY;
  auto finish_chunk = [&](bool recv, bool first, bool done, bool end) __attribute__((always_inline)) {
    const float tot = sum_halves(lsum);
    const float inv = tot > 0.f ? 1.f / tot : 0.f;
    const float lse = tot > 0.f ? row_lse(tot) : -INFINITY;
    float* const out = recv ? p.o_f32_recv : p.o_f32;
    float* const out_lse = recv ? p.lse_recv : p.lse;
    // the merged chunks in the output: this wave's nv rows of every head, taken
    // as nv * HPW * D floats in register order (instruction k holds 4 floats of
    // each lane with a row, side by side)
    // (lane-derived offsets from an opaque copy of the lane index: not held
    // across the key loop)
    const int ln = LEAN ? int(fresh_lane()) : int(opaque(uint32_t(lane))), pr = ln & 31;
    // (LEAN: what the epilogue needs of the lane's row, counted anew too)
    const int l31_ = LEAN ? pr : l31, half_ = LEAN ? ln >> 5 : half;
    const int h_ = LEAN ? kvh * p.group + hc * HPW + l31_ / RPW : h;
    const int qrow_ = LEAN ? q0 + wave * RPW + l31_ % RPW : qrow;
    const bool qvalid_ = LEAN ? qrow_ < q1 : qvalid;
    const int nv = min(RPW, q1 - (q0 + wave * RPW));
    const int ci = 2 * ((pr / RPW) * nv + pr % RPW) + (ln >> 5);
    float* const rows = out + (size_t(q0 + wave * RPW) * p.hq + kvh * p.group + hc * HPW) * D;
    auto raw = [&](int k) {
      const int L = k * (nv * HPW * 8) + 4 * ci;
      return rows + (L / (HPW * D)) * p.hq * D + L % (HPW * D);
    };
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[db][i] *= inv;
    if (first) {
      lse_acc = lse;
    } else {
      const Merge2 w = merge2(lse_acc, lse);
      lse_acc = w.lse;
      if (qvalid_) {
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          f32x4 y[4];
#pragma unroll
          for (int g = 0; g < 4; ++g) y[g] = *reinterpret_cast<const f32x4*>(raw(4 * db + g));
#pragma unroll
          for (int i = 0; i < 16; ++i)
            oacc[db][i] = merge2_value(w, y[i / 4][i % 4], oacc[db][i]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      // every row of the kept chunks has been read before any is written over
      wait_async();
    }
    if (end) return;
    if (!done) {
      if (qvalid_) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            f32x4 v;
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) v[jj] = oacc[db][4 * g + jj];
            *reinterpret_cast<f32x4*>(raw(4 * db + g)) = v;
          }
      }
    } else if (qvalid_) {
      const size_t ob = ((size_t)qrow_ * p.hq + h_) * D;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 v;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) v[jj] = oacc[db][4 * g + jj];
          *reinterpret_cast<f32x4*>(out + ob + 32 * db + 8 * g + 4 * half_) = v;
        }
      if (half_ == 0) out_lse[(size_t)h_ * p.t_q + qrow_] = lse_acc;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db] = zero16();
    m = -INFINITY;
    lsum = 0.f;
  };
  // CHUNKS: first key tile after the current chunk, the one that tile j begins (WIN: its
  // chunk may begin before, or end behind, what is taken of it); and whether it is the
  // source's first
  auto next_chunk = [&](int j) {
    if constexpr (WIN) {
      const bool rs = j < n_r;
      const KeyTiles k = rs ? wt.recv : wt.local;
      const int base = rs ? 0 : n_r;
      return base + k.before((k.at(j - base) & -p.chunk) + p.chunk);
    }
    return min(j + p.chunk, j < n_r ? n_r : n_t);
  };
  int chunk_end = CHUNKS ? next_chunk(0) : 0;
  bool first_chunk = true;

  // S^T = K Q^T for the K tile at byte offset ko (prologue only; the loop
  // interleaves the same products with the softmax), two independent
  // accumulator chains (32 keys each)
  auto scores = [&](f32x16 (&s)[2], uint32_t ko) {
    s[0] = zero16();
    s[1] = zero16();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
        s[mb] = mfma32(lds_b128(smem, pk[ks], ko + mb * 64 * D), qreg[ks], s[mb]);
  };
  // scores of tile j: keys past the range and, on diagonal tiles, keys after
  // the query are masked (element i of block mb is key k0 + 4*half +
  // cst(mb, i), visible iff cst < rel: one compare per score, edge tiles only)
  constexpr float kHidden = FIXED ? INFINITY : -INFINITY;  // no weight
  auto mask = [&](f32x16 (&s)[2], int j) {
    const bool rs = j < n_r;
    const int k0 = tile_at(j);
    const int hi = rs ? r1 : l1;
    const bool diag = !rs && k0 >= ldiag;
    const int sink = rs ? wt.sink_r : wt.sink_l;
    const bool cut_off = WIN && k0 < (rs ? wt.last_r : wt.last_l) && k0 + BN > sink;
    if (diag || k0 + BN > hi || cut_off) {
      const int ln = LEAN ? int(fresh_lane()) : lane, hf = LEAN ? ln >> 5 : half;
      const int qr = LEAN ? q0 + wave * RPW + (ln & 31) % RPW : qrow;
      const int rel = (diag ? min(hi, qr + 1) : hi) - k0 - 4 * hf;
      if constexpr (WIN) {
        // seen: in the window, or a sink
        const int from = *reinterpret_cast<const int*>(smem + OW + 8 * (32 * wave + (ln & 31)) + (rs ? 4 : 0)) -
                         k0 - 4 * hf;
        const uint32_t seen = seen_keys(rel, from, sink - k0 - 4 * hf);
#pragma unroll
        for (int n = 0; n < 32; ++n) s[n / 16][n % 16] = seen & (1u << n) ? s[n / 16][n % 16] : kHidden;
        return;
      }
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[mb][i] = mb * 32 + 8 * (i >> 2) + (i & 3) < rel ? s[mb][i] : kHidden;
    }
  };
  // SC: element e of a tile's products as a score in log2 units; kp: positions
  // of the keys of its group of four
  // (FIXED: up to r, which the exponential takes the rest of the way)
  auto score = [&](f32x16 (&s)[2], int e, const f32x4& kp) {
    if constexpr (FIXED)
      s[e / 16][e % 16] = cap_r(s[e / 16][e % 16], c);
    else
      s[e / 16][e % 16] = score_of<SC>(s[e / 16][e % 16], c, cap2,
                                     BIAS ? __builtin_fmaf(slope2, kp[e & 3], off2) : off2);
  };
  auto read_pos = [&](int e, uint32_t ofs) {  // of elements e & ~3 .. +3
    return *reinterpret_cast<const f32x4*>(smem + ofs + 4 * (32 * (e / 16) + 8 * ((e % 16) / 4) + 4 * half));
  };
  // row maximum of masked scores (scaled, log2 units)
  auto row_max = [&](const f32x16 (&s)[2]) {
    float mx = -INFINITY;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[mb][i]);
    return SC ? max_halves(mx) : max_halves(mx) * c;
  };
  // FIXED: the reference of the rows' exponentials, from a source's (or chunk's) first tile,
  // masked: cap_top, moved by at most a half so that the tile's best key has a whole
  // exponent. Its P is then a power of two, which bf16 holds: a single key's value comes out
  // whole, and so D, and a dS of 0. (With cap_top itself, documents of two or three tokens:
  // O 0.0020 off in the norm, dQ 0.0047, dK 0.0044; so 0.0012, 0.0019 and 0.0009, as
  // uncapped. 500 to 900 tokens: O 0.0023, so 0.0020.) What is left is fp32's rounding of
  // `top` and of the exponent, 2^-19 each. A row that sees nothing of the tile: any
  // reference does. It takes no time that shows: a forward of 32/8 heads of 128 over 64K
  // tokens and 8 ranks 441-443 us with it and without.
  auto set_top = [&](const f32x16 (&s)[2]) {
    float r0 = 1.f;
#pragma unroll
    for (int e = 0; e < 32; ++e) r0 = fminf(r0, s[e / 16][e % 16]);
    r0 = -max_halves(-r0);
    const float n = __builtin_rintf(__builtin_fmaf(r0, -2.f * cap2, p.cap_top));
    top = __builtin_fmaf(r0, 2.f * cap2, n);
  };

  wait_async();
  __syncthreads();
  f32x16 sa[2], sb[2];  // scores of the current and of the next tile
  float mxa = -INFINITY, mxb = -INFINITY;
  if (n_t > 0 && active) {
    scores(sa, 0);
    if constexpr (SC) {
      f32x4 kp = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        if (BIAS && e % 4 == 0) kp = read_pos(e, OP);
        score(sa, e, kp);
      }
    }
    mask(sa, 0);
    if constexpr (FIXED)
      set_top(sa);
    else
      mxa = row_max(sa);
  }
  // every wave has read K of tile 0 before iteration 0 copies tile 2 into
  // the same buffer
  if (n_t > 2) __syncthreads();

  // Iteration j runs the online softmax of tile j (scores sc and row maximum
  // mxc, both from the previous iteration) beside the MFMAs of tile j+1's
  // scores into sn, then O^T += V^T P^T for tile j beside tile j+1's mask
  // and row maximum (to mxn). The MFMAs form a fixed sequence of slots: a
  // slot issues the LDS reads of the slot two ahead, its MFMA and its share
  // of the vector work, then a scheduling barrier, so the softmax runs in
  // the MFMAs' shadow. The last iteration computes the scores of a tile that
  // does not exist (from whatever its K buffer holds: finite data or stale
  // bits, never read past the buffer) and drops them; one iteration body,
  // with no branch per slot and no second copy for the last tile.
  constexpr int NS = 2 * KS + 4 * DB;  // score slots, then PV slots
  constexpr int EX = 32 / (2 * KS);    // exponentials per score slot
  // SC: elements SS per slot become scores from PV slot 1 on, and the maxima follow
  // (FIXED: in every PV slot, with no maxima to follow)
  constexpr int SS = FIXED ? 8 / DB : 16 / DB, S0 = FIXED ? 0 : 1;
  constexpr int MX = FIXED ? 4 * DB : SC ? 2 + 32 / SS : 3;  // first PV slot that takes maxima
  constexpr int MPS = FIXED ? 0 : (32 + (4 * DB - MX) - 1) / (4 * DB - MX + FIXED);  // maxima per slot
  auto step = [&](int j, auto par, f32x16 (&sc)[2], float mxc, f32x16 (&sn)[2], float& mxn) {
    constexpr int PAR = decltype(par)::value;
    constexpr uint32_t KN = (1 - PAR) * TILE, VC = (2 + PAR) * TILE;
    if (j + 1 < n_t) fetch(j + 1, (3 - PAR) * TILE, true);   // V of tile j+1
    if (j + 2 < n_t) fetch(j + 2, PAR * TILE, false);        // K of tile j+2
    if (PAIRED && j == n_r) {
      switch_source();
      if (FIXED && active) set_top(sc);
    }
    if (CHUNKS && j == chunk_end) {
      const bool recv = j <= n_r;
      const int c0 = recv ? 0 : n_r;  // the source's first key tile
      if (active) finish_chunk(recv, WIN ? first_chunk : j - c0 <= p.chunk, j == n_r, false);
      first_chunk = j == n_r;
      chunk_end = next_chunk(j);
      if (FIXED && active) set_top(sc);
    }
    if (active) {
      // a row's output is rescaled only when its maximum grows by more than
      // the headroom; rows that do not grow keep their maximum and scale by 1
      const bool grow = !FIXED && mxc > m + kLazy;  // implies mxc > m
      if (!FIXED && __any(grow)) {
        const float alpha =
            !grow ? 1.f : m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mxc);
        m = grow ? mxc : m;
        lsum *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) oacc[db][i] *= alpha;
      }
      const float mref = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) pk[ks] = opaque(pk[ks]);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        pv[db][0] = opaque(pv[db][0]);
        pv[db][1] = opaque(pv[db][1]);
      }

      bf16x8 ring[3], pb[4];
      // operand of slot n: K rows of tile j+1 (score slots), V^T of tile j
      // (PV slots)
      auto rd = [&](int n) {
        if (n < 2 * KS) {
          ring[n % 3] = lds_b128(smem, pk[n / 2], KN + (n % 2) * 64 * D);
        } else {
          const int u = n - 2 * KS, kk = u / DB, db = u % DB;
          const uint32_t ro = VC + kk * 32 * D;  // rows 16*kk..
          ring[n % 3] = cat8(lds_tr(smem, pv[db][0], ro), lds_tr(smem, pv[db][1], ro));
        }
      };
      float ps = 0.f, mx = -INFINITY;
      constexpr int KP = SS < 4 ? 1 : SS / 4;
      f32x4 kp[KP];  // BIAS: positions of the next slot's keys
      sn[0] = zero16();
      sn[1] = zero16();
      rd(0);
      rd(1);
      static_for<0, NS>([&](auto nc) {
        constexpr int n = decltype(nc)::value;
        if (n + 2 < NS) rd(n + 2);
        if constexpr (n < 2 * KS) {
          sn[n % 2] = mfma32(ring[n % 3], qreg[n / 2], sn[n % 2]);
#pragma unroll
          for (int e = n * EX; e < (n + 1) * EX; ++e) {
            const float y = sc[e / 16][e % 16];
            const float x = __builtin_amdgcn_exp2f(FIXED ? __builtin_fmaf(y, -2.f * cap2, top)
                                                   : SC  ? y - mref
                                                         : __builtin_fmaf(y, c, -mref));
            sc[e / 16][e % 16] = x;
            ps += x;
            if (e % 8 == 7) {
              pb[e / 8] = pack8(sc[e / 16], 8 * ((e / 8) & 1));
              // complete here: keeps the exponentials in the score slots
              // rather than sunk past the masking branch into the PV slots
              asm volatile("" ::"v"(pb[e / 8]));
            }
          }
          if (n == 2 * KS - 1) {
            lsum += ps;
            asm volatile("" : "+v"(lsum));  // the row sum too, not sunk into the next step
          }
        } else {
          constexpr int u = n - 2 * KS;
          oacc[u % DB] = mfma32(ring[n % 3], pb[u / DB], oacc[u % DB]);
          if constexpr (SC && u < S0 + 32 / SS) {
            if constexpr (u >= S0) {
#pragma unroll
              for (int e = (u - S0) * SS; e < (u - S0 + 1) * SS; ++e) score(sn, e, kp[e / 4 % KP]);
            }
            if constexpr (BIAS && u < 32 / SS) {
#pragma unroll
              for (int i = 0; i < KP; ++i) kp[i] = read_pos(u * SS + 4 * i, OP + (1 - PAR) * 256);
            }
          }
          if constexpr (u == MX - 1) mask(sn, j + 1);
          if constexpr (u >= MX) {
#pragma unroll
            for (int e = (u - MX) * MPS; e < (u - MX + 1) * MPS && e < 32; ++e)
              mx = fmaxf(mx, sn[e / 16][e % 16]);
          }
          if constexpr (u == 4 * DB - 1 && !FIXED) mxn = SC ? max_halves(mx) : max_halves(mx) * c;
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    }
    wait_async();
    __syncthreads();
  };
  // no received key: the received partial (where one is asked for beside the
  // local one) is empty
  if (CHUNKS && n_r == 0 && p.o_f32 && p.o_f32_recv && active)
    finish_chunk(true, true, true, false);
  for (int j = 0; j < n_t; j += 2) {
    step(j, std::integral_constant<int, 0>(), sa, mxa, sb, mxb);
    if (j + 1 < n_t) step(j + 1, std::integral_constant<int, 1>(), sb, mxb, sa, mxa);
  }

  if (PAIRED && n_r == n_t) switch_source();  // no local tile (never empty in practice)
  if constexpr (CHUNKS) {
    // the last source's partial: in oacc, normalised, after its last chunk
    const bool recv = !p.o_f32;
    if (active) finish_chunk(recv, WIN ? first_chunk : n_t - (recv ? 0 : n_r) <= p.chunk, true, true);
    store_rows<D, RPW>(
        smem + size_t(wave) * (32 * D * 4), active,
        [&](int db, int g) {
          f32x4 v;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) v[jj] = oacc[db][4 * g + jj];
          return v;
        },
        q0 + wave * RPW, q1, p.hq, kvh * p.group + hc * HPW, recv ? p.o_f32_recv : p.o_f32,
        nullptr);
    if (qvalid && half == 0)
      (recv ? p.lse_recv : p.lse)[(size_t)h * p.t_q + qrow] = lse_acc;
    return;
  }
  // the local (or only) partial, normalised, and its LSE
  const float tot = sum_halves(lsum);
  const float inv = tot > 0.f ? 1.f / tot : 0.f;
  const float lse_own = tot > 0.f ? row_lse(tot) : -INFINITY;
  if constexpr (UNIT) {
    const size_t sl = (size_t(it[7]) * p.head_chunks + hc) * p.hkv + kvh;
    if (active) {
      float* const o = p.slots + (sl * 4 + wave) * (32 * D) + 4 * lane;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 v;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) v[jj] = oacc[db][4 * g + jj] * inv;
          *reinterpret_cast<f32x4*>(o + 256 * (4 * db + g)) = v;
        }
      if (half == 0) p.slot_lse[sl * 128 + 32 * wave + l31] = lse_own;
    }
    return;
  }
  // rows go out through the LDS tile buffers, free once the loop's last
  // barrier has passed: wave w's region is bytes 32*D*4*w ..
  char* const region = smem + size_t(wave) * (32 * D * 4);
  const int h0 = kvh * p.group + hc * HPW;
  if constexpr (MERGED) {
    // local partial (registers) merged with the received one (this wave's
    // slot, written at the switch; the waits since have completed it)
    wait_async();
    const Merge2 w = merge2(lse_own, lse_recv);
    // every read of the received partial is issued before the first use
    f32x4 y[DB][4];
    if (active) {  // (a wave without rows wrote no slot)
      const float* const sl = slot();
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          y[db][g] = *reinterpret_cast<const f32x4*>(sl + 256 * (4 * db + g));
    }
    store_rows<D, RPW>(
        region, active,
        [&](int db, int g) {
          f32x4 v;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) v[jj] = merge2_value(w, oacc[db][4 * g + jj] * inv, y[db][g][jj]);
          return v;
        },
        q0 + wave * RPW, q1, p.hq, h0, p.o_f32, p.o_bf16);
    if (qvalid && half == 0) p.lse[(size_t)h * p.t_q + qrow] = w.lse;
  } else {
    store_rows<D, RPW>(
        region, active,
        [&](int db, int g) {
          f32x4 v;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) v[jj] = oacc[db][4 * g + jj] * inv;
          return v;
        },
        q0 + wave * RPW, q1, p.hq, h0, p.o_f32, FINAL ? p.o_bf16 : nullptr);
    if (qvalid && half == 0) p.lse[(size_t)h * p.t_q + qrow] = lse_own;
  }
}

template <int D, int HPW, int OUT>
__global__ __launch_bounds__(256, 2) void attn_fwd_kernel(FwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[FwdLds<D, 0>::bytes];
  fwd_tile<D, HPW, OUT, 0>(p, smem);
}
template <int D, int HPW, int OUT, int SC>
__global__ __launch_bounds__(256, 2) void attn_fwd_scored_kernel(FwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[FwdLds<D, SC>::bytes];
  fwd_tile<D, HPW, OUT, SC>(p, smem);
}
// (Windows with slopes at head dim 128 take over 256 registers: one wave per SIMD, without
// scratch memory. Two waves with 1 to 28 registers spilled are faster: 32/8 heads of 128,
// 64K tokens over 8 ranks, window 1024, one pass 293-305 us and 213, two passes 336 and
// 234, where windows alone take 181 and 217; window 4096, 506 and 358, 537 and 368.)
template <int D, int HPW, int OUT, int KIND>
__global__ __launch_bounds__(256, D == 128 && (KIND & kScoreBias) ? 1 : 2) void attn_fwd_window_kernel(FwdParams p) {
  __shared__ __attribute__((aligned(16))) char smem[FwdLds<D, KIND>::bytes];
  fwd_tile<D, HPW, OUT, KIND>(p, smem);
}
template <int D, int HPW, int OUT, int KIND>
static void launch_fwd_kernel(const FwdParams& p, dim3 grid, hipStream_t s) {
  if constexpr (KIND & kWindow)
    hipLaunchKernelGGL((attn_fwd_window_kernel<D, HPW, OUT, KIND>), grid, dim3(256), 0, s, p);
  else if constexpr (KIND)
    hipLaunchKernelGGL((attn_fwd_scored_kernel<D, HPW, OUT, KIND>), grid, dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((attn_fwd_kernel<D, HPW, OUT>), grid, dim3(256), 0, s, p);
}

// The chunks as workgroups, then their merge.
template <int D, int HPW, int SC>
static hipError_t launch_units_t(const FwdParams& p, hipStream_t s) {
  launch_fwd_kernel<D, HPW, kOutUnit, SC>(p, dim3(unsigned(p.n_units) * p.hkv * p.head_chunks), s);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  return launch_fwd_combine(p, D, HPW, s);
}

// A partial pass of a split view in the view's own slots: after the last use
// of the slots (of each source it computes), before the next.
template <int D, int HPW, int SC>
static hipError_t launch_partial_units_t(const FwdParams& p, hipStream_t s) {
  std::unique_lock<std::mutex> lock[2];
  SlotGuard* used[2] = {p.o_f32 ? p.guard[0] : nullptr, p.o_f32_recv ? p.guard[1] : nullptr};
  for (int i = 0; i < 2; ++i) {
    SlotGuard* const g = used[i];
    if (!g) continue;
    lock[i] = std::unique_lock<std::mutex>(g->mu);
    if (const hipError_t e = g->wait(s); e != hipSuccess) return e;
  }
  if (const hipError_t e = launch_units_t<D, HPW, SC>(p, s); e != hipSuccess) return e;
  for (SlotGuard* g : used)
    if (g)
      if (const hipError_t e = g->used(s); e != hipSuccess) return e;
  return hipSuccess;
}

template <int D, int HPW, int SC>
static hipError_t launch_fwd_t(const FwdParams& p, int out, hipStream_t s) {
  if (out == kOutUnit)
    return p.o_bf16 ? launch_units_t<D, HPW, SC>(p, s) : launch_partial_units_t<D, HPW, SC>(p, s);
  const dim3 grid(unsigned(p.n_items) * p.hkv * p.head_chunks);
  if (out == kOutChunks)
    launch_fwd_kernel<D, HPW, kOutChunks, SC>(p, grid, s);
  else if (out == kOutFinal)
    launch_fwd_kernel<D, HPW, kOutFinal, SC>(p, grid, s);
  else if (out == kOutPaired)
    launch_fwd_kernel<D, HPW, kOutPaired, SC>(p, grid, s);
  else if (out == kOutMerged)
    launch_fwd_kernel<D, HPW, kOutMerged, SC>(p, grid, s);
  else
    launch_fwd_kernel<D, HPW, kOutPartial, SC>(p, grid, s);
  return hipGetLastError();
}

template <int D, int SC>
static hipError_t launch_fwd_d(const FwdParams& p, int hpw, int out, hipStream_t s) {
  switch (hpw) {
    case 1: return launch_fwd_t<D, 1, SC>(p, out, s);
    case 2: return launch_fwd_t<D, 2, SC>(p, out, s);
    case 4: return launch_fwd_t<D, 4, SC>(p, out, s);
    default: return hipErrorInvalidValue;
  }
}

// (one kind of view per source file)
template <int SC>
hipError_t launch_fwd_sc(const FwdParams& p, int d, int hpw, int out, hipStream_t s) {
  if (d == 64) return launch_fwd_d<64, SC>(p, hpw, out, s);
  if (d == 128) return launch_fwd_d<128, SC>(p, hpw, out, s);
  return hipErrorInvalidValue;
}

}  // namespace fck
