#pragma once
// Backward attention, dQ part (gfx950), query-major.
//
// Same work items and schedule as the fused forward: one workgroup takes a
// tile of query tokens of one piece for `heads_per_tile` query heads of one
// KV head, and walks the received key range (no mask) and then the local key
// range (intra-document causal). Key/value tiles of 64 keys are
// double-buffered in LDS (asynchronous HBM-to-LDS copies) and shared by the
// waves, i.e. by the heads of the group. Per tile, with a query per lane:
//   S^T = K Q^T, dP^T = V dO^T      Q and dO held in registers;
//   P = exp(S - LSE), dS = P (dP - D)  LSE and D are per-lane scalars;
//   dQ^T += K^T dS^T                 K^T read from LDS with transpose reads.
// dQ is produced whole by the workgroup that owns the query rows, so it is
// written once, without atomics, and is deterministic. Recomputing S and dP
// here costs two extra products per key tile compared with accumulating dQ
// inside the key-major kernel, but removes that kernel's dQ traffic and
// frees the registers and LDS that limit its occupancy.
//
// Scored views (SC, see score.hpp): S becomes the score before the exponential; with
// a cap, P (r - r^2) takes P's place in dS (its 4 is in the final scale), which
// needs no register more. A bias takes the keys' positions from LDS, put there per
// tile by the first wave, less the position of the workgroup's first row: its rows
// follow each other in the document, so a row's own share of the bias is at most 127
// slopes, wherever the document's rows lie. (Counted from the document's start its
// rounding alone, half a step of slope x position, takes P out of fp32's range: at a
// slope of 1024, from a million and a half tokens on.)
//
// Windowed views (WIN, see score.hpp) take the forward's tiles. A short window's P are
// large, and dQ is a difference of a few large terms: with dS as bf16 alone it is off by
// 0.0024 to 0.0036 of its root mean square (as against 64 bits), with the residuals of
// the halves that have a P above 1/16 by 0.0017 to 0.0024, at 226 -> 235 us (32/8 heads
// of 128, 8193 rows of 64K tokens over 8 ranks, window 1024). 16K rows, window 4096:
// 1205-1230 us.
#include "common.hpp"
#include "launch.hpp"
#include "score.hpp"

#include <type_traits>

namespace fck {

template <int D, int KIND = 0>
struct DqLds {
  // two K and two V tiles; with a bias the positions of two tiles' keys; windowed, those
  // of the rows
  static constexpr uint32_t bytes =
      4 * 64 * D * 2 + ((KIND & kScoreBias) ? 2 * 256 : 0) + ((KIND & kWindow) ? kWindowLds : 0);
};

// One workgroup's query tile (workgroup index b); smem: DqLds<D>::bytes of
// shared memory. HOLD: sixteen registers hold -D for dP's accumulators.
template <int D, int HPW, bool HOLD, int KIND = 0>
__device__ __forceinline__ void dq_tile(const DqParams& p, int b, char* smem) {
  constexpr int SC = KIND & kScores;
  constexpr bool WIN = KIND & kWindow, LEAN = KIND != 0;
  constexpr bool CAP = SC & kScoreCap, BIAS = SC & kScoreBias;
  constexpr int BN = 64;
  constexpr int RPW = 32 / HPW;  // query rows per wave and head
  constexpr int KS = D / 16;
  constexpr int DB = D / 32;
  constexpr uint32_t TILE = BN * D * 2;  // bytes of one K or V tile
  // LDS: K0 | V0 | K1 | V1 (double buffer); the loop is unrolled by two so
  // every read names its buffer with a compile-time offset
  constexpr uint32_t OP = 4 * TILE;  // BIAS: key positions
  constexpr uint32_t OW = OP + (BIAS ? 512 : 0);  // WIN: the rows' windows
  static_assert(OW + (WIN ? kWindowLds : 0) == DqLds<D, KIND>::bytes, "LDS layout");

  const int lane = threadIdx.x & 63, wave = wave_id();
  const int half = lane >> 5;
  int rest;
  const int kvh = kv_head<BIAS>(p, b, p.n_items * p.head_chunks, rest);
  const int hc = rest % p.head_chunks;
  const int32_t* it = p.items + 8 * (rest / p.head_chunks);
  const int q0 = it[0], q1 = it[1], r1 = it[3], l1 = it[5];
  int r0 = it[2], l0 = it[4];
  const int ldiag = it[6];

  // lane -> (query row, head) as in the forward: RPW rows of each of the
  // HPW heads per wave; a wave with no row skips the products
  const int l31 = lane & 31;
  const int h = kvh * p.group + hc * HPW + l31 / RPW;
  const int qrow = q0 + wave * RPW + l31 % RPW;
  const bool qvalid = qrow < q1;
  const bool active = q0 + wave * RPW < q1;  // wave-uniform
  const float sl2 = CAP ? p.cap_in : p.scale * kLog2e;
  const float gscale = CAP ? 4.f * p.scale : p.scale;

  int n_r = 0, n_t = 0;
  WindowTiles wt{};
  auto ranges = [&]() {
    if constexpr (WIN) wt = window_tiles(p.win, q0, q1, r0, r1, l0, l1);
    n_r = WIN ? wt.recv.n : (r1 - r0 + BN - 1) / BN;
    n_t = n_r + (WIN ? wt.local.n : (l1 - l0 + BN - 1) / BN);
  };
  ranges();
  if constexpr (WIN) put_window(smem + OW, 32 * wave + l31, p.win, min(qrow, q1 - 1));
  auto tile_at = [&](int j) {  // first key of the j-th tile taken
    const bool rs = j < n_r;
    const int t = rs ? j : j - n_r;
    return (rs ? r0 : l0) + (WIN ? (rs ? wt.recv : wt.local).at(t) : t) * BN;
  };
  const TileLoader<D, BN, 256, BN, LEAN> ld(p.hkv * D);
  // BIAS: position of the workgroup's first row, from which positions are counted here;
  // those of the next tile's keys go through a register of the first wave, a key per lane
  const float pos0 = BIAS ? p.q_pos[q0] : 0.f;
  float key_pos = 0.f;
  auto fetch = [&](int j, uint32_t kofs) {
    const bool rs = j < n_r;
    const int k0 = tile_at(j);
    const int hi = rs ? r1 : l1;
    const size_t base = (size_t(k0) * p.hkv + kvh) * D;
    ld.load_at(lds_addr(smem) + kofs, (rs ? p.k_recv : p.k_loc) + base, hi - k0);
    ld.load_at(lds_addr(smem) + kofs + TILE, (rs ? p.v_recv : p.v_loc) + base, hi - k0);
    if (BIAS && wave == 0)
      key_pos = ((rs ? p.recv_pos : p.q_pos) + k0)[min(int(fresh_lane()), hi - k0 - 1)];
  };
  auto put_pos = [&](uint32_t kofs) {
    if (BIAS && wave == 0)
      *reinterpret_cast<float*>(smem + OP + kofs / (2 * TILE / 256) + 4 * fresh_lane()) = key_pos - pos0;
  };

  const float cap2 = p.cap2, slope2 = BIAS ? p.slopes[h] : 0.f;

  // the workgroup's Q and dO rows through LDS first (Q over the second K/V
  // buffer, dO over the first), then key tile 0
  const int h0 = kvh * p.group + hc * HPW;
  load_pairs<D, RPW>(lds_addr(smem) + 2 * TILE, p.q, q0, q1, p.hq, h0);
  load_pairs<D, RPW>(lds_addr(smem), p.dout, q0, q1, p.hq, h0);

  bf16x8 qreg[KS], oreg[KS];
  float lse2 = 0.f, ndel = 0.f;
  if (qvalid) {
    lse2 = p.lse[(size_t)h * p.t_q + qrow] * kLog2e;
    ndel = -p.delta[(size_t)h * p.t_q + qrow];
  }
  // SC: the row's share of its scores less its LSE; what rounding it left out scales
  // every P of the row alike, and so its dQ
  // (row_scale, from values read again: not held across the loop)
  float off2 = CAP ? cap2 - lse2 : -lse2;
  if constexpr (BIAS) {
    float rest;
    off2 = row_offset(off2, slope2, p.q_pos[min(qrow, q1 - 1)] - pos0, rest);
  }

  // per-lane LDS byte offsets: K/V rows for k-step ks, and the two transpose
  // reads of K^T block db
  uint32_t pr[KS], pt[DB][2];
  {
    const int rb = row_base<D>(0, lane), tb = tr_base<D>(lane);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) pr[ks] = 2u * uint32_t(rb ^ (ks << 4));
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      pt[db][0] = 2u * uint32_t(tb ^ (db << 5));
      pt[db][1] = 2u * uint32_t((tb ^ ((db << 5) | 16)) + 8 * D);
    }
  }

  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = zero16();
  wait_async();
  __syncthreads();
  if (active) {
    const int qb = row_base<D>(32 * wave, lane);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qreg[ks] = lds_b128(smem, 2u * uint32_t(qb ^ (ks << 4)), 2 * TILE);
      oreg[ks] = lds_b128(smem, 2u * uint32_t(qb ^ (ks << 4)), 0);
    }
  }
  if (BIAS && p.norms) {
    // the ranges start, whole tiles on, at the first key within reach of a row of the
    // workgroup, given its LSE
    float n2 = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        n2 = __builtin_fmaf(active ? (float)qreg[ks][j] : 0.f, active ? (float)qreg[ks][j] : 0.f, n2);
    n2 = sum_halves(n2);
    const float qn = __builtin_sqrtf(n2 == n2 ? n2 : INFINITY), c = p.scale * kLog2e;
    const float bl = score_bound<SC>(c, qn, head_norm(p.norms, p.hq + kvh), cap2);
    const float br = score_bound<SC>(c, qn, head_norm(p.norms, p.hq + p.hkv + kvh), cap2);
    const float at = p.q_pos[min(qrow, q1 - 1)];
    skip_far<BN>(smem + OP, p.recv_pos, p.q_pos, qvalid ? at - reach(br - lse2, slope2) : INFINITY,
                 qvalid ? at - reach(bl - lse2, slope2) : INFINITY, r0, r1, l0, l1);
    ranges();
  }
  __syncthreads();  // every wave holds its rows before tile 0 overwrites them
  if (n_t > 0) {
    fetch(0, 0);
    put_pos(0);
  }
  wait_async();
  __syncthreads();

  // One key tile. Its MFMAs run as one software pipeline of slots:
  //   S^T, keys 0-31; S^T, keys 32-63 (with P of keys 0-31); dP^T, keys 0-31
  //   (with P of keys 32-63); dP^T, keys 32-63 (with dS of keys 0-31);
  //   dQ^T += K^T dS^T over keys 0-31 (with dS of keys 32-63), then 32-63.
  // Each slot issues the LDS reads of the slot two ahead, its MFMA and its
  // share of the vector work, which runs while the MFMA does; a scheduling
  // barrier after each slot keeps this order.
  constexpr int NS = 4 * KS + 4 * DB;        // slots per tile
  constexpr int EP = 16 / KS, EQ = 8 / DB;   // elements per slot (P, dS)
  constexpr int INIT0 = KS - 2, INIT1 = HOLD ? KS - 1 : 3 * KS - 2;  // of dP, see below
  auto step = [&](int j, auto buf) {
    constexpr uint32_t KO = decltype(buf)::value * 2 * TILE, VO = KO + TILE;
    if (j + 1 < n_t) fetch(j + 1, 2 * TILE - KO);
    const bool rs = j < n_r;
    const int k0 = tile_at(j);
    const int hi = rs ? r1 : l1;
    if (active) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) pr[ks] = opaque(pr[ks]);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        pt[db][0] = opaque(pt[db][0]);
        pt[db][1] = opaque(pt[db][1]);
      }
      // key k0 + 4*half + c (c = 32*mb + 8*(i/4) + i%4 for register i) is seen
      // iff c < rel: keys past the range, and later keys on diagonal tiles,
      // give P = 0. Only edge tiles (diagonal, or running past the range)
      // mask, in one branch before each half's dS.
      const bool diag = !rs && k0 >= ldiag;
      const int ln = LEAN ? int(fresh_lane()) : lane, hf = LEAN ? ln >> 5 : half;
      const int qr = LEAN ? q0 + wave * RPW + (ln & 31) % RPW : qrow;
      const int rel = (diag ? min(hi, qr + 1) : hi) - k0 - 4 * hf;
      const int sink = rs ? wt.sink_r : wt.sink_l;
      const bool edge = diag || k0 + BN > hi || (WIN && k0 < (rs ? wt.last_r : wt.last_l) && k0 + BN > sink);

      f32x16 s[2] = {zero16(), zero16()}, dp[2];
      bf16x8 ring[3], sb[4];
      auto rd = [&](int n) {
        bf16x8& a = ring[n % 3];
        if (n < 4 * KS) {  // K rows (S) or V rows (dP)
          const int ks = n % KS, mb = (n / KS) & 1;
          a = lds_b128(smem, pr[ks], (n < 2 * KS ? KO : VO) + mb * 64 * D);
        } else {  // K^T for dQ
          const int u = n - 4 * KS, kk = u / DB, db = u % DB;
          const uint32_t ro = KO + kk * 32 * D;
          a = cat8(lds_tr(smem, pt[db][0], ro), lds_tr(smem, pt[db][1], ro));
        }
      };
      // BIAS: positions of the EP keys of a slot's exponentials, read a slot ahead
      typedef float posv __attribute__((ext_vector_type(EP)));
      posv kp[2];
      auto rd_pos = [&](int t) {
        const int e = t % KS * EP;
        if (BIAS && t >= 0 && t < 2 * KS)
          kp[t & 1] = *reinterpret_cast<const posv*>(
              smem + OP + decltype(buf)::value * 256 + 16 * hf +
              4 * (32 * (t / KS) + 8 * (e / 4) + e % 4));
      };
      auto pexp = [&](int mb, int i) {
        float off = off2;
        if constexpr (BIAS) off = __builtin_fmaf(slope2, kp[(mb * KS + i / EP) & 1][i % EP], off);
        if constexpr (CAP) {
          float w;
          const float r = cap_r<0>(s[mb][i], sl2, w);
          s[mb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(r, -2.f * cap2, off)) * w;
          asm volatile("" : "+v"(s[mb][i]));  // here, not beyond the mask's branch with u and r kept
        } else {
          s[mb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mb][i], sl2, off));
        }
      };
      auto mask = [&](int mb) {
        if (WIN && edge) {  // seen: in the window, or a sink
          const int from = *reinterpret_cast<const int*>(smem + OW + 8 * (32 * wave + (ln & 31)) + (rs ? 4 : 0)) -
                           k0 - 4 * hf;
          const uint32_t seen = seen_keys(rel, from, sink - k0 - 4 * hf);
#pragma unroll
          for (int i = 0; i < 16; ++i) s[mb][i] = seen & (1u << (16 * mb + i)) ? s[mb][i] : 0.f;
        } else if (edge) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[mb][i] = 32 * mb + 8 * (i >> 2) + (i & 3) < rel ? s[mb][i] : 0.f;
        }
      };
      // dP's accumulators start from -D, as in the dK/dV workgroups (whose dS
      // has the same bits). With HOLD (head dim 64) sixteen registers hold it
      // for the first MFMA; at 128 there is no room for them, and the
      // accumulators are set: the first 32 keys' beside the first S products,
      // which have no other vector work, the others' two slots before they are
      // read (set together with the first, sixteen registers live through eight
      // more slots cost the grid a spill; either is as fast). Two registers per
      // move, named here (the compiler would write two moves); volatile, so that
      // they stay slots ahead of the MFMA that reads them. Layer of 16/8 heads of 64 over 32K
      // tokens: 349 -> 342 us (120 instead of 152 vector instructions beside 24
      // MFMAs); at 128, within noise.
      auto dp_init = [&](int mb) {
        if constexpr (HOLD) {
#pragma unroll
          for (int i = 0; i < 16; ++i) dp[mb][i] = ndel;
        } else {
          typedef uint64_t u64x8 __attribute__((ext_vector_type(8)));
          const uint32_t x = __builtin_bit_cast(uint32_t, ndel);
          u64x8 y;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            uint64_t r;
            asm volatile("v_mov_b64 %0, %1" : "=v"(r) : "v"(uint64_t(x) << 32 | x));
            y[i] = r;
          }
          dp[mb] = __builtin_bit_cast(f32x16, y);
        }
      };
      float pmax = 0.f;  // WIN: of the half's P (capped: times a quarter of 1 - tanh^2)
      auto dsv = [&](int mb, int i) {
        if (WIN) pmax = fmaxf(pmax, s[mb][i]);
        dp[mb][i] *= s[mb][i];
      };
      // WIN: where any P of a half tile is above 1/16, the bf16 residuals of its dS go
      // through the product too, as in dK/dV
      auto residual = [&](int mb) {
        if (!__any(pmax > (CAP ? 1.f / 64 : 1.f / 16))) return;
        const bf16x8 lo[2] = {lo8(dp[mb], 0, sb[2 * mb]), lo8(dp[mb], 8, sb[2 * mb + 1])};
        bf16x8 op[2];
        auto rk = [&](int m) {
          const uint32_t ro = KO + (2 * mb + m / DB) * 32 * D;
          op[m % 2] = cat8(lds_tr(smem, pt[m % DB][0], ro), lds_tr(smem, pt[m % DB][1], ro));
        };
        rk(0);
        static_for<0, 2 * DB>([&](auto mc) {
          constexpr int m = decltype(mc)::value;
          if (m + 1 < 2 * DB) rk(m + 1);
          dq[m % DB] = mfma32(op[m % 2], lo[m / DB], dq[m % DB]);
          __builtin_amdgcn_sched_barrier(0);
        });
      };
      rd(0);
      rd(1);
      static_for<0, NS>([&](auto nc) {
        constexpr int n = decltype(nc)::value;
        if (n + 2 < NS) rd(n + 2);
        rd_pos(n + 1 - KS);
        const bf16x8& a = ring[n % 3];
        if (n < 2 * KS) {
          const int ks = n % KS, mb = n / KS;
          s[mb] = mfma32(a, qreg[ks], s[mb]);
          if (n == INIT0) dp_init(0);
          if (n == INIT1) dp_init(1);
          if (mb == 1)
#pragma unroll
            for (int e = ks * EP; e < (ks + 1) * EP; ++e) pexp(0, e);
        } else if (n < 4 * KS) {
          const int ks = n % KS, mb = (n - 2 * KS) / KS;
          dp[mb] = mfma32(a, oreg[ks], dp[mb]);
          if (n == INIT1) dp_init(1);
          if (mb == 1 && ks == 0) mask(0);
          if (mb == 0) {
#pragma unroll
            for (int e = ks * EP; e < (ks + 1) * EP; ++e) pexp(1, e);
          } else {
#pragma unroll
            for (int e = ks * EP; e < (ks + 1) * EP; ++e) dsv(0, e);
            if ((ks + 1) * EP == 8) sb[0] = pack8(dp[0], 0);
            if ((ks + 1) * EP == 16) sb[1] = pack8(dp[0], 8);
            if (WIN && ks == KS - 1) {
              residual(0);
              pmax = 0.f;
            }
          }
        } else {
          const int u = n - 4 * KS, kk = u / DB, db = u % DB;
          dq[db] = mfma32(a, sb[kk], dq[db]);
          if (u == 0) mask(1);
          if (u < 2 * DB) {
#pragma unroll
            for (int e = u * EQ; e < (u + 1) * EQ; ++e) dsv(1, e);
            if ((u + 1) * EQ == 8) sb[2] = pack8(dp[1], 0);
            if ((u + 1) * EQ == 16) sb[3] = pack8(dp[1], 8);
            if (WIN && u == 2 * DB - 1) residual(1);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    }
    if (j + 1 < n_t) put_pos(2 * TILE - KO);
    wait_async();
    __syncthreads();
  };
  for (int j = 0; j < n_t; j += 2) {
    step(j, std::integral_constant<int, 0>());
    if (j + 1 < n_t) step(j + 1, std::integral_constant<int, 1>());
  }

  auto row_scale = [&](float f) {
    if constexpr (BIAS) {
      const int l = int(opaque(uint32_t(lane)) & 31), r = min(q0 + wave * RPW + l % RPW, q1 - 1);
      const int hh = kvh * p.group + hc * HPW + l / RPW;
      const float l2 = p.lse[(size_t)hh * p.t_q + r] * kLog2e;
      float rest;
      row_offset(CAP ? cap2 - l2 : -l2, p.slopes[hh], p.q_pos[r] - pos0, rest);
      f *= __builtin_amdgcn_exp2f(rest);
    }
    return f;
  };
  // a part of a split key range: the unscaled sums go to the part's slot, in
  // register order (1 KiB per store instruction), and are added up by
  // dq_combine_kernel
  if (p.part && it[7] >= 0) {
    if (active) {
      const size_t slot = (size_t(it[7]) * p.head_chunks + hc) * p.hkv + kvh;
      float* const sl = p.part + (slot * 4 + wave) * (32 * D) + 4 * lane;
      const float f = row_scale(1.f);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 v;
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) v[jj] = BIAS ? f * dq[db][4 * g + jj] : dq[db][4 * g + jj];
          *reinterpret_cast<f32x4*>(sl + 256 * (4 * db + g)) = v;
        }
    }
    return;
  }

  // dQ rows out through this wave's share of the (now free) K/V buffers,
  // 1 KiB per store instruction
  const float rscale = row_scale(gscale);
  store_rows<D, RPW>(
      smem + size_t(wave) * (32 * D * 4), active,
      [&](int db, int g) {
        f32x4 v;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) v[jj] = rscale * dq[db][4 * g + jj];
        return v;
      },
      q0 + wave * RPW, q1, p.hq, kvh * p.group + hc * HPW, p.dq, nullptr);
}

}  // namespace fck
