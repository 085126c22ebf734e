// C ABI entry points of the head norms with the rotation: the rank's own rows, the KV
// gather, and gradients. As in rope.cpp, everything is validated on the host before
// the launch, which is asynchronous on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "../kernels/norm.hpp"
#include "internal.hpp"
#include "rows.hpp"
#include "view.hpp"

using fc::check_rope;
using fc::fail;
using fc::Span;
using fc::turns;
using fc::View;

namespace {

// One tensor of a call.
struct Set {
  const fc_rows* rows;
  int32_t heads;
  bool recv, rotate, gather;  // gather: rows.in is a packed tensor
  const fc_norm* norm;
  const fc_norm_rows* x;      // backward, normalised
  int dw;                     // 0 of the queries' weights, 1 of the keys', -1 none
};

constexpr int64_t kMostStride = int64_t(1) << 28;

int check_norm(const fc_norm* n) {
  if (!n) return FC_OK;
  if (!(std::isfinite(n->eps) && n->eps >= FC_NORM_EPS_MIN))
    return fail(FC_ERR_INVALID_ARG, "eps must be finite and at least FC_NORM_EPS_MIN");
  if (!std::isfinite(n->offset)) return fail(FC_ERR_INVALID_ARG, "offset is not finite");
  if (n->weight && reinterpret_cast<uintptr_t>(n->weight) % (n->w_bf16 ? 2 : 4))
    return fail(FC_ERR_INVALID_ARG, "weights must be aligned to their type");
  return FC_OK;
}

// Rows of the weights' gradients: values of one.
int64_t width_of(const View& v, const fc_norm& n, int32_t heads) {
  return n.per_head ? int64_t(heads) * v.d : v.d;
}

// How workgroups share a tensor's rows: kNormSteps steps each, fewer where the whole call
// would leave most of the card without work. (A backward's workgroup leaves a row of
// partial weight gradients. Of 16, 8, 4 and 2 steps, with the weights' sums: gradients of
// 64K tokens over 8 ranks, 32/8 heads of 128, 208, 196, 192 and 202 us; of 50K over 4, 16/8
// heads of 64, weights per head, fp32, 108, 102, 98 and 104; own rows of the former 44, 43,
// 41 and 43; a gather of 135K rows of 8x128 217, 205, 193 and 204.)
int64_t share(fck::NormRows& k, int32_t d, bool back, int32_t steps) {
  const int32_t slots = 256 / fck::norm_lanes(d, back);
  k.head_groups = (k.heads + slots - 1) / slots;
  k.group_heads = (k.heads + k.head_groups - 1) / k.head_groups;
  k.head_groups = (k.heads + k.group_heads - 1) / k.group_heads;
  k.step_rows = std::min(slots / k.group_heads, fck::kNormRows);
  k.per_block = k.step_rows * steps;
  const int64_t blocks = (int64_t(k.rows) + k.per_block - 1) / k.per_block;
  k.blocks = int32_t(blocks * k.head_groups);
  return blocks * k.head_groups;
}
void share_all(fck::NormParams& p, int32_t d, bool back) {
  for (int32_t steps = fck::kNormSteps;; steps /= 2) {
    int64_t total = 0;
    for (int i = 0; i < p.n_sets; ++i) total += share(p.set[i], d, back, steps);
    if (total >= 1024 || steps == 1) return;
  }
}
// Rows of partial weight gradients that a tensor's workgroups leave.
int64_t part_rows(const fck::NormRows& k) {
  return k.w_stride ? k.blocks / k.head_groups : k.blocks;
}

// The tensors' rows and heads, without their addresses: what share_all goes by.
void add_set(fck::NormParams& p, const View& v, const Set& s) {
  fck::NormRows& k = p.set[p.n_sets++];
  const int32_t* m = v.dev_meta;
  k.rows = s.recv ? v.t_recv() : v.t_q();
  k.heads = s.heads;
  k.end = s.recv;
  if (m) {
    k.gpos = m + (s.recv ? v.off.recv_gpos : v.off.q_gpos);
    k.first = m + (s.recv ? v.off.first_r : v.off.first_q);
  }
  if (s.norm) {
    k.norm = 1;
    k.centred = s.norm->centred != 0;
    k.weight = s.norm->weight;
    k.w_stride = s.norm->per_head ? v.d : 0;
    k.w_bf16 = s.norm->w_bf16 != 0;
    k.offset = s.norm->offset;
    k.eps = s.norm->eps;
  }
}

int check_stride(int64_t stride, int64_t width, int64_t size) {
  if (stride < width || stride > kMostStride || stride * size % 16)
    return fail(FC_ERR_INVALID_ARG, "row strides must hold a row and be a multiple of 16 bytes");
  return FC_OK;
}

// Behind the partial rows, if there are many: the sums of their slices.
int64_t slice_bytes(int64_t rows, int64_t width) {
  const int32_t n = fck::norm_slices(rows);
  return n > 1 ? n * width * int64_t(sizeof(double)) : 0;
}

struct Weights {  // of a backward call
  void* dw[2];
  const fc_norm* norm[2];
  void* ws;
  size_t ws_bytes;
};

// The workspace of a backward call on these tensors: bytes of the queries' partial
// rows, and of the keys' behind them.
void part_sizes(const fck::NormParams& p, const std::initializer_list<Set>& sets, const View& v,
                int64_t (&rows)[2], int64_t (&bytes)[2]) {
  rows[0] = rows[1] = bytes[0] = bytes[1] = 0;
  int i = 0;
  for (const Set& s : sets) {
    if (!s.rows || !(s.recv ? v.t_recv() : v.t_q())) continue;
    const fck::NormRows& k = p.set[i++];
    if (s.dw < 0 || !s.norm) continue;
    rows[s.dw] += part_rows(k);
    bytes[s.dw] += part_rows(k) * width_of(v, *s.norm, s.heads) * int64_t(sizeof(float));
  }
}

// Validates the sets (null rows: skipped) and launches them together.
int run(const View& v, const fc_rope* rope, std::initializer_list<Set> sets, bool back, bool out_f32,
        const Weights* w, void* stream) {
  if (int rc = check_rope(rope, v.d)) return rc;
  fck::NormParams p{};
  // what is read (each tensor's rows, and a backward's x), and written
  Span in[fck::kNormSets], x[fck::kNormSets], out[fck::kNormSets];
  const int64_t isz = back ? 4 : 2, osz = out_f32 ? 4 : 2;
  bool given = false;
  for (const Set& s : sets) {
    if (!s.rows) continue;
    given = true;
    if (int rc = check_norm(s.norm)) return rc;
    const int32_t n = s.recv ? v.t_recv() : v.t_q();
    if (n == 0) continue;
    const fc_rows& r = *s.rows;
    if (!r.in || !r.out) return fail(FC_ERR_INVALID_ARG, "null tensor pointer");
    if (reinterpret_cast<uintptr_t>(r.in) % 16 || reinterpret_cast<uintptr_t>(r.out) % 16)
      return fail(FC_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
    const int64_t wd = int64_t(s.heads) * v.d;
    const int64_t is = r.in_stride ? r.in_stride : wd, os = r.out_stride ? r.out_stride : wd;
    if (int rc = check_stride(is, wd, isz)) return rc;
    if (int rc = check_stride(os, wd, osz)) return rc;
    const int i = p.n_sets;
    add_set(p, v, s);
    fck::NormRows& k = p.set[i];
    k.in = r.in;
    k.out = r.out;
    k.in_stride = is;
    k.out_stride = os;
    k.rotate = rope && s.rotate;
    const std::vector<int32_t>& gpos = s.recv ? v.recv_gpos : v.q_gpos;
    in[i] = {reinterpret_cast<uintptr_t>(r.in), is * isz, wd * isz, n};
    if (s.gather) {
      k.in_gather = k.gpos;
      in[i].rows = gpos.back() + 1;
    }
    out[i] = {reinterpret_cast<uintptr_t>(r.out), os * osz, wd * osz, n};
    x[i] = {0, 0, 0, 0};
    if (back && s.norm) {
      if (!s.x || !s.x->in) return fail(FC_ERR_INVALID_ARG, "the normalised rows are needed");
      if (reinterpret_cast<uintptr_t>(s.x->in) % 16)
        return fail(FC_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
      const int64_t xs = s.x->stride ? s.x->stride : wd;
      if (int rc = check_stride(xs, wd, 2)) return rc;
      k.x = s.x->in;
      k.x_stride = xs;
      x[i] = {reinterpret_cast<uintptr_t>(s.x->in), xs * 2, wd * 2, n};
      if (s.x->packed) {
        if (gpos.back() >= s.x->packed)
          return fail(FC_ERR_SHAPE, "a packed tensor has " + std::to_string(s.x->packed) +
                                        " rows, the view reads row " + std::to_string(gpos.back()));
        k.x_gather = k.gpos;
        x[i].rows = gpos.back() + 1;
      }
    }
  }
  if (!given) return fail(FC_ERR_INVALID_ARG, "no rows given");
  share_all(p, v.d, back);
  // weights' gradients: their partial rows, their slices' sums, and they themselves
  int64_t rows[2], bytes[2], width[2] = {0, 0};
  part_sizes(p, sets, v, rows, bytes);
  Span more[3];  // dw, dw, workspace
  int n_more = 0;
  if (back) {
    const int32_t heads[2] = {v.hq, v.hkv};
    int64_t need = 0;
    for (int i = 0; i < 2; ++i) {
      if (!w->dw[i]) {
        rows[i] = bytes[i] = 0;
        continue;
      }
      if (!w->norm[i] || !w->norm[i]->weight)
        return fail(FC_ERR_INVALID_ARG, "a gradient of weights without weights");
      if (int rc = check_norm(w->norm[i])) return rc;
      if (reinterpret_cast<uintptr_t>(w->dw[i]) % (w->norm[i]->w_bf16 ? 2 : 4))
        return fail(FC_ERR_INVALID_ARG, "weights must be aligned to their type");
      width[i] = width_of(v, *w->norm[i], heads[i]);
      const int64_t n = width[i] * (w->norm[i]->w_bf16 ? 2 : 4);
      more[n_more++] = {reinterpret_cast<uintptr_t>(w->dw[i]), n, n, 1};
      need += bytes[i] + slice_bytes(rows[i], width[i]);
    }
    if (need) {
      if (!w->ws || int64_t(w->ws_bytes) < need)
        return fail(FC_ERR_WORKSPACE, "workspace of " + std::to_string(w->ws ? w->ws_bytes : 0) +
                                          " bytes, need " + std::to_string(need));
      if (reinterpret_cast<uintptr_t>(w->ws) % 16)
        return fail(FC_ERR_INVALID_ARG, "tensor and workspace pointers must be 16-byte aligned");
      more[n_more++] = {reinterpret_cast<uintptr_t>(w->ws), need, need, 1};
    }
  }
  for (int i = 0; i < p.n_sets; ++i)
    for (int j = 0; j < p.n_sets; ++j) {
      const bool in_place = i == j && !p.set[i].in_gather && isz == osz && in[i].same(out[i]);
      if ((!in_place && in[i].touches(out[j])) || x[i].touches(out[j]) ||
          (i < j && out[i].touches(out[j])))
        return fail(FC_ERR_INVALID_ARG, "rows written overlap rows of another tensor");
    }
  for (int i = 0; i < n_more; ++i) {
    for (int j = 0; j < p.n_sets; ++j)
      if (more[i].touches(in[j]) || more[i].touches(x[j]) || more[i].touches(out[j]))
        return fail(FC_ERR_INVALID_ARG, "rows written overlap rows of another tensor");
    for (int j = 0; j < i; ++j)
      if (more[i].touches(more[j]))
        return fail(FC_ERR_INVALID_ARG, "weights' gradients or workspace overlap");
  }
  for (int i = 0; i < p.n_sets; ++i) {  // (nothing is written where a workgroup may still read weights)
    const fck::NormRows& k = p.set[i];
    if (!k.weight) continue;
    const int64_t n = (k.w_stride ? int64_t(k.heads) * v.d : v.d) * (k.w_bf16 ? 2 : 4);
    const Span ws{reinterpret_cast<uintptr_t>(k.weight), n, n, 1};
    for (int j = 0; j < p.n_sets; ++j)
      if (ws.touches(out[j])) return fail(FC_ERR_INVALID_ARG, "rows written overlap the weights");
    for (int j = 0; j < n_more; ++j)
      if (ws.touches(more[j])) return fail(FC_ERR_INVALID_ARG, "weights' gradients or workspace overlap");
  }
  fck::NormSum sum[2] = {};
  if (back) {
    char* at = static_cast<char*>(w->ws);
    float* part[2];
    for (int i = 0; i < 2; ++i) {
      part[i] = reinterpret_cast<float*>(at);
      at += bytes[i];
    }
    for (int i = 0; i < 2; ++i)
      if (w->dw[i]) {
        sum[i] = {part[i], int32_t(rows[i]), int32_t(width[i]), w->dw[i], w->norm[i]->w_bf16 != 0,
                  fck::norm_slices(rows[i]), reinterpret_cast<double*>(at)};
        at += slice_bytes(rows[i], width[i]);
      }
    int i = 0;
    for (const Set& s : sets) {
      if (!s.rows || !(s.recv ? v.t_recv() : v.t_q())) continue;
      fck::NormRows& k = p.set[i++];
      if (s.dw < 0 || !s.norm || !w->dw[s.dw]) continue;
      k.part_width = int32_t(width[s.dw]);
      k.part = part[s.dw];
      part[s.dw] += part_rows(k) * k.part_width;
    }
  }
  p.amplitude = 1.f;
  p.sign = back ? -1.f : 1.f;
  p.seg = v.dev_meta + v.off.seg;
  int layout = fck::kRopeHalves;
  if (rope) {
    p.pairs = rope->dim / 2;
    p.packed_pos = rope->packed_pos != 0;
    p.amplitude = rope->amplitude;
    turns(rope->inv_freq, p.pairs, p.turn);
    layout = rope->interleaved ? fck::kRopeNeighbours
             : p.pairs % 8     ? fck::kRopeHalvesOdd
                               : fck::kRopeHalves;
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  hipError_t e = back ? fck::launch_norm_bwd(p, v.d, layout, out_f32, st) : fck::launch_norm_fwd(p, v.d, layout, st);
  if (e == hipSuccess && back) e = fck::launch_norm_sum(sum[0], sum[1], st);
  if (e != hipSuccess) return fail(FC_ERR_HIP, std::string("norm launch: ") + hipGetErrorString(e));
  return FC_OK;
}

int bound(fc_view view, const View*& v) {
  if (!view) return fail(FC_ERR_INVALID_ARG, "view is null");
  v = reinterpret_cast<const View*>(view);
  if (!v->dev_meta) return fail(FC_ERR_WORKSPACE, "view is not bound to device metadata");
  return FC_OK;
}

}  // namespace

extern "C" {

int fc_norm_rope_fwd(fc_view view, const fc_rope* rope, const fc_norm* q_norm, const fc_norm* k_norm,
                     const fc_rows* q, const fc_rows* k, const fc_rows* v, void* stream) {
  if (!q_norm && !k_norm) return fc_rope_fwd(view, rope, q, k, v, stream);
  fc::clear_error();
  const View* w;
  if (int rc = bound(view, w)) return rc;
  return run(*w, rope,
             {{q, w->hq, false, true, false, q_norm, nullptr, -1},
              {k, w->hkv, false, true, false, k_norm, nullptr, -1},
              {v, w->hkv, false, false, false, nullptr, nullptr, -1}},
             false, false, nullptr, stream);
}

int fc_kv_gather_norm_rope(fc_view view, const fc_rope* rope, const fc_norm* k_norm, const void* k_packed,
                           const void* v_packed, int64_t t_packed, void* k_loc, void* v_loc, void* k_recv,
                           void* v_recv, void* stream) {
  if (!k_norm)
    return fc_kv_gather_rope(view, rope, k_packed, v_packed, t_packed, k_loc, v_loc, k_recv, v_recv, stream);
  fc::clear_error();
  const View* w;
  if (int rc = bound(view, w)) return rc;
  if (int rc = check_rope(rope, w->d)) return rc;
  if (int rc = check_norm(k_norm)) return rc;
  if (w->t_q() + w->t_recv() == 0) return FC_OK;
  // a part whose two outputs are both NULL is skipped
  const bool loc = k_loc || v_loc, rcv = k_recv || v_recv;
  if (!k_packed || !v_packed || (loc && (!k_loc || !v_loc)) || (rcv && (!k_recv || !v_recv)))
    return fail(FC_ERR_INVALID_ARG, "null tensor pointer");
  if (!loc && !rcv) return fail(FC_ERR_INVALID_ARG, "nothing to gather: every output is null");
  int64_t max_pos = -1;
  if (loc && w->t_q()) max_pos = std::max<int64_t>(max_pos, w->q_gpos.back());
  if (rcv && w->t_recv()) max_pos = std::max<int64_t>(max_pos, w->recv_gpos.back());
  if (max_pos >= t_packed)
    return fail(FC_ERR_SHAPE, "packed K/V have " + std::to_string(t_packed) +
                                  " rows, the view reads row " + std::to_string(max_pos));
  const fc_rows kl{k_packed, 0, k_loc, 0}, vl{v_packed, 0, v_loc, 0}, kr{k_packed, 0, k_recv, 0},
      vr{v_packed, 0, v_recv, 0};
  return run(*w, rope,
             {{loc ? &kl : nullptr, w->hkv, false, true, true, k_norm, nullptr, -1},
              {loc ? &vl : nullptr, w->hkv, false, false, true, nullptr, nullptr, -1},
              {rcv ? &kr : nullptr, w->hkv, true, true, true, k_norm, nullptr, -1},
              {rcv ? &vr : nullptr, w->hkv, true, false, true, nullptr, nullptr, -1}},
             false, false, nullptr, stream);
}

int fc_norm_rope_workspace(fc_view view, const fc_norm* q_norm, const fc_norm* k_norm, size_t* bytes) {
  fc::clear_error();
  if (!view || !bytes) return fail(FC_ERR_INVALID_ARG, "null argument");
  const View& v = *reinterpret_cast<const View*>(view);
  if (int rc = check_norm(q_norm)) return rc;
  if (int rc = check_norm(k_norm)) return rc;
  // the most that any choice of the tensors takes: a tensor's rows are shared among at
  // most as many workgroups with fewer others beside it (share_all)
  *bytes = 0;
  const Set each[3] = {{nullptr, v.hq, false, true, false, q_norm, nullptr, 0},
                       {nullptr, v.hkv, false, true, false, k_norm, nullptr, 1},
                       {nullptr, v.hkv, true, true, false, k_norm, nullptr, 1}};
  int64_t rows[2] = {0, 0}, width[2] = {0, 0};
  for (const Set& s : each) {
    if (!s.norm || !(s.recv ? v.t_recv() : v.t_q())) continue;
    fck::NormParams p{};
    add_set(p, v, s);
    share_all(p, v.d, true);
    rows[s.dw] += part_rows(p.set[0]);
    width[s.dw] = width_of(v, *s.norm, s.heads);
  }
  for (int i = 0; i < 2; ++i)
    *bytes += size_t(rows[i] * width[i] * int64_t(sizeof(float)) + slice_bytes(rows[i], width[i]));
  return FC_OK;
}

int fc_norm_rope_bwd(fc_view view, const fc_rope* rope, const fc_norm* q_norm, const fc_norm* k_norm,
                     int32_t out_bf16, const fc_rows* dq, const fc_rows* dk_loc, const fc_rows* dv_loc,
                     const fc_rows* dk_recv, const fc_rows* dv_recv, const fc_norm_rows* q_in,
                     const fc_norm_rows* k_in, const fc_norm_rows* k_recv_in, void* dw_q, void* dw_k, void* ws,
                     size_t ws_bytes, void* stream) {
  if (!q_norm && !k_norm && !dw_q && !dw_k)
    return fc_rope_bwd(view, rope, out_bf16, dq, dk_loc, dv_loc, dk_recv, dv_recv, stream);
  fc::clear_error();
  const View* w;
  if (int rc = bound(view, w)) return rc;
  const Weights weights{{dw_q, dw_k}, {q_norm, k_norm}, ws, ws_bytes};
  return run(*w, rope,
             {{dq, w->hq, false, true, false, q_norm, q_in, 0},
              {dk_loc, w->hkv, false, true, false, k_norm, k_in, 1},
              {dv_loc, w->hkv, false, false, false, nullptr, nullptr, -1},
              {dk_recv, w->hkv, true, true, false, k_norm, k_recv_in, 1},
              {dv_recv, w->hkv, true, false, false, nullptr, nullptr, -1}},
             true, !out_bf16, &weights, stream);
}

}  // extern "C"
