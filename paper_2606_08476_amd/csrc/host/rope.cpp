// C ABI entry points of the rotary rows: frequencies, the rank's own rows, the KV
// gather with rotated keys, and gradients. As in api.cpp, everything is validated
// on the host before the launch, which is asynchronous on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "../kernels/rope.hpp"
#include "internal.hpp"
#include "view.hpp"

using fc::fail;
using fc::View;

namespace {

// One tensor of a call: where its rows come from and go to.
struct Set {
  const fc_rows* rows;
  int32_t heads;
  bool recv, rotate, gather;
};

// A range of rows in memory, in bytes.
struct Span {
  uintptr_t base;
  int64_t stride, width, rows;
  uintptr_t end() const { return base + uintptr_t((rows - 1) * stride + width); }
  bool same(const Span& o) const { return base == o.base && stride == o.stride; }
  // whether any row of one touches a row of the other (slices of one buffer, rows
  // the same stride apart, touch where their columns do)
  bool touches(const Span& o) const {
    if (!rows || !o.rows || end() <= o.base || o.end() <= base) return false;
    if (stride != o.stride) return true;
    // columns from a row's start here to the start of the other's next row
    const int64_t ahead = o.base >= base ? int64_t(o.base - base) % stride
                                         : (stride - int64_t(base - o.base) % stride) % stride;
    return ahead < width || ahead + o.width > stride;
  }
};

int check_rope(const fc_rope* r, int32_t d) {
  if (!r) return FC_OK;
  if (r->dim < 2 || r->dim > d || r->dim % 2)
    return fail(FC_ERR_INVALID_ARG, "rotated values must be even and from 2 to the head dim");
  if (!r->inv_freq) return fail(FC_ERR_INVALID_ARG, "inv_freq is null");
  if (!std::isfinite(r->amplitude)) return fail(FC_ERR_INVALID_ARG, "amplitude is not finite");
  for (int32_t i = 0; i < r->dim / 2; ++i)
    if (!(std::fabs(r->inv_freq[i]) <= FC_ROPE_FREQ_MAX))
      return fail(FC_ERR_INVALID_ARG, "inv_freq must be within FC_ROPE_FREQ_MAX");
  return FC_OK;
}

// Radians per position as turns modulo 1, 64-bit fixed point (|w| is within
// FC_ROPE_FREQ_MAX, checked before).
uint64_t turns(double w) {
  constexpr long double kPerTurn = 0.15915494309189533576888376337251436L;
  const long double t = w * kPerTurn;
  const long double f = t - static_cast<int>(t);  // of w's sign, exact
  return static_cast<uint64_t>(static_cast<int64_t>(f * 9223372036854775808.0L)) << 1;
}

// Validates the sets (null rows: skipped) and launches them together.
int run(const View& v, const fc_rope* rope, std::initializer_list<Set> sets, bool in_f32,
        bool out_f32, bool back, void* stream) {
  if (int rc = check_rope(rope, v.d)) return rc;
  fck::RopeParams p{};
  Span in[fck::kRopeSets], out[fck::kRopeSets];
  const int64_t isz = in_f32 ? 4 : 2, osz = out_f32 ? 4 : 2;
  bool given = false;
  int64_t total = 0;  // workgroups at the most rows each
  for (const Set& s : sets) {
    if (!s.rows) continue;
    given = true;
    const int32_t n = s.recv ? v.t_recv() : v.t_q();
    if (n == 0) continue;
    const fc_rows& r = *s.rows;
    if (!r.in || !r.out) return fail(FC_ERR_INVALID_ARG, "null tensor pointer");
    if (reinterpret_cast<uintptr_t>(r.in) % 16 || reinterpret_cast<uintptr_t>(r.out) % 16)
      return fail(FC_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
    const int64_t w = int64_t(s.heads) * v.d, most = int64_t(1) << 28;
    const int64_t is = r.in_stride ? r.in_stride : w, os = r.out_stride ? r.out_stride : w;
    if (is < w || os < w || is > most || os > most || is * isz % 16 || os * osz % 16)
      return fail(FC_ERR_INVALID_ARG, "row strides must hold a row and be a multiple of 16 bytes");
    fck::RopeRows& k = p.set[p.n_sets];
    const int32_t* m = v.dev_meta;
    k.in = r.in;
    k.out = r.out;
    k.in_stride = is;
    k.out_stride = os;
    k.gpos = m + (s.recv ? v.off.recv_gpos : v.off.q_gpos);
    k.gather = s.gather ? k.gpos : nullptr;
    k.first = m + (s.recv ? v.off.first_r : v.off.first_q);
    k.end = s.recv;
    k.rows = n;
    k.heads = s.heads;
    k.rotate = rope && s.rotate;
    in[p.n_sets] = {reinterpret_cast<uintptr_t>(r.in), is * isz, w * isz, n};
    if (s.gather) {
      const std::vector<int32_t>& g = s.recv ? v.recv_gpos : v.q_gpos;
      in[p.n_sets].rows = g.back() + 1;
    }
    out[p.n_sets] = {reinterpret_cast<uintptr_t>(r.out), os * osz, w * osz, n};
    ++p.n_sets;
  }
  if (!given) return fail(FC_ERR_INVALID_ARG, "no rows given");
  for (int i = 0; i < p.n_sets; ++i)
    for (int j = 0; j < p.n_sets; ++j) {
      const bool in_place = i == j && !p.set[i].gather && isz == osz && in[i].same(out[i]);
      if ((!in_place && in[i].touches(out[j])) || (i < j && out[i].touches(out[j])))
        return fail(FC_ERR_INVALID_ARG, "rows written overlap rows of another tensor");
    }
  // rows per workgroup: four units per thread, fewer where the whole
  // call would leave most of the card without work
  auto blocks_of = [&](int64_t units) {
    total = 0;
    for (int i = 0; i < p.n_sets; ++i) {
      fck::RopeRows& k = p.set[i];
      const int64_t hu = int64_t(k.heads) * fck::rope_units(v.d, in_f32);
      int32_t per = 1;
      while (per < fck::kRopeRows && 2 * per * hu <= units) per *= 2;
      k.per_block = per;
      k.blocks = (k.rows + per - 1) / per;
      k.step_t = int32_t(256 / hu);
      k.step_q = int32_t(256 % hu);
      total += k.blocks;
    }
    return total;
  };
  for (int64_t units = 1024; blocks_of(units) < 1024 && units > 256;) units /= 2;
  p.amplitude = 1.f;
  p.sign = back ? -1.f : 1.f;
  p.seg = v.dev_meta + v.off.seg;
  int layout = fck::kRopeHalves;
  if (rope) {
    p.pairs = rope->dim / 2;
    p.packed_pos = rope->packed_pos != 0;
    p.amplitude = rope->amplitude;
    for (int32_t i = 0; i < p.pairs; ++i) p.turn[i] = turns(rope->inv_freq[i]);
    layout = rope->interleaved ? fck::kRopeNeighbours
             : p.pairs % 8     ? fck::kRopeHalvesOdd
                               : fck::kRopeHalves;
  }
  const hipError_t e = fck::launch_rope(p, v.d, layout, in_f32, out_f32,
                                        reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(FC_ERR_HIP, std::string("rope launch: ") + hipGetErrorString(e));
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

int fc_rope_freqs(int32_t dim, double base, int32_t scaling, double factor, double low, double high,
                  double context, double* inv_freq, float* amplitude) {
  fc::clear_error();
  if (!inv_freq || !amplitude) return fail(FC_ERR_INVALID_ARG, "null argument");
  if (dim < 2 || dim % 2 || dim > 128)
    return fail(FC_ERR_INVALID_ARG, "rotated values must be even and from 2 to 128");
  if (!(base > 1 && std::isfinite(base))) return fail(FC_ERR_INVALID_ARG, "base must be above 1");
  if (scaling < FC_ROPE_NONE || scaling > FC_ROPE_YARN)
    return fail(FC_ERR_INVALID_ARG, "unknown scaling");
  if (scaling != FC_ROPE_NONE && !(factor >= 1 && std::isfinite(factor)))
    return fail(FC_ERR_INVALID_ARG, "factor must be 1 or more");
  const bool by_turns = scaling == FC_ROPE_BANDS || scaling == FC_ROPE_YARN;
  if (by_turns && !(low > 0 && high > low && std::isfinite(high) && context > 0 && std::isfinite(context)))
    return fail(FC_ERR_INVALID_ARG, "need 0 < low < high and a trained context");
  if (scaling == FC_ROPE_BASE) {
    if (dim == 2) return fail(FC_ERR_INVALID_ARG, "one pair has no base to scale");
    base *= std::pow(factor, double(dim) / (dim - 2));
  }
  constexpr double kTurn = 6.283185307179586;
  // the pair, as a real number, that makes n turns in the trained context
  auto pair_of = [&](double n) { return dim * std::log(context / (n * kTurn)) / (2 * std::log(base)); };
  double first = 0, last = 0;
  if (scaling == FC_ROPE_YARN) {
    first = std::max(std::floor(pair_of(high)), 0.0);
    last = std::min(std::ceil(pair_of(low)), double(dim - 1));
  }
  for (int32_t i = 0; i < dim / 2; ++i) {
    const double w = std::pow(base, -2.0 * i / dim);
    double keep = 1;  // share of w; the rest is w / factor
    if (scaling == FC_ROPE_LINEAR) keep = 0;
    if (scaling == FC_ROPE_BANDS) keep = (context * w / kTurn - low) / (high - low);
    if (scaling == FC_ROPE_YARN) keep = 1 - (i - first) / std::max(last - first, 1e-3);
    keep = std::min(std::max(keep, 0.0), 1.0);
    inv_freq[i] = scaling == FC_ROPE_NONE || scaling == FC_ROPE_BASE ? w : w * keep + w / factor * (1 - keep);
  }
  *amplitude = scaling == FC_ROPE_YARN ? float(0.1 * std::log(factor) + 1) : 1.f;
  return FC_OK;
}

int fc_rope_fwd(fc_view view, const fc_rope* rope, const fc_rows* q, const fc_rows* k,
                const fc_rows* v, void* stream) {
  fc::clear_error();
  const View* w;
  if (int rc = bound(view, w)) return rc;
  return run(*w, rope, {{q, w->hq, false, true, false}, {k, w->hkv, false, true, false},
                        {v, w->hkv, false, false, false}},
             false, false, false, stream);
}

int fc_kv_gather_rope(fc_view view, const fc_rope* rope, const void* k_packed, const void* v_packed,
                      int64_t t_packed, void* k_loc, void* v_loc, void* k_recv, void* v_recv,
                      void* stream) {
  fc::clear_error();
  const View* w;
  if (int rc = bound(view, w)) return rc;
  if (int rc = check_rope(rope, w->d)) return rc;
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
  return run(*w, rope, {{loc ? &kl : nullptr, w->hkv, false, true, true},
                        {loc ? &vl : nullptr, w->hkv, false, false, true},
                        {rcv ? &kr : nullptr, w->hkv, true, true, true},
                        {rcv ? &vr : nullptr, w->hkv, true, false, true}},
             false, false, false, stream);
}

int fc_rope_bwd(fc_view view, const fc_rope* rope, int32_t out_bf16, const fc_rows* dq,
                const fc_rows* dk_loc, const fc_rows* dv_loc, const fc_rows* dk_recv,
                const fc_rows* dv_recv, void* stream) {
  fc::clear_error();
  const View* w;
  if (int rc = bound(view, w)) return rc;
  return run(*w, rope, {{dq, w->hq, false, true, false}, {dk_loc, w->hkv, false, true, false},
                        {dv_loc, w->hkv, false, false, false}, {dk_recv, w->hkv, true, true, false},
                        {dv_recv, w->hkv, true, false, false}},
             true, !out_bf16, true, stream);
}

}  // extern "C"
