// Host driver of the head norms for the sanitizer build: the entry points on bound
// views, with stub launchers that walk every table and check every row and partial
// row a kernel would touch. The "device" is host memory; tensors are addresses that
// nothing dereferences.
#define main host_driver_main
#include "host_driver.cpp"
#undef main

#include <cmath>
#include <limits>

#include "../../paper_2606_08476_amd/csrc/kernels/norm.hpp"

namespace fck {
hipError_t launch_rope(const RopeParams&, int, int, bool, bool, hipStream_t) { return hipSuccess; }
}  // namespace fck

namespace {

struct Bound {
  fc_view v = nullptr;
  std::vector<char> blob;
  fc_view_info i{};
  Bound(const std::vector<int32_t>& cu, int cp, int rank, int hq, int hkv, int d) {
    const auto plan = plan_of(cu, cp, "per_doc");
    CHECK(fc_view_create(cu.data(), int32_t(cu.size()) - 1, plan.data(), int64_t(plan.size()), cp, rank, hq,
                         hkv, d, nullptr, &v) == FC_OK);
    CHECK(fc_view_get_info(v, &i) == FC_OK);
    blob.resize(size_t(i.meta_bytes) + 256);
    char* base = blob.data() + ((256 - reinterpret_cast<uintptr_t>(blob.data()) % 256) % 256);
    CHECK(fc_view_bind(v, base, size_t(i.meta_bytes), nullptr) == FC_OK);
    g_blob = base;
    g_blob_bytes = size_t(i.meta_bytes);
  }
  ~Bound() {
    fc_view_destroy(v);
    g_blob = nullptr;
    g_blob_bytes = 0;
  }
};

void* at(uintptr_t a) { return reinterpret_cast<void*>(a); }

struct Freqs {
  double w[64];
  fc_rope r;
  explicit Freqs(int dim, int inter = 0) {
    float amp = 0;
    CHECK(fc_rope_freqs(dim, 10000.0, FC_ROPE_NONE, 1, 1, 4, 0, w, &amp) == FC_OK && amp == 1.f);
    r = {dim, inter, 0, amp, w};
  }
};

fck::NormParams g_norm;
fck::NormSum g_sum[2];
int g_sliced = 0;  // sums in more than one slice
int g_norm_layout = -1;
bool g_back = false, g_out32 = false;
uintptr_t g_ws = 0;
size_t g_ws_bytes = 0;

void check_norm_sets(const fck::NormParams& p, int d, bool back) {
  CHECK(d == 64 || d == 128);
  CHECK(p.n_sets >= 0 && p.n_sets <= fck::kNormSets && p.pairs >= 0 && p.pairs <= d / 2);
  std::vector<char> seen(g_ws_bytes / 4, 0);  // floats of the workspace that are written
  for (int i = 0; i < p.n_sets; ++i) {
    const fck::NormRows& s = p.set[i];
    const int slots = 256 / fck::norm_lanes(d, back);
    CHECK(s.rows > 0 && s.heads > 0 && s.group_heads >= 1 && s.group_heads <= slots);
    CHECK(s.group_heads * s.head_groups >= s.heads && s.group_heads * (s.head_groups - 1) < s.heads);
    CHECK(s.step_rows >= 1 && s.step_rows <= fck::kNormRows && s.step_rows * s.group_heads <= slots);
    CHECK(s.per_block % s.step_rows == 0 && s.blocks % s.head_groups == 0);
    const int64_t nb = s.blocks / s.head_groups;
    CHECK(nb * s.per_block >= s.rows && (nb - 1) * s.per_block < s.rows);
    CHECK(s.per_block / s.step_rows <= 16);  // (the tests' bound of a weight's gradient)
    in_blob(s.gpos, s.rows, "positions");
    in_blob(s.first, (s.rows + 63) / 64, "first segments");
    for (int r = 0; r < s.rows; ++r) {
      int k = s.first[r / 64];
      for (;; ++k) {
        in_blob(p.seg + 4 * k, 4, "segments");
        if (r < p.seg[4 * k + s.end]) break;
      }
      CHECK(s.gpos[r] >= p.seg[4 * k + 2]);
    }
    if (!s.part) continue;
    CHECK(back && s.norm && s.part_width == (s.w_stride ? s.heads * d : d));
    const int64_t rows = s.w_stride ? nb : s.blocks;
    const uintptr_t a = reinterpret_cast<uintptr_t>(s.part);
    CHECK(a >= g_ws && a + size_t(rows * s.part_width) * 4 <= g_ws + g_ws_bytes);
    for (int64_t e = 0; e < rows * s.part_width; ++e) CHECK(!seen[(a - g_ws) / 4 + size_t(e)]++);
  }
}
}  // namespace

namespace fck {
hipError_t launch_norm_fwd(const NormParams& p, int d, int layout, hipStream_t) {
  check_norm_sets(p, d, false);
  g_norm = p;
  g_norm_layout = layout;
  g_back = false;
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_norm_bwd(const NormParams& p, int d, int layout, bool out32, hipStream_t) {
  check_norm_sets(p, d, true);
  g_norm = p;
  g_norm_layout = layout;
  g_out32 = out32;
  g_back = true;
  ++g_launches;
  return hipSuccess;
}
hipError_t launch_norm_sum(const NormSum& a, const NormSum& b, hipStream_t) {
  g_sum[0] = a;
  g_sum[1] = b;
  for (const NormSum& s : g_sum) {
    CHECK(s.width % kSumCols == 0 && s.n >= 0 && (!s.width || s.slices == norm_slices(s.n)));
    if (!s.width || !s.n) continue;
    const uintptr_t end = g_ws + g_ws_bytes;
    CHECK(reinterpret_cast<uintptr_t>(s.part) >= g_ws);
    if (s.slices > 1) {
      // the slices' rows lie behind all partial rows, and not in each other's
      const uintptr_t r = reinterpret_cast<uintptr_t>(s.rows), z = r + size_t(s.slices) * s.width * 8;
      for (const NormSum& o : {a, b})
        if (o.width) CHECK(r >= reinterpret_cast<uintptr_t>(o.part) + size_t(o.n) * o.width * 4);
      if (a.slices > 1 && b.slices > 1)
        CHECK(reinterpret_cast<uintptr_t>(b.rows) >= reinterpret_cast<uintptr_t>(a.rows) + size_t(a.slices) * a.width * 8);
      CHECK(r % 8 == 0 && z <= end);
      ++g_sliced;
    }
    // every partial row summed is one that the launch before has written
    const uintptr_t p0 = reinterpret_cast<uintptr_t>(s.part);
    int64_t rows = 0;
    for (int i = 0; i < g_norm.n_sets; ++i) {
      const NormRows& k = g_norm.set[i];
      const uintptr_t q = reinterpret_cast<uintptr_t>(k.part);
      if (k.part && q >= p0 && q < p0 + size_t(s.n) * s.width * 4)
        rows += k.w_stride ? k.blocks / k.head_groups : k.blocks;
    }
    CHECK(rows == s.n);
  }
  return hipSuccess;
}
}  // namespace fck

namespace {

const uintptr_t X = uintptr_t(1) << 36, Y = uintptr_t(2) << 36, Wt = uintptr_t(5) << 36, Ws = uintptr_t(6) << 36,
                Dw = uintptr_t(7) << 36;

void forward_calls() {
  const std::vector<int32_t> cu = {0, 300, 301, 1000};
  Bound b(cu, 2, 1, 4, 2, 64);
  const int64_t T = b.i.t_q, W = 8 * 64;
  Freqs f(64);
  fc_rows q{at(X), W, at(Y), 0}, k{at(X + 512), W, at(Y + (1 << 24)), 0}, v{at(X + 768), W, at(Y + (2 << 24)), 0};
  fc_norm n{at(Wt), 1, 0, 0, 0.f, 1e-6f};
  CHECK(fc_norm_rope_fwd(b.v, &f.r, &n, &n, &q, &k, &v, nullptr) == FC_OK);
  CHECK(g_norm.n_sets == 3 && g_norm.set[0].norm && g_norm.set[1].norm && !g_norm.set[2].norm);
  CHECK(!g_norm.set[2].rotate && g_norm.set[0].w_stride == 0 && g_norm.set[0].w_bf16);
  CHECK(fc_norm_rope_fwd(b.v, nullptr, &n, nullptr, &q, &k, nullptr, nullptr) == FC_OK);
  CHECK(!g_norm.set[0].rotate && !g_norm.set[1].norm);
  fc_norm ph{at(Wt + 4), 0, 1, 1, 1.f, 1e-5f};
  CHECK(fc_norm_rope_fwd(b.v, &f.r, &ph, &ph, &q, &k, nullptr, nullptr) == FC_OK);
  CHECK(g_norm.set[0].w_stride == 64 && g_norm.set[0].centred && g_norm.set[0].offset == 1.f);
  fc_norm none{nullptr, 0, 0, 0, 5.f, 1e-6f};
  CHECK(fc_norm_rope_fwd(b.v, &f.r, &none, &none, &q, &k, nullptr, nullptr) == FC_OK);
  // in place
  fc_rows own{at(Y), 0, at(Y), 0};
  CHECK(fc_norm_rope_fwd(b.v, &f.r, &n, nullptr, &own, nullptr, nullptr, nullptr) == FC_OK);
  const int64_t before = g_launches;
  auto with = [&](fc_norm x) { return fc_norm_rope_fwd(b.v, &f.r, &x, nullptr, &q, nullptr, nullptr, nullptr); };
  for (float e : {0.f, -1.f, 1e-30f, std::nanf(""), std::numeric_limits<float>::infinity()})
    CHECK(with({at(Wt), 0, 0, 0, 0.f, e}) == FC_ERR_INVALID_ARG);
  for (float o : {std::nanf(""), std::numeric_limits<float>::infinity()})
    CHECK(with({at(Wt), 0, 0, 0, o, 1e-6f}) == FC_ERR_INVALID_ARG);
  CHECK(with({at(Wt + 1), 1, 0, 0, 0.f, 1e-6f}) == FC_ERR_INVALID_ARG);
  CHECK(with({at(Wt + 2), 0, 0, 0, 0.f, 1e-6f}) == FC_ERR_INVALID_ARG);
  CHECK(with({at(Y + 512), 1, 0, 0, 0.f, 1e-6f}) == FC_ERR_INVALID_ARG);  // weights that are written over
  CHECK(with({at(Y + size_t(T) * 512 - 2), 1, 0, 0, 0.f, 1e-6f}) == FC_ERR_INVALID_ARG);
  auto fwd = [&](fc_rows a) { return fc_norm_rope_fwd(b.v, &f.r, &n, nullptr, &a, nullptr, nullptr, nullptr); };
  CHECK(fc_norm_rope_fwd(b.v, &f.r, &n, &n, nullptr, nullptr, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  CHECK(fwd({nullptr, 0, at(Y), 0}) == FC_ERR_INVALID_ARG && fwd({at(X), 0, nullptr, 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(X + 8), 0, at(Y), 0}) == FC_ERR_INVALID_ARG && fwd({at(X), 0, at(Y + 2), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(X), 255, at(Y), 0}) == FC_ERR_INVALID_ARG && fwd({at(X), 260, at(Y), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(X), -512, at(Y), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(X), int64_t(1) << 40, at(Y), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(Y), 0, at(Y + 512), 0}) == FC_ERR_INVALID_ARG);
  fc_rope r = f.r;
  r.dim = 66;
  CHECK(fc_norm_rope_fwd(b.v, &r, &n, nullptr, &q, nullptr, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  CHECK(fc_norm_rope_fwd(nullptr, &f.r, &n, nullptr, &q, nullptr, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  // the gather
  const uintptr_t K = 1 << 24, V = 2 << 24, A = 3 << 24, B = 4 << 24, C = 5 << 24, E = 6 << 24;
  Bound g(cu, 2, 0, 4, 2, 64);
  CHECK(g.i.t_recv > 0);
  const int64_t there = g_launches;
  auto go = [&](uintptr_t a, uintptr_t c, uintptr_t e, uintptr_t h, int64_t t = 1000) {
    return fc_kv_gather_norm_rope(g.v, &f.r, &n, at(K), at(V), t, at(a), at(c), at(e), at(h), nullptr);
  };
  CHECK(go(A, B, C, E) == FC_OK && g_norm.n_sets == 4 && g_norm.set[2].in_gather == g_norm.set[2].gpos);
  CHECK(g_norm.set[0].norm && !g_norm.set[1].norm && g_norm.set[2].norm && g_norm.set[2].end == 1);
  CHECK(go(A, B, 0, 0) == FC_OK && g_norm.n_sets == 2 && go(0, 0, C, E) == FC_OK && g_norm.n_sets == 2);
  CHECK(g_launches == there + 3 && there == before);
  CHECK(go(A, 0, C, E) == FC_ERR_INVALID_ARG && go(0, 0, 0, 0) == FC_ERR_INVALID_ARG);
  CHECK(go(A, B, C, E, 10) == FC_ERR_SHAPE && go(K, B, C, E) == FC_ERR_INVALID_ARG);
  CHECK(go(A, A, C, E) == FC_ERR_INVALID_ARG && go(A + 8, B, C, E) == FC_ERR_INVALID_ARG);
  n.eps = 0;
  CHECK(go(A, B, C, E) == FC_ERR_INVALID_ARG);
  CHECK(g_launches == there + 3);
}

void gradient_calls() {
  const std::vector<int32_t> cu = {0, 300, 301, 1000};
  Bound b(cu, 2, 1, 4, 2, 64);
  Freqs f(64, 1);
  const int64_t W = 8 * 64;
  const uintptr_t I = uintptr_t(3) << 36, O = uintptr_t(4) << 36;
  fc_rows dq{at(I), 0, at(O), W}, dk{at(I + (1 << 24)), 0, at(O + 512), W}, dv{at(I + (2 << 24)), 0, at(O + 768), W},
      rk{at(I + (3 << 24)), 0, at(O + (1 << 24)), 0}, rv{at(I + (4 << 24)), 0, at(O + (2 << 24)), 0};
  fc_norm n{at(Wt), 1, 0, 0, 0.f, 1e-6f}, m{at(Wt + 4096), 0, 1, 0, 0.f, 1e-6f};
  fc_norm_rows xq{at(X), W, 0}, xk{at(X + 512), W, 0}, xr{at(X + (1 << 24)), 0, 1000};
  size_t need = 0, none = 1;
  CHECK(fc_norm_rope_workspace(b.v, &n, &m, &need) == FC_OK && need > 0);
  CHECK(fc_norm_rope_workspace(b.v, nullptr, nullptr, &none) == FC_OK && none == 0);
  g_ws = Ws;
  g_ws_bytes = need;
  void *wq = at(Dw), *wk = at(Dw + 4096);
  auto go = [&](const fc_norm* qn, const fc_norm* kn, const fc_rows* a, const fc_rows* c, const fc_rows* e,
                const fc_norm_rows* i, const fc_norm_rows* j, const fc_norm_rows* l, void* u, void* w, void* ws,
                size_t bytes, int bf = 1) {
    return fc_norm_rope_bwd(b.v, &f.r, qn, kn, bf, a, c, &dv, e, &rv, i, j, l, u, w, ws, bytes, nullptr);
  };
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(Ws), need) == FC_OK);
  CHECK(g_norm.n_sets == 5 && g_norm.sign == -1.f && !g_out32 && g_norm.set[3].x_gather == g_norm.set[3].gpos);
  CHECK(!g_norm.set[1].x_gather && g_norm.set[1].x_stride == W && g_sum[0].bf16 && !g_sum[1].bf16);
  CHECK(g_sum[0].width == 64 && g_sum[1].width == 128 && g_sum[0].n > 0 && g_sum[1].n > 0);
  // gradients of one's weights, of none's; without a tensor of one
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, nullptr, at(Ws), need) == FC_OK && !g_sum[1].width);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, nullptr, wk, at(Ws), need) == FC_OK && !g_sum[0].width);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, nullptr, nullptr, nullptr, 0) == FC_OK && !g_norm.set[0].part);
  CHECK(go(&n, &m, nullptr, &dk, &rk, nullptr, &xk, &xr, wq, wk, at(Ws), need) == FC_OK);
  CHECK(g_sum[0].width == 64 && g_sum[0].n == 0);  // (zeros)
  CHECK(go(&n, &m, &dq, nullptr, nullptr, &xq, nullptr, nullptr, wq, nullptr, at(Ws), need) == FC_OK);
  CHECK(go(nullptr, nullptr, &dq, &dk, &rk, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, 0) == FC_OK);
  fc_rows place{at(I), 0, at(I), 0};
  CHECK(fc_norm_rope_bwd(b.v, &f.r, &n, nullptr, 0, &place, nullptr, nullptr, nullptr, nullptr, &xq, nullptr, nullptr,
                         nullptr, nullptr, nullptr, 0, nullptr) == FC_OK);
  // refused
  const int64_t before = g_launches;
  CHECK(go(&n, &m, &dq, &dk, &rk, nullptr, &xk, &xr, wq, wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  fc_norm_rows bad = xq;
  bad.in = nullptr;
  CHECK(go(&n, &m, &dq, &dk, &rk, &bad, &xk, &xr, wq, wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  bad = {at(X + 8), W, 0};
  CHECK(go(&n, &m, &dq, &dk, &rk, &bad, &xk, &xr, wq, wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  bad = {at(X), 252, 0};
  CHECK(go(&n, &m, &dq, &dk, &rk, &bad, &xk, &xr, wq, wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  bad = {at(X), 0, 10};
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &bad, wq, wk, at(Ws), need) == FC_ERR_SHAPE);
  bad = {at(O), W, 0};  // written over
  CHECK(go(&n, &m, &dq, &dk, &rk, &bad, &xk, &xr, wq, wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(Ws), 64) == FC_ERR_WORKSPACE);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, nullptr, need) == FC_ERR_WORKSPACE);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(Ws + 4), need) == FC_ERR_INVALID_ARG);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(O), need) == FC_ERR_INVALID_ARG);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(X), need) == FC_ERR_INVALID_ARG);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, at(Dw + 1), wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, at(Dw), at(Ws), need) == FC_ERR_INVALID_ARG);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, at(Wt), wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, at(Ws), wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  CHECK(go(nullptr, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  fc_norm bare{nullptr, 0, 0, 0, 0.f, 1e-6f}, zero = n;
  zero.eps = 0;
  CHECK(go(&bare, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  CHECK(go(&zero, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(Ws), need) == FC_ERR_INVALID_ARG);
  CHECK(fc_norm_rope_workspace(b.v, &zero, nullptr, &none) == FC_ERR_INVALID_ARG);
  CHECK(fc_norm_rope_workspace(nullptr, &n, nullptr, &none) == FC_ERR_INVALID_ARG);
  CHECK(go(&n, &m, &dq, &dk, &rk, &xq, &xk, &xr, wq, wk, at(Ws), need, 0) == FC_ERR_INVALID_ARG);  // fp32 slices overlap
  CHECK(g_launches == before);
}

// Row shares and workspaces over random contexts, heads and choices of tensors.
void shares() {
  std::mt19937 rng(7);
  for (int c = 0; c < 200; ++c) {
    const int n = 1 + int(rng() % 30), cp = 1 + int(rng() % 4), top = c % 10 == 0 ? 20000 : 500;
    std::vector<int32_t> cu = {0};
    for (int j = 0; j < n; ++j) cu.push_back(cu.back() + 1 + int(rng() % unsigned(top)));
    const int shapes[][3] = {{4, 4, 64}, {16, 2, 128}, {64, 8, 128}, {1, 1, 64}, {40, 5, 128}, {12, 3, 64},
                             {200, 100, 64}, {8, 1, 128}, {36, 36, 128}};
    const int* sh = shapes[c % 9];
    Bound b(cu, cp, int(rng() % unsigned(cp)), sh[0], sh[1], sh[2]);
    Freqs f(2 * (1 + int(rng() % (sh[2] / 2))));
    auto big = [](int i) { return at((uintptr_t(16) + i) << 36); };
    fc_norm qn{big(0), int(rng() % 2), int(rng() % 2), int(rng() % 2), 0.f, 1e-6f}, kn = qn;
    kn.weight = big(1);
    kn.per_head = int(rng() % 2);
    fc_rows r[5];
    for (int i = 0; i < 5; ++i) r[i] = {big(2 + i), 0, big(7 + i), 0};
    const fc_norm_rows xq{big(12), 0, 0}, xk{big(13), 0, 0}, xr{big(14), 0, cu.back()};
    size_t need = 0;
    CHECK(fc_norm_rope_workspace(b.v, &qn, &kn, &need) == FC_OK);
    g_ws = reinterpret_cast<uintptr_t>(big(15));
    g_ws_bytes = need;
    const unsigned some = 1 + rng() % 31, dw = rng() % 4;
    CHECK(fc_norm_rope_bwd(b.v, c % 3 ? &f.r : nullptr, &qn, &kn, c % 2, some & 1 ? &r[0] : nullptr,
                           some & 2 ? &r[1] : nullptr, some & 4 ? &r[2] : nullptr, some & 8 ? &r[3] : nullptr,
                           some & 16 ? &r[4] : nullptr, &xq, &xk, &xr, dw & 1 ? big(30) : nullptr,
                           dw & 2 ? big(31) : nullptr, big(15), need, nullptr) == FC_OK);
    CHECK(fc_norm_rope_fwd(b.v, c % 3 ? &f.r : nullptr, &qn, &kn, &r[0], &r[1], &r[2], nullptr) == FC_OK);
    CHECK(fc_kv_gather_norm_rope(b.v, &f.r, &kn, big(2), big(3), cu.back(), big(7), big(8), big(9), big(10),
                                 nullptr) == FC_OK);
  }
}

}  // namespace

int main() {
  forward_calls();
  gradient_calls();
  shares();
  CHECK(g_sliced > 20);
  std::printf("norm driver: all checks passed\n");
  return 0;
}
