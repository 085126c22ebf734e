// Host driver of scored views and rotary rows for the sanitizer build: the stubs and
// the view driver of host_driver.cpp, whose entry points here run on views with a
// score function, and the rotary entry points with a stub launcher that walks every
// table a kernel would read, as the kernel reads it. The "device" is host memory;
// tensors are addresses that nothing dereferences.
#define main host_driver_main
#include "host_driver.cpp"
#undef main

#include <cmath>
#include <limits>

#include "../../paper_2606_08476_amd/csrc/kernels/rope.hpp"

namespace {
fck::RopeParams g_rope;
int g_layout = -1;
bool g_in32 = false, g_out32 = false;
}  // namespace

namespace fck {
hipError_t launch_rope(const RopeParams& p, int d, int layout, bool in32, bool out32, hipStream_t) {
  CHECK(d == 64 || d == 128);
  CHECK(p.n_sets >= 0 && p.n_sets <= kRopeSets && p.pairs >= 0 && p.pairs <= d / 2);
  for (int i = 0; i < p.n_sets; ++i) {
    const RopeRows& s = p.set[i];
    CHECK(s.rows > 0 && s.heads > 0 && s.per_block >= 1 && s.per_block <= kRopeRows);
    CHECK((s.per_block & (s.per_block - 1)) == 0 && 64 % s.per_block == 0);
    CHECK(int64_t(s.blocks) * s.per_block >= s.rows && int64_t(s.blocks - 1) * s.per_block < s.rows);
    in_blob(s.gpos, s.rows, "positions");
    in_blob(s.first, (s.rows + 63) / 64, "first segments");
    // the kernel's walk from a row to its document
    for (int r = 0; r < s.rows; ++r) {
      int k = s.first[r / 64];
      for (;; ++k) {
        in_blob(p.seg + 4 * k, 4, "segments");
        if (r < p.seg[4 * k + s.end]) break;
      }
      CHECK(s.gpos[r] >= p.seg[4 * k + 2]);
      CHECK(k == 0 || r >= p.seg[4 * (k - 1) + s.end]);
    }
  }
  g_rope = p;
  g_layout = layout;
  g_in32 = in32;
  g_out32 = out32;
  ++g_launches;
  return hipSuccess;
}
}  // namespace fck

namespace {

struct Bound {
  fc_view v = nullptr;
  std::vector<char> blob;
  fc_view_info i{};
  Bound(const std::vector<int32_t>& cu, int cp, int rank, int hq, int hkv, int d,
        const fc_score* score = nullptr) {
    const auto plan = plan_of(cu, cp, "per_doc");
    CHECK(fc_view_create_scored(cu.data(), int32_t(cu.size()) - 1, plan.data(), int64_t(plan.size()), cp,
                                rank, hq, hkv, d, nullptr, score, &v) == FC_OK);
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

void rows() {
  const std::vector<int32_t> cu = {0, 300, 301, 1000};
  Bound b(cu, 2, 1, 4, 2, 64);
  const int64_t T = b.i.t_q, W = 8 * 64;  // a fused row: 4 + 2 + 2 heads
  Freqs f(64);
  // slices of a fused buffer into tensors of their own
  const uintptr_t F0 = 1 << 24, O = 1 << 28;
  fc_rows q{at(F0), W, at(O), 0}, k{at(F0 + 512), W, at(O + (1 << 24)), 0},
      v{at(F0 + 768), W, at(O + (2 << 24)), 0};
  CHECK(fc_rope_fwd(b.v, &f.r, &q, &k, &v, nullptr) == FC_OK);
  CHECK(g_rope.n_sets == 3 && g_layout == fck::kRopeHalves && !g_in32 && !g_out32);
  CHECK(g_rope.set[0].rotate && g_rope.set[1].rotate && !g_rope.set[2].rotate);
  CHECK(g_rope.set[1].in_stride == W && g_rope.set[1].out_stride == 128 && g_rope.sign == 1.f);
  // (half a turn per position is 2^63)
  const double half_turn = 3.14159265358979323846;
  fc_rope one{2, 1, 1, 1.f, &half_turn};
  CHECK(fc_rope_fwd(b.v, &one, &q, nullptr, nullptr, nullptr) == FC_OK && g_rope.packed_pos == 1);
  CHECK(g_layout == fck::kRopeNeighbours && g_rope.pairs == 1);
  CHECK(std::llabs(int64_t(g_rope.turn[0] - (uint64_t(1) << 63))) < 4096);
  const double back = -half_turn / 2;  // three quarters forwards
  one.inv_freq = &back;
  CHECK(fc_rope_fwd(b.v, &one, &q, nullptr, nullptr, nullptr) == FC_OK);
  CHECK(std::llabs(int64_t(g_rope.turn[0] - (uint64_t(3) << 62))) < 4096);
  Freqs six(6);
  CHECK(fc_rope_fwd(b.v, &six.r, &q, nullptr, nullptr, nullptr) == FC_OK &&
        g_layout == fck::kRopeHalvesOdd);
  // no rotation: copies
  CHECK(fc_rope_fwd(b.v, nullptr, &q, &k, nullptr, nullptr) == FC_OK && !g_rope.set[0].rotate);
  // in place, in a tensor and in the fused buffer
  fc_rows own{at(O), 0, at(O), 0}, fq{at(F0), W, at(F0), W}, fk{at(F0 + 512), W, at(F0 + 512), W};
  CHECK(fc_rope_fwd(b.v, &f.r, &own, nullptr, nullptr, nullptr) == FC_OK);
  CHECK(fc_rope_fwd(b.v, &f.r, &fq, &fk, nullptr, nullptr) == FC_OK);
  // refused
  const int64_t before = g_launches;
  auto fwd = [&](fc_rows a) { return fc_rope_fwd(b.v, &f.r, &a, nullptr, nullptr, nullptr); };
  CHECK(fc_rope_fwd(b.v, &f.r, nullptr, nullptr, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  CHECK(fwd({nullptr, 0, at(O), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(F0), 0, nullptr, 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(F0 + 8), 0, at(O), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(F0), 0, at(O + 2), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(F0), 255, at(O), 0}) == FC_ERR_INVALID_ARG);       // less than a row
  CHECK(fwd({at(F0), 260, at(O), 0}) == FC_ERR_INVALID_ARG);       // not 16 bytes
  CHECK(fwd({at(F0), -512, at(O), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(F0), int64_t(1) << 40, at(O), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(O), 0, at(O + 512), 0}) == FC_ERR_INVALID_ARG);    // a row further
  CHECK(fwd({at(O), 512, at(O), 0}) == FC_ERR_INVALID_ARG);        // another stride
  CHECK(fwd({at(O + 512), 0, at(O), 0}) == FC_ERR_INVALID_ARG);
  CHECK(fwd({at(O), 0, at(O + size_t(T) * 512 - 16), 0}) == FC_ERR_INVALID_ARG);
  fc_rows to_k{at(F0), W, at(F0 + 512), W};                        // queries over keys
  CHECK(fc_rope_fwd(b.v, &f.r, &to_k, &fk, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  fc_rows same{at(F0 + 512), W, at(O + 1024), 0};                  // two outputs in one place
  CHECK(fc_rope_fwd(b.v, &f.r, &q, &same, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  for (int dim : {0, 1, 3, 66, -2}) {
    fc_rope r = f.r;
    r.dim = dim;
    CHECK(fc_rope_fwd(b.v, &r, &q, nullptr, nullptr, nullptr) == FC_ERR_INVALID_ARG);
    CHECK(fc_kv_gather_rope(b.v, &r, D, D, 1000, at(O), at(O), at(O), at(O), nullptr) ==
          FC_ERR_INVALID_ARG);
  }
  for (double w : {std::nan(""), 1.0 / 0.0 * 1.0, 9.0, -9.0}) {
    Freqs g(64);
    g.w[31] = w;
    CHECK(fc_rope_fwd(b.v, &g.r, &q, nullptr, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  }
  fc_rope r = f.r;
  r.amplitude = std::nanf("");
  CHECK(fc_rope_fwd(b.v, &r, &q, nullptr, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  r = f.r;
  r.inv_freq = nullptr;
  CHECK(fc_rope_fwd(b.v, &r, &q, nullptr, nullptr, nullptr) == FC_ERR_INVALID_ARG);
  CHECK(g_launches == before);
  // outputs that end where an input begins are apart
  CHECK(fwd({at(O + size_t(T) * 512), 0, at(O), 0}) == FC_OK);
}

void gather() {
  const std::vector<int32_t> cu = {0, 300, 301, 1000};
  Bound b(cu, 2, 0, 4, 2, 64);
  Freqs f(32);
  CHECK(b.i.t_recv > 0);
  const uintptr_t K = 1 << 24, V = 2 << 24, A = 3 << 24, B = 4 << 24, C = 5 << 24, E = 6 << 24;
  auto go = [&](uintptr_t a, uintptr_t c, uintptr_t e, uintptr_t g, int64_t t = 1000) {
    return fc_kv_gather_rope(b.v, &f.r, at(K), at(V), t, at(a), at(c), at(e), at(g), nullptr);
  };
  CHECK(go(A, B, C, E) == FC_OK && g_rope.n_sets == 4);
  CHECK(g_rope.set[2].gather == g_rope.set[2].gpos && g_rope.set[2].end == 1);
  CHECK(go(A, B, 0, 0) == FC_OK && g_rope.n_sets == 2);
  CHECK(go(0, 0, C, E) == FC_OK && g_rope.n_sets == 2 && g_rope.set[0].end == 1);
  CHECK(fc_kv_gather_rope(b.v, nullptr, at(K), at(V), 1000, at(A), at(B), at(C), at(E), nullptr) == FC_OK &&
        !g_rope.set[0].rotate);
  const int64_t before = g_launches;
  CHECK(go(A, 0, C, E) == FC_ERR_INVALID_ARG && go(A, B, C, 0) == FC_ERR_INVALID_ARG);
  CHECK(go(0, 0, 0, 0) == FC_ERR_INVALID_ARG);
  CHECK(go(A, B, C, E, 10) == FC_ERR_SHAPE);
  CHECK(go(K, B, C, E) == FC_ERR_INVALID_ARG && go(A, V + 256, C, E) == FC_ERR_INVALID_ARG);
  CHECK(go(A, A, C, E) == FC_ERR_INVALID_ARG && go(A + 8, B, C, E) == FC_ERR_INVALID_ARG);
  CHECK(g_launches == before);
}

void gradients() {
  const std::vector<int32_t> cu = {0, 300, 301, 1000};
  Bound b(cu, 2, 1, 4, 2, 64);
  Freqs f(64, 1);
  const int64_t W = 8 * 64;
  const uintptr_t I = 1 << 24, O = 1 << 29;
  fc_rows dq{at(I), 0, at(O), W}, dk{at(I + (1 << 24)), 0, at(O + 512), W},
      dv{at(I + (2 << 24)), 0, at(O + 768), W}, rk{at(I + (3 << 24)), 0, at(O + (1 << 24)), 0},
      rv{at(I + (4 << 24)), 0, at(O + (2 << 24)), 0};
  CHECK(fc_rope_bwd(b.v, &f.r, 1, &dq, &dk, &dv, &rk, &rv, nullptr) == FC_OK);
  CHECK(g_rope.n_sets == 5 && g_in32 && !g_out32 && g_rope.sign == -1.f && !g_rope.set[2].rotate);
  // (fp32 rows are twice as wide: the same slices now overlap)
  CHECK(fc_rope_bwd(b.v, &f.r, 0, &dq, &dk, &dv, &rk, &rv, nullptr) == FC_ERR_INVALID_ARG);
  fc_rows place{at(I), 0, at(I), 0};
  CHECK(fc_rope_bwd(b.v, &f.r, 0, &place, nullptr, nullptr, nullptr, nullptr, nullptr) == FC_OK && g_out32);
  CHECK(fc_rope_bwd(b.v, &f.r, 1, &place, nullptr, nullptr, nullptr, nullptr, nullptr) ==
        FC_ERR_INVALID_ARG);
  CHECK(fc_rope_bwd(b.v, &f.r, 1, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) ==
        FC_ERR_INVALID_ARG);
}

// Every table walk, over random contexts, with a score function or without; and
// the attention entry points on scored views.
void views() {
  std::mt19937 rng(99);
  std::vector<float> slopes(64, 0.25f);
  for (int c = 0; c < 80; ++c) {
    const int n = 1 + int(rng() % 40), cp = 1 + int(rng() % 6);
    std::vector<int32_t> cu = {0};
    for (int j = 0; j < n; ++j) cu.push_back(cu.back() + (rng() % 3 == 0 ? 1 : 1 + int(rng() % 700)));
    const int shapes[3][3] = {{4, 4, 64}, {16, 2, 128}, {64, 8, 128}};
    const int* sh = shapes[c % 3];
    const fc_score score{c % 2 ? 30.f : 0.f, c % 4 < 2 ? slopes.data() : nullptr};
    for (int r = 0; r < cp; ++r) {
      Bound b(cu, cp, r, sh[0], sh[1], sh[2], &score);
      Freqs f(2 * (1 + int(rng() % (sh[2] / 2))));
      const uintptr_t G = uintptr_t(1) << 36;
      fc_rows q{at(G), 0, at(2 * G), 0}, k{at(3 * G), 0, at(4 * G), 0}, v{at(5 * G), 0, at(6 * G), 0};
      CHECK(fc_rope_fwd(b.v, &f.r, &q, &k, &v, nullptr) == FC_OK);
      CHECK(fc_kv_gather_rope(b.v, &f.r, at(G), at(2 * G), cu.back(), at(3 * G), at(4 * G), at(5 * G),
                              at(6 * G), nullptr) == FC_OK);
      size_t fws = 0, bws = 0;
      CHECK(fc_workspace_size(b.v, FC_TWO_PASS, &fws, &bws, nullptr) == FC_OK);
      CHECK(fc_attn_fwd(b.v, D, D, D, D, D, 0.f, FC_TWO_PASS, D, Df, Df, D, fws, nullptr) == FC_OK);
      for (int det : {0, 1})
        CHECK(fc_attn_bwd(b.v, D, D, D, D, D, D, Df, Df, D, 0.f, det, Df, Df, Df, Df, Df, D, bws,
                          nullptr) == FC_OK);
      float cap = -1;
      int32_t biased = -1;
      std::vector<float> got(size_t(sh[0]), -1.f);
      CHECK(fc_view_get_score(b.v, &cap, &biased, got.data()) == FC_OK);
      CHECK(cap == score.cap && biased == (score.slopes != nullptr) && got[0] == (biased ? 0.25f : 0.f));
    }
  }
}

}  // namespace

int main() {
  rows();
  gather();
  gradients();
  views();
  std::printf("rows driver: all checks passed\n");
  return 0;
}
