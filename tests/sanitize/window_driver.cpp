// Host driver of windowed views for the sanitizer build: views over random contexts,
// and every attention entry point on them, with stub launchers that walk what the
// kernels would read: each work item's key tiles, every row's window, every wave's rows.
// The "device" is host memory; tensors are addresses that nothing dereferences.
// (The launchers of host_driver.cpp check the tables' extents, under other names.)
#define launch_fwd stub_launch_fwd
#define launch_bwd_dq stub_launch_bwd_dq
#define launch_bwd stub_launch_bwd
#define launch_bwd_atomic stub_launch_bwd_atomic
#define launch_bwd_grid stub_launch_bwd_grid
#define main host_driver_main
#include "host_driver.cpp"
#undef main
#undef launch_fwd
#undef launch_bwd_dq
#undef launch_bwd
#undef launch_bwd_atomic
#undef launch_bwd_grid

namespace {
bool g_windowed = false;
int64_t g_gaps = 0;  // query tiles that leave out tiles between sinks and window

void check_rows(const int32_t* win, int32_t t_q) {
  CHECK((win != nullptr) == g_windowed);
  if (win) in_blob(win, 4 * int64_t(t_q), "windows");
}

// The key tiles of a query-major item's source, as the kernels take them.
void walk(const int32_t* it, const int32_t* win, int src, int32_t extent) {
  const int32_t base = it[src ? 2 : 4], end = it[src ? 3 : 5];
  const int32_t *a = win + 4 * it[0], *b = win + 4 * (it[1] - 1);
  CHECK(a[src] <= b[src] && a[2 + src] == b[2 + src]);
  const fck::KeyTiles t = fck::key_tiles(base, end, a[src], a[2 + src]);
  CHECK(t.head >= 0 && t.skip >= 0 && t.n >= t.head);
  if (t.head && t.skip) ++g_gaps;
  for (int32_t i = 0; i < t.n; ++i) {
    const int32_t k0 = base + 64 * t.at(i);
    CHECK(k0 >= base && k0 < end && end <= extent);
    CHECK(t.before(t.at(i)) == i && t.before(t.at(i) + 1) == i + 1);
  }
  CHECK(t.before(0) == 0 && t.before(1 << 24) == t.n);
}
template <class P>
void walk_items(const P& p, const int32_t* items, int32_t n, int32_t t_r) {
  check_rows(p.win, p.t_q);
  if (!p.win) return;
  for (int32_t i = 0; i < n; ++i) {
    const int32_t* it = items + 8 * i;
    CHECK(0 <= it[0] && it[0] < it[1] && it[1] <= p.t_q);
    walk(it, p.win, 0, p.t_q);
    walk(it, p.win, 1, t_r);
  }
}
int32_t g_t_r = 0;
void walk_keys(const fck::BwdParams& p) {
  check_rows(p.win, p.t_q);
  CHECK((p.wave_end != nullptr) == g_windowed);
  if (!p.win) return;
  in_blob(p.wave_end, 8 * int64_t(p.n_items), "waves' last rows");
  for (int32_t i = 0; i < p.n_items; ++i) {
    const int32_t* it = p.items + 8 * i;
    for (int w = 0; w < 4; ++w) {
      const int32_t cut = p.wave_end[8 * i + 2 * w], end = p.wave_end[8 * i + 2 * w + 1];
      CHECK(cut <= end && cut >= 0 && (end == fck::kAlways || end <= p.t_q));
    }
    CHECK(it[2] < it[3]);
  }
}
}  // namespace

namespace fck {
hipError_t launch_fwd(const FwdParams& p, int d, int hpt, bool final_out, hipStream_t s) {
  walk_items(p, p.items, p.n_items, p.t_r);
  walk_items(p, p.units, p.n_units, p.t_r);
  return stub_launch_fwd(p, d, hpt, final_out, s);
}
hipError_t launch_bwd_dq(const DqParams& p, int d, int hpt, hipStream_t s) {
  walk_items(p, p.items, p.n_items, g_t_r);
  return stub_launch_bwd_dq(p, d, hpt, s);
}
hipError_t launch_bwd(const BwdParams& p, int d, hipStream_t s) {
  walk_keys(p);
  return stub_launch_bwd(p, d, s);
}
hipError_t launch_bwd_atomic(const BwdParams& p, int d, hipStream_t s) {
  walk_keys(p);
  return stub_launch_bwd_atomic(p, d, s);
}
hipError_t launch_bwd_grid(const BwdParams& b, const DqParams& q, int d, int hpt, hipStream_t s) {
  walk_keys(b);
  walk_items(q, q.items, q.n_items, g_t_r);
  return stub_launch_bwd_grid(b, q, d, hpt, s);
}
}  // namespace fck

int main() {
  std::mt19937 rng(4242);
  std::vector<float> slopes(64, 0.25f);
  int windowed = 0, whole = 0;
  for (int c = 0; c < 240; ++c) {
    const int n = 1 + int(rng() % 12), cp = 1 + int(rng() % 6), top = c % 5 == 0 ? 12000 : 900;
    std::vector<int32_t> cu = {0};
    for (int j = 0; j < n; ++j) cu.push_back(cu.back() + 1 + int(rng() % unsigned(top)));
    const int shapes[5][3] = {{4, 4, 64}, {16, 2, 128}, {64, 8, 128}, {4, 1, 128}, {8, 8, 64}};
    const int* sh = shapes[c % 5];
    const fc_score score{c % 3 == 1 ? 30.f : 0.f, c % 4 == 3 ? slopes.data() : nullptr};
    const fc_window win{1 + int(rng() % unsigned(c % 2 ? 200 : 3000)), int(rng() % 3 ? rng() % 300 : 0)};
    const char* kinds[3] = {"per_doc", "whole_lpt", "per_doc"};
    const auto plan = plan_of(cu, cp, kinds[c % 3]);
    for (int r = 0; r < cp; ++r) {
      fc_view v = nullptr;
      CHECK(fc_view_create_windowed(cu.data(), n, plan.data(), int64_t(plan.size()), cp, r, sh[0], sh[1], sh[2],
                                    nullptr, &score, &win, &v) == FC_OK);
      fc_view_info i;
      CHECK(fc_view_get_info(v, &i) == FC_OK);
      int32_t on = -1, w = 0, k = -1;
      CHECK(fc_view_export_window(v, &on, nullptr, nullptr) == FC_OK);
      CHECK(fc_view_get_window(v, &w, &k) == FC_OK && w == win.window && k == win.sinks);
      std::vector<int32_t> a(size_t(i.t_q) * 4 + 1), b(size_t(i.n_bwd_launch) * 8 + 1);
      CHECK(fc_view_export_window(v, &on, a.data(), b.data()) == FC_OK);
      ++(on ? windowed : whole);
      g_windowed = on;
      g_t_r = i.t_recv;
      for (bool slots : {true, false}) {
        std::vector<char> blob(size_t(i.meta_bytes) + 256);
        char* base = blob.data() + ((256 - reinterpret_cast<uintptr_t>(blob.data()) % 256) % 256);
        const size_t bytes = size_t(slots ? i.meta_bytes : i.table_bytes);
        CHECK(fc_view_bind(v, base, bytes, nullptr) == FC_OK);
        g_blob = base;
        g_blob_bytes = bytes;
        size_t fws = 0, bws = 0, kws = 0;
        for (int mode : {FC_TWO_PASS, FC_FUSED}) {
          CHECK(fc_workspace_size(v, mode, &fws, &bws, &kws) == FC_OK);
          CHECK(fc_attn_fwd(v, D, D, D, D, D, 0.f, mode, D, Df, Df, D, fws, nullptr) == FC_OK);
        }
        CHECK(fc_attn_fwd(v, D, D, D, D, D, 0.f, FC_FUSED, D, Df, Df, nullptr, 0, nullptr) == FC_OK);
        CHECK(fc_attn_fwd_partials(v, D, D, D, D, D, 0.f, Df, Df, Df, Df, nullptr) == FC_OK);
        CHECK(fc_attn_fwd_partial(v, 0, D, D, D, 0.f, Df, Df, nullptr) == FC_OK);
        CHECK(fc_attn_fwd_partial(v, 1, D, D, D, 0.f, Df, Df, nullptr) == FC_OK);
        for (int det : {0, 1})
          CHECK(fc_attn_bwd(v, D, D, D, D, D, D, Df, Df, D, 0.f, det, Df, Df, Df, Df, Df, D, bws, nullptr) == FC_OK);
        CHECK(fc_attn_bwd_dkdv(v, D, D, D, D, D, Df, Df, D, 0.f, Df, Df, Df, Df, D, kws, nullptr) == FC_OK);
        CHECK(fc_attn_bwd_dq(v, D, D, D, D, D, Df, Df, D, 0.f, Df, nullptr) == FC_OK);
        CHECK(fc_kv_gather(v, D, D, cu.back(), D, D, D, D, nullptr) == FC_OK);
      }
      fc_view_destroy(v);
      g_blob = nullptr;
      g_blob_bytes = 0;
    }
  }
  CHECK(windowed > 100 && whole > 20 && g_gaps > 1000);
  // refused
  const int32_t cu[2] = {0, 10};
  const fc_shard plan[1] = {{0, 0, 0, 10}};
  for (fc_window bad : {fc_window{-1, 0}, fc_window{0, 1}, fc_window{4, -1}}) {
    fc_view v = reinterpret_cast<fc_view>(1);
    CHECK(fc_view_create_windowed(cu, 1, plan, 1, 1, 0, 4, 2, 64, nullptr, nullptr, &bad, &v) == FC_ERR_INVALID_ARG);
    CHECK(v == nullptr);
  }
  const fc_window ok{4, 1};
  CHECK(fc_view_create_windowed(cu, 1, plan, 1, 1, 0, 4, 2, 64, nullptr, nullptr, &ok, nullptr) == FC_ERR_INVALID_ARG);
  std::printf("window driver: all checks passed\n");
  return 0;
}
