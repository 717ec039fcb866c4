// plan_check.cpp for the scoring calls: PLAN_CHECK is a copy of it whose backward is vp_score_backward
// and whose main is plan_check_main.  Adds the scoring forward: that every chunk's tiles cover the
// shards, that partial states and maxima lie inside the workspace, apart from each other, and that
// the chunks' outputs follow one another.
#include PLAN_CHECK

static std::vector<vpce::ScoreArgs> scored;
static std::vector<vpce::ScoreCombArgs> joined_tokens;
static std::vector<vpce::TopArgs> tops;

namespace vpce {
bool run_score(int, const ScoreArgs& a, hipStream_t) {
  scored.push_back(a);
  return true;
}
bool run_score_comb(int, const ScoreCombArgs& a, const ScoreArgs&, hipStream_t) {
  joined_tokens.push_back(a);
  return true;
}
bool run_top(int, const TopArgs& a, hipStream_t) {
  tops.push_back(a);
  return true;
}
}  // namespace vpce

static bool check_score(const vp_problem& p, int top) {
  scored.clear();
  joined_tokens.clear();
  tops.clear();
  const bool f8 = p.dtype == VP_E4M3;
  const int64_t eb = (int64_t)elem_bytes(p.dtype), nb = ceil_div(p.d, 128);
  const vp_score score{top};
  size_t bytes = 0;
  CHECK(vp_score_workspace_size(&p, &score, &bytes) == VP_OK);
  char* ws = (char*)(1ll << 44);
  const char* H = (const char*)(2ll << 44);
  const uint8_t* hs = (const uint8_t*)(6ll << 44);
  float *loss = (float*)(7ll << 44), *lse = loss + (1 << 26), *entropy = lse + (1 << 26);
  int64_t* ids = (int64_t*)(8ll << 44);
  float* top_loss = (float*)(9ll << 44);
  std::vector<const void*> W(p.P);
  std::vector<const uint8_t*> scales(p.P);
  for (int q = 0; q < p.P; ++q) {
    W[q] = (const void*)((4ll << 44) + ((int64_t)q << 38));
    scales[q] = (const uint8_t*)((5ll << 44) + ((int64_t)q << 38));
  }
  const int64_t* targets = (const int64_t*)(10ll << 44);
  CHECK((f8 ? vp_score_forward_f8(&p, &score, H, hs, W.data(), scales.data(), targets, loss, lse, entropy, ids, top_loss,
                                  ws, bytes, nullptr)
            : vp_score_forward(&p, &score, H, W.data(), targets, loss, lse, entropy, ids, top_loss, ws, bytes,
                               nullptr)) == VP_OK);
  const bool maxima = top || f8;
  CHECK(!scored.empty() && tops.size() == (maxima ? scored.size() : 0) && joined_tokens.size() == (maxima ? 0 : scored.size()));
  int64_t t0 = 0, V = 0;
  for (int q = 0; q < p.P; ++q) V += p.shard_rows[q];
  for (size_t k = 0; k < scored.size(); ++k) {
    const vpce::ScoreArgs& a = scored[k];
    const vpce::FwdArgs& f = a.f;
    const vpce::FwdTile t = vpce::score_tile(p.dtype, f.kind);
    CHECK(f.T > 0 && t0 + f.T <= p.T && f.H == (const void*)(H + t0 * p.d * eb) && f.targets == targets + t0);
    CHECK((f.counter != nullptr) == (t0 == 0));
    CHECK(f.n_tok_blocks == ceil_div(f.T, t.bn) && f.n_splits >= 1 && (int64_t)f.n_tok_blocks * f.n_splits < (1ll << 31));
    int64_t off = 0, tiles = 0;
    for (int q = 0; q < p.P; ++q) {  // shards in order, whole
      CHECK(f.st.w[q] == W[q] && f.st.off[q] == off && f.st.rows[q] == p.shard_rows[q] && f.st.tile0[q] == tiles);
      off += p.shard_rows[q];
      tiles += ceil_div(p.shard_rows[q], t.bm);
    }
    CHECK(f.n_tiles == tiles && off == V);
    std::vector<std::pair<const char*, int64_t>> parts = {{ws, 8},
                                                          {(const char*)f.m_part, f.n_splits * f.T * 4},
                                                          {(const char*)f.s_part, f.n_splits * f.T * 4},
                                                          {(const char*)a.u_part, f.n_splits * f.T * 4}};
    const vpce::ScoreCombArgs& c = maxima ? tops[k].comb : joined_tokens[k];
    CHECK(c.c.m_part == f.m_part && c.c.s_part == f.s_part && c.u_part == a.u_part && c.c.n_splits == f.n_splits);
    CHECK(c.c.T == f.T && c.c.V == V && c.c.loss == loss + t0 && c.c.lse == lse + t0 && c.entropy == entropy + t0);
    CHECK(c.c.targets == f.targets && (char*)c.c.bad_counter == ws);
    if (maxima) {
      const vpce::TopArgs& x = tops[k];
      CHECK(x.bm == t.bm && (x.cpt == 4 || x.cpt == 8) && x.tok >= 1 && x.ids == (top ? ids + t0 * top : nullptr) && x.loss == (top ? top_loss + t0 * top : nullptr));
      parts.push_back({(const char*)a.fine, tiles * round_up(f.T, x.tok) * t.bm});
      parts.push_back({(const char*)a.coarse, tiles * f.T * x.cpt * 4});
    } else {
      CHECK(!a.fine && !a.coarse);
    }
    for (size_t i = 0; i < parts.size(); ++i) {
      CHECK(parts[i].first >= ws && parts[i].first + parts[i].second <= ws + bytes);
      if (i) CHECK(parts[i - 1].first + parts[i - 1].second <= parts[i].first && (uintptr_t)parts[i].first % 16 == 0);
    }
    if (f8) {
      CHECK(a.nb == nb && a.h_scale == hs + t0 * nb);
      for (int q = 0; q < p.P; ++q) CHECK(a.w_scale[q] == scales[q]);
    }
    t0 += f.T;
  }
  CHECK(t0 == p.T);
  return true;
}

int main(int argc, char** argv) {
  if (plan_check_main(argc, argv)) return 1;
  std::mt19937_64 r(17);
  auto log_int = [&](double lo, double hi) {
    return (int64_t)exp(std::uniform_real_distribution<double>(log(lo), log(hi))(r));
  };
  int kinds[3][vpce::kScoreKinds] = {{0}}, chunks = 0;
  for (int n = 0; n < 1500; ++n) {
    vp_problem p;
    memset(&p, 0, sizeof(p));
    p.dtype = (int)(r() % 3);
    p.T = log_int(1, n % 10 == 0 ? 1e6 : n % 3 ? 3000 : 20000);
    p.d = p.dtype == VP_E4M3 ? log_int(16, vpce::kF8MaxD) / 16 * 16 : log_int(8, 8192) / 8 * 8;
    p.P = 1 + (int)(r() % (n % 10 == 1 ? VP_MAX_SHARDS : 9));
    std::vector<int64_t> rows(p.P);
    for (auto& x : rows) x = r() % 8 == 0 ? 0 : log_int(1, 60000);
    rows[r() % p.P] = log_int(1, 200000);
    p.shard_rows = rows.data();
    p.ignore_index = -100;
    const int top = n % 3 ? (int)(r() % (VP_MAX_TOP + 1)) : 0;
    if (!check_score(p, top)) {
      printf("T=%lld d=%lld P=%d dtype=%d top=%d rows:", (long long)p.T, (long long)p.d, p.P, p.dtype, top);
      for (auto x : rows) printf(" %lld", (long long)x);
      printf("\n");
      return 1;
    }
    for (const auto& a : scored) ++kinds[p.dtype][a.f.kind];
    chunks += scored.size() > 1;
  }
  bool all = chunks > 0;
  for (int t = 0; t < 3; ++t)
    for (int k = 0; k < vpce::kScoreKinds; ++k) {
      printf("%d ", kinds[t][k]);
      all = all && (kinds[t][k] > 0) == (vpce::score_tile(t, k).per_cu > 0);
    }
  printf("launches by type and kind; %d in chunks\n", chunks);
  return all ? 0 : 1;
}
