// Runs the C entries of the losses of whole sequences on the CPU, the kernels of vpce_seq.hip as
// they stand, over arrays that end (or begin) at a page that faults: a read or a write outside an
// array ends the program.
//   ordered     outputs against plain loops in double, for layouts of every kind
//   disordered  offsets that decrease or leave the tokens: NaN for the sequences that they bound,
//               every gradient written, nothing outside the arrays touched
//   runs        long runs of empty sequences, in order and not
//   no tokens   empty sequences alone, more of them than one workgroup takes among them
#include <sys/mman.h>

#include <random>

#include "../paper_2609_14306_amd/csrc/vpce_head_api.cpp"
#include "../paper_2609_14306_amd/csrc/vpce_seq.hip"

namespace vpce {  // (the layer norm's kernels are not part of this program)
int norm_parts(int64_t, int) { return 1; }
bool run_norm_forward(int, bool, const NormArgs&, hipStream_t) { return false; }
bool run_norm_backward(int, bool, const NormGradArgs&, hipStream_t) { return false; }
}  // namespace vpce

static bool at_end;  // which end of an array lies at the page that faults

// n elements, all bytes 0xff (NaN, -1).
template <class T>
struct Array {
  T* p;
  char* map;
  size_t bytes, n;
  explicit Array(size_t count, size_t align = alignof(T)) : n(count) {
    const size_t page = 4096, size = (count * sizeof(T) + align - 1) / align * align;
    const size_t inner = max<size_t>(1, (size + page - 1) / page) * page;
    bytes = inner + 2 * page;
    map = (char*)mmap(nullptr, bytes, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
    if (map == MAP_FAILED || mprotect(map + page, inner, PROT_READ | PROT_WRITE) != 0) abort();
    memset(map + page, 0xff, inner);
    p = (T*)(at_end ? map + page + inner - size : map + page);
  }
  Array(const Array&) = delete;
  ~Array() { munmap(map, bytes); }
  T& operator[](size_t i) { return p[i]; }
  operator T*() { return p; }
};

static char what[200];
#define CHECK(...)                                                          \
  do {                                                                      \
    if (!(__VA_ARGS__)) {                                                   \
      printf("FAILED line %d, %s: %s\n", __LINE__, what, #__VA_ARGS__);     \
      return false;                                                         \
    }                                                                       \
  } while (0)

// One float32 rounding, and what double sums in another order leave.
static bool close(double got, double want, double size) {
  if (want != want) return got != got;
  return std::fabs(got - want) <= std::ldexp(std::fabs(want), -24) + std::ldexp(size, -40) + 1e-44;
}

struct Options {
  bool mean, old, ref, per_token;
  int kind;
};

// Calls both losses, forward and backward, on tokens of T in sequences of `offsets`.
static bool run(int T, const std::vector<int>& offsets, const Options& o, unsigned seed) {
  const int S = (int)offsets.size() - 1;
  std::mt19937_64 rng(seed);
  std::uniform_real_distribution<float> uniform(0.f, 1.f);
  Array<int32_t> start(S + 1), clipped(S), tokens(S);
  Array<int64_t> targets(T);
  Array<float> loss(T), old(T), ref(T), adv(o.per_token ? T : S), seq_loss(S), seq_kl(S), up(S), grad(T);
  Array<float> pair(S / 2), reward(S), coef(S), up_pair(S / 2), pair_grad(T);
  const float kUnwritten = 12345.f;
  for (float* out : {seq_loss.p, seq_kl.p, reward.p}) std::fill(out, out + S, kUnwritten);
  std::fill(pair.p, pair.p + S / 2, kUnwritten);
  std::fill(grad.p, grad.p + T, kUnwritten);
  std::fill(pair_grad.p, pair_grad.p + T, kUnwritten);
  bool ordered = true;
  for (int s = 0; s <= S; ++s) {
    start[s] = offsets[s];
    ordered = ordered && offsets[s] >= (s ? offsets[s - 1] : 0) && offsets[s] <= T;
  }
  for (int t = 0; t < T; ++t) {
    targets[t] = uniform(rng) < 0.3f ? -100 : 7;
    const bool junk = targets[t] == -100;  // (NaN stays in the masked tokens)
    const float l = 4.f * uniform(rng), a = 0.4f * (uniform(rng) - 0.5f), b = 0.4f * (uniform(rng) - 0.5f);
    if (!junk) loss[t] = l, old[t] = l + a, ref[t] = l + b;
  }
  for (size_t i = 0; i < adv.n; ++i) adv[i] = 2.f * uniform(rng) - 1.f;
  for (int s = 0; s < S; ++s) up[s] = uniform(rng) - 0.3f;
  for (int i = 0; i < S / 2; ++i) up_pair[i] = uniform(rng) - 0.3f;

  const vp_sequences seq = {T, S, -100, o.mean ? VP_SEQ_MEAN : 0u};
  const vp_policy pol = {0.08, 0.1, 0.3, o.per_token ? VP_ADV_PER_TOKEN : 0u};
  const vp_preference pref = {o.kind, o.mean ? 1.5 : 0.01, 0.2, 0.0};
  size_t bytes = 0;
  CHECK(vp_seq_workspace_size(&seq, &bytes) == VP_OK);
  Array<char> ws(bytes, 16), ws2(bytes, 16);
  CHECK(vp_policy_forward(&seq, &pol, start, targets, loss, o.old ? old.p : nullptr, o.ref ? ref.p : nullptr, adv,
                          seq_loss, seq_kl, clipped, tokens, ws, bytes, nullptr) == VP_OK);
  CHECK(vp_policy_backward(&seq, &pol, start, targets, loss, o.old ? old.p : nullptr, o.ref ? ref.p : nullptr, adv,
                           tokens, up, grad, nullptr) == VP_OK);
  const bool pairs = S % 2 == 0;
  if (pairs) {
    CHECK(vp_pref_forward(&seq, &pref, start, targets, loss, o.ref ? ref.p : nullptr, pair, reward, coef, ws2, bytes,
                          nullptr) == VP_OK);
    CHECK(vp_pref_backward(&seq, start, targets, coef, up_pair, pair_grad, nullptr) == VP_OK);
  }

  if (!ordered) {
    for (int s = 0; s < S; ++s)
      if (offsets[s] < 0 || offsets[s] > offsets[s + 1] || offsets[s + 1] > T) {
        CHECK(seq_loss[s] != seq_loss[s] && seq_kl[s] != seq_kl[s]);
        if (pairs) CHECK(pair[s / 2] != pair[s / 2]);
      }
    for (int t = 0; t < T; ++t) {
      CHECK(grad[t] != kUnwritten && (targets[t] != -100 || grad[t] == 0.f));
      if (pairs) CHECK(pair_grad[t] != kUnwritten && (targets[t] != -100 || pair_grad[t] == 0.f));
    }
    return true;
  }
  std::vector<double> want(T, 0.0), size(T, 0.0), want_pair(T, 0.0), ratio(S), weight(S);
  for (int s = 0; s < S; ++s) {
    double l = 0, kl = 0, R = 0, mag = 0;
    int n = 0, c = 0;
    for (int t = start[s]; t < start[s + 1]; ++t)
      if (targets[t] != -100) ++n;
    weight[s] = !o.mean ? 1.0 : n ? 1.0 / n : 0.0;
    for (int t = start[s]; t < start[s + 1]; ++t) {
      if (targets[t] == -100) continue;
      const double A = adv[o.per_token ? t : s], x = o.old ? (double)old[t] - loss[t] : 0.0, rho = std::exp(x);
      const double q = o.ref ? (double)loss[t] - ref[t] : 0.0;
      const bool cut = A > 0 ? rho > 1.1 : A < 0 ? rho < 0.92 : false;
      const double k = std::expm1(q) - q;
      l += -min(rho * A, max(0.92, min(1.1, rho)) * A) + 0.3 * k;
      kl += k;
      c += cut;
      R += (o.ref ? ref[t] : 0.f) - (double)loss[t];
      mag += 2 * std::fabs(A) + std::fabs(loss[t]) + 1;
      want[t] = up[s] * weight[s] * ((cut ? 0.0 : rho * A) + 0.3 * std::expm1(q));
      size[t] = std::fabs(up[s]) * weight[s] * (2 * std::fabs(A) + 1);
    }
    ratio[s] = weight[s] * R;
    CHECK(tokens[s] == n && clipped[s] == c);
    CHECK(close(seq_loss[s], weight[s] * l, weight[s] * mag) && close(seq_kl[s], weight[s] * kl, weight[s] * mag));
    if (pairs) CHECK(close(reward[s], pref.beta * ratio[s], pref.beta * weight[s] * mag));
  }
  for (int t = 0; t < T; ++t) CHECK(close(grad[t], want[t], size[t]));
  for (int i = 0; pairs && i < S / 2; ++i) {
    const double z = pref.beta * (ratio[2 * i] - ratio[2 * i + 1]) - pref.margin;
    const double big = 1 + std::fabs(z) + pref.beta * (std::fabs(ratio[2 * i]) + std::fabs(ratio[2 * i + 1]));
    double slope, value, scale = 1;
    if (o.kind == VP_PREF_LOGISTIC) {
      value = std::log1p(std::exp(-std::fabs(z))) + max(-z, 0.0);
      slope = -1 / (1 + std::exp(z));
    } else {
      value = (z - 0.5) / pref.beta * ((z - 0.5) / pref.beta);
      slope = 2 * (z - 0.5) / pref.beta / pref.beta;
      scale = 2 * big / pref.beta / pref.beta;
    }
    CHECK(close(pair[i], value, scale * big));
    for (int k = 0; k < 2; ++k) {
      const int s = 2 * i + k;
      const double g = (k ? slope : -slope) * pref.beta * weight[s];
      for (int t = start[s]; t < start[s + 1]; ++t)
        if (targets[t] != -100) want_pair[t] = up_pair[i] * g;
    }
    for (int s = 2 * i; s < 2 * i + 2; ++s)
      for (int t = start[s]; t < start[s + 1]; ++t) {
        // two roundings to float32: coef and the product
        const double w = want_pair[t];
        CHECK(std::fabs(pair_grad[t] - w) <=
              std::ldexp(std::fabs(w), -23) + std::ldexp(std::fabs(up_pair[i]) * pref.beta * scale * big, -40) + 1e-44);
      }
  }
  for (int t = 0; pairs && t < T; ++t)
    if (t < start[0] || t >= start[S]) CHECK(pair_grad[t] == 0.f);
  return true;
}

// S + 1 offsets in 0..T: some empty sequences, tokens before the first and behind the last.
static std::vector<int> offsets_of(std::mt19937_64& rng, int T, int S, int style) {
  std::vector<int> v(S + 1);
  const int lo = style == 1 ? T / 7 : 0, hi = style == 1 ? T - T / 9 : T;
  for (int& x : v) x = lo + (int)(rng() % (uint64_t)(hi - lo + 1));
  std::sort(v.begin(), v.end());
  if (style == 2)  // runs of empty sequences
    for (size_t i = 1; i < v.size(); ++i)
      if (i % 90) v[i] = v[i - 1];
  if (style != 1 && S > 0) v[0] = 0, v[S] = T;
  return v;
}

static bool all(bool disordered) {
  const int sizes[] = {1, 64, 65, 700, 2048, 2049, 3300}, counts[] = {0, 1, 2, 63, 65, 200, 2050, 4200};
  std::mt19937_64 rng(disordered ? 11 : 5);
  unsigned seed = 0;
  for (int T : sizes)
    for (int S : counts)
      for (int style = 0; style < 3; ++style) {
        if ((S >= 2050 && style != (T + S) % 3) || (S == 0 && style)) {
          ++seed;
          continue;
        }
        std::vector<int> v = offsets_of(rng, T, S, style);
        if (disordered) {
          const int bad[] = {-5, T + 9, INT32_MAX, INT32_MIN, 0, T / 2, T, -1};
          for (int i = 0; i <= S / 3; ++i) v[rng() % v.size()] = bad[rng() % 8];
        }
        const Options o = {(seed & 1) != 0, (seed & 2) == 0, (seed & 4) == 0, (seed & 8) != 0, (int)(seed / 2 % 2)};
        at_end = seed % 2 == 0;
        snprintf(what, sizeof what, "T %d S %d style %d seed %u", T, S, style, seed);
        if (!run(T, v, o, seed++)) return false;
      }
  return true;
}

// Rounds of several tokens a lane and chunks of several rounds, which the entries take for more
// than a million tokens, on a few thousand: the same results as with one.
static bool longer() {
  using namespace vpce;
  std::mt19937_64 rng(3);
  for (int S : {1, 2, 40, 300}) {
    const int T = 5000 + S;
    snprintf(what, sizeof what, "longer, S %d", S);
    const std::vector<int> v = offsets_of(rng, T, S, S % 3);
    Array<int32_t> start(S + 1);
    Array<int64_t> targets(T);
    Array<float> coef(S + 1), up(S + 1), a(T), b(T);
    std::copy(v.begin(), v.end(), start.p);
    for (int t = 0; t < T; ++t) targets[t] = rng() % 3 ? 1 : -100;
    for (int s = 0; s <= S; ++s) coef[s] = 1.f + s, up[s] = 0.5f + s;
    SeqArgs q = {start, targets, -100, T, S, 0, 64, nullptr};
    launch_grad<1>(PrefGrad{q, coef, up, a}, nullptr);
    launch_grad<4>(PrefGrad{q, coef, up, b}, nullptr);
    for (int t = 0; t < T; ++t) CHECK(cpu::bits(a[t]) == cpu::bits(b[t]));

    Array<float> loss(T), adv(S), l1(S), k1(S), l2(S), k2(S);
    Array<int32_t> c1(S), n1(S), c2(S), n2(S);
    for (int t = 0; t < T; ++t) loss[t] = (float)(rng() % 64) / 16;  // (sums without a rounding)
    for (int s = 0; s < S; ++s) adv[s] = (float)(s % 5) - 2;
    for (int chunk : {64, 192, 512}) {
      q.chunk = chunk;
      Array<double> part(((T + chunk - 1) / chunk + S) * kMaxSeqSums);
      q.part = part;
      PolicyArgs p = {};
      p.q = q;
      p.loss = p.old = p.ref = p.adv_tok = loss;
      p.adv = adv;
      p.high = 1.2, p.low = 0.8, p.log_high = std::log1p(0.2), p.log_low = std::log1p(-0.2);
      p.seq_loss = chunk == 64 ? l1.p : l2.p, p.seq_kl = chunk == 64 ? k1.p : k2.p;
      p.clipped = chunk == 64 ? c1.p : c2.p, p.tokens = chunk == 64 ? n1.p : n2.p;
      const int chunks = (T + chunk - 1) / chunk;
      hipLaunchKernelGGL((chunk_kernel<PolicyOp, PolicyArgs>), dim3((chunks + 3) / 4), dim3(256), 0, nullptr, p);
      if (chunk == 64)
        launch_finish<PolicyOp, PolicyArgs, 64>(p, S, nullptr);
      else if (chunk == 192)
        launch_finish<PolicyOp, PolicyArgs, 256>(p, S, nullptr);
      else
        launch_finish<PolicyOp, PolicyArgs, 8>(p, S, nullptr);
      for (int s = 0; chunk > 64 && s < S; ++s)
        CHECK(l1[s] == l2[s] && k1[s] == k2[s] && c1[s] == c2[s] && n1[s] == n2[s]);
    }
    int counting = 0, mine = 0;
    for (int t = v[0]; t < v[S]; ++t) counting += targets[t] != -100;
    for (int s = 0; s < S; ++s) mine += n1[s];
    CHECK(mine == counting);
    CHECK(hipGetLastError() == hipSuccess);
  }
  return true;
}

// Runs of empty sequences longer than a window of offsets, between any two tokens, also where the
// offsets behind a run go back.
static bool runs() {
  std::mt19937_64 rng(8);
  unsigned seed = 0;
  for (int T : {3, 130, 2500})
    for (int S : {64, 130, 1000, 2300})
      for (int wrong = 0; wrong < 2; ++wrong) {
        snprintf(what, sizeof what, "runs, T %d S %d seed %u", T, S, seed);
        std::vector<int> v(S + 1);
        int at = (int)(rng() % 3);
        for (int i = 0; i <= S;) {
          for (int n = 1 + (int)(rng() % 300); n > 0 && i <= S; --n) v[i++] = min(at, T);
          at += 1 + (int)(rng() % (1 + T / 8));
        }
        if (wrong)
          for (int k = 0; k < 4; ++k) v[rng() % v.size()] = (int)(rng() % (T + 1));
        at_end = seed % 2 == 0;
        const Options o = {(seed & 1) != 0, (seed & 2) == 0, (seed & 4) == 0, (seed & 8) != 0, (int)(seed / 2 % 2)};
        if (!run(T, v, o, seed++)) return false;
      }
  return true;
}

// Sequences without any tokens, from a few to more than one workgroup takes.
static bool no_tokens() {
  unsigned seed = 0;
  for (int S : {0, 1, 2, 2048, 2049, 2050, 4096, 4098, 20000})
    for (int wrong = 0; wrong < (S ? 2 : 1); ++wrong) {
      snprintf(what, sizeof what, "no tokens, S %d%s", S, wrong ? ", wrong offsets" : "");
      std::vector<int> v(S + 1, 0);
      if (wrong) v[S / 2] = -1, v[S] = 9;
      const Options o = {(seed & 1) != 0, (seed & 2) == 0, (seed & 4) == 0, (seed & 8) != 0, (int)(seed / 2 % 2)};
      if (!run(0, v, o, seed++)) return false;
    }
  return true;
}

int main(int argc, char** argv) {
  const bool ok = argc > 1 && (!strcmp(argv[1], "ordered")      ? all(false)
                               : !strcmp(argv[1], "disordered") ? all(true)
                               : !strcmp(argv[1], "longer")     ? longer()
                               : !strcmp(argv[1], "no tokens")  ? no_tokens()
                               : !strcmp(argv[1], "runs")       ? runs()
                                                                : false);
  printf("%s, %ld launches\n", ok ? "ok" : "FAILED", cpu::launches);
  return ok ? 0 : 1;
}
