// One call of the attention weights' kernels on the CPU, in buffers of exact sizes, twice in other orders of
// its waves and work groups, against a sum in 64 bits.
//   weigh name=value ... lens=a,b,... [new=a,b,...]
// Prints the launch, and with dry=1 no more than that.  Ends with 1 where a weight is off by more than its roundings, or goes by the order.
#include "cache_weigh.hip"

#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <string>
#include <vector>

#include "lanes.hpp"

using namespace cqsa;

static std::map<std::string, std::string> args;
static int arg(const char* name, int standard) { return args.count(name) ? atoi(args[name].c_str()) : standard; }
static std::vector<int> list(const char* name) {
  std::vector<int> out;
  const std::string& s = args[name];
  for (size_t at = 0; at < s.size(); at = s.find(',', at) == std::string::npos ? s.size() : s.find(',', at) + 1)
    out.push_back(atoi(s.c_str() + at));
  return out;
}

// Exactly n elements, so that the first one behind them is no one's.
template <typename T>
struct Buffer {
  T* p;
  int64_t n;
  explicit Buffer(int64_t n) : p((T*)malloc(n * sizeof(T))), n(n) {}
  ~Buffer() { free(p); }
  T& operator[](int64_t i) { return p[i]; }
};

int main(int argc, char** argv) {
  for (int i = 1; i < argc; ++i) {
    const std::string s = argv[i];
    args[s.substr(0, s.find('='))] = s.substr(s.find('=') + 1);
  }
  const std::vector<int> lens = list("lens");
  std::vector<int> fresh = list("new");
  const int B = int(lens.size()), L = arg("L", 1), H = arg("H", 1), G = arg("G", 1), d = arg("d", 32);
  const cqsa_dtype dt = cqsa_dtype(arg("dtype", CQSA_BF16));
  const int page_log2 = arg("page_log2", 6), P = 1 << page_log2, causal = arg("causal", 1), Hq = G * H;
  const bool packed = !fresh.empty(), counted = arg("counted", 0), in_place = arg("in_place", 0), prior = arg("prior", 1);
  if (!packed) fresh.assign(B, L);
  const int max_len = arg("max_len", *std::max_element(lens.begin(), lens.end()));
  const float decay = 0.75f, scale = 0.25f;
  std::mt19937 g(arg("seed", 1));
  auto real = [&]() { return float(int(g() % 2001) - 1000) / 1000; };

  WeighPlan p = plan_weigh(B, H, int64_t(L) * G, max_len, dt, d);
  if (const int tiles = arg("tiles", 0)) {  // fewer work groups over the tokens, so that each goes through several tiles
    if (p.row_groups == 0 && !p.resident) return 2;
    p.tiles = tiles, p.groups = int64_t(B) * H * tiles;
  }
  const int each = p.row_groups ? 32 : 64;  // tokens of a wave's tile
  printf("row_groups %d resident %d waves %d tiles %d splits %d a_wave %d\n", p.row_groups, p.resident, p.waves, p.tiles, p.splits,
         (max_len + each * p.waves * p.tiles - 1) / (each * p.waves * p.tiles));
  fflush(stdout);
  if (arg("dry", 0)) return 0;

  const int columns = std::max(1, (max_len + P - 1) / P);
  int64_t n_pages = 1, rows = packed ? 0 : L;
  for (int n : lens) n_pages += (n + P - 1) / P;
  for (int n : fresh) rows += packed ? n : 0;
  const int64_t page_bytes = int64_t(H) * (P / 32) * tile_bytes(d), QB = packed ? 1 : B, heads = int64_t(B) * H;
  Buffer<uint8_t> data(n_pages * page_bytes);
  for (int64_t i = 0; i < data.n; ++i) data[i] = i % tile_bytes(d) < 32 * d ? g() : 123 + g() % 3;
  Buffer<int32_t> pages(int64_t(B) * columns), lengths(B), start(B + 1), counts(B);
  start[0] = 0;
  int64_t next = 0;
  for (int b = 0; b < B; ++b) {
    for (int i = 0; i < columns; ++i) pages[b * columns + i] = i < (lens[b] + P - 1) / P ? int(next++) : -1;
    if (arg("holes", 0) && lens[b] > 2 * P) pages[b * columns + lens[b] / P / 2] = b % 2 ? -1 : 1 << 30;
    lengths[b] = lens[b];
    start[b + 1] = start[b] + fresh[b];
    counts[b] = fresh[b] - int(g() % 3);
  }
  const int bytes = dt == CQSA_F32 ? 4 : 2;
  const int64_t nq = QB * rows * Hq * d, nl = QB * Hq * rows;
  Buffer<uint8_t> q(nq * bytes);
  std::vector<float> q_value(nq);
  for (int64_t i = 0; i < nq; ++i) {
    const float x = real();
    if (dt == CQSA_F32) ((float*)q.p)[i] = x, q_value[i] = x;
    if (dt == CQSA_F16) ((_Float16*)q.p)[i] = (_Float16)x, q_value[i] = ((_Float16*)q.p)[i];
    if (dt == CQSA_BF16) ((__bf16*)q.p)[i] = (__bf16)x, q_value[i] = ((__bf16*)q.p)[i];
  }
  Buffer<float> lse(nl), before(heads * max_len), W(heads * max_len);
  for (int64_t i = 0; i < nl; ++i) lse[i] = i % 37 == 36 ? (i & 1 ? NAN : -INFINITY) : 3 + real();
  for (int64_t i = 0; i < before.n; ++i) before[i] = 1 + real();

  WeighArgs a{};
  a.c = {(char*)data.p, pages.p, lengths.p, packed ? start.p : nullptr, n_pages, columns, page_bytes, page_log2, H, d, B,
         max_len, packed ? L : 0, int32_t(rows)};
  a.q = {q.p, rows * Hq * d, int64_t(Hq) * d, d};
  a.lse = lse.p;
  a.counts = counted ? counts.p : nullptr;
  a.w = {W.p, int64_t(H) * max_len, max_len};
  if (prior) a.prior = in_place ? a.w : TokenWeights{before.p, int64_t(H) * max_len, max_len};
  a.Hq = Hq, a.G = G, a.causal = causal, a.decay = decay;
  a.scale_log2 = scale * 1.4426950408889634f;
  Buffer<float> part(p.splits > 1 ? p.splits * heads * max_len : 0);
  a.part = p.splits > 1 ? part.p : nullptr;

  std::vector<float> first;
  for (int run = 0; run < 2; ++run) {
    lanes::order.seed(100 * run + 7);
    for (int64_t i = 0; i < W.n; ++i) W[i] = in_place ? before[i] : 7.f;
    for (int64_t i = 0; i < part.n; ++i) part[i] = NAN;
    launch_cache_weigh(dt, a, p, nullptr);
    if (run == 0) first.assign(W.p, W.p + W.n);
    if (memcmp(first.data(), W.p, W.n * 4) != 0) return printf("the order of waves changes results\n"), 1;
  }

  static const double level[8] = {0, .5, 1, 1.5, 2, 3, 4, 6};
  double worst = 0;
  for (int b = 0; b < B; ++b) {
    const int n = lens[b], m = packed ? std::min(fresh[b], L) : L, old = std::max(0, n - m);
    const int live = counted ? std::min(std::max(counts[b], 0), m) : m;
    for (int h = 0; h < H; ++h) {
      std::vector<double> sum(n), big(n), add(n);
      for (int t = 0; t < n; ++t) {
        const int32_t page = pages[b * columns + t / P];
        if (page < 0 || page >= n_pages) continue;
        const uint8_t* tile = data.p + page * page_bytes + (int64_t(h) * (P / 32) + t % P / 32) * tile_bytes(d);
        std::vector<double> k(d);
        for (int e = 0; e < d; ++e) {
          const int code = tile[e / 32 * 512 + t % 32 * 16 + e % 32 / 2] >> (4 * (e % 2)) & 15;
          k[e] = ldexp(level[code & 7], tile[32 * d + t % 16 * (d / 16) + 2 * (e / 32) + t % 32 / 16] - 127) * (code & 8 ? -1 : 1);
        }
        for (int i = 0; i < live; ++i) {
          if (causal && t > n - m + i) continue;
          const int64_t row = packed ? start[b] + i : i, tb = packed ? 0 : b;
          for (int u = h * G; u < h * G + G; ++u) {
            const float l = lse[(tb * Hq + u) * rows + row];
            if (!std::isfinite(l)) continue;
            double s = 0, size = 0;
            const float* x = &q_value[((tb * rows + row) * Hq + u) * d];
            for (int e = 0; e < d; ++e) s += x[e] * k[e], size += fabs(x[e] * k[e]);
            sum[t] += exp(s * scale - l);
            big[t] = std::max({big[t], size * scale, fabs(double(l))});
            add[t] += 1;
          }
        }
      }
      for (int t = 0; t < max_len; ++t) {
        const int64_t i = (int64_t(b) * H + h) * max_len + t;
        if (t >= n) {
          if (W[i] != (in_place ? before[i] : 7.f)) return printf("token %d behind sequence %d was written\n", t, b), 1;
          continue;
        }
        const double want = sum[t] + (prior && t < old ? decay * double(before[i]) : 0.0);
        // half steps: the exponent's by the sizes in it, the exponential's, and the sum's
        const double bound = want * ldexp(1, -24) * ((d + 8) * big[t] + add[t] + 16) + 1e-36;
        const double off = fabs(W[i] - want);
        if (!(off <= bound)) return printf("sequence %d head %d token %d: %g instead of %g\n", b, h, t, W[i], want), 1;
        worst = std::max(worst, off / bound);
      }
    }
  }
  printf("ok %.3f\n", worst);
}
