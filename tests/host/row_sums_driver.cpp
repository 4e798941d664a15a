// CPU-only check of csrc/row_sums.h over the range of logits and temperatures that the log-prob calls accept: rows are walked in
// chunks by several threads, their sums merged, and ln S and the entropy compared with sums in 64 and more bits.  Built
// and run by tests/test_host_row_sums.py.
//
// Tolerances (u = 2^-24): S is a sum of n additions one after another (n = values of a thread + merges), each off by u of the
// sum, of terms 2^y whose exponent is off by 4 u |y| (c = log2(e) / T is rounded twice, the difference and the product
// once each) with |y| 2^y < 0.54, the exponential itself and a scaling by 2 u: ln S is off by (n + 8) u.  The entropy is
// ln S + a sum of the same kind, of at most n + 16 roundings of a value no larger than ln V each.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../paper_2506_06122_amd/csrc/row_sums.h"

static long long checks = 0;

struct Row {
  const char* kind;
  float at;  // what the kind is made of
  std::vector<float> x;
};

// Values `threads` apart in chunks of 8, then one by one (walk 0), or each thread a contiguous share (walk 1); threads joined in
// order (join 0) or pairwise (join 1)
static RowSums sums_of(const std::vector<float>& x, float c, int threads, int walk, int join) {
  const int V = (int)x.size(), share = (V + threads - 1) / threads;
  std::vector<RowSums> part;
  for (int k = 0; k < threads; ++k) {
    std::vector<float> mine;
    for (int i = 0; i < V; ++i)
      if (walk ? i / share == k : i % threads == k) mine.push_back(x[i]);
    RowSums r{kLowest, 0.f, 0.f};
    size_t i = 0;
    for (; i + 8 <= mine.size(); i += 8) add_chunk<8>(r, &mine[i], c);
    for (; i < mine.size(); ++i) add_chunk<1>(r, &mine[i], c);
    part.push_back(r);
  }
  if (join) {
    for (size_t n = part.size(); n > 1; n = (n + 1) / 2)
      for (size_t k = 0; k < n / 2; ++k) part[k] = merge(part[k], part[n - 1 - k], c);
    return part[0];
  }
  RowSums all = part[0];
  for (size_t k = 1; k < part.size(); ++k) all = merge(all, part[k], c);
  return all;
}

static void check(const Row& row, float T) {
  const int V = (int)row.x.size();
  const float inv = 1.0f / T, c = inv * kLog2e;
  if (!std::isfinite(c)) return;  // refused by the calls
  float m = -INFINITY;
  for (float v : row.x) m = std::fmax(m, v);
  long double S = 0, A = 0;
  for (float v : row.x) {
    const long double d = ((long double)v - m) / T, e = expl(d);
    if (e > 0) S += e, A += e * d;
  }
  const bool empty = m == -INFINITY;
  const double log_s = empty ? -INFINITY : (double)logl(S), entropy = empty ? 0 : (double)(logl(S) - A / S);
  for (int threads : {1, 4, 7})
    for (int walk = 0; walk < 2; ++walk)
      for (int join = 0; join < 2; ++join) {
        const RowSums r = sums_of(row.x, c, threads, walk, join);
        const double u = std::ldexp(1.0, -24), n = V / threads + threads + 8;
        const float got_s = row_log_sum(r, c), got_h = row_entropy(r);
        const double off_s = empty ? (got_s == -INFINITY ? 0 : 1) : std::fabs(got_s - log_s), off_h = std::fabs(got_h - entropy);
        const double tol_s = (n + 8) * u + u * std::fabs(empty ? 0 : log_s), tol_h = tol_s + (2 * n + 32) * u * std::log(V + 1.0);
        for (int i = 0; i < V && !empty; i += 1 + V / 16) {  // ln p: the difference's, the product's and 1 / T's roundings beside ln S
          const double lp = (double)(((long double)row.x[i] - m) / T) - log_s, got = row_logp(row.x[i], r.m, inv, got_s);
          const bool past = lp < -0x1.fffffep127;  // below fp32's range
          if (past ? got > -0x1.ffffe0p127 : !(std::fabs(got - lp) <= tol_s + 4 * u * (std::fabs(lp) + 2 * std::fabs(log_s)) || got == lp)) {
            std::fprintf(stderr, "%s %g, %d values, T %g: ln p of %g is %g of %g\n", row.kind, row.at, V, T, row.x[i], got, lp);
            std::exit(1);
          }
        }
        if (!(off_s <= tol_s) || !(off_h <= tol_h) || (!empty && r.m != m)) {
          std::fprintf(stderr, "%s %g, %d values, T %g, %d threads, walk %d, join %d: max %g of %g, ln S %g of %g, entropy %g of %g\n", row.kind,
                       row.at, V, T, threads, walk, join, r.m, m, got_s, log_s, got_h, entropy);
          std::exit(1);
        }
        ++checks;
      }
}

static float uniform(unsigned& seed) {
  seed = seed * 1664525u + 1013904223u;
  return (float)(seed >> 8) * 0x1p-24f;
}

int main() {
  unsigned seed = 1;
  std::vector<float> temperatures = {3e38f, 1e30f, 1e9f, 1e3f, 3.f, 2.f, 1.5f, 1.3f, 1.f, 0.9f, 0.8f, 0.7f, 0.6f, 0.25f, 1e-2f};
  for (int e = -3; e >= -37; --e) temperatures.push_back(std::pow(10.f, (float)e));
  for (float T : temperatures) {
    for (int V : {1, 2, 9, 130, 601}) {
      // a value everywhere; all but a few of them; a block of them at either end; every third
      for (float fill : {-1e4f, -65504.f, -1e5f, -1e6f, -1e7f, -1e8f, -1e9f, -1e10f, -1e12f, -1e15f, -1e20f, -1e28f, -7e29f, -1e30f, -1e31f, -1e38f, kLowest,
                         -INFINITY, 0.f, 1e4f, 1e9f, 1e20f, 3.4e38f}) {
        check({"all", fill, std::vector<float>(V, fill)}, T);
        for (int part = 0; part < 4; ++part) {
          std::vector<float> x(V);
          for (int i = 0; i < V; ++i) {
            const bool masked = part == 0 ? i != V / 2 : part == 1 ? i < V * 9 / 10 : part == 2 ? i >= V / 10 : i % 3 == 0;
            x[i] = masked ? fill : 5.f * uniform(seed) - 2.5f;
          }
          check({"partly", fill, x}, T);
        }
      }
      // differences past fp32's range
      for (int i = 0; i < V; i += 1 + V / 8) {
        std::vector<float> x(V, 2.5f);
        x[i] = kLowest;
        x[V - 1 - i] = 3.3e38f;
        check({"wide", (float)i, x}, T);
      }
      // ordinary logits, and larger ones
      for (float size : {1.f, 25.f, 1e3f, 6e4f, 1e9f, 1e30f}) {
        std::vector<float> x(V);
        for (float& v : x) v = size * (2.f * uniform(seed) - 1.f);
        check({"spread", size, x}, T);
      }
    }
    // exponents next to 2^k, neighbouring values: on both sides of every limit of magnitude, with a share below it in most threads
    for (int k = 15; k <= 34; ++k)
      for (float sign : {1.f, -1.f}) {
        const float c = (1.0f / T) * kLog2e, at = std::ldexp(sign, k) / c;
        if (!std::isfinite(at) || !std::isnormal(at)) continue;
        for (int V : {3, 40, 300}) {
          std::vector<float> x(V);
          for (int i = 0; i < V; ++i) x[i] = at * (1.f + 0x1p-23f * (float)((i * 37) % 61 - 30));
          check({"beside 2^", std::ldexp(sign, k), x}, T);
          for (int i = 0; i < V; i += 3) x[i] = at * (1.f - sign * 0x1p-10f);
          check({"below 2^", std::ldexp(sign, k), x}, T);
        }
      }
  }
  std::printf("%lld rows\n", checks);
  return 0;
}
