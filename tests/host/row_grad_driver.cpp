// CPU-only check of the logits' gradient in csrc/row_sums.h over the range of logits and temperatures that the calls accept,
// against the formula in 64 and more bits.  Built and run by tests/test_host_row_sums.py.
//
// Tolerances (u = 2^-24): log2 p = (x - m) c - ln S / ln 2 is off by 4 u of the first term and 3 u of the second, so with `mag` the sum
// of both in nats p is off by 4 u mag, and its factor g + h (ln p + H) by 4 u of |g| + |h| (mag + H); what is added at the target
// and the division by T are a few roundings of |g| / T.  p is held in fp32: below its least normal value, 2^-126, off by up to that.  The result once more by half a step of fp32, 2^-150 at the least.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../paper_2506_06122_amd/csrc/row_sums.h"

static long long checks = 0;

static void check(const char* kind, const std::vector<float>& x, float T, float g, float h, int target) {
  const int V = (int)x.size();
  const float inv = 1.0f / T, c = inv * kLog2e;
  if (!std::isfinite(c)) return;  // refused by the calls
  float m = -INFINITY;
  for (float v : x) m = std::fmax(m, v);
  if (m == -INFINITY) return;
  long double S = 0, A = 0;
  for (float v : x) {
    const long double d = ((long double)v - m) / T, e = expl(d);
    if (e > 0) S += e, A += e * d;
  }
  const long double log_s = logl(S), H = log_s - A / S, u = ldexpl(1, -24);
  const RowGrad r = row_grad_of(m, (float)log_s, (float)H, g, h, target, inv);
  for (int i = 0; i < V; ++i) {
    const long double lp = ((long double)x[i] - m) / T - log_s, p = expl(lp), gt = target < 0 ? 0 : g;
    const long double want = r.none ? 0 : (gt * (i == target) - gt * p - (p > 0 ? h * p * (lp + H) : 0)) / T;
    const long double mag = (p > 0 ? fabsl(lp) + 2 * log_s : 0) + 4, size = fabsl(gt) + fabsl(h) * (mag + H);
    const long double tol = (size * (p * (4 * u * mag + 8 * u) + ldexpl(1, -126)) + 8 * u * fabsl(gt)) / T + u * fabsl(want) + ldexpl(1, -126);
    if (fabsl(want) + tol > 3.4e38L) continue;  // not a value of the type
    const float got = r.none ? 0.f : grad_at(x[i], i, r);
    if (!(fabsl(got - want) <= tol)) {
      std::fprintf(stderr, "%s, %d values, T %g, g %g, h %g, target %d: value %d, logit %g, is %g of %Lg +- %Lg\n", kind, V, T, g, h, target, i, x[i], got,
                   want, tol);
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
  std::vector<float> temperatures = {3e38f, 1e30f, 1e9f, 1e3f, 2.f, 1.f, 0.7f, 0.25f, 1e-2f};
  for (int e = -3; e >= -38; --e) temperatures.push_back(std::pow(10.f, (float)e));
  temperatures.push_back(4.3e-39f);
  for (float T : temperatures)
    for (float h : {0.f, 0.01f, -1.f, 8.f, 1e4f})
      for (float g : {0.f, 1e-6f, 1.f, -30.f})
        for (int V : {1, 2, 33}) {
          for (float fill : {-1e4f, -1e9f, -1e20f, -1e31f, kLowest, -INFINITY, 1e9f, 3.4e38f}) {
            std::vector<float> x(V);
            for (int i = 0; i < V; ++i) x[i] = i % 3 == 1 ? fill : 5.f * uniform(seed) - 2.5f;
            for (int target : {-1, 0, V - 1}) check("masked", x, T, g, h, target);
          }
          for (int i = 0; i < V; ++i) {  // differences past fp32's range
            std::vector<float> x(V, 2.5f);
            x[i] = kLowest;
            x[V - 1 - i] = 3.3e38f;
            check("wide", x, T, g, h, i);
          }
          for (float size : {1.f, 1e3f, 1e30f}) {
            std::vector<float> x(V);
            for (float& v : x) v = size * (2.f * uniform(seed) - 1.f);
            check("spread", x, T, g, h, V / 2);
          }
          if (T > 1e30f) continue;
          std::vector<float> x(V);  // differences of a few units of an exponent
          for (int i = 0; i < V; ++i) x[i] = 1.5f + (float)(i % 7) * T * 0.7f;
          check("near", x, T, g, h, V / 2);
        }
  std::printf("%lld values\n", checks);
  return 0;
}
