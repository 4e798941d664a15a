// The arithmetic of a row's softmax sums (kernels_vocab.hip, kernels_head.hip), used by the kernels and - without a GPU - by
// the test of its range.
#pragma once
#include <cmath>

#ifdef __HIPCC__
#define ROW_SUMS_FN __host__ __device__ inline
#define ROW_SUMS_UNROLL _Pragma("unroll")
#else
#define ROW_SUMS_FN inline
#define ROW_SUMS_UNROLL
#endif

constexpr float kLog2e = 0x1.715476p+0f, kLn2 = 0x1.62e430p-1f;

ROW_SUMS_FN float row_exp2(float y) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_exp2f(y);
#else
  return exp2f(y);
#endif
}

// What one pass leaves of (a part of) a row: m = the maximum (at least the lowest finite float), and over y = (x - m) c + offset(m)
// the sums of 2^y and y 2^y, c = log2(e) / T.  Where the maximum's exponent m c is small enough (plain_exponent), the offset makes
// up for rounding it to a whole number r: one fused multiply-add, x c - r, then gives y without a rounding of r, and moving to
// another such maximum is exact.  Beyond, the product's own rounding would be a share of an exponent and soon hundreds of them,
// so that the maximum's 2^y overflows or vanishes: there the difference is taken first, and the offset is 0.
struct RowSums {
  float m, s, t;
};
constexpr float kLowest = -3.402823466e38f;

// m c is then rounded by at most an eighth, so that |offset| < 1
ROW_SUMS_FN bool plain_exponent(float mc) { return fabsf(mc) < 0x1p22f; }
ROW_SUMS_FN float offset(float m, float c) {
  const float mc = m * c;
  return plain_exponent(mc) ? fmaf(m, c, -rintf(mc)) : 0.f;
}
// binary orders of magnitude from the reference of maximum `from` up to that of `to` >= from, m c - offset(m) each; past 1e30 it
// is as good as infinite, and 0 x infinity would be NaN
ROW_SUMS_FN float raise(float from, float to, float c) {
  const float a = from * c, b = to * c;
  const float d = plain_exponent(a) && plain_exponent(b) ? rintf(b) - rintf(a) : (to - from) * c + (offset(from, c) - offset(to, c));
  return fminf(d, 1e30f);
}
ROW_SUMS_FN RowSums merge(const RowSums& p, const RowSums& q, float c) {
  const float m = fmaxf(p.m, q.m), dp = raise(p.m, m, c), dq = raise(q.m, m, c);
  const float fp = row_exp2(-dp), fq = row_exp2(-dq);
  return RowSums{m, p.s * fp + q.s * fq, (p.t - dp * p.s) * fp + (q.t - dq * q.s) * fq};
}
// s and t with N more values, none above m.  The quick form is of no use past the plain exponents, and makes a NaN of 0 x -inf for
// values whose y is -inf: such chunks are summed again with care, and what is NaN or +inf among the values stays NaN.
template <int N>
ROW_SUMS_FN RowSums sum_below(float m, float s0, float t0, const float* v, float c) {
  const float ref = rintf(m * c);
  const bool plain = plain_exponent(m * c);
  float s = s0, t = t0;
  ROW_SUMS_UNROLL
  for (int i = 0; i < N; ++i) {
    const float y = fmaf(v[i], c, -ref), e = row_exp2(y);
    s += e;
    t = fmaf(e, y, t);
  }
  if (!plain || !(fabsf(t) < 1e30f)) {
    s = s0;
    t = t0;
    ROW_SUMS_UNROLL
    for (int i = 0; i < N; ++i) {
      const float y = plain ? fmaf(v[i], c, -ref) : (v[i] - m) * c, e = row_exp2(y);
      s += e;
      t = fmaf(e, fmaxf(y, -1e30f), t);
    }
  }
  return RowSums{m, s, t};
}
// N more values; returns their maximum
template <int N>
ROW_SUMS_FN float add_chunk(RowSums& r, const float* v, float c) {
  float top = v[0];
  ROW_SUMS_UNROLL
  for (int i = 1; i < N; ++i) top = fmaxf(top, v[i]);
  const float m = fmaxf(r.m, top), d = raise(r.m, m, c), f = row_exp2(-d);
  r = sum_below<N>(m, r.s * f, (r.t - d * r.s) * f, v, c);
  return top;
}
// ln of the sum of exp((x - m) / T), from s relative to the reference; -inf for a row of nothing but -inf
ROW_SUMS_FN float row_log_sum(const RowSums& r, float c) {
  return r.s == 0.f ? -INFINITY : logf(r.s) - kLn2 * offset(r.m, c);
}
ROW_SUMS_FN float row_entropy(const RowSums& r) { return r.s == 0.f ? 0.f : logf(r.s) - kLn2 * (r.t / r.s); }

// (x - m) scale as fma(x, part, -m part) (scale / part): where the scale is below 1 a difference past fp32's range may yet give a
// value inside it, and halves leave every other difference as it is.
ROW_SUMS_FN float part_of(float scale) { return scale < 1.f ? 0.5f : 1.f; }
// ln p of a value whose x is given
ROW_SUMS_FN float row_logp(float x, float m, float inv_temp, float log_s) {
  if (log_s == -INFINITY) return -INFINITY;  // a row of nothing but -inf
  const float k = part_of(inv_temp);
  return fmaf(fmaf(x, k, -m * k), inv_temp / k, -log_s);
}

// What a row's gradient needs beside its logits: T dx = p (a + b y2) (+ at_target at the target), y2 = log2 p.  1 / T comes last:
// with small temperatures the factors would leave fp32's range where the result does not, and make a NaN of p = 0.
struct RowGrad {
  float k, mk, ck;  // part, maximum times part, log2(e) / T / part
  float l2, a, b, at_target, inv_temp;
  int target;       // -1: none
  bool none;        // the whole row is zero
};
ROW_SUMS_FN RowGrad row_grad_of(float m, float log_s, float entropy, float grad_logp, float grad_entropy, int target, float inv_temp) {
  RowGrad r;
  const float g = target < 0 ? 0.f : grad_logp, h = grad_entropy, c = inv_temp * kLog2e;
  r.target = target;
  r.k = part_of(c);
  r.mk = m * r.k;
  r.ck = c / r.k;
  r.l2 = log_s * kLog2e;
  r.none = (g == 0.f && h == 0.f) || log_s == -INFINITY;
  r.a = -g - h * entropy;
  r.b = -h * kLn2;
  r.at_target = g;
  r.inv_temp = inv_temp;
  return r;
}
// T dx away from the target.  Where p = 0, a banned id's x = -inf among others, log2 p must not meet that 0 as an infinity: 2^-256
// is 0 in fp32 already.  A NaN stays one.
ROW_SUMS_FN float grad_of(float x, const RowGrad& r) {
  const float y = fmaf(fmaf(x, r.k, -r.mk), r.ck, -r.l2);
  return row_exp2(y) * fmaf(r.b, fmaxf(y, -256.f), r.a);
}
ROW_SUMS_FN float grad_at(float x, int id, const RowGrad& r) {
  return (grad_of(x, r) + (id == r.target ? r.at_target : 0.f)) * r.inv_temp;
}
