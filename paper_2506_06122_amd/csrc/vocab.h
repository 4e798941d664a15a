// Host-callable launchers of the operators at the vocabulary's two ends of a policy-gradient pass (api_vocab.hip):
// log-probs of given tokens from logits with their gradient, the same from hidden states and the lm_head matrix, embedding
// lookup and gradient.  All launches are asynchronous on the given stream; every pointer is device memory the caller owns.
#pragma once
#include "common.h"
#include "row_sums.h"

// Element type of a caller's tensor: ROLLOUT_DTYPE_*.
enum { VT_F32 = 0, VT_BF16 = 1, VT_F16 = 2 };
constexpr size_t vt_size(int dtype) { return dtype == VT_F32 ? 4 : 2; }

constexpr long long kLastCache = 256ll << 20;  // bytes of the cache before memory

// Workgroups of 256 threads: a launch counts the threads along x in 32 bits, so that more than 2^23 workgroups go into rows
// of the grid.  The last row may reach past `blocks`.
inline dim3 many_blocks(long long blocks) {
  const long long x = 1ll << 23;
  return blocks <= x ? dim3((unsigned)blocks) : dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

// ---- logits ------------------------------------------------------------------------------
constexpr int kTopMax = 64;        // alternatives per row
constexpr int kTokenThreads = 256;

struct TokenRows {
  const void* logits;
  long long stride;  // elements between rows
  int dtype, rows, vocab;
  float inv_temp;
  const int* targets;  // [rows] or NULL; ids outside [0, vocab): no target
};
struct TokenOut {
  float* logp;       // [rows]
  float* entropy;    // [rows]
  float* row_stats;  // [rows][2]: maximum, ln of the sum of exp((x - maximum) / T)
  int top;
  int* top_ids;      // [rows][top]
  float* top_logp;   // [rows][top]
};
// workgroups a row is cut into
int token_parts(int rows, int vocab);
size_t token_workspace(int rows, int vocab, int top);
void launch_token_logprobs(const TokenRows& in, const TokenOut& out, void* workspace, hipStream_t s);

struct TokenGrad {
  TokenRows in;
  const float *row_stats, *entropy;          // as launch_token_logprobs left them; entropy only with grad_entropy
  const float *grad_logp, *grad_entropy;     // [rows]; grad_entropy may be NULL
  void* out;                                 // [rows][vocab], in.dtype; may be in.logits
  long long out_stride;
};
void launch_token_logprobs_grad(const TokenGrad& a, hipStream_t s);

__device__ inline RowGrad row_grad(const float* row_stats, const float* entropy, const float* grad_logp,
                                   const float* grad_entropy, const int* targets, float inv_temp, int vocab, int row) {
  const int t = targets ? targets[row] : -1;
  return row_grad_of(row_stats[2 * row], row_stats[2 * row + 1], grad_entropy ? entropy[row] : 0.f, grad_logp[row],
                     grad_entropy ? grad_entropy[row] : 0.f, t >= 0 && t < vocab ? t : -1, inv_temp);
}

// Over a wavefront without a trip through LDS; every lane gets the result.  The lanes' order is fixed.
template <int CTRL, int ROWS = 0xf>
__device__ inline float dpp(float v, float other) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <typename F>
__device__ inline float across_wave(float v, float none, F&& f) {
  v = f(v, dpp<0x111>(v, none));       // the lane 1 below in the row of 16, then 2, 4, 8
  v = f(v, dpp<0x112>(v, none));
  v = f(v, dpp<0x114>(v, none));
  v = f(v, dpp<0x118>(v, none));
  v = f(v, dpp<0x142, 0xa>(v, none));  // the last lane of the row before, into rows 1 and 3
  v = f(v, dpp<0x143, 0xc>(v, none));  // lane 31 into rows 2 and 3
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ inline RowSums merge_wave(const RowSums& r, float c) {
  const float m = across_wave(r.m, kLowest, [](float a, float b) { return fmaxf(a, b); });
  const float d = raise(r.m, m, c), f = __builtin_amdgcn_exp2f(-d);
  const auto add = [](float a, float b) { return a + b; };
  return RowSums{m, across_wave(r.s * f, 0.f, add), across_wave((r.t - d * r.s) * f, 0.f, add)};
}

// A row's results from its sums, written by one thread; x_target is read only with a target.  Returns ln S.
__device__ inline float finish_row(const RowSums& r, const TokenOut& o, int row, bool has_target, float x_target, float inv_temp) {
  const bool empty = r.s == 0.f;  // nothing but -inf
  const float log_s = row_log_sum(r, inv_temp * kLog2e);
  o.logp[row] = has_target ? row_logp(x_target, r.m, inv_temp, log_s) : 0.f;
  o.entropy[row] = row_entropy(r);
  o.row_stats[2 * row] = empty ? -INFINITY : r.s != r.s ? r.s : r.m;  // (the maximum passes NaN by)
  o.row_stats[2 * row + 1] = log_s;
  return log_s;
}

// ---- embedding ---------------------------------------------------------------------------
struct EmbedArgs {
  const void* table;
  long long table_stride;
  int dtype, vocab, hidden;
  const int* tokens;
  int n;
  float scale;
  void* out;  // [n][hidden]
};
void launch_embed_rows(const EmbedArgs& a, hipStream_t s);

struct EmbedGrad {
  const void* grad_rows;  // [n][hidden]
  long long row_stride;
  int dtype;
  const int* tokens;
  int n, vocab, hidden;
  float scale;
  const void* base;       // [vocab][hidden], out_dtype, or NULL; may be out
  int out_dtype;
  void* out;              // [vocab][hidden]
};
size_t embed_grad_workspace(int n, int vocab, int hidden);
void launch_embed_grad(const EmbedGrad& a, void* workspace, hipStream_t s);

// ---- lm_head -----------------------------------------------------------------------------
struct HeadArgs {
  const void* hidden_states;  // bf16 [rows][hidden]
  long long hidden_stride;
  const void* lm_head;        // bf16 [vocab][hidden]
  long long head_stride;
  int rows, vocab, hidden;
  float inv_temp;
  const int* targets;
};
size_t head_workspace(int rows, int vocab, int hidden);
void launch_head_logprobs(const HeadArgs& in, const TokenOut& out, void* workspace, hipStream_t s);

struct HeadGrad {
  HeadArgs in;
  const float *row_stats, *entropy, *grad_logp, *grad_entropy;
  void* grad_hidden;  // bf16 [rows][hidden]
  void* grad_head;    // bf16 [vocab][hidden]
};
size_t head_grad_workspace(int rows, int vocab, int hidden);
void launch_head_logprobs_grad(const HeadGrad& a, void* workspace, hipStream_t s);
