// extern "C" entry points of the vocabulary's two ends of a policy-gradient pass: argument checks and launches.  See
// include/rollout.h for the contract of each.
#include <cmath>

#include "api_guard.h"
#include "vocab.h"

static_assert(VT_F32 == ROLLOUT_DTYPE_F32 && VT_BF16 == ROLLOUT_DTYPE_BF16 && VT_F16 == ROLLOUT_DTYPE_F16, "one numbering");
static_assert(kTopMax == ROLLOUT_TOP_MAX, "one limit");

namespace {

constexpr int kMaxRows = 1 << 24, kMaxVocab = 1 << 24, kMaxHidden = 1 << 20;

void check_sizes(int rows, int vocab, int hidden) {
  if (rows < 0 || rows > kMaxRows) fail(ROLLOUT_E_INVAL, "rows must be within 0 .. 2^24");
  if (vocab < 1 || vocab > kMaxVocab) fail(ROLLOUT_E_INVAL, "vocab must be within 1 .. 2^24");
  if (hidden < 1 || hidden > kMaxHidden) fail(ROLLOUT_E_INVAL, "hidden must be within 1 .. 2^20");
}
// launches of a workgroup to a row count their threads in 32 bits
void check_row_launch(int rows) {
  if (rows > kMaxRows - 64) fail(ROLLOUT_E_INVAL, "rows must not exceed 2^24 - 64");
}
// what the launches count in 32 bits
void check_product(int rows, int hidden) {
  if ((int64_t)rows * hidden > (int64_t)1 << 38) fail(ROLLOUT_E_INVAL, "rows x hidden must not exceed 2^38");
}
void check_tiles(int rows, int vocab) {
  if ((int64_t)(rows / 128 + 1) * (vocab / 128 + 1) > (int64_t)1 << 28)
    fail(ROLLOUT_E_INVAL, "rows x vocab must not exceed 2^42");
}
void check_dtype(int dtype) {
  if (dtype != VT_F32 && dtype != VT_BF16 && dtype != VT_F16) fail(ROLLOUT_E_INVAL, "unknown dtype");
}
void check_array(const void* p, size_t align, const char* name) {
  if (!p) fail(ROLLOUT_E_INVAL, std::string(name) + " is null");
  if ((size_t)p % align) fail(ROLLOUT_E_INVAL, std::string(name) + " must be aligned to " + std::to_string(align) + " bytes");
}
void check_optional(const void* p, size_t align, const char* name) {
  if (p) check_array(p, align, name);
}
constexpr int64_t kMaxStride = (int64_t)1 << 36;
void check_stride(int64_t stride, int width, const char* name) {
  if (stride < width || stride > kMaxStride) fail(ROLLOUT_E_INVAL, std::string(name) + " must be from the row's length to 2^36");
}
// operands of matrix products: 256 rows are reached by a 32-bit offset in bytes
void check_operand_stride(int64_t stride, int width, const char* name) {
  if (stride < width || stride > (int64_t)1 << 22 || stride % 8)
    fail(ROLLOUT_E_INVAL, std::string(name) + " must be a multiple of 8 from the row's length to 2^22");
}
float inverse(float temperature) {
  const float inv = 1.0f / temperature;
  if (!(temperature > 0.f) || !(temperature <= 3.0e38f) || !std::isfinite(inv * kLog2e))
    fail(ROLLOUT_E_INVAL, "temperature must be positive and finite, and so its inverse");
  return inv;
}
void check_scale(float scale) {
  if (!std::isfinite(scale)) fail(ROLLOUT_E_INVAL, "scale must be finite");
}
void check_workspace(const void* p, size_t bytes, size_t need) {
  if (need == 0) return;
  if (bytes < need)
    fail(ROLLOUT_E_INVAL, "workspace of " + std::to_string(bytes) + " bytes, " + std::to_string(need) + " are needed");
  check_array(p, 16, "workspace");
}
// Two arrays of `rows` rows each, in bytes, that must not share any: rows of one stride may lie between each other's.
struct Extent {
  size_t at;
  int64_t rows, width, stride;
  size_t end() const { return at + (size_t)((rows - 1) * stride + width); }
};
Extent extent(const void* p, int64_t rows, int64_t width, int64_t stride, size_t size) {
  return Extent{(size_t)p, rows, width * (int64_t)size, stride * (int64_t)size};
}
void check_apart(const Extent& a, const Extent& b, const char* names) {
  if (a.rows <= 0 || b.rows <= 0 || a.end() <= b.at || b.end() <= a.at) return;
  if (a.stride == b.stride && a.rows > 1 && b.rows > 1) {
    const int64_t d = (int64_t)((b.at > a.at ? b.at - a.at : a.at - b.at) % (size_t)a.stride);
    const int64_t first = b.at > a.at ? a.width : b.width, second = b.at > a.at ? b.width : a.width;
    if (d >= first && d + second <= a.stride) return;
  }
  fail(ROLLOUT_E_INVAL, std::string(names) + " must not overlap");
}
void check_top(int top, int vocab) {
  if (top < 0 || top > ROLLOUT_TOP_MAX || top > vocab) fail(ROLLOUT_E_INVAL, "top must be within 0 .. min(vocab, ROLLOUT_TOP_MAX)");
}

template <typename F>
void enqueue(F&& launches) {
  (void)hipGetLastError();  // an older error of the thread is not this launch's
  launches();
  HIP_TRY(hipGetLastError());
}

// bytes, or the error code of what `body` refuses
template <typename F>
int64_t bytes_of(F&& body) {
  int64_t bytes = 0;
  const int rc = guarded(nullptr, [&] { bytes = (int64_t)body(); });
  return rc == ROLLOUT_OK ? bytes : rc;
}

void check_gradients(const float* row_stats, const float* entropy, const float* grad_logp, const float* grad_entropy) {
  check_array(row_stats, 4, "row_stats");
  check_array(grad_logp, 4, "grad_logp");
  check_optional(grad_entropy, 4, "grad_entropy");
  if (grad_entropy) check_array(entropy, 4, "entropy");
}

HeadArgs head_args(const void* hidden_states, int64_t hidden_stride, const void* lm_head, int64_t head_stride, int rows,
                   int vocab, int hidden, float temperature, const int32_t* targets) {
  check_sizes(rows, vocab, hidden);
  if (hidden % 64) fail(ROLLOUT_E_INVAL, "hidden must be a multiple of 64");
  check_product(rows, hidden);
  check_tiles(rows, vocab);
  check_row_launch(rows);
  check_operand_stride(hidden_stride, hidden, "hidden_stride");
  check_operand_stride(head_stride, hidden, "head_stride");
  check_optional(targets, 4, "targets");
  check_array(lm_head, 16, "lm_head");
  if (rows > 0) check_array(hidden_states, 16, "hidden_states");
  return HeadArgs{hidden_states, hidden_stride, lm_head, head_stride, rows, vocab, hidden, inverse(temperature), targets};
}

}  // namespace

extern "C" {

int64_t rollout_token_logprobs_workspace(int32_t rows, int32_t vocab, int32_t top) {
  return bytes_of([&] {
    check_sizes(rows, vocab, 1);
    check_row_launch(rows);
    check_top(top, vocab);
    return token_workspace(rows, vocab, top);
  });
}

int rollout_token_logprobs(const void* logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride,
                           float temperature, const int32_t* targets, int32_t top, void* workspace,
                           size_t workspace_bytes, void* hip_stream, float* logp, float* entropy, float* row_stats,
                           int32_t* top_ids, float* top_logp) {
  return guarded(nullptr, [&] {
    check_sizes(rows, vocab, 1);
    check_row_launch(rows);
    check_dtype(dtype);
    check_top(top, vocab);
    check_stride(row_stride, vocab, "row_stride");
    const float inv_temp = inverse(temperature);
    if (rows == 0) return;
    check_array(logits, vt_size(dtype), "logits");
    check_optional(targets, 4, "targets");
    check_array(logp, 4, "logp");
    check_array(entropy, 4, "entropy");
    check_array(row_stats, 4, "row_stats");
    if (top) {
      check_array(top_ids, 4, "top_ids");
      check_array(top_logp, 4, "top_logp");
    }
    check_workspace(workspace, workspace_bytes, token_workspace(rows, vocab, top));
    const TokenRows in{logits, row_stride, dtype, rows, vocab, inv_temp, targets};
    const TokenOut out{logp, entropy, row_stats, top, top_ids, top_logp};
    enqueue([&] { launch_token_logprobs(in, out, workspace, (hipStream_t)hip_stream); });
  });
}

int rollout_token_logprobs_grad(const void* logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride,
                                float temperature, const int32_t* targets, const float* row_stats, const float* entropy,
                                const float* grad_logp, const float* grad_entropy, void* hip_stream, void* grad_logits,
                                int64_t grad_row_stride) {
  return guarded(nullptr, [&] {
    check_sizes(rows, vocab, 1);
    check_row_launch(rows);
    check_dtype(dtype);
    check_stride(row_stride, vocab, "row_stride");
    check_stride(grad_row_stride, vocab, "grad_row_stride");
    const float inv_temp = inverse(temperature);
    if (rows == 0) return;
    check_array(logits, vt_size(dtype), "logits");
    check_array(grad_logits, vt_size(dtype), "grad_logits");
    check_optional(targets, 4, "targets");
    check_gradients(row_stats, entropy, grad_logp, grad_entropy);
    if (grad_logits != logits)
      check_apart(extent(logits, rows, vocab, row_stride, vt_size(dtype)),
                  extent(grad_logits, rows, vocab, grad_row_stride, vt_size(dtype)), "logits and grad_logits");
    else if (grad_row_stride != row_stride)
      fail(ROLLOUT_E_INVAL, "gradients in place of the logits need their row stride");
    const TokenGrad a{{logits, row_stride, dtype, rows, vocab, inv_temp, targets}, row_stats, entropy, grad_logp,
                      grad_entropy, grad_logits, grad_row_stride};
    enqueue([&] { launch_token_logprobs_grad(a, (hipStream_t)hip_stream); });
  });
}

int rollout_embed(const void* table, int32_t dtype, int32_t vocab, int32_t hidden, int64_t table_stride,
                  const int32_t* tokens, int32_t n, float scale, void* hip_stream, void* out) {
  return guarded(nullptr, [&] {
    check_sizes(n, vocab, hidden);
    check_dtype(dtype);
    check_stride(table_stride, hidden, "table_stride");
    check_scale(scale);
    if (n == 0) return;
    check_array(table, vt_size(dtype), "table");
    check_array(tokens, 4, "tokens");
    check_array(out, vt_size(dtype), "out");
    check_product(n, hidden);
    check_apart(extent(table, vocab, hidden, table_stride, vt_size(dtype)), extent(out, n, hidden, hidden, vt_size(dtype)),
                "table and out");
    const EmbedArgs a{table, table_stride, dtype, vocab, hidden, tokens, n, scale, out};
    enqueue([&] { launch_embed_rows(a, (hipStream_t)hip_stream); });
  });
}

int64_t rollout_embed_grad_workspace(int32_t n, int32_t vocab, int32_t hidden) {
  return bytes_of([&] {
    check_sizes(n, vocab, hidden);
    return embed_grad_workspace(n, vocab, hidden);
  });
}

int rollout_embed_grad(const void* grad_rows, int32_t dtype, int32_t n, int32_t vocab, int32_t hidden, int64_t row_stride,
                       const int32_t* tokens, float scale, const void* base, int32_t table_dtype, void* workspace,
                       size_t workspace_bytes, void* hip_stream, void* grad_table) {
  return guarded(nullptr, [&] {
    check_sizes(n, vocab, hidden);
    check_dtype(dtype);
    if (table_dtype != dtype && table_dtype != VT_F32) fail(ROLLOUT_E_INVAL, "table_dtype must be dtype or ROLLOUT_DTYPE_F32");
    check_stride(row_stride, hidden, "row_stride");
    check_scale(scale);
    if (n > 0) {
      check_array(grad_rows, vt_size(dtype), "grad_rows");
      check_array(tokens, 4, "tokens");
    }
    check_optional(base, vt_size(table_dtype), "base");
    check_array(grad_table, vt_size(table_dtype), "grad_table");
    const Extent result = extent(grad_table, vocab, hidden, hidden, vt_size(table_dtype));
    check_apart(extent(grad_rows, n, hidden, row_stride, vt_size(dtype)), result, "grad_rows and grad_table");
    if (base && base != grad_table) check_apart(extent(base, vocab, hidden, hidden, vt_size(table_dtype)), result, "base and grad_table");
    check_workspace(workspace, workspace_bytes, embed_grad_workspace(n, vocab, hidden));
    const EmbedGrad a{grad_rows, row_stride, dtype, tokens, n, vocab, hidden, scale, base, table_dtype, grad_table};
    enqueue([&] { launch_embed_grad(a, workspace, (hipStream_t)hip_stream); });
  });
}

int64_t rollout_head_logprobs_workspace(int32_t rows, int32_t vocab, int32_t hidden) {
  return bytes_of([&] {
    check_sizes(rows, vocab, hidden);
    check_product(rows, hidden);
    check_tiles(rows, vocab);
    check_row_launch(rows);
    return head_workspace(rows, vocab, hidden);
  });
}

int rollout_head_logprobs(const void* hidden_states, int64_t hidden_stride, const void* lm_head, int64_t head_stride,
                          int32_t rows, int32_t vocab, int32_t hidden, float temperature, const int32_t* targets,
                          void* workspace, size_t workspace_bytes, void* hip_stream, float* logp, float* entropy,
                          float* row_stats) {
  return guarded(nullptr, [&] {
    const HeadArgs in = head_args(hidden_states, hidden_stride, lm_head, head_stride, rows, vocab, hidden, temperature, targets);
    if (rows == 0) return;
    check_array(logp, 4, "logp");
    check_array(entropy, 4, "entropy");
    check_array(row_stats, 4, "row_stats");
    check_workspace(workspace, workspace_bytes, head_workspace(rows, vocab, hidden));
    const TokenOut out{logp, entropy, row_stats, 0, nullptr, nullptr};
    enqueue([&] { launch_head_logprobs(in, out, workspace, (hipStream_t)hip_stream); });
  });
}

int64_t rollout_head_logprobs_grad_workspace(int32_t rows, int32_t vocab, int32_t hidden) {
  return bytes_of([&] {
    check_sizes(rows, vocab, hidden);
    check_product(rows, hidden);
    check_tiles(rows, vocab);
    check_row_launch(rows);
    return head_grad_workspace(rows, vocab, hidden);
  });
}

int rollout_head_logprobs_grad(const void* hidden_states, int64_t hidden_stride, const void* lm_head, int64_t head_stride,
                               int32_t rows, int32_t vocab, int32_t hidden, float temperature, const int32_t* targets,
                               const float* row_stats, const float* entropy, const float* grad_logp,
                               const float* grad_entropy, void* workspace, size_t workspace_bytes, void* hip_stream,
                               void* grad_hidden, void* grad_head) {
  return guarded(nullptr, [&] {
    const HeadArgs in = head_args(hidden_states, hidden_stride, lm_head, head_stride, rows, vocab, hidden, temperature, targets);
    check_array(grad_head, 16, "grad_head");
    if (rows > 0) {
      check_array(grad_hidden, 16, "grad_hidden");
      check_gradients(row_stats, entropy, grad_logp, grad_entropy);
    }
    const Extent states = extent(hidden_states, rows, hidden, hidden_stride, 2), head = extent(lm_head, vocab, hidden, head_stride, 2);
    const Extent d_states = extent(grad_hidden, rows, hidden, hidden, 2), d_head = extent(grad_head, vocab, hidden, hidden, 2);
    check_apart(states, d_states, "hidden_states and grad_hidden");
    check_apart(states, d_head, "hidden_states and grad_head");
    check_apart(head, d_states, "lm_head and grad_hidden");
    check_apart(head, d_head, "lm_head and grad_head");
    check_apart(d_states, d_head, "grad_hidden and grad_head");
    check_workspace(workspace, workspace_bytes, head_grad_workspace(rows, vocab, hidden));
    const HeadGrad a{in, row_stats, entropy, grad_logp, grad_entropy, grad_hidden, grad_head};
    enqueue([&] { launch_head_logprobs_grad(a, workspace, (hipStream_t)hip_stream); });
  });
}

}  // extern "C"
