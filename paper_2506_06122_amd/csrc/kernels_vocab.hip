// Log-probs of given tokens from logits, with entropy and the most likely alternatives, and the gradient of the logits.
//
//   y_v = x_v log2(e) / T - r,  S = sum 2^y,  ln p_v = ln2 y_v - ln S,  H = ln S - ln2 (sum y 2^y) / S, for any r
//
// One pass over the row: every thread keeps the maximum it has seen, and its two sums relative to that (row_sums.h); a chunk of
// values is taken relative to the new maximum, the old sums are scaled once a chunk.  The pass is bound by memory; the
// arithmetic (9 issue slots per value, the exponential counting four) comes next.  Chunks that hold a value of -inf are summed
// twice (a fiftieth of the values, so nearly every chunk: 2048 x 152064 bf16 146 us instead of 96).
//
// Alternatives ride along: every thread notes the maximum of each of kSegments runs of its values.  The K-th largest of
// these is a bound that K values reach, and every value that reaches it lies in a run whose maximum does.  So only those
// runs are read again, spread over the workgroup, and what reaches the bound - a few more than K - is ranked.  Rows that
// defeat this (long stretches of equal values, NaN) are found one alternative per sweep instead.
//
// A row belongs to one workgroup where rows are enough; fewer are cut into parts whose results a second launch joins.
//
// 2048 x 152064 bf16, calls in a loop: 95 us without alternatives, 6.5 TB/s (some processes 117); 109 to 111 with 8, a first call
// after other work 118.  A lone row of 151936 fp32 with 20: 7.5 to 8.6 and 7.0 us.
#include "vocab.h"
#include "vocab_vec.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int T = kTokenThreads, NW = T / WAVE;
constexpr int kListed = 1024;       // candidates a workgroup can rank
constexpr int kSegments = 4;        // runs of a thread's vectors whose maxima are kept, where each has at least kRun vectors
constexpr int kRun = 8;
constexpr int kPartValues = 2048;   // fewest values worth a workgroup
// workgroups that fill the card: two to a CU (x 152064 bf16 with 8 alternatives, us by 512 / 1024: 300 rows 31.5 / 30.7, 513 rows
// 37.3 / 48.4, 900 rows 53.0 / 65.4)
constexpr int kFill = 512;

// Order of the alternatives: greater values first, then lower ids; -0 and 0 are equal, NaN comes last.  Key 0 is nothing.
__device__ inline unsigned value_key(float x) {
  if (x != x) return 1;
  const unsigned u = __float_as_uint(x + 0.f);  // -0 + 0 = 0
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float key_value(unsigned k) {
  if (k <= 1) return __uint_as_float(0x7fc00000u);
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
__device__ inline unsigned long long full_key(unsigned key, int id) { return (unsigned long long)key << 32 | (unsigned)~id; }

// How a row lies in memory: `head` values up to the first 16-byte boundary, `vecs` vectors, `tail` values.  A part takes
// vectors [begin, end), the first part the head, the last the tail.
template <typename V>
struct RowSlice {
  const V* x;
  int head, begin, end, tail_at, tail;
  __device__ RowSlice(const V* row, int vocab, int part, int parts) {
    constexpr int E = kVec<V>;
    x = row;
    head = min(vocab, (int)((16 - ((size_t)row & 15)) & 15) / (int)sizeof(V));
    const int vecs = (vocab - head) / E, per = (vecs + parts - 1) / parts;
    begin = min(vecs, part * per);
    end = min(vecs, begin + per);
    tail_at = head + vecs * E;
    tail = part == parts - 1 ? vocab - tail_at : 0;
    if (part) head_here = 0;
    else head_here = head;
  }
  int head_here;
  __device__ u32x4 vec(int i) const { return *(const u32x4*)(x + head + (long long)i * kVec<V>); }
  __device__ int id(int i) const { return head + i * kVec<V>; }
  // the single value of thread `tid`: one of the head, or one of the tail; -1: none
  __device__ int single(int tid) const {
    if (tid < head_here) return tid;
    return tid >= WAVE && tid - WAVE < tail ? tail_at + tid - WAVE : -1;
  }
  __device__ int values() const { return head_here + (end - begin) * kVec<V> + tail; }
};

struct TopShared {
  unsigned max_key[kSegments * T];
  unsigned short hot[kSegments * T];
  unsigned bound;
  int n_hot, n_listed;
  unsigned long long best[NW];
  unsigned long long listed[kListed];
};

// A key that K or a few more of the keys reach, as near to the K-th greatest as that takes; 0 where they are fewer.  One
// wavefront, N keys to a lane.
template <int N>
__device__ inline unsigned bound_of(const unsigned* keys, int K, int lane) {
  unsigned k[N], bound = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) k[i] = keys[lane + i * WAVE];
  for (int bit = 31; bit >= 0; --bit) {
    const unsigned trial = bound | 1u << bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __popcll(__ballot(k[i] >= trial));
    if (n >= K) bound = trial;
    if (n >= K && n <= K + K / 4) break;
  }
  return bound;
}

// The K greatest keys of the slice, greatest first, through emit(rank, key); ranks past the slice's values get key 0.
// sh.max_key holds the maxima of the threads' `runs` runs of `steps` vectors, T apart.
template <typename V, typename Emit>
__device__ void top_of_slice(const RowSlice<V>& row, int runs, int steps, int K, TopShared& sh, Emit&& emit) {
  constexpr int E = kVec<V>, U = 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) sh.n_hot = sh.n_listed = 0;
  __syncthreads();
  if (wave == 0) {
    const unsigned bound = runs > 1 ? bound_of<kSegments * T / WAVE>(sh.max_key, K, lane) : bound_of<T / WAVE>(sh.max_key, K, lane);
    if (lane == 0) sh.bound = max(bound, 1u);
  }
  __syncthreads();
  const unsigned bound = sh.bound;
  for (int i = 0; i < runs; ++i)
    if (sh.max_key[i * T + tid] >= bound) sh.hot[atomicAdd(&sh.n_hot, 1)] = (unsigned short)(i * T + tid);
  auto consider = [&](float x, int id) {
    const unsigned key = value_key(x);
    if (key >= bound) {
      const int at = atomicAdd(&sh.n_listed, 1);
      if (at < kListed) sh.listed[at] = full_key(key, id);
    }
  };
  const int one = row.single(tid);
  if (one >= 0) consider(to_f32(row.x[one]), one);
  __syncthreads();
  // vector w of the runs to read: step w % steps of run hot[w / steps]; the quotient by a product is at most one off, in
  // rows of millions of values, and the remainder tells
  const int n_vecs = sh.n_hot * steps;
  const float by = 1.0f / (float)steps;
  for (int w0 = tid; w0 < n_vecs; w0 += U * T) {
    u32x4 v4[U];
    int at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int w = w0 + u * T, about = (int)(((float)w + 0.5f) * by), over = w - about * steps;
      const int h = about + (over >= steps) - (over < 0), hot = sh.hot[min(h, sh.n_hot - 1)];
      at[u] = row.begin + ((hot / T) * steps + w - h * steps) * T + hot % T;
      if (w >= n_vecs || at[u] >= row.end) at[u] = -1;
      else v4[u] = row.vec(at[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at[u] >= 0) {
        float v[E];
        widen(v4[u], v, V{});
#pragma unroll
        for (int e = 0; e < E; ++e) consider(v[e], row.id(at[u]) + e);
      }
  }
  __syncthreads();
  const int n = sh.n_listed, want = min(K, row.values());
  if (n <= kListed && n >= want) {
    for (int i = tid; i < n; i += T) {
      const unsigned long long mine = sh.listed[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += sh.listed[j] > mine;
      if (rank < want) emit(rank, mine);
    }
  } else {
    unsigned long long last = ~0ull;
    for (int k = 0; k < want; ++k) {  // the greatest key below the last one
      unsigned long long best = 0;
      auto take = [&](float x, int id) {
        const unsigned long long key = full_key(value_key(x), id);
        if (key < last && key > best) best = key;
      };
      if (one >= 0) take(to_f32(row.x[one]), one);
      for (int i = row.begin + tid; i < row.end; i += T) {
        float v[E];
        widen(row.vec(i), v, V{});
#pragma unroll
        for (int e = 0; e < E; ++e) take(v[e], row.id(i) + e);
      }
#pragma unroll
      for (int o = 1; o < WAVE; o <<= 1) best = max(best, (unsigned long long)__shfl_xor(best, o, WAVE));
      if (lane == 0) sh.best[wave] = best;
      __syncthreads();
      last = max(max(sh.best[0], sh.best[1]), max(sh.best[2], sh.best[3]));
      if (tid == 0) emit(k, last);
      __syncthreads();
    }
  }
  for (int k = want + tid; k < K; k += T) emit(k, 0ull);
}

struct TokenParts {
  int parts;
  RowSums* sums;             // [rows][parts]
  unsigned long long* keys;  // [rows][parts][top]
};

__device__ inline void store_top(const TokenOut& o, int row, int rank, unsigned long long key, float m, float log_s, float inv_temp) {
  const long long at = (long long)row * o.top + rank;
  o.top_ids[at] = (int)~(unsigned)key;
  o.top_logp[at] = row_logp(key_value((unsigned)(key >> 32)), m, inv_temp, log_s);
}

// STREAM: past the caches
template <typename V, bool TOP, bool STREAM>
__global__ __launch_bounds__(T) void token_logprobs_kernel(TokenRows in, TokenOut out, TokenParts p) {
  // vectors in flight: eight where nothing else holds registers (x 152064 bf16, 2048 rows 94 us, four 99; but through the caches 300
  // rows 23.2 and 21.5, with 8 alternatives 2048 rows 129 and 122)
  constexpr int E = kVec<V>, U = STREAM && !TOP ? 8 : 4;
  __shared__ RowSums wave_s[NW];
  __shared__ float log_s_s;
  __shared__ std::conditional_t<TOP, TopShared, int> sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = blockIdx.x / p.parts, part = blockIdx.x % p.parts;
  const RowSlice<V> row((const V*)in.logits + r * in.stride, in.vocab, part, p.parts);
  const float c = in.inv_temp * kLog2e;
  const int target = in.targets ? in.targets[r] : -1;
  const bool has_target = target >= 0 && target < in.vocab;
  const float x_target = has_target && p.parts == 1 ? to_f32(row.x[target]) : 0.f;
  // the reference starts at the lowest finite value: a row of -inf then has differences of -inf, not NaN
  RowSums sums{kLowest, 0.f, 0.f};
  const int one = row.single(tid);
  const int vecs = row.end - row.begin, runs = TOP && vecs >= kSegments * kRun * T ? kSegments : 1;
  const int steps = max(1, (vecs + runs * T - 1) / (runs * T));
  for (int q = 0; q < runs; ++q) {
    int i = row.begin + q * steps * T + tid;
    const int end = min(row.end, row.begin + (q + 1) * steps * T);
    const bool has = i < end;
    float top = -INFINITY;
    for (; i + (U - 1) * T < end; i += U * T) {
      u32x4 w[U];
      float v[U * E];
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = STREAM ? __builtin_nontemporal_load((const u32x4*)(row.x + row.id(i + u * T))) : row.vec(i + u * T);
#pragma unroll
      for (int u = 0; u < U; ++u) widen(w[u], v + u * E, V{});
      top = fmaxf(top, add_chunk<U * E>(sums, v, c));
    }
    u32x4 w[U - 1];
    float v[E];
#pragma unroll
    for (int u = 0; u < U - 1; ++u)
      if (i + u * T < end) w[u] = row.vec(i + u * T);
#pragma unroll
    for (int u = 0; u < U - 1; ++u)
      if (i + u * T < end) {
        widen(w[u], v, V{});
        top = fmaxf(top, add_chunk<E>(sums, v, c));
      }
    if constexpr (TOP) sh.max_key[q * T + tid] = has ? value_key(top) : 0;
  }
  if (one >= 0) {
    const float x = to_f32(row.x[one]);
    add_chunk<1>(sums, &x, c);
  }
  const RowSums all = merge_wave(sums, c);
  if (lane == 0) wave_s[wave] = all;
  __syncthreads();
  RowSums total = wave_s[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) total = merge(total, wave_s[w], c);
  if (p.parts == 1) {
    if (tid == 0) log_s_s = finish_row(total, out, r, has_target, x_target, in.inv_temp);
  } else if (tid == 0) {
    p.sums[(long long)r * p.parts + part] = total;
  }
  if constexpr (TOP) {
    __syncthreads();
    const float log_s = p.parts == 1 ? log_s_s : 0.f;
    top_of_slice(row, runs, steps, out.top, sh, [&](int rank, unsigned long long key) {
      if (p.parts == 1) store_top(out, r, rank, key, total.m, log_s, in.inv_temp);
      else p.keys[((long long)r * p.parts + part) * out.top + rank] = key;
    });
  }
}

// Joins a row's parts.  An alternative of the row is one of its part's.
template <typename V, bool TOP>
__global__ __launch_bounds__(T) void token_join_kernel(TokenRows in, TokenOut out, TokenParts p) {
  __shared__ RowSums wave_s[NW];
  __shared__ float log_s_s;
  __shared__ unsigned long long least_s;
  __shared__ int n_s;
  extern __shared__ unsigned long long listed[];  // [parts * top]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x;
  const float c = in.inv_temp * kLog2e;
  const int target = in.targets ? in.targets[r] : -1;
  const bool has_target = target >= 0 && target < in.vocab;
  const float x_target = has_target ? to_f32(((const V*)in.logits + r * in.stride)[target]) : 0.f;
  if (tid == 0) n_s = 0;
  // what is looked at later is on its way meanwhile: the first keys of every thread, and of every part's `deep` greatest the
  // last (see below)
  constexpr int AHEAD = 5;
  const unsigned long long* keys = p.keys + (long long)r * p.parts * out.top;
  const int n_keys = p.parts * out.top, deep = (2 * out.top + p.parts - 1) / p.parts, wide = TOP ? (out.top + deep - 1) / deep : 0;
  unsigned long long ahead[AHEAD], deep_key = 0;
  if constexpr (TOP) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) ahead[u] = tid + u * T < n_keys ? keys[tid + u * T] : 0;
    if (tid < p.parts) deep_key = keys[(long long)tid * out.top + deep - 1];
  }
  RowSums mine{kLowest, 0.f, 0.f};
  for (int i = tid; i < p.parts; i += T) mine = merge(mine, p.sums[(long long)r * p.parts + i], c);
  mine = merge_wave(mine, c);
  if (lane == 0) wave_s[wave] = mine;
  __syncthreads();
  RowSums total = wave_s[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) total = merge(total, wave_s[w], c);
  if (tid == 0) log_s_s = finish_row(total, out, r, has_target, x_target, in.inv_temp);
  if constexpr (TOP) {
    // Of every part's `deep` greatest keys the last: the `wide`-th greatest of these is a bound that K keys reach, and
    // with about half the parts above it few more do
    if (wave == 0) {
      const unsigned long long key = deep_key;
      int rank = 0;
      for (int j = 0; j < p.parts; ++j) {
        const unsigned long long other = (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(key >> 32), j) << 32 |
                                         (unsigned)__builtin_amdgcn_readlane((int)key, j);
        rank += other > key || (other == key && j < lane);
      }
      if (lane < p.parts && rank == wide - 1) least_s = key;
    }
    __syncthreads();
    const unsigned long long least = max(least_s, 1ull);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (ahead[u] >= least) listed[atomicAdd(&n_s, 1)] = ahead[u];
    for (int i = tid + AHEAD * T; i < n_keys; i += T) {
      const unsigned long long key = keys[i];
      if (key >= least) listed[atomicAdd(&n_s, 1)] = key;
    }
    __syncthreads();
    const int n = n_s;
    for (int i = tid; i < n; i += T) {
      const unsigned long long key = listed[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += listed[j] > key;
      if (rank < out.top) store_top(out, r, rank, key, total.m, log_s_s, in.inv_temp);
    }
  }
}

// dx_v = [g (1{v = t} - p_v) - h p_v (ln p_v + H)] / T, value by value; a row without a gradient is written without being
// read.  SAME: rows of both arrays lie alike relative to 16 bytes.
//
// Bound by memory: a thread takes one vector, so that the workgroups that run at a time read and write neighbouring
// addresses, and what does not fit the last cache passes it by (STREAM).  6144 x 152064 bf16, all rows with a
// gradient: 601 us, 6.2 TB/s; with four vectors to a thread, through the caches, 736.
template <typename V, bool SAME, bool STREAM>
__global__ __launch_bounds__(T) void token_grad_kernel(TokenGrad a, int parts) {
  constexpr int E = kVec<V>;
  const int tid = threadIdx.x, r = blockIdx.x / parts, part = blockIdx.x % parts;
  const RowSlice<V> row((const V*)a.in.logits + r * a.in.stride, a.in.vocab, part, parts);
  V* out = (V*)a.out + r * a.out_stride;
  const RowGrad g = row_grad(a.row_stats, a.entropy, a.grad_logp, a.grad_entropy, a.in.targets, a.in.inv_temp, a.in.vocab, r);
  auto store = [&](int i, const float* v) {
    if constexpr (SAME) {
      u32x4* to = (u32x4*)(out + row.id(i));
      const u32x4 w = narrow(v, V{});
      if constexpr (STREAM) __builtin_nontemporal_store(w, to);
      else *to = w;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) out[row.id(i) + e] = narrow1(v[e], V{});
    }
  };
  const int one = row.single(tid);
  if (g.none) {
    float zero[E] = {};
    for (int i = row.begin + tid; i < row.end; i += T) store(i, zero);
    if (one >= 0) out[one] = narrow1(0.f, V{});
    return;
  }
  for (int i = row.begin + tid; i < row.end; i += T) {
    float v[E];
    widen(STREAM ? __builtin_nontemporal_load((const u32x4*)(row.x + row.id(i))) : row.vec(i), v, V{});
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = grad_of(v[e], g);
    const unsigned at = (unsigned)(g.target - row.id(i));
    if (at < E) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += at == e ? g.at_target : 0.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= g.inv_temp;
    store(i, v);
  }
  if (one >= 0) out[one] = narrow1(grad_at(to_f32(row.x[one]), one, g), V{});
}

TokenParts layout(int rows, int vocab, int top, void* ws) {
  TokenParts p{};
  p.parts = token_parts(rows, vocab);
  p.keys = (unsigned long long*)ws;
  p.sums = (RowSums*)(p.keys + (size_t)rows * p.parts * top);
  return p;
}

template <typename V>
void launch(const TokenRows& in, const TokenOut& out, const TokenParts& p, hipStream_t s) {
  const int grid = in.rows * p.parts;
  // logits larger than the last cache (x 152064 bf16, us past / through the caches: 2048 rows 99 / 107, 1300 rows with 8
  // alternatives 85 / 91, 1000 rows 58 / 58)
  const bool stream = (long long)in.rows * in.vocab * (long long)sizeof(V) > kLastCache;
  const auto pass = [&](auto top, auto past) {
    token_logprobs_kernel<V, decltype(top)::value, decltype(past)::value><<<grid, T, 0, s>>>(in, out, p);
  };
  const auto by_size = [&](auto top) { stream ? pass(top, std::true_type{}) : pass(top, std::false_type{}); };
  out.top ? by_size(std::true_type{}) : by_size(std::false_type{});
  if (p.parts == 1) return;
  if (out.top) token_join_kernel<V, true><<<in.rows, T, (size_t)p.parts * out.top * 8, s>>>(in, out, p);
  else token_join_kernel<V, false><<<in.rows, T, 0, s>>>(in, out, p);
}

template <typename V>
void launch_grad(const TokenGrad& a, hipStream_t s) {
  const size_t size = sizeof(V);
  const bool same = (((size_t)a.in.logits - (size_t)a.out) & 15) == 0 && ((a.in.stride - a.out_stride) * size & 15) == 0;
  // both arrays together larger than the last cache (512 x 152064 bf16: 51 us past it, 57 through; 128 rows 15.4 and 14.7)
  const bool stream = 2ll * a.in.rows * a.in.vocab * size > kLastCache;
  // a vector to a thread, as long as 32 bits count the threads
  int parts = std::max(1, ceil_div(a.in.vocab, T * kVec<V>));
  while (parts > 1 && (long long)a.in.rows * parts > 0xffffff) parts = (parts + 1) / 2;
  const int grid = a.in.rows * parts;
  if (same && stream) token_grad_kernel<V, true, true><<<grid, T, 0, s>>>(a, parts);
  else if (same) token_grad_kernel<V, true, false><<<grid, T, 0, s>>>(a, parts);
  else token_grad_kernel<V, false, false><<<grid, T, 0, s>>>(a, parts);
}

}  // namespace

// Parts of a row: as many workgroups as fill the card, none with fewer than kPartValues values, at most 64 (64 x 64 keys
// are 32 KB of LDS in the join).
int token_parts(int rows, int vocab) {
  return std::max(1, std::min({ceil_div(kFill, std::max(rows, 1)), vocab / kPartValues, 64}));
}
size_t token_workspace(int rows, int vocab, int top) {
  const int parts = token_parts(rows, vocab);
  return parts == 1 ? 0 : (size_t)rows * parts * (sizeof(RowSums) + 8 * (size_t)top);
}
void launch_token_logprobs(const TokenRows& in, const TokenOut& out, void* ws, hipStream_t s) {
  const TokenParts p = layout(in.rows, in.vocab, out.top, ws);
  if (in.dtype == VT_F32) launch<float>(in, out, p, s);
  else if (in.dtype == VT_BF16) launch<bf16_t>(in, out, p, s);
  else launch<f16_t>(in, out, p, s);
}
void launch_token_logprobs_grad(const TokenGrad& a, hipStream_t s) {
  if (a.in.dtype == VT_F32) launch_grad<float>(a, s);
  else if (a.in.dtype == VT_BF16) launch_grad<bf16_t>(a, s);
  else launch_grad<f16_t>(a, s);
}
