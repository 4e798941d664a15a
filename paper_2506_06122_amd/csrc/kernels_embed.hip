// Embedding lookup with scaling, and the gradient of the embedding matrix.
//
//   out_r = scale E[id_r];     dE_v = base_v + scale sum over r with id_r = v of dy_r
//
// Both are bound by memory.  The gradient takes three launches.  The first sorts the rows by id and meanwhile writes
// every row of the matrix (zeros, or the base), which is most of the bytes of a large vocabulary.  The second sums runs
// of equal ids in fp32, in the order of the rows, so the result does not depend on scheduling.  It takes a chunk of sorted
// rows to a workgroup whatever the ids are: a run that crosses the edge of a chunk leaves partial sums, and the third
// launch joins those in order.
//
// Lookup of 16384 rows x 3584 bf16: 34.5 us, 6.8 TB/s of results and rows that the caches hold in part.  Gradient of as many
// rows, 152064 ids: 175 us of sorting and filling (6.2 TB/s), 35 of sums, 8 of joins.
#include "vocab.h"
#include "vocab_vec.h"

#include <algorithm>

namespace {

// ---- lookup --------------------------------------------------------------------------------
// One thread per 16 bytes of the result (VEC), or per value where rows are not whole, aligned vectors.
template <typename V, bool VEC, bool STREAM>
__global__ __launch_bounds__(256) void embed_rows_kernel(EmbedArgs a, int per_row) {
  constexpr int E = VEC ? kVec<V> : 1;
  const long long at = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
  const long long r = at / per_row;
  if (r >= a.n) return;
  const int col = (int)(at - r * per_row) * E;
  const int id = a.tokens[r];
  const bool inside = id >= 0 && id < a.vocab;
  const V* src = (const V*)a.table + (inside ? (long long)id * a.table_stride : 0) + col;
  V* dst = (V*)a.out + r * a.hidden + col;
  if constexpr (VEC) {
    u32x4 w = {0, 0, 0, 0};
    if (inside) {
      w = *(const u32x4*)src;
      if (a.scale != 1.f) {
        float v[E];
        widen(w, v, V{});
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= a.scale;
        w = narrow(v, V{});
      }
    }
    if constexpr (STREAM) __builtin_nontemporal_store(w, (u32x4*)dst);
    else *(u32x4*)dst = w;
  } else {
    *dst = !inside ? narrow1(0.f, V{}) : a.scale == 1.f ? *src : narrow1(to_f32(*src) * a.scale, V{});
  }
}

template <typename V>
void launch_rows(const EmbedArgs& a, hipStream_t s) {
  constexpr int E = kVec<V>;
  const bool vec = a.hidden % E == 0 && a.table_stride % E == 0 && (((size_t)a.table | (size_t)a.out) & 15) == 0;
  const int per_row = vec ? a.hidden / E : a.hidden;
  const dim3 grid = many_blocks(((long long)a.n * per_row + 255) / 256);
  // results larger than the XCDs' own caches go past them (x 3584 bf16, us past / through: 1024 rows 7.03 / 7.02, 4096 rows
  // 8.6 / 10.5, 16384 rows 34.5 / 43.5)
  const bool stream = (long long)a.n * a.hidden * sizeof(V) > 16 << 20;
  if (vec && stream) embed_rows_kernel<V, true, true><<<grid, 256, 0, s>>>(a, per_row);
  else if (vec) embed_rows_kernel<V, true, false><<<grid, 256, 0, s>>>(a, per_row);
  else embed_rows_kernel<V, false, false><<<grid, 256, 0, s>>>(a, per_row);
}

// ---- gradient ------------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / WAVE;
constexpr int kRange = 512;   // ids of a sorting workgroup at most: kSortWaves counters each are 32 KB of LDS
// sorted rows of a summing workgroup: as many rows as fill the card, each workgroup with a few in flight; with many rows more,
// since each chunk may leave two rows of partial sums (152064 x 3584 bf16 on top of a base, us with 4 / 16: 1021 rows 14.5 / 17.8,
// 4096 rows 26.2 / 27.8, 8192 rows 43.0 / 40.3)
constexpr int chunk_rows(int n) { return n <= 4096 ? 4 : 16; }
// 16-byte vectors of the matrix that a filling workgroup writes (`filled`): one to a thread where they are many, so that the workgroups that
// run at a time write neighbouring addresses (whole calls, us by 1 / 8 to a thread: 1021 rows, 152064 x 3584 bf16 184 / 194, with a base in fp32
// 822 / 860, but 4096 rows, 32001 x 1536 28.8 / 24.5)
// (past 32 GB again eight: 32 bits count a launch's threads)
constexpr int fill_vectors(long long bytes) { return bytes > kLastCache && bytes <= 32ll << 30 ? kSortThreads : 8 * kSortThreads; }

struct EmbedSort {
  int* row;        // [n] rows sorted by id, equal ids in the order of the rows
  int* id;         // [n] their ids
  int* n_inside;   // rows whose id is inside the vocabulary
  float* first;    // [chunks][hidden]: a chunk's share of the run that began in an earlier chunk
  float* last;     // [chunks][hidden]: its share of the run that it begins and a later chunk ends
};
struct EmbedPlan {
  int ranges, range;  // sorting workgroups and the ids of each
  int chunk, chunks;
};
EmbedPlan plan(int n, int vocab) {
  EmbedPlan p;
  // up to 256 workgroups, one to a CU, unless a range would outgrow its LDS; with few rows fewer, wider ranges
  const int wanted = std::max(ceil_div(vocab, kRange), std::min(256, ceil_div(n, 16)));
  p.range = ceil_div(vocab, std::min(wanted, vocab));
  p.ranges = ceil_div(vocab, p.range);
  p.chunk = chunk_rows(n);
  p.chunks = ceil_div(n, p.chunk);
  return p;
}

// Workgroup b of the first `ranges` takes the ids [lo, hi) of its range.  Its wavefronts count a contiguous share of the
// rows each, per id, and the rows with lower ids; so each knows where its first row of every id belongs, and a second
// walk puts them there: the order within an id is the order of the rows, and no workgroup waits for another.  The
// workgroups behind them fill the matrix.
template <typename G>
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(EmbedGrad a, EmbedSort q, int ranges, int range, int filled, bool fill, bool large) {
  __shared__ int count_s[kSortWaves][kRange];
  __shared__ int below_s[kSortWaves], scan_s[kSortWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if ((int)blockIdx.x >= ranges) {  // out = base, or 0
    if (!fill) return;
    constexpr int E = kVec<G>;
    const long long total = (long long)a.vocab * a.hidden;
    const long long block = blockIdx.x - ranges, me = block * kSortThreads + tid;
    G* out = (G*)a.out;
    const G* base = (const G*)a.base;
    const G zero = narrow1(0.f, G{});
    const long long head = min(total, (long long)((16 - ((size_t)out & 15)) & 15) / (long long)sizeof(G));
    const long long vecs = (total - head) / E, tail = head + vecs * E;
    if (me < head) out[me] = base ? base[me] : zero;
    if (me < total - tail) out[tail + me] = base ? base[tail + me] : zero;
    u32x4* o = (u32x4*)(out + head);
    const u32x4* b = (const u32x4*)(base + head);
    const u32x4 none = {0, 0, 0, 0};
    const long long first = block * filled + tid, end = min(vecs, (block + 1) * (long long)filled);
    // what is larger than the last cache passes it by (152064 x 3584 in bf16, the whole call: 248 -> 232 us)
    if (!base && large) {
#pragma unroll 4
      for (long long i = first; i < end; i += kSortThreads) __builtin_nontemporal_store(none, o + i);
    } else if (!base) {
#pragma unroll 4
      for (long long i = first; i < end; i += kSortThreads) o[i] = none;
    } else if (large && (((size_t)base - (size_t)out) & 15) == 0) {
#pragma unroll 4
      for (long long i = first; i < end; i += kSortThreads) __builtin_nontemporal_store(__builtin_nontemporal_load(b + i), o + i);
    } else if ((((size_t)base - (size_t)out) & 15) == 0) {
#pragma unroll 4
      for (long long i = first; i < end; i += kSortThreads) o[i] = b[i];
    } else {
      for (long long i = head + first * E; i < head + end * E; i += kSortThreads * E)
        for (int e = 0; e < E; ++e) out[i + e] = base[i + e];
    }
    return;
  }
  const int lo = blockIdx.x * range, hi = min(a.vocab, lo + range);
  for (int i = tid; i < kSortWaves * kRange; i += kSortThreads) (&count_s[0][0])[i] = 0;
  __syncthreads();
  const int share = (a.n + kSortWaves * WAVE - 1) / (kSortWaves * WAVE) * WAVE;
  const int begin = min(a.n, wave * share), end = min(a.n, begin + share);
  int below = 0;
  for (int i = begin + lane; i < end; i += WAVE) {
    const int id = a.tokens[i];
    if (id >= lo && id < hi) atomicAdd(&count_s[wave][id - lo], 1);
    else if (id >= 0 && id < lo) ++below;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) below += __shfl_xor(below, o, WAVE);
  if (lane == 0) below_s[wave] = below;
  __syncthreads();
  // exclusive scan over the ids, and per id over the wavefronts
  int mine = 0;
  if (tid < kRange)
    for (int w = 0; w < kSortWaves; ++w) mine += count_s[w][tid];
  int up = mine;
#pragma unroll
  for (int o = 1; o < WAVE; o <<= 1) {
    const int v = __shfl_up(up, o, WAVE);
    if (lane >= o) up += v;
  }
  if (lane == WAVE - 1) scan_s[wave] = up;
  __syncthreads();
  int at = up - mine, all = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    at += below_s[w] + (w < wave ? scan_s[w] : 0);
    all += below_s[w] + scan_s[w];
  }
  if (tid == 0 && (int)blockIdx.x == ranges - 1) *q.n_inside = all;
  if (tid < kRange)
    for (int w = 0; w < kSortWaves; ++w) {
      const int n = count_s[w][tid];
      count_s[w][tid] = at;
      at += n;
    }
  __syncthreads();
  for (int i0 = begin; i0 < end; i0 += WAVE) {
    const int i = i0 + lane, id = i < end ? a.tokens[i] : -1;
    const bool inside = id >= lo && id < hi;
    unsigned long long left = __ballot(inside);
    while (left) {  // one id at a time; lanes are rows in order
      const int leader = __builtin_ctzll(left), its = __builtin_amdgcn_readlane(id, leader);
      const unsigned long long same = __ballot(inside && id == its);
      int base = 0;
      if (lane == leader) base = atomicAdd(&count_s[wave][its - lo], __popcll(same));
      base = __builtin_amdgcn_readlane(base, leader);
      if (same >> lane & 1) {
        const int to = base + __popcll(same & ((1ull << lane) - 1));
        q.row[to] = i;
        q.id[to] = id;
      }
      left &= ~same;
    }
  }
}

// E values of a gradient row (VEC), or one
template <typename V, bool VEC, int E>
__device__ inline void load_row(const V* p, float* v) {
  if constexpr (VEC) {
    if constexpr (E == kVec<V>) {
      widen(*(const u32x4*)p, v, V{});
    } else {  // 8 floats
      widen(((const u32x4*)p)[0], v, V{});
      widen(((const u32x4*)p)[1], v + 4, V{});
    }
  } else {
    v[0] = to_f32(*p);
  }
}
template <typename G, bool VEC, int E>
__device__ inline void store_row(const EmbedGrad& a, int id, int col, const float* sum) {
  const long long at = (long long)id * a.hidden + col;
  G* out = (G*)a.out + at;
  float v[E];
  if (a.base) load_row<G, VEC, E>((const G*)a.base + at, v);
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = a.base ? fmaf(sum[e], a.scale, v[e]) : sum[e] * a.scale;
  if constexpr (VEC) {
#pragma unroll
    for (int e = 0; e < E; e += kVec<G>) *(u32x4*)(out + e) = narrow(v + e, G{});
  } else {
    *out = narrow1(v[0], G{});
  }
}

template <typename V, typename G, bool VEC, int kChunk>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedGrad a, EmbedSort q) {
  constexpr int E = VEC ? 8 : 1;
  __shared__ int row_s[kChunk], id_s[kChunk + 2];  // ids from the one before the chunk to the one behind it
  const int tid = threadIdx.x, chunk = blockIdx.x, col = (blockIdx.y * blockDim.x + tid) * E;
  const int n = *q.n_inside, begin = chunk * kChunk, end = min(n, begin + kChunk);
  if (begin >= end) return;
  if (tid < kChunk + 2) {
    const int i = begin + tid - 1;
    id_s[tid] = i >= 0 && i < n ? q.id[i] : -1;
    if (tid < kChunk) row_s[tid] = begin + tid < n ? q.row[begin + tid] : 0;
  }
  __syncthreads();
  if (col >= a.hidden) return;
  const V* src = (const V*)a.grad_rows + col;
  const int count = end - begin;
  constexpr int A = 4;  // rows in flight
  float v[A][E], sum[E] = {};
  bool began = id_s[0] != id_s[1];  // the current run begins in this chunk
#pragma unroll
  for (int j = 0; j < kChunk; j += A) {
    if (j >= count) break;
#pragma unroll
    for (int u = 0; u < A; ++u)
      if (j + u < count) load_row<V, VEC, E>(src + (long long)row_s[j + u] * a.row_stride, v[u]);
#pragma unroll
    for (int u = 0; u < A; ++u) {
      if (j + u >= count) break;
      const int id = id_s[j + u + 1];
      const bool ends = id != id_s[j + u + 2];
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += v[u][e];
      if (ends || j + u == count - 1) {
        if (began && ends) {
          store_row<G, VEC, E>(a, id, col, sum);
        } else {
          float* part = (began ? q.last : q.first) + (long long)chunk * a.hidden + col;
          if constexpr (VEC) {
            *(float4*)part = make_float4(sum[0], sum[1], sum[2], sum[3]);
            *(float4*)(part + 4) = make_float4(sum[4], sum[5], sum[6], sum[7]);
          } else {
            *part = sum[0];
          }
        }
        began = true;
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.f;
      }
    }
  }
}

// A run that leaves its chunk: the chunk in which it begins takes the shares of the following ones, in order, a wavefront to 512
// columns: a long run is a chain of loads (x 3584 bf16, all three launches in place, us: 16384 rows of one id 150, of mixed ids
// 118; 10^5 rows of mixed ids 454, a fifth of them one id 630, all of them 1228).
template <typename G, bool VEC>
__global__ __launch_bounds__(64) void embed_join_kernel(EmbedGrad a, EmbedSort q, int kChunk) {
  constexpr int E = VEC ? 8 : 1;
  const int chunk = blockIdx.x, col = (blockIdx.y * 64 + threadIdx.x) * E;
  const int n = *q.n_inside, next = (chunk + 1) * kChunk;
  if (next >= n) return;
  const int id = q.id[next];
  if (q.id[next - 1] != id) return;                          // nothing crosses
  if (chunk > 0 && q.id[chunk * kChunk - 1] == id) return;   // it began earlier
  int end = chunk;  // the last chunk that the run reaches: ids are sorted, so those at the chunks' first places tell
  for (;;) {
    const long long first = (long long)(end + 1 + (int)threadIdx.x % WAVE) * kChunk;
    const unsigned long long in_run = __ballot(first < n && q.id[first < n ? first : 0] == id);
    const int more = ~in_run ? __builtin_ctzll(~in_run) : WAVE;
    end += more;
    if (more < WAVE) break;
  }
  if (col >= a.hidden) return;
  float sum[E];
  load_row<float, VEC, E>(q.last + (long long)chunk * a.hidden + col, sum);
#pragma unroll 4
  for (int k = chunk + 1; k <= end; ++k) {
    float v[E];
    load_row<float, VEC, E>(q.first + (long long)k * a.hidden + col, v);
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += v[e];
  }
  store_row<G, VEC, E>(a, id, col, sum);
}

constexpr size_t piece(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

template <typename V, typename G>
void launch_grad(const EmbedGrad& a, void* ws, hipStream_t s) {
  const EmbedPlan p = plan(a.n, a.vocab);
  char* at = (char*)ws;
  auto take = [&](size_t bytes) {
    void* r = at;
    at += piece(bytes);
    return r;
  };
  EmbedSort q;
  q.n_inside = (int*)take(4);
  q.row = (int*)take((size_t)a.n * 4);
  q.id = (int*)take((size_t)a.n * 4);
  q.first = (float*)take((size_t)p.chunks * a.hidden * 4);
  q.last = (float*)take((size_t)p.chunks * a.hidden * 4);
  const bool fill = a.base != a.out;
  const long long bytes = (long long)a.vocab * a.hidden * sizeof(G);
  const int filled = fill_vectors(bytes), fillers = fill ? ceil_div(bytes, filled * 16) : 0;
  embed_sort_kernel<G><<<p.ranges + fillers, kSortThreads, 0, s>>>(a, q, p.ranges, p.range, filled, fill, bytes > kLastCache);
  if (p.chunks == 0) return;
  // whole vectors of 8 values: every row starts on 16 bytes
  const bool vec = a.hidden % 8 == 0 && a.row_stride % 8 == 0 && (((size_t)a.grad_rows | (size_t)a.base | (size_t)a.out) & 15) == 0;
  const int cols = vec ? a.hidden / 8 : a.hidden, threads = std::min(256, ceil_div(cols, 64) * 64);
  const dim3 grid(p.chunks, ceil_div(cols, threads)), join(p.chunks - 1, ceil_div(cols, 64));
  if (vec) p.chunk == 4 ? embed_sum_kernel<V, G, true, 4><<<grid, threads, 0, s>>>(a, q) : embed_sum_kernel<V, G, true, 16><<<grid, threads, 0, s>>>(a, q);
  else p.chunk == 4 ? embed_sum_kernel<V, G, false, 4><<<grid, threads, 0, s>>>(a, q) : embed_sum_kernel<V, G, false, 16><<<grid, threads, 0, s>>>(a, q);
  if (p.chunks == 1) return;
  if (vec) embed_join_kernel<G, true><<<join, 64, 0, s>>>(a, q, p.chunk);
  else embed_join_kernel<G, false><<<join, 64, 0, s>>>(a, q, p.chunk);
}

}  // namespace

void launch_embed_rows(const EmbedArgs& a, hipStream_t s) {
  if (a.dtype == VT_F32) launch_rows<float>(a, s);
  else if (a.dtype == VT_BF16) launch_rows<bf16_t>(a, s);
  else launch_rows<f16_t>(a, s);
}

size_t embed_grad_workspace(int n, int vocab, int hidden) {
  const EmbedPlan p = plan(n, vocab);
  return piece(4) + 2 * piece((size_t)n * 4) + 2 * piece((size_t)p.chunks * hidden * 4);
}

void launch_embed_grad(const EmbedGrad& a, void* ws, hipStream_t s) {
  if (a.dtype == VT_F32) launch_grad<float, float>(a, ws, s);
  else if (a.dtype == VT_BF16) a.out_dtype == VT_F32 ? launch_grad<bf16_t, float>(a, ws, s) : launch_grad<bf16_t, bf16_t>(a, ws, s);
  else a.out_dtype == VT_F32 ? launch_grad<f16_t, float>(a, ws, s) : launch_grad<f16_t, f16_t>(a, ws, s);
}
