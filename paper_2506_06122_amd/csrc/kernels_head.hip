// Log-probs of given tokens straight from hidden states and the lm_head matrix, and the gradients of both.
//
//   x = h W^T (never stored);  sums of every row as in kernels_vocab.hip
//   g = the logits' gradient;  dh = g W;  dW = g^T h
//
// Three products of 2 R H V operations each, one of them twice (the gradient needs the logits again), so matrix-core
// bound for more than a few rows; with a few the walk over W is.  One kernel does all of them: C = A B^T over tiles, where
// each operand lies with its rows or with the summed index outermost, as the caller or the previous launch left it -
// fragments of the second kind are transposed on their way out of LDS - so that nothing is transposed in memory.
//
// 4096 x 152064 x 3584: 3.25 to 3.37 ms, 1.32 to 1.37 PFLOP/s by the card (matrix instructions two thirds of the time, the
// clock at 1.9 to 2.0 GHz under them); its gradients with respect to three quarters of the rows, three products, 8.0 to 8.4 ms, 1.20 to 1.25 PFLOP/s: slices with K
// outermost take a tenth longer.  7 x 151936 x 1536: 90 us, 5.2 TB/s of W.  In between a tile's start and end show, with 5 to 24
// stages to it and one workgroup to a CU: 160 x 151936 x 1536 136 us, 300 192, 613 305; W's bytes take 74, the products 51 to 197.
#include "vocab.h"

#include <algorithm>
#include <utility>

#include "head_tile.h"
#include "vocab_vec.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// What becomes of a tile of C
//   TO_SUMS   the logits of a row over the tile's columns become one RowSums; the target's logit is stored
//   TO_GRAD   logits become their gradients, bf16
//   TO_PLANE  fp32, one plane per split of K; with `add` on top of what is there
//   TO_BF16   bf16
enum { TO_SUMS, TO_GRAD, TO_PLANE, TO_BF16 };

struct Operand {
  const void* p;
  int pitch;  // elements between rows, or with the summed index outermost between its steps
};
struct Product {
  Operand a, b;
  int M, N, K;            // b with K outermost has exactly K steps; anything else is padded to whole slices
  const HeadActive* plan; // device: TO_GRAD's M, TO_PLANE's M and cuts of K, TO_BF16's K
  HeadGrid grid;
  bool stream_b;          // STREAM
  void* out;
  long long out_pitch;
  int room;               // rows of the panels that the gradients of logits lie in: TO_GRAD's result, the next products' A
  bool add;
  float inv_temp;
  // TO_SUMS
  const int* targets;
  RowSums* sums;        // [M][grid.n_tiles]
  float* target_logit;  // [M]
  // TO_GRAD: rows of A are rows active[.] of the caller's arrays; columns start at col0 of the vocabulary
  const int* active;
  const float *row_stats, *entropy, *grad_logp, *grad_entropy;
  int col0, vocab, row_capacity, planes;
};

__device__ __forceinline__ void load_to_lds(unsigned lds, unsigned voff, const void* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(base)
               : "memory");
}
// past the caches
__device__ __forceinline__ void load_to_lds_once(unsigned lds, unsigned voff, const void* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(lds), "v"(voff), "s"(base)
               : "memory");
}
// this wavefront's loads but the last N have arrived and its LDS reads are done; then the barrier
template <int N>
__device__ __forceinline__ void wait_and_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// over the four lanes that hold a row's columns, 16 and 32 lanes apart, in each of them
__device__ __forceinline__ float column_max(float x) {
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
  const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float column_sum(float x) {
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(h[0]) + __uint_as_float(h[1]);
  const auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
template <class F, int... I>
__device__ __forceinline__ void unrolled(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// Fragment i of half a slice in LDS
template <int C, bool KM>
__device__ __forceinline__ u32x4 fragment(const char* slice, int i, int half, int lane) {
  const char* p = slice + HeadSlice<C, KM>::fragment(i, half, lane);
  if constexpr (KM) {
    typedef __attribute__((address_space(3))) s16x4* lds_t;
    struct Two {
      s16x4 a, b;
    } v;
    v.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)p);
    v.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(p + 4 * HeadSlice<C, KM>::pitch));
    return __builtin_bit_cast(u32x4, v);
  } else {
    return *(const u32x4*)p;
  }
}

// A workgroup computes BM = 16 WM MT rows x BN = 16 WN NT columns of C; its WM x WN wavefronts own MT x NT tiles of 16 x 16
// each.  Slices of 64 steps of K go straight from memory into a ring of S LDS stages.  A stage is multiplied in two halves:
// while the first is, the second's fragments are read; then one barrier says that every wavefront holds the whole stage
// in registers, so that its buffer takes the copies of stage s + S, and that stage s + 1 has arrived (loads are counted
// in order, later stages stay in flight), whose first half is read while the second is multiplied.  The copies past the
// end of K repeat the last slice, so that every stage counts the same number of them.
// STREAM: past the caches goes a B that one row of tiles reads, once, and that is larger than the last cache (16 rows x
// 152064 x 3584 209 -> 191 us; the gradients' products 704 -> 654, 64 rows 779 -> 733).
template <int WM, int WN, int MT, int NT, int S, int TO, bool AK, bool BK, bool STREAM>
__global__ __launch_bounds__(WM* WN * 64, MT * NT >= 32 || S > 2 ? 1 : 2) void head_product_kernel(Product p) {
  constexpr bool WIDE = MT * NT >= 32;
  constexpr int NW = WM * WN, BM = WM * MT * 16, BN = WN * NT * 16;
  using A = HeadSlice<BM, AK>;
  using B = HeadSlice<BN, BK>;
  constexpr int U = A::units + B::units, L = (U + NW - 1) / NW, STAGE = U * 1024;
  // results on their way out: a wavefront's rows of bf16, 16 bytes past its width so that rows do not share banks
  constexpr int OUT_ROW = NT * 32 + 16, OUT_WAVE = MT * 16 * OUT_ROW, OUT = TO == TO_BF16 || TO == TO_GRAD ? NW * OUT_WAVE : 0;
  constexpr int EXTRA = TO == TO_GRAD ? BM * (int)sizeof(RowGrad) : TO == TO_SUMS ? WN * BM * (int)sizeof(RowSums) : 0;
  constexpr int LDS = S * STAGE > OUT + EXTRA ? S * STAGE : OUT + EXTRA;
  static_assert(LDS <= 160 * 1024 && S >= 2 && (S - 1) * L < 64, "fits the CU and the load counter");
  __shared__ __attribute__((aligned(1024))) char lds[LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int M = TO == TO_GRAD ? p.plan->count : TO == TO_PLANE ? p.plan->stacked : p.M, K = TO == TO_BF16 ? p.plan->stacked : p.K;
  HeadGrid grid = p.grid;
  const int pad = TO == TO_GRAD ? head_pad(p.planes) : 0, rows = TO == TO_GRAD ? head_up(M, pad) : M;
  if constexpr (TO == TO_GRAD || TO == TO_PLANE) grid = head_grid_rows(grid, head_ceil(rows, BM));
  if constexpr (TO == TO_PLANE) grid.splits = p.plan->splits;
  const HeadBlock block = head_block(blockIdx.y * gridDim.x + blockIdx.x, grid);
  if (!block.inside) return;
  const int bn = block.n, bz = block.z;
  const int m0 = block.m * BM, n0 = bn * BN;
  const HeadExtent x = head_extent(AK, BK, pad, m0, n0, bz, M, p.N, K, TO == TO_PLANE ? head_ceil(head_ceil(K, kHeadDeep), grid.splits) : head_ceil(K, kHeadDeep),
                                   p.row_capacity);
  if (m0 >= x.m_end) return;
  const int k_tiles = x.k_tiles, kt_begin = x.kt_begin, kt_end = x.kt_end;

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int wm = wave / WN, wn = wave % WN;
  if (kt_begin < kt_end && m0 < M) {  // (rows of zeros that pad the next product's K take no product)
    // this wavefront's loads of a stage: units wave, wave + NW, ... of A's, then B's; their sources move on with the slices
    unsigned voff[L], tail[L], dst[L];
    bool is_b[L];
    constexpr bool PANELS = TO == TO_PLANE || TO == TO_BF16;
    const int a_pitch = PANELS ? kHeadPanel : p.a.pitch;
    const long long b_step = (BK ? (long long)p.b.pitch : 1) * 2 * kHeadDeep;
    const auto a_slice = [&](int kt) __attribute__((always_inline)) {
      return (const char*)p.a.p + 2 * (PANELS ? head_panel_slice(AK, m0, kt, p.room) : (long long)m0 * p.a.pitch + kt * kHeadDeep);
    };
    const char* pa = a_slice(kt_begin);
    const char* pb = (const char*)p.b.p + 2 * (BK ? n0 : (long long)n0 * p.b.pitch) + kt_begin * b_step;
#pragma unroll
    for (int s = 0; s < L; ++s) {
      const int u = __builtin_amdgcn_readfirstlane(min(s * NW + wave, U - 1));  // an uneven last round loads the last one again
      is_b[s] = u >= A::units;
      dst[s] = u * 1024;
      if (!is_b[s]) {
        tail[s] = voff[s] = A::source(u, lane, x.a_limit, kHeadDeep, a_pitch);
      } else {
        voff[s] = B::source(u - A::units, lane, x.b_limit, kHeadDeep, p.b.pitch);
        tail[s] = BK ? B::source(u - A::units, lane, x.b_limit, x.b_last, p.b.pitch) : voff[s];
      }
    }
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) void*)lds;
    int ahead = kt_begin;  // slice of the next copies
    auto issue = [&](int s, int buf) __attribute__((always_inline)) {
      const unsigned to = __builtin_amdgcn_readfirstlane(lds0 + buf * STAGE + dst[s]);
      const unsigned from = BK && ahead == k_tiles - 1 ? tail[s] : voff[s];
      if (STREAM && is_b[s]) load_to_lds_once(to, from, pb);
      else load_to_lds(to, from, is_b[s] ? pb : pa);
    };
    auto move_on = [&]() __attribute__((always_inline)) {
      if (ahead + 1 < kt_end) {
        ++ahead;
        pa = a_slice(ahead);
        pb += b_step;
      }
    };
#pragma unroll
    for (int q = 0; q < S; ++q) {
#pragma unroll
      for (int s = 0; s < L; ++s) issue(s, q);
      move_on();
    }
    u32x4 a[2][MT], b[2][NT];
    constexpr int NR = MT + NT, NM = MT * NT;
    auto read = [&](int half, const char* st, int f) __attribute__((always_inline)) {  // in the order in which they are multiplied
      if (f < 1) a[half][0] = fragment<BM, AK>(st, wm * MT, half, lane);
      else if (f < 1 + NT) b[half][f - 1] = fragment<BN, BK>(st + A::units * 1024, wn * NT + f - 1, half, lane);
      else a[half][f - NT] = fragment<BM, AK>(st, wm * MT + f - NT, half, lane);
    };
    auto mul = [&](int half, int q) __attribute__((always_inline)) {
      const int i = q / NT, j = q % NT;
      acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b[half][j]),
                                                          __builtin_bit_cast(bf16x8, a[half][i]), acc[i][j], 0, 0, 0);
    };
    auto keep_sums = [&]() __attribute__((always_inline)) {  // in the accumulation registers at the end of each half
      if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) asm volatile("" : "+a"(acc[i][j]));
      }
    };
    keep_sums();
    wait_and_barrier<(S - 1) * L>();
#pragma unroll
    for (int f = 0; f < NR; ++f) read(0, lds, f);
    int buf = 0;
    // products of one half; spread between them, the reads of the other half from st and, with COPIES, a stage's copies
    auto half_stage = [&](auto halfc, auto copiesc, const char* st) __attribute__((always_inline)) {
      constexpr int H = decltype(halfc)::value, NS = NR + (decltype(copiesc)::value ? L : 0);
      unrolled([&](auto qc) __attribute__((always_inline)) {
        // reads alone are through in half the time, so that the barrier need not wait for the last of them (no difference that two runs
        // in turn would show: 4096 x 152064 x 3584 3.32 ms, reads spread over all of it 3.33); copies evenly, as fast as the CU
        // takes them (both within half the time 3.42)
        constexpr int q = decltype(qc)::value, OVER = decltype(copiesc)::value ? NM : NM / 2;
        constexpr int u0 = q >= OVER ? NS : (q * NS + OVER - 1) / OVER, u1 = q + 1 >= OVER ? NS : ((q + 1) * NS + OVER - 1) / OVER;
        mul(H, q);
#pragma unroll
        for (int u = u0; u < u1; ++u) {
          // copies and reads in turn, until either is through
          constexpr int C = NS - NR, both = 2 * (C < NR ? C : NR);
          const bool copy = u < both ? u & 1 : C > NR;
          if (copy) issue(u < both ? u >> 1 : u - NR, buf);
          else read(H ^ 1, st, u < both ? u >> 1 : u - C);
        }
        __builtin_amdgcn_sched_barrier(0);
      }, std::make_integer_sequence<int, NM>{});
      keep_sums();
    };
    using First = std::integral_constant<int, 0>;
    using Second = std::integral_constant<int, 1>;
    for (int left = kt_end - kt_begin; left > 1; --left) {
      half_stage(First{}, std::false_type{}, lds + buf * STAGE);
      wait_and_barrier<(S - 2) * L>();
      const int next = buf == S - 1 ? 0 : buf + 1;
      half_stage(Second{}, std::true_type{}, lds + next * STAGE);
      move_on();
      buf = next;
    }
    half_stage(First{}, std::false_type{}, lds + buf * STAGE);
    unrolled([&](auto qc) __attribute__((always_inline)) { mul(1, decltype(qc)::value); }, std::make_integer_sequence<int, NM>{});
    keep_sums();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing may still be on its way into LDS
  }
  __syncthreads();
  // acc[i][j][e]: row 16 (wm MT + i) + r, column 16 (wn NT + j) + 4 g + e of the tile
  const int col0 = n0 + wn * NT * 16, col = col0 + 4 * g;
  const bool whole = n0 + BN <= p.N;

  if constexpr (TO == TO_SUMS) {
    const float c = p.inv_temp * kLog2e;
    RowSums* part = (RowSums*)lds;  // [WN][BM]
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int ml = (wm * MT + i) * 16 + r, m = m0 + ml;
      const int target = p.targets && m < M ? p.targets[m] : -1, from = target - col0;
      if (__any(target < p.N && from >= 0 && from < NT * 16)) {  // some row's target is among these columns
        const int place = (from >> 4) * 4 + (from & 3);
        float x_target = 0.f;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) x_target = place == 4 * j + e ? acc[i][j][e] : x_target;
        if (target >= 0 && target < p.N && from >= 0 && from < NT * 16 && (from >> 2 & 3) == g) p.target_logit[m] = x_target;
      }
      float v[4 * NT];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * j + e] = whole || col + j * 16 + e < p.N ? acc[i][j][e] : -INFINITY;
      float top = v[0];
#pragma unroll
      for (int k = 1; k < 4 * NT; ++k) top = fmaxf(top, v[k]);
      RowSums s = sum_below<4 * NT>(column_max(fmaxf(top, kLowest)), 0.f, 0.f, v, c);
      s.s = column_sum(s.s);
      s.t = column_sum(s.t);
      if (g == 0) part[wn * BM + ml] = s;
    }
    __syncthreads();
    for (int ml = threadIdx.x; ml < BM && m0 + ml < M; ml += NW * 64) {
      RowSums s = part[ml];
#pragma unroll
      for (int w = 1; w < WN; ++w) s = merge(s, part[w * BM + ml], c);
      p.sums[(long long)(m0 + ml) * p.grid.n_tiles + bn] = s;
    }
  } else if constexpr (TO == TO_PLANE) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = m0 + (wm * MT + i) * 16 + r;
      if (m < M) {
        f32x4* o = (f32x4*)((float*)p.out + ((long long)bz * M + m) * p.out_pitch);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int n = col + j * 16;
          if (n < p.N) o[n / 4] = p.add ? o[n / 4] + acc[i][j] : acc[i][j];  // N is a multiple of 64
        }
      }
    }
  } else {
    // bf16, through LDS so that rows leave as whole lines
    char* mine = lds + wave * OUT_WAVE;
    const RowGrad* row_grads = (const RowGrad*)(lds + OUT);
    if constexpr (TO == TO_GRAD) {
      for (int ml = threadIdx.x; ml < BM; ml += NW * 64) {
        RowGrad q{};
        q.none = true;
        if (m0 + ml < M)
          q = row_grad(p.row_stats, p.entropy, p.grad_logp, p.grad_entropy, p.targets, p.inv_temp, p.vocab, p.active[m0 + ml]);
        ((RowGrad*)(lds + OUT))[ml] = q;
      }
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if constexpr (TO == TO_GRAD) {
        const RowGrad q = row_grads[(wm * MT + i) * 16 + r];
        const int from = q.target - p.col0 - col0, place = (from >> 4) * 4 + (from & 3);
        const bool here = q.target >= 0 && from >= 0 && from < NT * 16 && (from >> 2 & 3) == g;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][j][e] = grad_of(acc[i][j][e], q);
        if (__any(here)) {
          const float add = here ? q.at_target : 0.f;
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] += place == 4 * j + e ? add : 0.f;
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] *= q.inv_temp;
        if (__any(q.none || !whole)) {
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (q.none || col + j * 16 + e >= p.N) acc[i][j][e] = 0.f;
        }
      }
    }
    // columns that exist: the product's, or as far as the padding of K in the product that follows
    constexpr int LANES = NT * 2, ROWS = 64 / LANES;  // lanes to a row, rows at a time
    const int n = col0 + lane % LANES * 8, n_end = TO == TO_GRAD ? head_up(p.N, kHeadPanel) : p.N;
    const long long out_pitch = TO == TO_GRAD ? kHeadPanel : p.out_pitch;
    uint16_t* out = (uint16_t*)p.out + (TO == TO_GRAD ? head_panel_at(0, n, p.room) : n);
    constexpr bool TWO = TO == TO_GRAD && BM <= 128;  // tiles of few rows
#pragma unroll 1
    for (int plane = 0; plane < (TWO ? p.planes : 1); ++plane) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          uint2 w;
          w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32_pair{acc[i][j][0], acc[i][j][1]}), bf16_pair));
          w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32_pair{acc[i][j][2], acc[i][j][3]}), bf16_pair));
          *(uint2*)(mine + (i * 16 + r) * OUT_ROW + j * 32 + g * 8) = w;
          if constexpr (TWO)  // the rest
            acc[i][j] -= f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
        }
      // (only this wavefront's own writes are read: the compiler waits for them)
#pragma unroll 4
      for (int q = 0; q < MT * 16; q += ROWS) {
        const int ml = q + lane / LANES, m = m0 + wm * MT * 16 + ml;
        const u32x4 w = *(const u32x4*)(mine + ml * OUT_ROW + lane % LANES * 16);
        // past the caches, which the operands need (all three products: 7 rows 404 -> 324 us, 613 rows 832 -> 783, 151936 x 1536)
        if (m < x.m_end && n < n_end) __builtin_nontemporal_store(w, (u32x4*)(out + m * out_pitch));
      }
      out += rows * out_pitch;
    }
  }
}

// ---- a row's parts -> its results: one workgroup per row, up to 1024 parts with all loads at once ------------------------
__global__ __launch_bounds__(256) void head_finish_kernel(HeadArgs in, TokenOut out, const RowSums* sums, const float* target_logit, int parts) {
  __shared__ RowSums wave_s[4];
  const int row = blockIdx.x, tid = threadIdx.x;
  const float c = in.inv_temp * kLog2e;
  const int t = in.targets ? in.targets[row] : -1;
  const bool has = t >= 0 && t < in.vocab;
  const float x_target = has ? target_logit[row] : 0.f;
  constexpr int U = 4;
  RowSums mine{kLowest, 0.f, 0.f};
  for (int i = tid; i < parts; i += U * 256) {
    RowSums v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = i + u * 256 < parts ? sums[(long long)row * parts + i + u * 256] : RowSums{kLowest, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < U; ++u) mine = merge(mine, v[u], c);
  }
  mine = merge_wave(mine, c);
  if ((tid & 63) == 0) wave_s[tid >> 6] = mine;
  __syncthreads();
  if (tid) return;
  RowSums s = wave_s[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) s = merge(s, wave_s[w], c);
  finish_row(s, out, row, has, x_target, in.inv_temp);
}

// ---- rows that have a gradient ---------------------------------------------------------------
// active[i] = i-th row with a gradient, place[row] = its i or -1, *plan = what follows from their number.  One workgroup.
__global__ __launch_bounds__(1024) void head_active_kernel(HeadGrad a, HeadGradPlan g, HeadActive* plan, int* active, int* place) {
  __shared__ int wave_s[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int done = 0;
  for (int r0 = 0; r0 < a.in.rows; r0 += 1024) {
    const int r = r0 + tid;
    bool has = false;
    if (r < a.in.rows)
      has = !row_grad(a.row_stats, a.entropy, a.grad_logp, a.grad_entropy, a.in.targets, a.in.inv_temp, a.in.vocab, r).none;
    const unsigned long long mask = __ballot(has);
    if (lane == 0) wave_s[wave] = __popcll(mask);
    __syncthreads();
    int at = done, all = 0;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) at += wave_s[w];
      all += wave_s[w];
    }
    at += __popcll(mask & ((1ull << lane) - 1));
    if (r < a.in.rows) place[r] = has ? at : -1;
    if (has) active[at] = r;
    done += all;
    __syncthreads();
  }
  if (tid == 0) *plan = head_active(done, g, a.in.vocab, a.in.hidden);
}
// The rows of hidden_states that go with the stacked gradients, zeros in between; one row per workgroup
__global__ __launch_bounds__(256) void head_gather_kernel(HeadArgs in, int planes, const HeadActive* plan, const int* active, uint16_t* out) {
  const int n = plan->count, rows = head_up(n, head_pad(planes)), row = blockIdx.x;
  if (row >= rows * planes) return;
  const int i = row >= rows ? row - rows : row;
  const u32x4* src = i < n ? (const u32x4*)((const uint16_t*)in.hidden_states + active[i] * in.hidden_stride) : nullptr;
  u32x4* dst = (u32x4*)(out + (long long)row * in.hidden);
  const u32x4 zero = {0, 0, 0, 0};
  for (int v = threadIdx.x; v < in.hidden / 8; v += 256) dst[v] = src ? src[v] : zero;
}
// grad_hidden[row] = sum over the cuts of K of the rows that go with place[row]; zeros where it has none.  A workgroup takes 64 quads of columns, a
// wavefront a quarter of the planes, in their order; the quarters meet in LDS.
__global__ __launch_bounds__(256) void head_planes_kernel(const float* part_rows, int planes, const HeadActive* plan, int rows, int hidden, const int* place, uint16_t* out) {
  __shared__ f32x4 part[3][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per_row = hidden / 4;
  const long long at = ((long long)blockIdx.y * gridDim.x + blockIdx.x) * 64 + lane;
  const int row = (int)min(at / per_row, (long long)rows - 1), col = (int)(at % per_row) * 4;
  const int stacked = plan->stacked, second = planes == 2 ? stacked / 2 : 0;
  const int i = place[row], splits = plan->splits, share = (splits + 3) / 4, end = min(splits, (wave + 1) * share);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (i >= 0) {
#pragma unroll 8
    for (int z = wave * share; z < end; ++z) {
      const float* at_row = part_rows + ((long long)z * stacked + i) * hidden + col;
      s += *(const f32x4*)at_row;
      if (second) s += *(const f32x4*)(at_row + (long long)second * hidden);
    }
  }
  if (wave) part[wave - 1][lane] = s;
  __syncthreads();
  if (wave || at >= (long long)rows * per_row) return;
  s += part[0][lane];
  s += part[1][lane];
  s += part[2][lane];
  uint2 w;
  w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32_pair{s[0], s[1]}), bf16_pair));
  w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32_pair{s[2], s[3]}), bf16_pair));
  *(uint2*)(out + (long long)row * hidden + col) = w;
}

// ---- shapes ------------------------------------------------------------------------------------
template <int WM, int WN, int MT, int NT, int S, int TO, bool AK, bool BK>
void launch_shape(Product p, int blocks, hipStream_t s) {
  p.grid = head_grid(head_ceil(TO == TO_GRAD ? p.row_capacity : p.M, WM * MT * 16), head_ceil(p.N, WN * NT * 16), 1);
  const dim3 grid = many_blocks(blocks ? blocks : head_blocks(p.grid));
  if constexpr (WM == 1) {
    if (p.stream_b) return head_product_kernel<WM, WN, MT, NT, S, TO, AK, BK, true><<<grid, WM * WN * 64, 0, s>>>(p);
  }
  head_product_kernel<WM, WN, MT, NT, S, TO, AK, BK, false><<<grid, WM * WN * 64, 0, s>>>(p);
}
static_assert(kHeadTwoPlanes <= 256, "two planes leave tiles of up to 128 rows");
template <int TO, bool AK, bool BK>
void launch_product(const Product& p, HeadTile t, int blocks, hipStream_t s) {
  if (t.m == 256) return launch_shape<2, 2, 8, 8, 2, TO, AK, BK>(p, blocks, s);
  if (t.m == 128 && t.n == 128) return launch_shape<2, 2, 4, 4, TO == TO_SUMS ? 3 : 2, TO, AK, BK>(p, blocks, s);
  if constexpr (TO == TO_SUMS) {
    if (t.m == 160) return launch_shape<2, 2, 5, 8, 2, TO, AK, BK>(p, blocks, s);
    if (t.m == 192) return launch_shape<2, 2, 6, 8, 2, TO, AK, BK>(p, blocks, s);
    if (t.m == 224) return launch_shape<2, 2, 7, 8, 2, TO, AK, BK>(p, blocks, s);
  }
  // one row of tiles: three stages in flight in one workgroup per CU (two stages and two workgroups: x 152064 x 3584, 16
  // rows 236 -> 211 us, 32 rows 224 -> 192, 64 rows 229 -> 201)
  if constexpr (!AK) {
    if (t.m == 128) return launch_shape<1, 4, 8, 4, 3, TO, AK, BK>(p, blocks, s);
  }
  if constexpr (!BK) {
    if (t.m == 64) return launch_shape<1, 4, 4, 4, 3, TO, AK, BK>(p, blocks, s);
    if constexpr (TO == TO_SUMS) {
      if (t.m == 32) return launch_shape<1, 4, 2, 4, 3, TO, AK, BK>(p, blocks, s);
      return launch_shape<1, 4, 1, 4, 3, TO, AK, BK>(p, blocks, s);
    }
  }
}

constexpr size_t piece(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

}  // namespace

size_t head_workspace(int rows, int vocab, int) {
  const HeadTile t = head_tile(rows, vocab);
  return piece((size_t)rows * 4) + (size_t)rows * ceil_div(vocab, t.n) * sizeof(RowSums);
}
void launch_head_logprobs(const HeadArgs& in, const TokenOut& out, void* ws, hipStream_t s) {
  const HeadTile t = head_tile(in.rows, in.vocab);
  Product p{};
  p.a = {in.hidden_states, (int)in.hidden_stride};
  p.b = {in.lm_head, (int)in.head_stride};
  p.M = in.rows;
  p.N = in.vocab;
  p.K = in.hidden;
  p.stream_b = in.rows <= 128 && (long long)in.vocab * in.hidden * 2 > kLastCache;
  p.inv_temp = in.inv_temp;
  p.targets = in.targets;
  p.target_logit = (float*)ws;
  p.sums = (RowSums*)((char*)ws + piece((size_t)in.rows * 4));
  launch_product<TO_SUMS, false, false>(p, t, 0, s);
  head_finish_kernel<<<in.rows, 256, 0, s>>>(in, out, p.sums, p.target_logit, ceil_div(in.vocab, t.n));
}

size_t head_grad_workspace(int rows, int vocab, int hidden) {
  const HeadGradPlan g = head_grad_plan(rows, vocab);
  const size_t room = (size_t)g.rows * g.planes;
  return piece(sizeof(HeadActive)) + 2 * piece((size_t)rows * 4) + piece(room * hidden * 2) + piece(room * g.chunk * 2) +
         piece((size_t)head_most(g, rows, vocab, hidden).plane_rows * hidden * 4);
}
void launch_head_logprobs_grad(const HeadGrad& a, void* ws, hipStream_t s) {
  const HeadArgs& in = a.in;
  const HeadGradPlan g = head_grad_plan(in.rows, in.vocab);
  const HeadMost most = head_most(g, in.rows, in.vocab, in.hidden);
  const size_t room = (size_t)g.rows * g.planes;
  char* at = (char*)ws;
  auto take = [&](size_t bytes) {
    void* r = at;
    at += piece(bytes);
    return r;
  };
  HeadActive* plan = (HeadActive*)take(sizeof(HeadActive));
  int* active = (int*)take((size_t)in.rows * 4);
  int* place = (int*)take((size_t)in.rows * 4);
  uint16_t* h = (uint16_t*)take(room * in.hidden * 2);
  uint16_t* dx = (uint16_t*)take(room * g.chunk * 2);
  float* part_rows = (float*)at;
  head_active_kernel<<<1, 1024, 0, s>>>(a, g, plan, active, place);
  head_gather_kernel<<<(int)room, 256, 0, s>>>(in, g.planes, plan, active, h);
  for (int v0 = 0; v0 < in.vocab; v0 += g.chunk) {
    const int v = std::min(g.chunk, in.vocab - v0);
    const uint16_t* w = (const uint16_t*)in.lm_head + v0 * in.head_stride;
    if (in.rows > 0) {
      Product p{};  // logits of the chunk and their gradients
      p.a = {h, in.hidden};
      p.b = {w, (int)in.head_stride};
      p.M = in.rows;
      p.N = v;
      p.K = in.hidden;
      p.stream_b = room <= 128 && (long long)v * in.hidden * 2 > kLastCache;
      p.plan = plan;
      p.out = dx;
      p.room = (int)room;
      p.inv_temp = in.inv_temp;
      p.targets = in.targets;
      p.active = active;
      p.row_stats = a.row_stats;
      p.entropy = a.entropy;
      p.grad_logp = a.grad_logp;
      p.grad_entropy = a.grad_entropy;
      p.col0 = v0;
      p.vocab = in.vocab;
      p.row_capacity = g.rows;
      p.planes = g.planes;
      launch_product<TO_GRAD, false, false>(p, head_tile_logits(in.rows, v), 0, s);
      Product q{};  // + dx W
      q.a = {dx, kHeadPanel};
      q.room = (int)room;
      q.b = {w, (int)in.head_stride};
      q.M = (int)room;
      q.N = in.hidden;
      q.K = v;
      q.stream_b = p.stream_b;
      q.plan = plan;
      q.out = part_rows;
      q.out_pitch = in.hidden;
      q.add = v0 > 0;
      launch_product<TO_PLANE, false, true>(q, head_tile_hidden((int)room), most.blocks, s);
    }
    Product q{};  // dx^T h
    q.a = {dx, kHeadPanel};
    q.room = (int)room;
    q.b = {h, in.hidden};
    q.M = v;
    q.N = in.hidden;
    q.plan = plan;
    q.out = (uint16_t*)a.grad_head + (long long)v0 * in.hidden;
    q.out_pitch = in.hidden;
    launch_product<TO_BF16, true, true>(q, head_tile_head(in.rows), 0, s);
  }
  if (in.rows > 0)
    head_planes_kernel<<<many_blocks(((long long)in.rows * (in.hidden / 4) + 63) / 64), 256, 0, s>>>(part_rows, g.planes, plan, in.rows, in.hidden,
                                                                                              place, (uint16_t*)a.grad_hidden);
}
