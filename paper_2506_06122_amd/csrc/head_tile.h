// Where the products of the lm_head operators (kernels_head.hip) read and write: tiles, slices of operands and their places
// in LDS.  Plain integers, used by the kernel, by its launcher and - without a GPU - by the test that every access of
// every launch stays inside its array and every fragment holds the values it should.
#pragma once

constexpr int head_min(int a, int b) { return a < b ? a : b; }
constexpr int head_max(int a, int b) { return a > b ? a : b; }
constexpr int head_ceil(long long a, long long b) { return (int)((a + b - 1) / b); }
constexpr int head_up(int v, int to) { return (v + to - 1) / to * to; }

// The 32-deep slice of an operand of C columns (rows of C's other side): 64 C bytes of LDS, C / 16 loads of 1 KiB.
//   rows outermost (KM = false): row by row 64 bytes; the 16-byte chunk c of row r lies in slot c ^ (r / 4 % 4), so that the
//     16 rows a fragment read touches at a time fill all banks
//   K outermost (KM = true): step by step 2 C bytes; chunk c of step k lies in slot c ^ 2 (k % 4 + 4 (k / 8 % 2)), which
//     spreads the eight steps that half a wavefront reads
template <int C, bool KM>
struct HeadSlice {
  static constexpr int units = C / 16, pitch = 2 * C, chunks = C / 8;
  static constexpr int swizzle(int k) { return 2 * ((k & 3) + 4 * (k >> 3 & 1)) & (chunks - 1); }
  // byte offset in memory, from the slice's first value, of lane's 16 bytes of unit u; rows (columns) past `limit` and
  // steps past k_left read the last one
  static constexpr long long source(int u, int lane, int limit, int k_left, long long op_pitch) {
    if (KM) {
      const int at = u * 1024 + lane * 16, k = at / pitch, slot = at % pitch / 16, col = (slot ^ swizzle(k)) * 8;
      return (head_min(k, k_left - 1) * op_pitch + head_min(col, limit - 8)) * 2;
    }
    const int row = u * 16 + (lane >> 2), chunk = (lane & 3) ^ (lane >> 4);
    return (head_min(row, limit - 1) * op_pitch + chunk * 8) * 2;
  }
  // LDS byte of a lane's part of the fragment of columns 16 i ..: lane = 16 g + r.  Rows outermost: the 16 bytes of
  // column r, steps 8 g ...  K outermost: 8 bytes of step 8 g + r / 4, columns 4 (r % 4) ..., and again four steps on;
  // the transposing read exchanges them among the 16 lanes of g, so that lane r gets column r of the four steps.
  static constexpr int fragment(int i, int lane) {
    const int r = lane & 15, g = lane >> 4;
    if (KM) {
      const int k = 8 * g + (r >> 2), chunk = (2 * i + (r >> 1 & 1)) ^ swizzle(k);
      return k * pitch + chunk * 16 + (r & 1) * 8;
    }
    return i * 1024 + r * 64 + (g ^ (r >> 2)) * 16;
  }
};

// Workgroup -> tile.  Consecutive workgroups go to the eight XCDs in turn: each XCD takes a contiguous share of the tiles,
// all row blocks of a column block before the next, so that a column block's slices are fetched into one L2.
struct HeadBlock {
  int m, n, z;
  bool inside;
};
constexpr int head_blocks(int tiles) { return 8 * head_ceil(tiles, 8); }
constexpr HeadBlock head_block(unsigned index, int m_tiles, int n_tiles, int splits) {
  const int tiles = m_tiles * n_tiles * splits, per = (tiles + 7) / 8, t = (int)(index & 7) * per + (int)(index >> 3);
  return HeadBlock{t % m_tiles, t / m_tiles % n_tiles, t / (m_tiles * n_tiles), t < tiles};
}

// Rows and columns of the tiles that an M x N product is cut into
struct HeadTile {
  int m, n;
};
constexpr HeadTile head_tile(int M, int N) {
  if (M <= 16) return {16, 256};
  if (M <= 32) return {32, 256};
  if (M <= 64) return {64, 256};
  if (head_ceil(M, 256) * (long long)head_ceil(N, 256) < 192) return {128, 128};
  return {256, 256};
}

struct HeadGradPlan {
  int rows;    // room for the rows of the logits' gradients: a whole number of k-tiles
  int chunk;   // columns of the vocabulary at a time, a multiple of 256
  int splits;  // of K in grad_hidden's product
};
constexpr HeadGradPlan head_grad_plan(int rows, int vocab, int hidden) {
  HeadGradPlan g{};
  g.rows = head_up(head_max(rows, 1), 32);
  // up to 4 GiB of gradients of logits at a time
  const long long fit = ((long long)4 << 30) / (2ll * g.rows) / 256 * 256, all = head_up(vocab, 256);
  g.chunk = (int)(fit < 256 ? 256 : fit < all ? fit : all);
  const HeadTile t = head_tile(rows, hidden);
  const int tiles = head_max(1, head_ceil(rows, t.m) * head_ceil(hidden, t.n));
  g.splits = head_max(1, head_min(head_ceil(1024, tiles), g.chunk / 1024));
  return g;
}
// columns between the rows of a chunk's gradients: the padding of K in the product that follows, and of its tiles
constexpr int head_grad_pitch(int columns) { return head_up(columns, 256); }

// One tile's share of a product, with the sizes that only the device knows filled in.
struct HeadExtent {
  int m_end;             // rows of C to write; past M they are zeros that pad a later product's K
  int k_tiles, kt_begin, kt_end;
  int a_limit, b_limit;  // rows or columns of the slices that exist, from the tile's first
  int b_last;            // steps of B's last slice that exist
};
constexpr HeadExtent head_extent(bool a_km, bool b_km, bool pad_rows, int m0, int n0, int z, int M, int N, int K, int per_split,
                                 long long a_pitch, int row_capacity) {
  HeadExtent x{};
  x.m_end = pad_rows ? head_min(row_capacity, head_up(M, 32)) : M;
  x.k_tiles = (K + 31) >> 5;
  x.kt_begin = z * per_split;
  x.kt_end = head_min(x.k_tiles, x.kt_begin + per_split);
  // (with K outermost a row of A ends at its pitch, past the last column that is stored; with rows outermost the padding
  // rows exist too, as zeros)
  x.a_limit = (a_km ? (int)a_pitch : x.m_end) - m0;
  x.b_limit = N - n0;
  x.b_last = b_km ? K - (x.k_tiles - 1) * 32 : 32;
  return x;
}
