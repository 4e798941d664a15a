// Where the products of the lm_head operators (kernels_head.hip) read and write: tiles, slices of operands and their places
// in LDS.  Plain integers, used by the kernel, by its launcher and - without a GPU - by the test that every access of
// every launch stays inside its array and every fragment holds the values it should.
#pragma once

constexpr int head_min(int a, int b) { return a < b ? a : b; }
constexpr int head_max(int a, int b) { return a > b ? a : b; }
constexpr int head_ceil(long long a, long long b) { return (int)((a + b - 1) / b); }
constexpr int head_up(int v, int to) { return (v + to - 1) / to * to; }

constexpr int kHeadDeep = 64;  // steps of K in a stage: with rows outermost a whole line of each row

// The 64-deep slice of an operand of C columns (rows of C's other side): 128 C bytes of LDS, C / 8 loads of 1 KiB.
//   rows outermost (KM = false): row by row 128 bytes; the 16-byte chunk c of row r lies in slot c ^ (r % 8), so that the
//     8 rows a fragment read touches at a time fill all banks
//   K outermost (KM = true): step by step 2 C bytes; chunk c of step k lies in slot c ^ 2 (k % 4 + 4 (k / 8 % 2)), which
//     spreads the eight steps that half a wavefront reads
template <int C, bool KM>
struct HeadSlice {
  static constexpr int units = C / 8, pitch = 2 * C, chunks = C / 8;
  static constexpr int swizzle(int k) { return 2 * ((k & 3) + 4 * (k >> 3 & 1)) & (chunks - 1); }
  // byte offset in memory, from the slice's first value, of lane's 16 bytes of unit u; rows (columns) past `limit` and
  // steps past k_left read the last one
  static constexpr unsigned source(int u, int lane, int limit, int k_left, int op_pitch) {
    if (KM) {
      const int at = u * 1024 + lane * 16, k = at / pitch, slot = at % pitch / 16, col = (slot ^ swizzle(k)) * 8;
      return ((unsigned)head_min(k, k_left - 1) * (unsigned)op_pitch + (unsigned)head_min(col, limit - 8)) * 2;
    }
    const int row = u * 8 + (lane >> 3), chunk = (lane & 7) ^ (row & 7);
    return ((unsigned)head_min(row, limit - 1) * (unsigned)op_pitch + chunk * 8) * 2;
  }
  // LDS byte of a lane's part of the fragment of columns 16 i .., steps 32 half ..: lane = 16 g + r.  Rows outermost: the
  // 16 bytes of column r, steps 8 g ...  K outermost: 8 bytes of step 8 g + r / 4, columns 4 (r % 4) ..., and again four
  // steps on; the transposing read exchanges them among the 16 lanes of g, so that lane r gets column r of the four steps.
  static constexpr int fragment(int i, int half, int lane) {
    const int r = lane & 15, g = lane >> 4;
    if (KM) {
      const int k = 8 * g + (r >> 2), chunk = (2 * i + (r >> 1 & 1)) ^ swizzle(k);
      return (32 * half + k) * pitch + chunk * 16 + (r & 1) * 8;
    }
    return i * 2048 + r * 128 + ((4 * half + g) ^ (r & 7)) * 16;
  }
};

// Workgroup -> tile.  Consecutive workgroups go to the eight XCDs in turn, each with an L2 of its own.  Tiles come in groups of
// group_m x group_n that run side by side on an XCD and share their operands' slices.  Groups go down the rows first and
// round the XCDs, so that what these fetch at a time lies together (grad_head of 4096 rows, 152064 x 3584: 2.9 ms;
// across first, or each XCD a contiguous share, 3.3); with cuts of K each XCD takes a contiguous share, because the tiles
// of a cut share all of its slices (grad_hidden of 1500 rows, 151936 x 2048, six cuts: round the XCDs 0.79 ms, in
// shares 0.67).
struct HeadGrid {
  int m_tiles, n_tiles, splits;
  int group_m, group_n, m_groups, n_groups;
};
struct HeadBlock {
  int m, n, z;
  bool inside;
};
constexpr HeadGrid head_grid(int m_tiles, int n_tiles, int splits) {
  // 32 tiles side by side, one to a CU, about as many rows as columns; smaller groups where the XCDs would get too few
  HeadGrid g{m_tiles, n_tiles, splits, head_min(8, m_tiles), 0, 0, 0};
  g.group_n = head_min(32 / g.group_m, n_tiles);
  for (;;) {
    g.m_groups = head_ceil(m_tiles, g.group_m);
    g.n_groups = head_ceil(n_tiles, g.group_n);
    if (g.m_groups * g.n_groups * splits >= 64 || (g.group_m == 1 && g.group_n == 1)) return g;
    (g.group_n >= g.group_m ? g.group_n : g.group_m) = (head_max(g.group_n, g.group_m) + 1) / 2;
  }
}
// the same for the first rows of it alone: never more workgroups
constexpr HeadGrid head_grid_rows(HeadGrid g, int m_tiles) {
  g.m_tiles = m_tiles;
  g.m_groups = head_max(1, head_ceil(m_tiles, g.group_m));
  g.group_m = head_max(1, head_ceil(m_tiles, g.m_groups));
  return g;
}
constexpr int head_blocks(const HeadGrid& g) { return head_up(g.m_groups * g.n_groups * g.splits, 8) * g.group_m * g.group_n; }
constexpr HeadBlock head_block(unsigned index, const HeadGrid& g) {
  const int per = g.group_m * g.group_n, idx = (int)(index >> 3), in = idx % per, share = (g.m_groups * g.n_groups * g.splits + 7) / 8;
  if (idx / per >= share) return HeadBlock{0, 0, 0, false};
  const int group = g.splits > 1 ? (int)(index & 7) * share + idx / per : idx / per * 8 + (int)(index & 7);
  const int across = group / g.m_groups, z = across / g.n_groups;
  const int m = group % g.m_groups * g.group_m + in % g.group_m, n = across % g.n_groups * g.group_n + in / g.group_m;
  return HeadBlock{m, n, z, m < g.m_tiles && n < g.n_tiles && z < g.splits};
}

// Rows and columns of the tiles that an M x N product is cut into.  Up to 128 rows are one tile, so that W is read once
// (128 x 152064 x 3584: 219 us, in 128 x 128 tiles 245), unless that leaves many CUs without one (128 x 32000 x 4096: 55 us,
// in 128 x 128 tiles 52).  More than 128 rows take tiles of 160 to 256 rows, so that
// neither the last row of tiles nor the last round of 256 workgroups stands half empty: a round costs as much as its
// rows and some 150 more (151936 x 1536: 160 rows in one tile 138 us, in two of 128 161; 300 in two of 160 196, in two of
// 256 236; 613 in three of 224 316, of 256 345; 512 in two of 256 239, in three of 192 286).
struct HeadTile {
  int m, n;
};
constexpr HeadTile head_tile(int M, int N) {
  if (M <= 16) return {16, 256};
  if (M <= 32) return {32, 256};
  if (M <= 64) return {64, 256};
  const int across = head_ceil(N, 256);
  if (M <= 128 && across >= 192) return {128, 256};
  if (M <= 128 || head_ceil(M, 160) * (long long)across < 192) return {128, 128};
  int best = 256;
  long long best_time = 0;
  for (int m = 256; m >= 160; m -= 32) {
    const long long time = (long long)head_ceil((long long)head_ceil(M, m) * across, 256) * (m + 150);
    if (m == 256 || time < best_time) {
      best_time = time;
      best = m;
    }
  }
  return {best, 256};
}
// the gradients' first product writes whole slices of rows, zeros included (16 x 256 tiles, 7 rows: 208 us, four times the
// workgroups, where 64 x 256 take 119), and the device alone knows how many rows there are (160 rows, a quarter without
// gradient, 151936 x 1536, all three products: 445 us with 128 x 128 tiles here, 474 with 256 x 256; 128 x 256 a
// little less than 128 x 128, seven runs in turn each: 187 rows 468-488 and 473-487, 128 rows x 152064 x 3584 951-957 and 960-974)
constexpr HeadTile head_tile_logits(int M, int N) {
  if (M <= 64) return {64, 256};
  if (M <= 256 && head_ceil(N, 256) >= 192) return {128, 256};
  if (M <= 256 || head_ceil(M, 256) * (long long)head_ceil(N, 256) < 192) return {128, 128};
  return {256, 256};
}
// the gradients' second and third product: K is long in grad_hidden's, which is cut along it instead, and short in
// grad_head's with few rows, where two small workgroups to a CU hide each other's start and end (32 rows x 152064 x 3584 723
// -> 655 us in all, 151936 x 1536 with 187 rows 497 -> 469, with 400 691 -> 675, but with 613 775 to 782 either way)
// (one row of tiles of grad_hidden: 128 x 256 and three stages, 64 rows x 152064 x 3584 715 -> 690 us in all)
constexpr HeadTile head_tile_hidden(int M) { return M <= 128 ? HeadTile{128, 256} : M <= 256 ? HeadTile{128, 128} : HeadTile{256, 256}; }
constexpr HeadTile head_tile_head(int K) { return K <= 512 ? HeadTile{128, 128} : HeadTile{256, 256}; }

// Cuts of K for `tiles` tiles of a product with k_tiles slices: rounds over the card's places for workgroups, in slices.  A cut
// costs the tile's partial results, written and read again, as much as some twenty slices of a tile that fills a CU.
constexpr int head_splits(int tiles, int k_tiles, HeadTile t) {
  const int places = t.n == 256 ? 256 : 512, cost = t.n == 256 ? 20 : 8;
  int best = 1, best_time = head_ceil(tiles, places) * (k_tiles + cost);
  for (int rounds = 1; rounds <= 4; ++rounds) {
    const int s = head_min(places * rounds / tiles, k_tiles / 8);
    if (s <= 1) continue;
    const int time = head_ceil((long long)tiles * s, places) * (head_ceil(k_tiles, s) + cost);
    if (time < best_time) {
      best_time = time;
      best = s;
    }
  }
  return best;
}

// The gradients of the logits are bf16.  One rounding of the given token's, by far the row's largest, moves the whole row
// of both results; over many rows that averages out to the size of the results' own rounding, with few it does not, and
// the gradients are kept as a bf16 value and the bf16 rest, below the first values' rows: twice the rows for
// grad_hidden's product, twice the K for grad_head's, which few rows do not notice much.
constexpr int kHeadTwoPlanes = 128;  // rows up to which
// a plane's rows are padded to this, so that all planes are whole slices
constexpr int head_pad(int planes) { return kHeadDeep / planes; }
struct HeadGradPlan {
  int rows;    // room for the rows of the logits' gradients: a whole number of slices
  int planes;  // 1 or 2
  int chunk;   // columns of the vocabulary at a time, a multiple of 256
};
constexpr HeadGradPlan head_grad_plan(int rows, int vocab) {
  HeadGradPlan g{};
  g.rows = head_up(head_max(rows, 1), kHeadDeep);
  g.planes = rows <= kHeadTwoPlanes ? 2 : 1;
  // up to 4 GiB of gradients of logits at a time
  const long long fit = ((long long)4 << 30) / (2ll * g.rows * g.planes) / 256 * 256, all = head_up(vocab, 256);
  g.chunk = (int)(fit < 256 ? 256 : fit < all ? fit : all);
  return g;
}
// What `count` rows with a gradient make of it, known to the device only
struct HeadActive {
  int count;   // rows
  int stacked; // rows of the logits' gradients as the products see them: the planes below each other, padded with zeros
  int splits;  // of K in grad_hidden's product
};
constexpr HeadActive head_active(int count, const HeadGradPlan& g, int vocab, int hidden) {
  HeadActive a{count, g.planes == 1 ? count : 2 * head_up(count, head_pad(2)), 1};
  // (the tile is chosen by the rows there is room for: the launch does not know the count)
  const HeadTile t = head_tile_hidden(g.rows * g.planes);
  const int tiles = head_ceil(a.stacked, t.m) * head_ceil(hidden, t.n), slices = head_ceil(head_min(vocab, g.chunk), kHeadDeep);
  if (tiles > 0) a.splits = head_splits(tiles, slices, t);
  return a;
}
// the most that any count needs: rows of partial results, and workgroups of grad_hidden's product
struct HeadMost {
  long long plane_rows;
  int blocks;
};
constexpr HeadMost head_most(const HeadGradPlan& g, int rows, int vocab, int hidden) {
  const HeadTile t = head_tile_hidden(g.rows * g.planes);
  const int m_tiles = head_ceil(g.rows * g.planes, t.m);
  const HeadGrid grid = head_grid(m_tiles, head_ceil(hidden, t.n), 1);
  HeadMost most{0, 0};
  // splits change with the number of row tiles alone; the last count of each has the most rows
  for (int i = 1; i <= m_tiles; ++i) {
    const int end = head_min(rows, g.planes == 1 ? i * t.m : i * t.m / 2);
    const HeadActive a = head_active(head_max(end, 1), g, vocab, hidden);
    HeadGrid some = head_grid_rows(grid, head_ceil(a.stacked, t.m));
    some.splits = a.splits;
    const long long plane_rows = (long long)a.splits * a.stacked;
    if (plane_rows > most.plane_rows) most.plane_rows = plane_rows;
    if (head_blocks(some) > most.blocks) most.blocks = head_blocks(some);
    if (i > 600 && i < m_tiles - 1) i = m_tiles - 2;  // (far beyond that many tiles K is not cut)
  }
  return most;
}
// The gradients of logits lie in panels of 256 columns, row below row, so that both products that read them find a slice
// together: 64 rows of 512 bytes one behind the other, or 256 rows 512 bytes apart, where rows of a vocabulary's length
// put every one on a page of its own.
constexpr int kHeadPanel = 256;
constexpr long long head_panel_at(int row, int col, int room) {
  return ((long long)(col / kHeadPanel) * room + row) * kHeadPanel + col % kHeadPanel;
}
// The slice kt of a panelled operand, from its first row (rows outermost) or column (K outermost)
constexpr long long head_panel_slice(bool km, int first, int kt, int room) {
  return km ? head_panel_at(kt * kHeadDeep, first, room) : head_panel_at(first, kt * kHeadDeep, room);
}

// One tile's share of a product, with the sizes that only the device knows filled in.
struct HeadExtent {
  int m_end;             // rows of C to write; past M they are zeros that pad a later product's K
  int k_tiles, kt_begin, kt_end;
  int a_limit, b_limit;  // rows or columns of the slices that exist, from the tile's first
  int b_last;            // steps of B's last slice that exist
};
constexpr HeadExtent head_extent(bool a_km, bool b_km, int pad, int m0, int n0, int z, int M, int N, int K, int per_split,
                                 int row_capacity) {
  HeadExtent x{};
  x.m_end = pad ? head_min(row_capacity, head_up(M, pad)) : M;
  x.k_tiles = head_ceil(K, kHeadDeep);
  x.kt_begin = z * per_split;
  x.kt_end = head_min(x.k_tiles, x.kt_begin + per_split);
  // (A with K outermost is panelled, whole tiles; with rows outermost the padding rows exist too, as zeros)
  x.a_limit = a_km ? kHeadPanel - m0 % kHeadPanel : x.m_end - m0;
  x.b_limit = N - n0;
  x.b_last = b_km ? K - (x.k_tiles - 1) * kHeadDeep : kHeadDeep;
  return x;
}
