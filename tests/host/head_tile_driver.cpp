// CPU-only check of csrc/head_tile.h: every load and store that the products of the lm_head operators make, for tiles at the
// corners of many sizes, stays inside its array; every tile is visited once; and what fragments read from LDS is what
// they should hold.  Built and run by tests/test_host_head_tile.py.
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>

#include "../../paper_2506_06122_amd/csrc/head_tile.h"

static long long checks = 0;
[[noreturn]] static void bad(const char* what, const char* product, long long a, long long b, long long c, long long d) {
  std::fprintf(stderr, "%s: %s (%lld, %lld, %lld, %lld)\n", product, what, a, b, c, d);
  std::exit(1);
}

struct Array {
  long long bytes;
};
struct Product {
  const char* name;
  HeadTile tile;
  int pad_rows;
  Array a, b, out;
  long long a_pitch, b_pitch, out_pitch, out_size;
  int m_room, M, N, K, capacity, splits, blocks;  // M, K, splits: as the device finds them
  long long out_row;                              // rows before the first one's
  bool panels;                                    // A is panelled; with pad_rows the result is
  int room;
};

template <int C, bool KM>
static void loads(const char* name, long long base, int limit, int k_left, long long pitch, const Array& arr) {
  using S = HeadSlice<C, KM>;
  for (int u = 0; u < S::units; ++u)
    for (int lane = 0; lane < 64; ++lane) {
      const long long off = S::source(u, lane, limit, k_left, (int)pitch), at = base + off;
      if (off < 0 || off >= 1ll << 32) bad("offset does not fit", name, u, lane, limit, off);
      if (at < 0 || at + 16 > arr.bytes) bad("load out of range", name, u, lane, at, arr.bytes);
      if (at % 16) bad("load not aligned", name, u, lane, at, 0);
      ++checks;
    }
}

template <int BM, int BN, bool AK, bool BK>
static void walk(const Product& p) {
  const int M = p.M, K = p.K, per = p.splits > 1 ? head_ceil(head_ceil(K, kHeadDeep), p.splits) : head_ceil(K, kHeadDeep);
  const HeadGrid room = head_grid(head_ceil(p.pad_rows ? p.capacity : p.m_room, BM), head_ceil(p.N, BN), 1);
  const int m_tiles = head_ceil(p.pad_rows ? head_up(M, p.pad_rows) : M, BM), n_tiles = room.n_tiles, tiles = m_tiles * n_tiles * p.splits;
  const int blocks = p.blocks ? p.blocks : head_blocks(room);
  HeadGrid grid = head_grid_rows(room, m_tiles);
  grid.splits = p.splits;
  if (head_blocks(grid) > blocks) bad("too few workgroups", p.name, head_blocks(grid), blocks, m_tiles, p.splits);
  if (blocks < 200000) {
    std::vector<char> seen(tiles, 0);
    for (int i = 0; i < blocks; ++i) {
      const HeadBlock b = head_block(i, grid);
      if (!b.inside) continue;
      if (b.m < 0 || b.m >= m_tiles || b.n >= n_tiles || b.z >= p.splits || seen[(b.z * n_tiles + b.n) * m_tiles + b.m]++) bad("tile twice", p.name, i, b.m, b.n, b.z);
    }
    for (char c : seen)
      if (!c) bad("tile missing", p.name, tiles, 0, 0, 0);
  }
  if (!m_tiles) return;
  std::set<int> ms{0, m_tiles / 2, m_tiles - 1, head_max(0, m_tiles - 2)}, ns{0, n_tiles - 1}, zs{0, p.splits / 2, p.splits - 1};
  for (int i = head_max(0, M / BM - 1); i < head_min(m_tiles, M / BM + 2); ++i) ms.insert(i);  // around the end of the rows
  for (int m : ms)
    for (int n : ns)
      for (int z : zs) {
        const int m0 = m * BM, n0 = n * BN;
        const HeadExtent x = head_extent(AK, BK, p.pad_rows, m0, n0, z, M, p.N, K, per, p.capacity);
        if (m0 >= x.m_end) continue;
        std::set<int> kts;
        if (x.kt_begin < x.kt_end && m0 < M) kts = {x.kt_begin, x.kt_end - 1, (x.kt_begin + x.kt_end) / 2};
        for (int kt : kts) {
          const long long a0 = 2 * (p.panels ? head_panel_slice(AK, m0, kt, p.room) : m0 * p.a_pitch + kt * kHeadDeep), b0 = 2 * (BK ? n0 + kt * kHeadDeep * p.b_pitch : n0 * p.b_pitch + kt * kHeadDeep);
          loads<BM, AK>(p.name, a0, x.a_limit, kHeadDeep, p.a_pitch, p.a);
          loads<BN, BK>(p.name, b0, x.b_limit, BK && kt == x.k_tiles - 1 ? x.b_last : kHeadDeep, p.b_pitch, p.b);
        }
        // stores of four values: last row of the tile, last column that passes the kernel's test
        const int row = head_min(m0 + BM, x.m_end) - 1;
        const int cols = p.pad_rows ? head_up(p.N, kHeadPanel) : p.N, col = head_min(n0 + BN, cols) - 8;
        const long long at = (p.pad_rows ? head_panel_at((int)p.out_row + row, col, p.room)
                                         : (p.splits > 1 ? (long long)z * M + row : p.out_row + row) * p.out_pitch + col) * p.out_size;
        if (p.out.bytes && (at < 0 || at + 8 * p.out_size > p.out.bytes)) bad("store out of range", p.name, row, col, at, p.out.bytes);
        ++checks;
      }
}
template <bool AK, bool BK>
static void by_tile(const Product& p) {
  const HeadTile t = p.tile;
  if (t.m == 16 && t.n == 256) walk<16, 256, AK, BK>(p);
  else if (t.m == 32 && t.n == 256) walk<32, 256, AK, BK>(p);
  else if (t.m == 64 && t.n == 256) walk<64, 256, AK, BK>(p);
  else if (t.m == 128 && t.n == 256 && !AK) walk<128, 256, AK, BK>(p);
  else if (t.m == 128 && t.n == 128) walk<128, 128, AK, BK>(p);
  else if (t.m == 160 && t.n == 256 && !AK && !BK) walk<160, 256, AK, BK>(p);
  else if (t.m == 192 && t.n == 256 && !AK && !BK) walk<192, 256, AK, BK>(p);
  else if (t.m == 224 && t.n == 256 && !AK && !BK) walk<224, 256, AK, BK>(p);
  else if (t.m == 256 && t.n == 256) walk<256, 256, AK, BK>(p);
  else bad("unknown tile", p.name, t.m, t.n, 0, 0);
}

static void sizes(int rows, int vocab, int hidden, int pad) {
  const long long hp = hidden + pad;
  const Array states{(rows - 1) * hp * 2 + hidden * 2}, head{(vocab - 1) * hp * 2 + hidden * 2ll};
  by_tile<false, false>({"logits", head_tile(rows, vocab), 0, states, head, {0}, hp, hp, 0, 0, rows, rows, vocab, hidden, 0, 1, 0, 0, false, 0});
  const HeadGradPlan g = head_grad_plan(rows, vocab);
  const HeadMost most = head_most(g, rows, vocab, hidden);
  const int room = g.rows * g.planes;
  const Array h{(long long)room * hidden * 2}, dx{(long long)room * g.chunk * 2}, parts{most.plane_rows * hidden * 4};
  std::set<int> counts{0, 1, rows / 5, rows / 3, rows / 2 + 1, rows - 1, rows};
  for (int c = 0; c < rows && c < 700; c += 64) counts.insert({c, c + 1});
  for (int count : counts) {
    if (count < 0 || count > rows) continue;
    const HeadActive a = head_active(count, g, vocab, hidden);
    if (a.stacked > room || a.splits < 1) bad("plan", "active", count, a.stacked, room, a.splits);
    for (int v0 = 0; v0 < vocab; v0 += g.chunk) {
      const int v = head_min(g.chunk, vocab - v0);
      const Array w{(long long)(v - 1) * hp * 2 + hidden * 2ll + (long long)(vocab - v0 - v) * hp * 2};
      for (int plane = 0; plane < g.planes; ++plane)
        by_tile<false, false>({"gradients", head_tile_logits(rows, v), head_pad(g.planes), h, w, dx, hidden, hp, 0, 2, rows, count, v, hidden, g.rows, 1, 0,
                               (long long)plane * head_up(count, head_pad(g.planes)), false, room});
      by_tile<false, true>({"grad_hidden", head_tile_hidden(room), 0, dx, w, parts, kHeadPanel, hp, hidden, 4, room, a.stacked, hidden, v, 0, a.splits, most.blocks, 0, true, room});
      by_tile<true, true>({"grad_head", head_tile_head(rows), 0, dx, h, {(long long)v * hidden * 2}, kHeadPanel, hidden, hidden, 2, v, v, hidden, a.stacked, 0, 1, 0, 0, true, room});
    }
  }
}

// LDS after the loads of a slice, then what fragments read from it: value (row, step) as row * 64 + step
template <int C, bool KM>
static void fragments() {
  using S = HeadSlice<C, KM>;
  const long long pitch = KM ? 1000 * 8 : 64;  // any
  std::vector<int> lds(C * 64, -1);
  for (int u = 0; u < S::units; ++u)
    for (int lane = 0; lane < 64; ++lane) {
      const long long v = S::source(u, lane, C, 64, pitch) / 2;
      for (int e = 0; e < 8; ++e) {
        const int row = KM ? (int)(v % pitch) + e : (int)(v / pitch), k = KM ? (int)(v / pitch) : (int)(v % pitch) + e;
        lds[(u * 1024 + lane * 16) / 2 + e] = row * 64 + k;
      }
    }
  for (int i = 0; i < C / 8; ++i)
    for (int lane = 0; lane < 64; ++lane) {
      const int half = i & 1, r = lane & 15, g = lane >> 4;
      for (int e = 0; e < 8; ++e) {
        int got;
        if (KM) {  // element e of lane r: value r % 4 of what lane 4 (e % 4) + r / 4 of the group points at, the second half four steps on
          const int from = S::fragment(i >> 1, half, g * 16 + 4 * (e & 3) + (r >> 2)) + (e >> 2) * 4 * S::pitch;
          got = lds[from / 2 + (r & 3)];
        } else {
          got = lds[S::fragment(i >> 1, half, lane) / 2 + e];
        }
        if (got != (16 * (i >> 1) + r) * 64 + 32 * half + 8 * g + e) bad("fragment", KM ? "K outermost" : "rows outermost", C, i, lane, e);
        ++checks;
      }
    }
}

int main() {
  fragments<16, false>();
  fragments<32, false>();
  fragments<64, false>();
  fragments<128, false>();
  fragments<160, false>();
  fragments<192, false>();
  fragments<224, false>();
  fragments<256, false>();
  fragments<16, true>();
  fragments<32, true>();
  fragments<64, true>();
  fragments<128, true>();
  fragments<256, true>();
  for (int rows : {1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 160, 187, 255, 256, 257, 300, 400, 511, 613, 1500, 4096, 70001})
    for (int vocab : {1, 33, 100, 256, 257, 513, 4099, 32001, 152064})
      for (int hidden : {64, 192, 1536, 3584})
        sizes(rows, vocab, hidden, hidden % 128 ? 8 : 0);
  std::printf("%lld checks\n", checks);
}
