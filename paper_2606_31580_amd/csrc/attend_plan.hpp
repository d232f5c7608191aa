// Which kernel takes a span of laser_attend, and over how many workgroups its keys are split (host;
// plain C++).
#pragma once

#include <algorithm>
#include <cstdint>

namespace laser {

constexpr int kAttendKinds = 3;  // row kernel with 16 columns, with 32; tile kernel
constexpr int kAttendFewCols = 64;
// All partials of a call, at most.  Splits beyond it are not made, whichever kernel takes the rows: calls that would
// make them have workgroups enough without (30,000 rows of the 8B heads are 3,752 tiles).
constexpr int64_t kAttendPartBytes = (int64_t)288 << 20;

// A span as the planner sees it, and what it decides.
struct AttendSize {
  int n, pages;    // query rows; pages that any of them sees
  int rows_pages;  // pages that the last row sees and the first does not (causal)
  int kind;      // the kernel
  int tiles;     // query tiles
  int nsplit;    // workgroups over a tile's pages
};

inline int attend_ceil(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Columns (rows x query heads of a kv head) of a tile of each kernel.
inline int attend_cols(int kind) { return kind == 0 ? 16 : kind == 1 ? 32 : 256; }

// Splits of a span of the tile kernel at `run` pages a workgroup, a step of 4 at least.
inline int tile_split(const AttendSize& s, int run) { return std::max(1, std::min(attend_ceil(s.pages, run), s.pages / 4)); }
inline int tile_run(const AttendSize* s, int n, int kv_heads, int heads, int hd, int cus, int64_t part_bytes);
// Bytes of a span's partials at `splits` workgroups a tile: O, m and l per row, head and split.
inline int64_t span_part_bytes(const AttendSize& s, int splits, int heads, int hd) {
  return splits > 1 ? (int64_t)s.n * heads * splits * (hd + 2) * 4 : 0;
}

// es: bytes of a cached element (i8: integers); io16: 16-bit rows.  fp32 pools have only the row kernel with 16 columns,
// and fp32 rows not the one with 32 (three parts of everything would not fit the registers).
//
// The tile kernel converts a page once for 256 columns and not for 32, but has 8 times fewer, longer workgroups: it
// pays from some work on, counted in pages x 32-column tiles per CU (us, tiles and rows, 7B heads, INT8, bf16 rows: a
// prompt of 512 rows, 28 per CU, 26.2 and 15.8, of 1,024, 112, 41 and 34, of 2,048, 450, 68 and 84; 512 rows
// behind 2,000 positions, 246, 44 and 57; bf16 pools: 20 rows behind 14,000, 68, 24 and 32; fp32 rows: a prompt of
// 1,024 70 and 49, of 2,048 137 and 139).
// A tile takes about as long with few of its 256 columns in use as with all, a row kernel as many times longer as it
// has tiles: a span goes through tiles if these are filled to 6 of 8 parts with INT8 pools and bf16 rows, 4 with E4M3
// or bf16 pools; fp32 rows: 7.5, 6 with E4M3, 5 with bf16 (us, tiles and rows, 8B heads, 16 sequences of 1,000-9,000:
// INT8, 120 columns, 4 parts, 122 and 100, 192, 6, 121 and 142; E4M3, 96, 3, 111 and 114, 160, 5, 104 and 153;
// bf16, 3, 125 and 120, 4, 123 and 131; fp32 rows: INT8, 7, 308 and 252, 8, 308 and 307, a chunk of 1,000 rows 253 and
// 298; E4M3, 5, 205 and 183, 8, 218 and 278; bf16, 5, 234 and 248).
//
// Row kernels: pages per wave.  Every CU runs one workgroup of 4 waves, or two on 8-bit pools (fewer
// registers).  Long runs stream best when two workgroups per CU share the pages; where that leaves a wave only
// a few pages, one per CU with twice the pages has fewer splits to join and, on wider pools, no second
// round (us, two and one per CU: 7B heads, 4 sequences of 3,000-14,000, bf16 pool, 4 pages a wave 23.9 and 19.4; 8B
// heads, 8 sequences, 17 pages 50.5 and 60.8; INT8, 16 sequences of 100-2,000, 2 pages 13.4 and 11.5; 6 of
// 3,000-9,000, 9 pages 20.5 and 26.6).  Runs end at 32 pages: more rounds even out ragged lengths (64 sequences of
// 3,000-14,000: 219 us with runs of 133 pages, 192 with 33).
// A span of up to 32 pages stays whole, since joining splits is a launch of its own, up to 64 where there
// are spans enough to fill the CUs (64 sequences of 50-600 positions: 18.2 us split, 14.4 whole) or rows enough to
// make the join long.
// All splits together are at most 64 workgroups per CU beyond one per tile: more rounds than that even out nothing (16
// per CU cost 4% at 128 sequences of 3,000-14,000 and 256 of 1,000-6,000 positions).  And no span has more than the
// number of splits at which all partials (8 or 17 KB per workgroup) fit kAttendPartBytes.
// Tile kernel: see tile_run.
// mode: 0 the kernels as above, 1 only row kernels, 2 the tile kernel wherever it can be (laser_model_set_attend_kernel).
inline void plan_attend(AttendSize* s, int n, int q_heads, int kv_heads, int hd, int cus, int es, bool i8, bool io16, int mode) {
  int64_t work = 0, wide = 0, wgs = 0;
  const int half_parts = io16 ? (i8 ? 12 : 8) : i8 ? 15 : es == 1 ? 12 : 10;
  auto fills = [&](int64_t cols) {  // tiles filled far enough
    return cols > kAttendFewCols && (mode == 2 || 2 * (int64_t)attend_ceil(cols, 32) >= half_parts * (int64_t)attend_ceil(cols, 256));
  };
  for (int i = 0; i < n; ++i) {
    const int64_t cols = (int64_t)s[i].n * (q_heads / kv_heads);
    if (fills(cols)) wide += (int64_t)attend_ceil(cols, 32) * kv_heads * (s[i].pages - s[i].rows_pages / 2);
  }
  const bool tiles = es <= 2 && mode != 1 && (mode == 2 || wide > (int64_t)cus * (io16 ? (es == 1 ? 130 : 60) : 300));
  for (int i = 0; i < n; ++i) {
    const int64_t cols = (int64_t)s[i].n * (q_heads / kv_heads);
    s[i].kind = tiles && fills(cols) ? 2 : es == 4 || cols <= 16 || !io16 ? 0 : 1;
    s[i].tiles = attend_ceil(cols, attend_cols(s[i].kind));
    if (s[i].kind == 2) continue;
    work += (int64_t)s[i].pages * s[i].tiles * kv_heads;
    wgs += (int64_t)s[i].tiles * kv_heads;
  }
  const int two = attend_ceil(work, (int64_t)cus * 8);  // pages per wave, two workgroups per CU
  const int run = two <= (es == 1 ? 4 : 8) ? std::max(2, attend_ceil(work, (int64_t)cus * 4)) : std::min(two, 32);
  const int most = std::max(1, attend_ceil(64 * (int64_t)cus, std::max<int64_t>(wgs, 1)));
  int widest = 1;
  for (int i = 0; i < n; ++i) {
    if (s[i].kind == 2) continue;
    s[i].nsplit = s[i].pages <= (two >= 4 || (int64_t)s[i].n * q_heads > 512 ? 64 : 32) ? 1 : std::min({128, attend_ceil(s[i].pages, 4 * run), most});
    widest = std::max(widest, s[i].nsplit);
  }
  auto row_bytes = [&](int cap) {
    int64_t bytes = 0;
    for (int i = 0; i < n; ++i)
      if (s[i].kind != 2) bytes += span_part_bytes(s[i], std::min(s[i].nsplit, cap), q_heads, hd);
    return bytes;
  };
  int cap = widest;
  if (row_bytes(cap) > kAttendPartBytes) {  // the largest cap that fits (1 does)
    int over = cap;
    cap = 1;
    while (over - cap > 1) {
      const int mid = (cap + over) / 2;
      (row_bytes(mid) <= kAttendPartBytes ? cap : over) = mid;
    }
  }
  const int tile = tile_run(s, n, kv_heads, q_heads, hd, cus, kAttendPartBytes - row_bytes(cap));
  for (int i = 0; i < n; ++i) s[i].nsplit = s[i].kind == 2 ? tile_split(s[i], tile) : std::min(s[i].nsplit, cap);
}

// Pages of a workgroup of the tile kernel, the same for all spans (8B heads, INT8, 16 sequences of 1,000-9,000, 60
// rows: 127 us, 150 with the same number of splits for all): those that make the call shortest, counting 2.2 us for a step of a CU's workgroup, 5 us to start and end one, the
// partials written and read at 7 TB/s (mostly from the memory-side cache) and 9 us for joining them (eleven calls with 1 to 32 splits took that, most within 15%).
// Only runs whose partials take part_bytes at most (the longest, one per span, has none).
inline int tile_run(const AttendSize* s, int n, int kv_heads, int heads, int hd, int cus, int64_t part_bytes) {
  int longest_span = 1, best = 0;
  for (int i = 0; i < n; ++i)
    if (s[i].kind == 2) longest_span = std::max(longest_span, s[i].pages);
  double best_us = 1e300;
  for (int k : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
    const int run = attend_ceil(longest_span, k);
    double all = 0, longest = 0, parts = 0, wgs = 0;
    int64_t bytes = 0;
    for (int i = 0; i < n; ++i) {
      if (s[i].kind != 2) continue;
      const int mine = tile_split(s[i], run);
      const double us = 5 + 2.2 * attend_ceil(s[i].pages, 4 * mine);
      const double mean = 5 + 2.2 * (s[i].pages - 0.5 * s[i].rows_pages) / (4.0 * mine);
      const double w = (double)s[i].tiles * kv_heads * mine;
      all += w * mean;
      wgs += w;
      longest = std::max(longest, us);
      if (mine > 1) parts += (double)s[i].n * heads * mine;
      bytes += span_part_bytes(s[i], mine, heads, hd);
    }
    if (wgs == 0) break;
    if (bytes > part_bytes) continue;
    // workgroups of like length run in whole rounds; many of them even out but for the last
    const double rounds = wgs / cus;
    const double busy = wgs > 3.0 * cus ? all / cus + longest / 2 : all / cus * (rounds > 1 ? attend_ceil((int64_t)wgs, cus) / rounds : 1.0);
    const double us = std::max(busy, longest) + (parts > 0 ? 9 + parts * (hd + 2) * 8 / 7e6 : 0);
    if (us < best_us) {
      best = run;
      best_us = us;
    }
  }
  return best;
}

}  // namespace laser
