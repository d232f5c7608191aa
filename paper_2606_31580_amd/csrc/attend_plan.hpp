// Which kernel takes a span of laser_attend, and over how many workgroups its keys are split (host;
// plain C++).
#pragma once

#include <algorithm>
#include <cstdint>

namespace laser {

constexpr int kAttendKinds = 3;  // row kernel with 16 columns, with 32; tile kernel
constexpr int kAttendFewCols = 64;

// A span as the planner sees it, and what it decides.
struct AttendSize {
  int n, pages;  // query rows; pages that any of them sees
  int kind;      // the kernel
  int tiles;     // query tiles
  int nsplit;    // workgroups over a tile's pages
};

inline int attend_ceil(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Columns (rows x query heads of a kv head) of a tile of each kernel.
inline int attend_cols(int kind) { return kind == 0 ? 16 : kind == 1 ? 32 : 256; }

// es: bytes of a cached element; io16: 16-bit rows.  fp32 pools have only the row kernel with 16 columns,
// and fp32 rows not the one with 32 (three parts of everything would not fit the registers).
//
// Row kernels: pages per wave.  Every CU runs one workgroup of 4 waves, or two on 8-bit pools (fewer
// registers).  Long runs stream best when two workgroups per CU share the pages; where that leaves a wave only
// a few pages, one per CU with twice the pages has fewer splits to join and, on wider pools, no second
// round (us, two and one per CU: 7B heads, 4 sequences of 3,000-14,000, bf16 pool, 4 pages a wave 23.9 and 19.4; 8B
// heads, 8 sequences, 17 pages 50.5 and 60.8; INT8, 16 sequences of 100-2,000, 2 pages 13.4 and 11.5; 6 of
// 3,000-9,000, 9 pages 20.5 and 26.6).  Runs end at 32 pages: more rounds even out ragged lengths (64 sequences of
// 3,000-14,000: 219 us with runs of 133 pages, 192 with 33).
// A span of up to 32 pages stays whole, since joining splits is a launch of its own, up to 64 where there
// are spans enough to fill the CUs (64 sequences of 50-600 positions: 18.2 us split, 14.4 whole).
// Tile kernel: one workgroup per CU, each with at least 16 pages.
inline void plan_attend(AttendSize* s, int n, int group, int kv_heads, int cus, int es, bool io16) {
  int64_t work = 0, wgs = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t cols = (int64_t)s[i].n * group;
    s[i].kind = es == 4 || cols <= 16 ? 0 : cols > kAttendFewCols ? 2 : io16 ? 1 : 0;
    s[i].tiles = attend_ceil(cols, attend_cols(s[i].kind));
    if (s[i].kind == 2)
      wgs += (int64_t)s[i].tiles * kv_heads;
    else
      work += (int64_t)s[i].pages * s[i].tiles * kv_heads;
  }
  const int two = attend_ceil(work, (int64_t)cus * 8);  // pages per wave, two workgroups per CU
  const int run = two <= (es == 1 ? 4 : 8) ? std::max(2, attend_ceil(work, (int64_t)cus * 4)) : std::min(two, 32);
  const int whole = two >= 4 ? 64 : 32;
  const int tile_splits = wgs > 0 ? std::max(1, attend_ceil(cus, wgs)) : 1;
  for (int i = 0; i < n; ++i) {
    if (s[i].kind == 2)
      s[i].nsplit = std::max(1, std::min({128, tile_splits, s[i].pages / 16}));
    else
      s[i].nsplit = s[i].pages <= whole ? 1 : std::min(128, attend_ceil(s[i].pages, 4 * run));
  }
}

}  // namespace laser
