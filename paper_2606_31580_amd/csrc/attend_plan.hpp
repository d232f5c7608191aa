// Which kernel takes a span of laser_attend, and over how many workgroups its keys are split (host;
// plain C++).
#pragma once

#include <algorithm>
#include <cstdint>

namespace laser {

constexpr int kAttendKinds = 2;  // row kernel with 16 columns, with 32

// A span as the planner sees it, and what it decides.
struct AttendSize {
  int n, pages;  // query rows; pages that any of them sees
  int kind;      // AttendArgs' kernel
  int tiles;     // query tiles
  int nsplit;    // workgroups over a tile's pages
};

inline int attend_ceil(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Columns (rows x query heads of a kv head) of a tile of each kernel.
inline int attend_cols(int kind) { return kind == 0 ? 16 : 32; }

// wide: 16-bit rows and at most 16-bit K and V, for which the 32-column row kernel fits its registers.
// Splits: enough workgroups of 4 waves that every CU has two of them, a wave with at least 2 pages (they
// are computed in pairs); a span of up to 32 pages stays whole, since joining splits is a launch of
// its own.
inline void plan_attend(AttendSize* s, int n, int group, int kv_heads, int cus, bool wide) {
  int64_t work = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t cols = (int64_t)s[i].n * group;
    s[i].kind = cols <= 16 || !wide ? 0 : 1;
    s[i].tiles = attend_ceil(cols, attend_cols(s[i].kind));
    work += (int64_t)s[i].pages * s[i].tiles * kv_heads;
  }
  const int run = std::max(2, attend_ceil(work, (int64_t)cus * 8));  // pages per wave
  for (int i = 0; i < n; ++i)
    s[i].nsplit = s[i].pages <= 32 ? 1 : std::min(128, attend_ceil(s[i].pages, 4 * run));
}

}  // namespace laser
