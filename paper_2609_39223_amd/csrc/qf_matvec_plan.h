// How a product of few rows with packed weights is laid out on the device (qf_matvec.hip): rows of X
// and tiles a workgroup takes, waves that share a tile, copies, and how many row groups one launch
// holds.  Plain host code without HIP, so the rules can be checked without a device.
#ifndef QF_MATVEC_PLAN_H_
#define QF_MATVEC_PLAN_H_

#include <stdint.h>

#include <algorithm>

#include "qf.h"

namespace qf {

constexpr int kMatvecMaxWaves = 8;
constexpr int kMatvecMaxRows = 16;
constexpr int64_t kMatvecLdsBytes = 160 * 1024;

// LDS of 16 rows x 512 codes.
constexpr int matvec_code_bytes(int fmt) { return fmt == QF_FMT_Q4K ? 5120 : 4096; }

// Copies of codes: through the caches, past them, or in words (rows that are only 8-byte aligned).
enum Copy { kCopy = 0, kCopyNt = 1, kCopyWords = 2 };
// Forms of the kernel by rows of X; see matvec_kernel.
enum Rows { kAll = 0, kSmall = 1, kTwice = 2 };

struct MatvecPlan {
  int nt;               // tiles of 16 weight rows a workgroup takes (1 or 2)
  int copy, rows;       // Copy, Rows
  int xmax;             // rows of X a workgroup takes at most (1 .. 16)
  int xrows;            // rows of X that lie in LDS at once: xmax, or 8 of 16
  int waves;            // waves that share a tile's slices
  int64_t tiles;        // workgroups side by side over N
  int64_t items;        // row groups
  int64_t per_launch;   // row groups one launch holds (a grid has fewer than 2^32 lanes)
};

// R rows against one weight [N, K] (grouped false), or split over E of them by offsets on the device.
// R, N > 0; N < 2^30.
inline MatvecPlan matvec_plan(int fmt, bool grouped, int64_t E, int64_t N, int64_t K, int64_t R, int64_t cus) {
  MatvecPlan p{};
  // Rows a workgroup takes.  Experts: more than the mean, since LDS for rows that most experts do not
  // have costs waves, and an expert with more rows is read again from the last-level cache (3072 x
  // 3072 NVFP4, 32 tokens to 8 of 128: 4 rows 117 us, 8 rows 111; 2048 x 2048 Q4_K, 16 to 4 of 64: 4
  // rows 33.2, 8 rows 34.7; 3072 x 1536 MXFP4, 64 to 8 of 128: 8 rows 71.8, 16 rows 77.7).
  const int64_t xmax = !grouped ? kMatvecMaxRows : 2 * R <= 3 * E ? 4 : R <= 4 * E ? 8 : kMatvecMaxRows;
  p.xmax = p.xrows = (int)std::min(R, xmax);
  // 16 through LDS for 8, from 4 rows an expert on, or 2.5 of many experts, whose rows spread wider (us,
  // 8 or 16 rows / 16 through 8: 3072 x 1536 MXFP4, 64 tokens to 8 of 128 64.6 / 60.4, 44 to 8 52.6 / 51.5, 36
  // to 8 54.9 / 55.5 with 1536 x 3072; 14336 x 4096 MXFP4, 60 to 2 of 8 109.6 / 104.6, 16 to 2 60.1 / 57.6,
  // 12 to 2 52.7 / 55.2; 1024 x 2048 NVFP4, 100 to 8 of 256 76.4 / 68.7).  Dense calls gain or lose by
  // shape (MXFP4, 24576 x 4096, 40 rows 44.6 / 36.0; 4096 x 4096, 64 rows 11.4 / 13.3) and do without.
  if (grouped && fmt != QF_FMT_Q4K && R > 8 && (R >= 4 * E || (E >= 32 && 2 * R >= 5 * E))) {
    p.xrows = 8;
    p.xmax = (int)std::min<int64_t>(R, kMatvecMaxRows);
  }
  p.rows = fmt == QF_FMT_NVFP4 && p.xmax <= 4 ? kSmall : p.xrows < p.xmax ? kTwice : kAll;
  // row groups: of a dense call ceil(R / xmax); of E experts at most one more each
  p.items = grouped ? std::min(E, R) + R / p.xmax : (R + p.xmax - 1) / p.xmax;
  // Tile height and waves a tile: the least of rounds of resident workgroups (whole ones up to four,
  // then as they overlap) x (slices a wave takes + 1 for start and end) x what a slice copies.
  // Measured against it, us: 24576 x 4096 NVFP4, 1 row, 8 / 4 / 2 waves 15.4 / 14.8 / 15.4; 4096 x 4096 8
  // / 4 / 2 waves 5.1 / 5.8 / 7.4; 24576 x 4096, 16 rows, one tile 4 waves / two tiles 4 / 2 waves 24.3 /
  // 28.3 / 21.2; 64 rows x 4096 x 4096 MXFP4, 8 / 4 / 2 waves 15.9 / 12.9 / 11.4.
  const int64_t busy = grouped ? std::min(E, R) : p.items;   // row groups that are likely there
  const int64_t slices = std::max<int64_t>(1, (K + 511) / 512);
  double least = 0;
  for (int t = 1; t <= 2; ++t) {
    const int64_t unit = t * matvec_code_bytes(fmt) + p.xrows * 1024, tiles = (N + 16 * t - 1) / (16 * t);
    const int64_t blocks = tiles * busy;
    for (int64_t most = std::min<int64_t>(kMatvecMaxWaves, slices); most > 0; --most) {
      const int64_t each = (slices + most - 1) / most, waves = (slices + each - 1) / each;
      // (two tiles and one wave always pass both: N < 2^30)
      if (waves * unit > kMatvecLdsBytes || tiles > UINT32_MAX / (64 * waves)) continue;
      const int64_t resident = cus * std::min(kMatvecLdsBytes / (waves * unit), 32 / waves);
      const double rounds = blocks > 4 * resident ? (double)blocks / resident : (double)((blocks + resident - 1) / resident);
      const double cost = rounds * (each + 1) * unit;
      if (least == 0 || cost < least) {
        least = cost;
        p.nt = t;
        p.waves = (int)waves;
        p.tiles = tiles;
      }
    }
  }
  p.per_launch = UINT32_MAX / (64 * p.waves) / p.tiles;
  // Codes that are read once, and are many, past the caches (24576 x 4096 NVFP4, one row, 14.9 -> 14.4
  // us; 12288-deep MXFP4 9.9 -> 9.5); small weights may still be there from before, and further row
  // groups read them again (4096 x 4096: 16 rows 6.8 -> 7.0 us, 64 rows 13.5 -> 14.6).
  const bool many = (double)busy * (double)N * (double)K >= (double)(1 << 25);
  p.copy = (grouped || p.items == 1) && many ? kCopyNt : kCopy;
  if (fmt == QF_FMT_NVFP4 && K % 32) p.copy = kCopyWords;
  return p;
}

}  // namespace qf

#endif  // QF_MATVEC_PLAN_H_
