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
  // Rows a workgroup takes, 16 of a dense call.  Of experts more than the mean: LDS for rows that most of
  // them do not have costs waves, and an expert with more rows is read again from the last-level cache.
  // All us below: graph replays over sets of inputs in turn, 230 MB of 4096 x 4096, else more than the
  // last-level cache holds; experts' rows of X read through the sort.
  //   4 or 8 rows at 1.5 / 2 / 3 rows an expert.  MXFP4, 3072 x 3072, 128 experts: 81, 78 / 97, 89 / 128,
  //   108; 4096 x 4096, 8 experts: 14.9, 16.3 / 16.5, 16.7 / 18.6, 17.9.  Q4_K: 121, 122 / 148, 140 / 194,
  //   172; 21.3, 26.8 / 23.9, 27.1 / 28.8, 28.6.  NVFP4 has a cheaper form for 4 rows; at 2 / 2.5 / 3: 95,
  //   101 / 112, 114 / 126, 123; 15.8, 20.5 / 17.3, 20.9 / 18.1, 21.7.
  //   8 or 16 rows of Q4_K at 4 / 5 / 6 rows an expert.  14336 x 4096, 8 experts: 89, 101 / 94, 102 / -;
  //   4096 x 4096, 8: 31.2, 35.4 / 38.2, 36.6 / 43.1, 38.5; 3072 x 1536, 128: 117, 118 / - / 150, 139.
  // FP4 takes 16 through LDS for 8 rather than 16 in LDS, from 4 rows an expert on, or 2.5 of many
  // experts, whose rows spread wider (8 rows / 16 / 16 through 8).  3072 x 1536 MXFP4, 64 tokens to 8 of
  // 128: 74 / 79 / 68; 44 to 8: 59.7 / - / 58.9; 36 to 8, 1536 x 3072: 55.2 / - / 55.7; 14336 x 4096 MXFP4,
  // 60 to 2 of 8: 138 / 109.6 / 104.3; 16 to 2: 60.4 / - / 57.7; 12 to 2: 53.4 / - / 55.4; 1024 x 2048
  // NVFP4, 100 to 8 of 256: 76.7 / 76.4 / 68.7.  Dense calls gain or lose by shape (MXFP4, 24576 x 4096, 40
  // rows 45.3 / 36.6 with 16 in LDS / through 8; 4096 x 4096, 64 rows 11.6 / 13.3) and do without.
  const bool twice = grouped && fmt != QF_FMT_Q4K && R > 8 && (R >= 4 * E || (E >= 32 && 2 * R >= 5 * E));
  const bool few = 2 * R <= (fmt == QF_FMT_NVFP4 ? 5 : 3) * E;
  const int64_t xmax = !grouped || twice ? kMatvecMaxRows : few ? 4 : fmt != QF_FMT_Q4K || R <= 4 * E ? 8 : kMatvecMaxRows;
  p.xmax = (int)std::min(R, xmax);
  p.xrows = twice ? 8 : p.xmax;
  p.rows = fmt == QF_FMT_NVFP4 && p.xmax <= 4 ? kSmall : p.xrows < p.xmax ? kTwice : kAll;
  // row groups: of a dense call ceil(R / xmax); of E experts at most one more each
  p.items = grouped ? std::min(E, R) + R / p.xmax : (R + p.xmax - 1) / p.xmax;
  // Tile height and waves a tile: the least of rounds of resident workgroups (whole ones up to four,
  // then as they overlap) x (slices a wave takes + 1 for start and end) x what a slice copies.
  // Measured against it, us: 24576 x 4096 NVFP4, 1 row, 8 / 4 / 2 waves 13.7 / 12.5 / 12.8; 4096 x 4096 8
  // / 4 / 2 waves 4.9 / 5.5 / 6.8; 24576 x 4096, 16 rows, one tile 4 waves / two tiles 4 / 2 waves 22.9 /
  // 28.6 / 21.2; 64 rows x 4096 x 4096 MXFP4, 8 / 4 / 2 waves 16.5 / 13.3 / 11.6.
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
  // Codes that are read once, and are many, past the caches (24576 x 4096 NVFP4, one row, 13.1 -> 12.5
  // us; 4096 x 12288 MXFP4, 8 rows 10.7 -> 10.0); small weights may still be there from before, and
  // further row groups read them again (4096 x 4096 MXFP4: 16 rows 5.8 -> 6.1 us, 64 rows 11.6 -> 12.6).
  const bool many = (double)busy * (double)N * (double)K >= (double)(1 << 25);
  p.copy = (grouped || p.items == 1) && many ? kCopyNt : kCopy;
  if (fmt == QF_FMT_NVFP4 && K % 32) p.copy = kCopyWords;
  return p;
}

}  // namespace qf

#endif  // QF_MATVEC_PLAN_H_
