// Attention over the 4-bit cache for sequences with many new tokens (a prompt, or a piece of one): the
// mathematics, types and operand layouts of qf_attend.hip, with the decoded keys and values shared.
//
// A workgroup takes 128 rows (queries of the tokens and heads that share a head of the cache), 32 a wave, and all
// of its waves go through the same tokens, 64 at a time.  Decoding a tile once for each 32 rows costs more vector
// operations than the products themselves take; here each wave decodes a quarter of the tile, 16 tokens of K and
// a quarter of V's tiles of d, and leaves the matrix cores' operands in LDS (1 KB blocks, lane i's 16 bytes at 16 i),
// from which every wave reads all of them.  The tile that is multiplied, the one that is decoded and the one whose
// codes are on their way are three different ones, so there is one barrier a tile:
//   step k   copies of V's codes of tile k + 2 to LDS, its scales to FP16 in LDS; K's codes of k + 1 (loaded in
//            step k - 1) and V's (in LDS since then) decoded; tile k multiplied.
// 2048 new tokens behind 8192, 32 heads over 8, 128 wide (NVFP4): 353 us, 0.88 PFLOP/s (MXFP4 374); 32 rows a wave that each decode
// for themselves took 502, 16 rows 601, 64 rows 608.  Bound by what the two waves of a SIMD do one after the other:
// vector units busy half of the time (per row and token an exponent, a maximum, a sum, conversions; the decode),
// matrix units 30 %, LDS 30 % (32 KB of operands a wave and tile).  Scores of the next tile between the
// exponents of this one need more registers than there are (spilled, 487 us for 405 then).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "qf_attend.h"

namespace qf {
namespace attend {
namespace {

template <int FMT, int D>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_rows_kernel(AttendArgs p) {
  typedef Tile<FMT, D> T;
  constexpr int NQ = 2, NB = T::VS, CS = D / 32, DT = D / 16, SB = T::VS;
  __shared__ uint4 keys[2][4 * CS][64];                 // operand s of 16 tokens u at u CS + s
  __shared__ uint4 values[2][2 * DT][64];               // operands 0, 1 of d's tile d at 2 d
  __shared__ __align__(16) char raw[2][kTile * D / 2];  // V's codes on their way
  __shared__ __align__(16) _Float16 vscale[2][NB * kTile];
  __shared__ uint64_t special_of[4][4];                 // of tile k % 4, 16 tokens: bits 4 r .. 4 r + 3 of token r
  __shared__ __align__(4) uint8_t flags_of[4][4];       // of 16 tokens: 1 no page, 2 some are special
  __shared__ __align__(16) uint32_t nan_of[2][4];       // of 16 tokens: keys with NaN scales (MXFP4)
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const KvCache& c = p.c;
  uint32_t bid = blockIdx.x;
  const int h = (int)(bid % (uint32_t)c.H);
  bid /= (uint32_t)c.H;
  const int grp = (int)(bid % (uint32_t)p.groups);
  bid /= (uint32_t)p.groups;
  const int split = (int)(bid % (uint32_t)p.splits);
  int b, tok0, first, n;
  // (the last row tiles, which see most, first: 405 -> 387 us)
  const int items = (int)(gridDim.x / (uint32_t)(c.H * p.groups * p.splits)), item = p.item0 + items - 1 - (int)(bid / (uint32_t)p.splits);
  if (!find_tile(p.q, p.tpt, item, b, tok0, first, n)) return;

  const int page_log = c.page_log;
  const int len = max(__builtin_amdgcn_readfirstlane(p.q.lens[b]), 0), pos0 = len - n + first, toks = min(p.tpt, n - first);
  const Reach reach = reach_of(p, len, pos0, pos0 + toks - 1);
  const int a0 = reach.lo + split * p.chunk, todo = max(min(a0 + p.chunk, reach.hi) - a0, 0), tiles = (todo + kTile - 1) / kTile;

  // this wave's 32 rows
  int row_at[NQ], row_pos[NQ];
  bool row_ok[NQ];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    const int r = 32 * wv + 16 * j + l16, i = r / p.Gg, gh = grp * p.Gg + r % p.Gg;
    row_ok[j] = i < toks && gh < p.G;
    row_pos[j] = pos0 + (row_ok[j] ? i : toks - 1);     // (what a row that is none sees is not stored)
    row_at[j] = (tok0 + (row_ok[j] ? i : 0)) * (int)p.a.Hq + h * p.G + (row_ok[j] ? gh : 0);
  }
  // positions from which on no row of this wave sees anything
  int wave_end = max(row_pos[0], row_pos[1]) + 1;
#pragma unroll
  for (int d = 1; d < 16; d *= 2) wave_end = max(wave_end, __shfl_xor(wave_end, d, 64));
  wave_end = __builtin_amdgcn_readfirstlane(wave_end);

  // ids of the pages of this wave's 16 tokens of 64 tiles, -1 for a bad one
  const int32_t* const table = p.q.table + b * p.q.cols;
  int tile_base = 0, ids = -1;
  auto fetch_ids = [&](int tile) {
    const int pos = a0 + min((tile + lane) * kTile + 16 * wv, (todo - 1) & ~15);
    const int id = table[pos >> page_log];
    tile_base = tile;
    ids = id >= 0 && id < c.pages ? id : -1;
  };
  // where this wave's 16 tokens of a tile lie, counted in tokens; past the end the last ones
  auto place = [&](int tile, uint32_t& bad) -> int64_t {
    if (tile - tile_base >= 64) fetch_ids(tile);
    const int pos = a0 + min(tile * kTile + 16 * wv, (todo - 1) & ~15);
    const int id = __builtin_amdgcn_readlane(ids, tile - tile_base);
    bad = (uint32_t)id >> 31;
    return (((int64_t)max(id, 0) * c.H + h) << page_log) + (pos & ((1 << page_log) - 1));
  };
  auto quarter = [&](int q4) { return FMT == QF_FMT_MXFP4 && D == 64 ? q4 >> 1 : q4 * T::KS; };
  const uint32_t row_k = l16 * (D / 2) + g * (D / 8), row_ks = l16 * SB + quarter(g), row_vs = (lane >> 2) * SB + quarter(lane & 3);
  auto load_scales = [&](global_byte* sp) -> uint32_t {
    return T::KS == 4 ? load_as<uint32_t>(sp) : T::KS == 2 ? load_as<uint16_t>(sp) : *sp;
  };
  uint32_t kw[T::W], ks = 0, vs = 0, bad_vs = 0;        // K of the tile to be decoded next, V's scales of the one after it
  int64_t at_v = 0;                                     // the place of vs
  auto load_k = [&](int64_t at) {
    load_words<T::W>(lane_at(c.codes[0] + at * (D / 2), row_k), kw);
    ks = load_scales(lane_at(c.scales[0] + at * SB, row_ks));
  };
  auto load_vs = [&](int tile) {
    at_v = place(tile, bad_vs);
    vs = load_scales(lane_at(c.scales[1] + at_v * SB, row_vs));
  };
  auto copy_v = [&](int64_t at, char* to) { copy_values<D>(c.codes[1] + at * (D / 2), wv, lane, to); };
  auto put_scales = [&](int tile) {
    const bool seen = tile * kTile + 16 * wv + (lane >> 2) < todo && !bad_vs;
    const uint64_t special = __ballot(store_scales<FMT, T::KS>(seen ? vs : 0u, quarter(lane & 3), wv, lane, vscale[tile & 1]));
    if (lane == 0) {
      special_of[tile & 3][wv] = special;
      flags_of[tile & 3][wv] = (uint8_t)(bad_vs | (special ? 2u : 0u));
    }
  };
  auto put_keys = [&](int tile) {
#pragma unroll
    for (int s = 0; s < CS; ++s) keys[tile & 1][wv * CS + s][lane] = decode_key<FMT>(kw[s], ks, s);
    if constexpr (FMT == QF_FMT_MXFP4) {
      const uint32_t nan = nan_keys<FMT, T::KS>(ks);
      if (lane == 0) nan_of[tile & 1][wv] = nan;
    }
  };
  auto put_values = [&](int tile) {
#pragma unroll
    for (int i = 0; i < DT / 4; ++i) {
      const int d = wv * (DT / 4) + i;
      uint4 v0, v1;
      decode_values<FMT, D>(raw[tile & 1], vscale[tile & 1], d, lane, v0, v1);
      values[tile & 1][2 * d][lane] = v0;
      values[tile & 1][2 * d + 1][lane] = v1;
    }
  };
  auto arrived = [&]() {                                // this wave's copies and everybody's LDS writes
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);                 // vmcnt(0)
    asm volatile("" ::: "memory");
    __syncthreads();
  };

  int64_t at_next = 0;                                  // the place of tile k + 2 at the top of step k
  if (tiles > 0) {
    fetch_ids(0);
    load_vs(0);
    copy_v(at_v, raw[0]);
    load_k(at_v);
    put_scales(0);
    put_keys(0);
    if (tiles > 1) {
      load_vs(1);
      copy_v(at_v, raw[1]);
      load_k(at_v);
      put_scales(1);
    }
    if (tiles > 2) {
      load_vs(2);
      at_next = at_v;
    }
  }

  uint4 q[NQ][CS];
  float cz[NQ], m[NQ], l[NQ];
  int far = 0;
  f32x4_t acc[NQ][DT];
  const float S_k = FMT == QF_FMT_NVFP4 ? c.S[0][h] : 1.0f;
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    cz[j] = load_query<FMT, D>(p, row_at[j], g, S_k, q[j]);
    m[j] = neg_inf();
    l[j] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[j][d] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }
  if (tiles > 0) {
    arrived();
    put_values(0);
    __syncthreads();
  }

  // A wave on its way to the barrier, from its outputs through the next tile's decode, goes before the other workgroup's
  // wave that scores: 387 -> 357 us (the other way round, products first, 410; softmax first 378).
  for (int k = 0; k < tiles; ++k) {
    __builtin_amdgcn_s_setprio(1);
    if (k + 2 < tiles) put_scales(k + 2);
    if (k + 1 < tiles) {
      put_keys(k + 1);
      put_values(k + 1);
    }
    if (k + 2 < tiles) {                                // (after the use of what was loaded a step ago, or that would wait for these)
      copy_v(at_next, raw[k & 1]);                      // (V's codes of tile k were decoded a step ago)
      load_k(at_next);
    }
    if (k + 3 < tiles) {
      load_vs(k + 3);
      at_next = at_v;
    }

    __builtin_amdgcn_s_setprio(0);
    const int t0 = k * kTile, base = a0 + t0;
    if (base < wave_end) {
      f32x4_t zz[NQ][4];
#pragma unroll
      for (int j = 0; j < NQ; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) zz[j][u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int s = 0; s < CS; ++s) {
          const uint4 a = keys[k & 1][u * CS + s][lane];
#pragma unroll
          for (int j = 0; j < NQ; ++j) zz[j][u] = mfma_z<FMT>(a, q[j][s], zz[j][u]);
        }
      const uint32_t flags = __builtin_amdgcn_readfirstlane(*reinterpret_cast<const uint32_t*>(flags_of[k & 3]));
      const uint32_t bad = (flags & 1u) | (flags >> 7 & 2u) | (flags >> 14 & 4u) | (flags >> 21 & 8u);
      float z[NQ][16];
#pragma unroll
      for (int j = 0; j < NQ; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) z[j][i] = zz[j][i >> 2][i & 3];
      if constexpr (FMT == QF_FMT_MXFP4) {
        const uint4 nan4 = *reinterpret_cast<const uint4*>(nan_of[k & 1]);
        if (__builtin_amdgcn_readfirstlane(nan4.x | nan4.y | nan4.z | nan4.w)) {
          const uint32_t nan[4] = {nan4.x, nan4.y, nan4.z, nan4.w};
#pragma unroll
          for (int j = 0; j < NQ; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if ((nan[i >> 2] >> (4 * g + (i & 3))) & 1u) z[j][i] = __builtin_nanf("");
        }
      }
      const bool whole = t0 + kTile <= todo && bad == 0;
      uint32_t pw[NQ][8];
      int from[NQ], to[NQ];
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        from[j] = p.window > 0 ? row_pos[j] - p.window + 1 - base : 0;
        to[j] = min(row_pos[j] + 1 - base, todo - t0);
      }
      softmax_step<DT>(z, cz, from, to, whole, bad, g, m, l, acc, pw, far);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const uint4 v0 = values[k & 1][2 * d][lane], v1 = values[k & 1][2 * d + 1][lane];
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
          acc[j][d] = mfma_o(v0, make_uint4(pw[j][0], pw[j][1], pw[j][2], pw[j][3]), acc[j][d]);
          acc[j][d] = mfma_o(v1, make_uint4(pw[j][4], pw[j][5], pw[j][6], pw[j][7]), acc[j][d]);
        }
      }
      if (flags & 0x02020202u) {
#pragma unroll 1
        for (int u = 0; u < 4; ++u) {
          uint64_t those = special_of[k & 3][u];
#pragma unroll 1
          while (__any(those != 0)) {
            const int r = __builtin_amdgcn_readfirstlane(__builtin_ctzll(those) >> 2), pos = base + 16 * u + r;
            those &= ~(15ull << (4 * r));
            const int64_t at = (((int64_t)table[pos >> page_log] * c.H + h) << page_log) + (pos & ((1 << page_log) - 1));
            const uint8_t* const codes = c.codes[1] + at * (D / 2) + 2 * g;
            add_special<FMT, D, NQ>(p, c.scales[1] + at * SB, [&](int d) -> uint32_t {
              return *reinterpret_cast<const uint16_t*>(codes + 8 * d);
            }, u, r, pos, l16, pw, row_pos, acc);
          }
        }
      }
    }
    arrived();
  }
  __builtin_amdgcn_s_setprio(0);

#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    l[j] += __shfl_xor(l[j], 16, 64);
    l[j] += __shfl_xor(l[j], 32, 64);
    if (row_ok[j]) emit_row<FMT, D>(p, split, row_at[j], h, g, acc[j], m[j], l[j]);
  }
}

template <int FMT, int D>
hipError_t launch(AttendArgs a, int64_t items, hipStream_t s) {
  const int64_t each = (int64_t)a.splits * a.groups * a.c.H, most = std::max<int64_t>(1, ((int64_t)1 << 23) / each);
  for (int64_t i = 0; i < items; i += most) {
    a.item0 = (int)i;
    hipLaunchKernelGGL((attend_rows_kernel<FMT, D>), dim3((unsigned)(std::min(most, items - i) * each)), dim3(64 * kWaves), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_rows(const AttendArgs& a, int64_t items, hipStream_t s) {
  if (a.c.fmt == QF_FMT_NVFP4) return a.c.D == 64 ? launch<QF_FMT_NVFP4, 64>(a, items, s) : launch<QF_FMT_NVFP4, 128>(a, items, s);
  return a.c.D == 64 ? launch<QF_FMT_MXFP4, 64>(a, items, s) : launch<QF_FMT_MXFP4, 128>(a, items, s);
}

}  // namespace attend
}  // namespace qf
