// Attention of new tokens over the 4-bit cache of keys and values (qf_kv.h):
//   z_t = scale q . k_t,  O = sum exp(z_t - lse) v_t,  lse = log sum exp z_t
// over the positions t that the query sees, in one pass with a running maximum and sum.
//
// A workgroup takes 16 NQ rows, the queries of tpt tokens and Gg heads that share a head of the cache,
// and a piece of the tokens they see; each of its four waves takes a quarter of the piece on its own, 64
// tokens at a time, and their sums meet in LDS.  Pieces of one row meet in a second kernel (merge).
// On v_mfma_f32_16x16x32 both products are taken transposed, Z^T = K Q^T and O^T = V^T P^T: a row's
// scores, maximum, sum and outputs then all belong to lane % 16, so P goes from the first product
// into the second without leaving its registers.
//   K  lane (token l16, group g) holds d = g D / 4 ..: a token's bytes as they lie in memory, four
//      groups side by side.  (Any bijection of d is fine as long as Q uses it.)
//   V  64 tokens' codes go through LDS and are read back transposed (ds_read_b64_tr_b4): lane (d l16,
//      g) gets the 16 tokens 16 u + 4 g + i, which are the ones whose P it holds.
// What is exact:  NVFP4  V s in FP16 (E2M1 has 2 significant bits, E4M3 4; 2^-10 <= |V s| <= 2688); the
// head's S multiplies scores and outputs.  Queries are FP16 (MXFP4: bf16), each row times a power of two that
// takes its largest element to 2^14 .. 2^15: bits below 2^-38 of that are lost, less than FP32 sums lose.
//                 MXFP4  keys V 2^p in bf16.  Values V 2^(p + 6) in FP16 for
// -20 <= p <= 7; blocks with any other scale (but 0, the code of a block of zeros), and under both
// formats blocks with NaN scales, are "special" and added one by one in FP32, which also keeps an
// infinity or NaN away from the rows that do not see it.
// Probabilities are rounded to FP16 as 2^14 exp(z - max): relative 2^-11 down to 2^-28 of the row's
// largest and absolute 2^-38 of it below, so that many small ones still sum.  The sum of
// probabilities is of the unrounded ones, in FP32.
// Bound by memory where the batch fills the card: 64 sequences x 8192 tokens x 8 heads of 128 (NVFP4, 4 rows a
// head) 117 us, 5.2 TB/s (MXFP4 114); its loads alone take 103.  One sequence of 131072: 39 us, 3.9 TB/s, loads alone 33.  With
// several rows a head (5 drafted tokens) by the softmax, 16 exponents a lane, row and 64 tokens, and by what
// decoding costs each wave; short sequences by trips to memory one after the other (row, length, page, codes), 7 us.  Prompts with heads of
// 256 (32 rows that each wave decodes for, one wave a SIMD: 2048 new tokens behind 8192, NVFP4, 1276 us, 0.48 PFLOP/s) by
// what that wave does one after the other, vector units half of the time, matrix units a fifth.
// What did not pay: four or two workgroups a compute unit for three (registers spilled at 128: 127 us for 117),
// waves taking every fourth tile of the piece instead of a quarter of it (129), workgroups of 8 or 16 waves
// (129 - 144), 64 rows a wave.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "qf_attend.h"

namespace qf {
namespace attend {
namespace {

template <int FMT, int D, int NQ>
__global__ __launch_bounds__(64 * kWaves, NQ == 2 && D == 256 ? 1 : NQ == 2 || D == 256 ? 2 : 3) void attend_kernel(AttendArgs p) {
  typedef Tile<FMT, D> T;
  constexpr int NB = T::VS, CS = D / 32, DT = D / 16;   // V's blocks, steps of a score, tiles of d
  constexpr int kCodes = kTile * D / 2, kStage = kCodes + NB * kTile * 2;   // a wave's LDS: codes, scales in FP16
  constexpr int kSum = DT * 64 * 16;                    // a wave's outputs of 16 rows on their way to another
  __shared__ __align__(16) char smem[std::max(kWaves * kStage, 2 * kSum)];
  __shared__ uint4 queries[NQ][CS][64];                 // the rows of Q as the products take them
  __shared__ float rows_m[kWaves][16 * NQ], rows_l[kWaves][16 * NQ];
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
  if (!find_tile(p.q, p.tpt, p.item0 + (int)(bid / (uint32_t)p.splits), b, tok0, first, n)) return;

  const int page_log = c.page_log;
  const int len = max(__builtin_amdgcn_readfirstlane(p.q.lens[b]), 0), pos0 = len - n + first, toks = min(p.tpt, n - first);
  const Reach reach = reach_of(p, len, pos0, pos0 + toks - 1);

  // this lane's row of each 16
  int row_at[NQ], row_pos[NQ];                          // row of [T, Hq]; position
  bool row_ok[NQ];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    const int r = 16 * j + l16, i = r / p.Gg, gh = grp * p.Gg + r % p.Gg;
    row_ok[j] = i < toks && gh < p.G;
    row_pos[j] = pos0 + (row_ok[j] ? i : toks - 1);     // (what a row that is none sees is not stored)
    row_at[j] = (tok0 + (row_ok[j] ? i : 0)) * (int)p.a.Hq + h * p.G + (row_ok[j] ? gh : 0);
  }
  if (p.splits > 1 && split >= live_pieces(reach, p.chunk)) {   // a piece that the sequence does not have
    if (wv == 0 && g == 0)
#pragma unroll
      for (int j = 0; j < NQ; ++j)
        if (row_ok[j]) row_sums(p, split, row_at[j], D) = f32x2_t{neg_inf(), 0.0f};
    return;
  }
  // this wave's tokens
  const int a0 = reach.lo + split * p.chunk, a1 = min(a0 + p.chunk, reach.hi);
  const int per = (max(a1 - a0, 0) + kWaves * kTile - 1) / (kWaves * kTile) * kTile;
  const int w0 = a0 + wv * per, todo = max(min(w0 + per, a1) - w0, 0);

  char* const mine = smem + wv * kStage;
  _Float16* const vscale = reinterpret_cast<_Float16*>(mine + kCodes);

  // ids of 64 pages in the lanes of one register, -1 for a bad one
  const int page_first = w0 >> page_log, page_last = (w0 + todo - 1) >> page_log;
  const int32_t* const table = p.q.table + b * p.q.cols;
  int page_base = page_first, ids = -1;
  auto fetch_ids = [&](int base) {
    const int id = table[min(base + lane, page_last)];
    page_base = base;
    ids = id >= 0 && id < c.pages ? id : -1;
  };

  T x;
  uint32_t bad_now = 0, bad_next = 0;                 // bit u: the tile's tokens 16 u .. have no page
  constexpr int SB = T::VS;                           // scale bytes of a token
  const uint32_t row_k = l16 * (D / 2) + g * (D / 8);
  auto quarter = [&](int q4) { return FMT == QF_FMT_MXFP4 && D == 64 ? q4 >> 1 : q4 * T::KS; };
  const uint32_t row_ks = l16 * SB + quarter(g), row_vs = (lane >> 2) * SB + quarter(lane & 3);
  auto load_scales = [&](global_byte* sp) -> uint32_t {
    return T::KS == 4 ? load_as<uint32_t>(sp) : T::KS == 2 ? load_as<uint16_t>(sp) : *sp;
  };

  // where the 16 tokens from w0 + t on lie, counted in tokens, and whether they have a page; past the end
  // the last ones again
  auto place = [&](int t, uint32_t& bad) -> int64_t {
    const int pos = w0 + min(t, (todo - 1) & ~15);
    const int id = __builtin_amdgcn_readlane(ids, (pos >> page_log) - page_base);
    bad = (uint32_t)id >> 31;
    return (((int64_t)max(id, 0) * c.H + h) << page_log) + (pos & ((1 << page_log) - 1));
  };
  auto load_k = [&](int t) {
    if (((w0 + min(t + 48, (todo - 1) & ~15)) >> page_log) - page_base >= 64) fetch_ids((w0 + t) >> page_log);
    bad_next = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint32_t bad;
      const int64_t at = place(t + 16 * u, bad);
      bad_next |= bad << u;
      load_words<T::W>(lane_at(c.codes[0] + at * (D / 2), row_k), x.k[u]);
      x.ks[u] = load_scales(lane_at(c.scales[0] + at * SB, row_ks));
    }
  };
  // V's codes to LDS, rows back to back as the copies lay them down; the scales of token 16 u + lane / 4
  auto load_v = [&](int t) {
    int64_t at[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      uint32_t bad;
      at[u] = place(t + 16 * u, bad);
      x.vs[u] = load_scales(lane_at(c.scales[1] + at[u] * SB, row_vs));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) copy_values<D>(c.codes[1] + at[u] * (D / 2), u, lane, mine);
  };

  if (todo > 0) {
    fetch_ids(page_first);
    load_k(0);
    load_v(0);
  }

  float cz[NQ];                                         // times this scores are in units of log 2
  const float S_k = FMT == QF_FMT_NVFP4 ? c.S[0][h] : 1.0f;
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    uint4 q[CS];
    cz[j] = load_query<FMT, D>(p, row_at[j], g, S_k, q);
#pragma unroll
    for (int s = 0; s < CS; ++s)
      if (s % kWaves == wv) queries[j][s][lane] = q[s];
  }
  __syncthreads();

  float m[NQ], l[NQ];
  int far = 0;
  f32x4_t acc[NQ][DT];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    m[j] = neg_inf();
    l[j] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[j][d] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  if (todo > 0) {
    for (int t0 = 0; t0 < todo; t0 += kTile) {
      bad_now = bad_next;
      // ---- scores
      f32x4_t zz[NQ][4];
#pragma unroll
      for (int j = 0; j < NQ; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) zz[j][u] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < CS; ++s) {
        uint4 q[NQ];
#pragma unroll
        for (int j = 0; j < NQ; ++j) q[j] = queries[j][s][lane];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint4 a = decode_key<FMT>(x.k[u][s], x.ks[u], s);
#pragma unroll
          for (int j = 0; j < NQ; ++j) zz[j][u] = mfma_z<FMT>(a, q[j], zz[j][u]);
        }
      }
      float z[NQ][16];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t nan_rows = nan_keys<FMT, T::KS>(x.ks[u]);
#pragma unroll
        for (int j = 0; j < NQ; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            z[j][4 * u + i] = zz[j][u][i];
            if (nan_rows && ((nan_rows >> (4 * g + i)) & 1u)) z[j][4 * u + i] = __builtin_nanf("");
          }
      }
      // the scales, in the order in which the products take them; zeros for tokens that no row sees and
      // for special ones
      uint32_t special = 0;                             // bit u: one of this quarter of token 16 u + lane / 4
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool seen = t0 + 16 * u + (lane >> 2) < todo && !((bad_now >> u) & 1u);
        if (store_scales<FMT, T::KS>(seen ? x.vs[u] : 0u, quarter(lane & 3), u, lane, vscale)) special |= 1u << u;
      }
      // ---- which positions a row sees, its maximum, its probabilities
      const int base = w0 + t0;
      const bool whole = t0 + kTile <= todo && bad_now == 0;
      uint32_t pw[NQ][8];
      int from[NQ], to[NQ];
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        from[j] = p.window > 0 ? row_pos[j] - p.window + 1 - base : 0;
        to[j] = min(row_pos[j] + 1 - base, todo - t0);
      }
      softmax_step<DT>(z, cz, from, to, whole, bad_now, g, m, l, acc, pw, far);
      // ---- outputs
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0F70);               // vmcnt(0): this wave's copies of V are in its region
      asm volatile("" ::: "memory");
      if (t0 + kTile < todo) load_k(t0 + kTile);
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        uint4 v0, v1;
        decode_values<FMT, D>(mine, vscale, d, lane, v0, v1);
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
          acc[j][d] = mfma_o(v0, make_uint4(pw[j][0], pw[j][1], pw[j][2], pw[j][3]), acc[j][d]);
          acc[j][d] = mfma_o(v1, make_uint4(pw[j][4], pw[j][5], pw[j][6], pw[j][7]), acc[j][d]);
        }
      }
      // ---- blocks with special scales, one token after the other
      if (__any(special != 0)) {
#pragma unroll 1
        for (int u = 0; u < 4; ++u) {
          uint64_t those = __ballot((special >> u) & 1u);
#pragma unroll 1
          while (those) {
            const int r = __builtin_ctzll(those) >> 2, t = 16 * u + r, pos = base + t;
            those &= ~(15ull << (4 * r));
            const int id = table[pos >> page_log];      // (a good page: it was seen)
            const uint8_t* const sp = c.scales[1] + ((((int64_t)id * c.H + h) << page_log) + (pos & ((1 << page_log) - 1))) * SB;
            const char* const codes = mine + t * (D / 2) + 2 * g;
            add_special<FMT, D, NQ>(p, sp, [&](int d) -> uint32_t {
              return *reinterpret_cast<const uint16_t*>(codes + 8 * (d ^ (v_swap<D>(t) << 1)));
            }, u, r, pos, l16, pw, row_pos, acc);
          }
        }
      }
      if (t0 + kTile < todo) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the next copies land
        load_v(t0 + kTile);
      }
    }
  }

  // ---- the four waves' sums
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    l[j] += __shfl_xor(l[j], 16, 64);
    l[j] += __shfl_xor(l[j], 32, 64);
    if (g == 0) {
      rows_m[wv][16 * j + l16] = m[j];
      rows_l[wv][16 * j + l16] = l[j];
    }
  }
  __syncthreads();
  float lt[NQ], mt[NQ];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    const int r = 16 * j + l16;
    float top = rows_m[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, rows_m[w][r]);
    const float ref = top == neg_inf() ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sum += rows_l[w][r] * __builtin_amdgcn_exp2f(rows_m[w][r] - ref);
    lt[j] = sum;
    mt[j] = top;
    const float f = __builtin_amdgcn_exp2f(m[j] - ref);
#pragma unroll
    for (int d = 0; d < DT; ++d) acc[j][d] *= f;
  }
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    auto give = [&](char* to) {
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4_t*>(to + (d * 64 + lane) * 16) = acc[j][d];
    };
    auto take = [&](const char* from) {
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[j][d] += *reinterpret_cast<const f32x4_t*>(from + (d * 64 + lane) * 16);
    };
    if (wv >= 2) give(smem + (wv - 2) * kSum);
    __syncthreads();
    if (wv < 2) take(smem + wv * kSum);
    __syncthreads();
    if (wv == 1) give(smem);
    __syncthreads();
    if (wv == 0) take(smem);
    if (j + 1 < NQ) __syncthreads();
  }
  if (wv != 0) return;

#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    if (row_ok[j]) emit_row<FMT, D>(p, split, row_at[j], h, g, acc[j], mt[j], lt[j]);
  }
}

// A row's pieces' sums, brought to the largest maximum.  A lane takes 4 of the row's elements of every P-th piece with
// a running maximum of its own, so no load waits for another; D / 4 P lanes have a row, all of a workgroup
// (P = 256 / (D / 4), its parts meet in LDS) or, for few pieces, a wave or less (P = 1).
template <int FMT, int D, int P>
__global__ __launch_bounds__(256) void merge_kernel(AttendArgs p) {
  constexpr int L = D / 4, ROWS = 256 / (L * P);
  __shared__ f32x4_t sum[P][L];
  __shared__ float top_of[P], l_of[P];
  const int tid = threadIdx.x, e = tid % L, part = P == 1 ? 0 : tid / L;
  const int64_t R = p.q.T * p.a.Hq, row = (int64_t)p.item0 + (int64_t)blockIdx.x * ROWS + (P == 1 ? tid / L : 0), t = row / p.a.Hq;
  if (P == 1 && row >= R) return;
  const int hq = (int)(row - t * p.a.Hq);
  f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
  float top = neg_inf(), l = 0.0f;
  constexpr int U = 4;                                  // pieces whose loads are in flight together
  for (int s0 = part; s0 < p.splits; s0 += U * P) {
    f32x2_t w[U];
    f32x4_t v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int s = min(s0 + i * P, p.splits - 1);      // (past the last: the last again, which does not count)
      w[i] = row_sums(p, s, row, D);
      v[i] = *reinterpret_cast<const f32x4_t*>(p.part + (s * R + row) * D + 4 * e);
      if (s0 + i * P >= p.splits) w[i][1] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      // (a piece without tokens holds no outputs; its sum says so, for a maximum of -inf has one that saw NaN alone too)
      if (w[i][1] == 0.0f) continue;
      const float now = fmaxf(top, w[i][0]), down = __builtin_amdgcn_exp2f(top - now), f = __builtin_amdgcn_exp2f(w[i][0] - now);
      l = l * down + f * w[i][1];
      acc = acc * down + f * v[i];
      top = now;
    }
  }
  if (p.q.off && t >= p.q.off[p.q.B]) return;           // a row of nobody: nothing was written for it
  if constexpr (P > 1) {
    sum[part][e] = acc;
    if (e == 0) {
      top_of[part] = top;
      l_of[part] = l;
    }
    __syncthreads();
    if (tid >= L) return;
#pragma unroll
    for (int i = 0; i < P; ++i) top = fmaxf(top, top_of[i]);
    const float ref = top == neg_inf() ? 0.0f : top;
    acc = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    l = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float f = __builtin_amdgcn_exp2f(top_of[i] - ref);
      acc += f * sum[i][tid];
      l += f * l_of[i];
    }
  }
  const float f = 1.0f / l, S = FMT == QF_FMT_NVFP4 ? p.c.S[1][hq / p.G] : 0x1p-6f;   // (S / l may have few bits left)
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = codec::bf16_rne(l == 0.0f ? 0.0f : acc[k] * f * S);
  *reinterpret_cast<uint2*>(p.a.O + t * p.a.ldo + (int64_t)hq * D + 4 * e) = make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
  if (p.a.lse && e == 0) p.a.lse[row] = l == 0.0f ? neg_inf() : (top + (__builtin_log2f(l) - kUp)) * kLn2;
}

// ------------------------------------------------------------------------------ the launch rules
struct Plan {
  int nq, G, Gg, groups, tpt, splits, chunk, most;      // nq: 16 rows a wave takes; 0: qf_attend_rows.hip
  int64_t items;
};

Plan plan_of(const KvCache& c, const KvSeqs& q, const AttendCall& a) {
  Plan p;
  p.G = (int)(a.Hq / c.H);
  p.groups = (p.G + 15) / 16;
  p.Gg = (p.G + p.groups - 1) / p.groups;
  // rows a sequence has on average: from 17 on 32 a wave, so that keys and values are decoded once for both
  // halves; from 128 on the kernel that shares the decoded ones between waves (heads of 256 do not fit it).  16
  // sequences x 4096 tokens x 8 heads of 128, us with 16 a wave / 32 a wave / shared:  16 rows 27 / 29 / 53,
  // 20 rows 40 / 30 / 53, 64 rows 65 / 45 / 59, 128 rows 87 / 69 / 62, 512 rows 295 / 243 / 156
  const int64_t rows = q.off ? q.T / std::max<int64_t>(q.B, 1) * p.Gg : 1;
  p.nq = rows <= 16 ? 1 : rows < kManyRows || c.D == 256 ? 2 : 0;
  p.tpt = (p.nq ? 16 * p.nq : kManyRows) / p.Gg;
  p.items = q.off ? q.T / p.tpt + q.B : q.B;
  // pieces of the tokens: two workgroups a compute unit (one sequence of 131072: one 48 us, two 38, three 38, four
  // 42, eight 47; 20 of 8192: 59, 47, 47, 50, 51), none of less than one tile a wave (4 of 2048: pieces of 256
  // 10.2 us, of 512 11.9)
  p.most = c.pages == 0 ? 0 : (int)std::min(a.max_len, q.cols << c.page_log);
  const int64_t longest = std::max<int64_t>(1, a.window > 0 ? std::min<int64_t>(p.most, a.window + p.tpt + 15) : p.most);
  // (the row tiles of sequences with as many rows each: p.items, the most that there can be, has up to twice as
  // many, and 16 sequences of 8 new tokens took 45 us for 32)
  const int64_t each = q.off ? (q.T + q.B * p.tpt - 1) / (q.B * p.tpt) : 1;
  const int64_t tiles = std::max<int64_t>(1, q.B * each * p.groups * c.H), goal = 2 * compute_units();
  int64_t want = (goal + tiles - 1) / tiles;
  if (want > 1 && tiles * want > (p.nq == 1 ? 3 : 2) * compute_units()) --want;
  // (no more than run at one time: 16 sequences of 24 new tokens in 768 workgroups, 512 of them at a time, took 86
  // us, in 384 69)
  const int64_t least = kWaves * kTile;
  const int64_t chunk = (longest + want - 1) / want;
  p.chunk = (int)((chunk + least - 1) / least * least);
  p.splits = (int)((longest + p.chunk - 1) / p.chunk);
  return p;
}

template <int FMT, int D, int P>
hipError_t merge(AttendArgs a, hipStream_t s) {
  constexpr int64_t rows = 256 / (D / 4 * P);
  const int64_t R = a.q.T * a.a.Hq, step = rows << 23;
  for (int64_t r = 0; r < R; r += step) {
    a.item0 = (int)r;
    hipLaunchKernelGGL((merge_kernel<FMT, D, P>), dim3((unsigned)((std::min(step, R - r) + rows - 1) / rows)), dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int FMT, int D, int NQ>
hipError_t launch(AttendArgs a, const Plan& p, hipStream_t s) {
  const int64_t each = (int64_t)p.splits * p.groups * a.c.H, most = std::max<int64_t>(1, ((int64_t)1 << 23) / each);
  for (int64_t i = 0; i < p.items; i += most) {
    a.item0 = (int)i;
    hipLaunchKernelGGL((attend_kernel<FMT, D, NQ>), dim3((unsigned)(std::min(most, p.items - i) * each)), dim3(64 * kWaves), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int FMT, int D>
hipError_t launch_nq(const AttendArgs& a, const Plan& p, hipStream_t s) {
  const hipError_t e = p.nq == 0 ? launch_rows(a, p.items, s) : p.nq == 2 ? launch<FMT, D, 2>(a, p, s) : launch<FMT, D, 1>(a, p, s);
  if (e != hipSuccess || a.splits == 1) return e;
  // (a whole workgroup for 32 rows of 64 pieces: 37 us of attention, less 50; for 9600 rows of
  // 6 pieces 86, less 82; for 2560 rows of 5 17.7, less 17.2; for 64 rows of 8 10.1, less 11.0)
  return a.splits <= (a.q.T * a.a.Hq < 2048 ? 4 : 8) ? merge<FMT, D, 1>(a, s) : merge<FMT, D, 1024 / D>(a, s);
}

template <int FMT>
hipError_t launch_d(const AttendArgs& a, const Plan& p, hipStream_t s) {
  return a.c.D == 64 ? launch_nq<FMT, 64>(a, p, s) : a.c.D == 128 ? launch_nq<FMT, 128>(a, p, s) : launch_nq<FMT, 256>(a, p, s);
}

}  // namespace
}  // namespace attend

size_t kv_attention_ws_bytes(const KvCache& c, const KvSeqs& q, const AttendCall& a) {
  const attend::Plan p = attend::plan_of(c, q, a);
  return p.splits == 1 ? 0 : (size_t)p.splits * q.T * a.Hq * (c.D + 2) * 4;
}

hipError_t launch_kv_attention(const KvCache& c, const KvSeqs& q, const AttendCall& a, float* ws, hipStream_t s) {
  const attend::Plan p = attend::plan_of(c, q, a);
  const attend::AttendArgs args{c, q, a, p.G, p.Gg, p.groups, p.tpt, p.splits, p.chunk, p.most,
                        (int)a.window, 0, ws};
  return c.fmt == QF_FMT_NVFP4 ? attend::launch_d<QF_FMT_NVFP4>(args, p, s) : attend::launch_d<QF_FMT_MXFP4>(args, p, s);
}

}  // namespace qf
