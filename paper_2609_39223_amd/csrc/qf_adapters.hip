// Low-rank adapters of many requests beside a shared projection: Y[m] = base[m] + s_a (x_m A_a^T) B_a^T
// with a = ids[m] (QATFactory Eq. qad-lora's factors, served without merging them).
//
// Two products on v_mfma_f32_16x16x32_bf16: down, z = x A^T, and up, which adds s z B^T to base with s z as two bf16
// halves.  Few rows leave z in FP32 slices of K, which up adds in order; with more rows there are workgroups enough
// without slices, and down leaves the halves themselves.  A workgroup takes one adapter's rows, 16 at a time:
//   up to 64 rows   the z-th adapter among them and the rows that have it (ballots, no memory but the ids);
//   more            16 RB places in the order of the rows' adapters, which a launch of one workgroup makes (a
//                   counting sort in LDS; the places of equal ones do not matter to any result).  Rows of other
//                   adapters among them ride along in the products and are not stored.
// More rows or adapters than the sort takes (2^16, 2^13) are taken as they come.
// Bound by memory: base and Y of many rows (4099 of 6 adapters, rank 32, 4096 x 24576, bf16: 118 us, of them 97 up at
// 4.2 TB/s, 19 down, 7 the order; factors read again by every 32 rows from L2), the factors in use of few (61 of
// 24, rank 64, 4096 x 4096: 16 us, two launches of 8), and launches (16 of 16, rank 16, 4096 x 6144: 9.7 us).  What did not
// pay: a wave that goes over columns with the next ones on their way (186 us for 143 then), base and Y past the caches
// (149, 150, both 156), 16 rows a workgroup for 32 (155).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "qf.h"
#include "qf_codecs.h"
#include "qf_internal.h"

namespace qf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kRankTiles = 4;                // 64 ranks a workgroup of the first product
constexpr int kDownWaves = 8, kUpWaves = 4;
constexpr int kCols = 64;                    // columns of Y a wave takes at a time
constexpr int kFew = 64;                     // rows without an order
constexpr int kSortRows = 1 << 16, kSortAdapters = 1 << 13;

struct RowsArgs {
  AdapterSet s;
  const int32_t* ids;
  int M;
  const uint16_t* X;
  int64_t ldx;
  const void* base;
  int64_t ldb;
  void* Y;
  int64_t ldy;
  float* z;                                  // FP32 [slices, M, r], or bf16 [M, 2, r]: the halves of s z
  int2* order;                               // [M]: row and adapter (-1: none) of each place, or null
  int slices, kc;                            // slices of K, their size
  int abreast;                               // adapters of a group of rows that workgroups take side by side
  int cols;                                  // workgroups of the second product that share a row
  int group0;                                // the launch's first group
};

__device__ __forceinline__ f32x4_t mfma(uint4 a, uint4 b, f32x4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
#else
  return c;
#endif
}

__device__ __forceinline__ int adapter_of(const RowsArgs& p, int row) {
  const int id = p.ids[row];
  return id >= 0 && id < p.s.n ? id : -1;
}
__device__ __forceinline__ int rank_of(const AdapterSet& s, int a) {
  return s.ranks ? min(max(s.ranks[a], 0), s.r) : s.r;
}

// Adds one to the bin of every lane's adapter; returns the bin's count before that lane.  A wave of one adapter (rows
// side by side, as prompts are) adds once: 64 additions to one address come one after the other.
__device__ __forceinline__ int take_place(int* bins, int bin) {
  const int first = __builtin_amdgcn_readfirstlane(bin);
  const uint64_t active = __ballot(true);
  if (__all(bin == first)) {
    const int before = __popcll(active & ((1ull << (threadIdx.x & 63)) - 1));
    int base = 0;
    if (before == 0) base = atomicAdd(&bins[first], __popcll(active));
    return __builtin_amdgcn_readfirstlane(base) + before;
  }
  return atomicAdd(&bins[bin], 1);
}

// The rows in the order of their adapters, those without one last.  One workgroup: counts of the adapters in LDS,
// their prefix sums, then every row takes the next place of its adapter.
__global__ __launch_bounds__(1024) void order_kernel(RowsArgs p) {
  extern __shared__ int count[];             // [n + 1]
  __shared__ int sums[16];
  const int tid = threadIdx.x, lane = tid & 63, n = (int)p.s.n;
  for (int i = tid; i <= n; i += 1024) count[i] = 0;
  __syncthreads();
  for (int m = tid; m < p.M; m += 1024) {
    const int a = adapter_of(p, m);
    take_place(count, a < 0 ? n : a);
  }
  __syncthreads();
  // thread t owns bins t per .. t per + per - 1
  const int per = n / 1024 + 1;
  int mine = 0;
  for (int i = 0; i < per; ++i)
    if (tid * per + i <= n) mine += count[tid * per + i];
  int inc = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(inc, d, 64);
    if (lane >= d) inc += o;
  }
  if (lane == 63) sums[tid >> 6] = inc;
  __syncthreads();
  int at = inc - mine;
  for (int w = 0; w < tid >> 6; ++w) at += sums[w];
  for (int i = 0; i < per; ++i)
    if (tid * per + i <= n) {
      const int c = count[tid * per + i];
      count[tid * per + i] = at;
      at += c;
    }
  __syncthreads();
  for (int m = tid; m < p.M; m += 1024) {
    const int a = adapter_of(p, m);
    p.order[take_place(count, a < 0 ? n : a)] = make_int2(m, a);
  }
}

// Row and adapter (-1: none) of lane % 16 among 16; no row: -1, -1.
struct Group {
  int row, id;
};
__device__ __forceinline__ Group group_at(const RowsArgs& p, int place) {
  const int at = place + (threadIdx.x & 15);
  if (at >= p.M) return {-1, -1};
  if (p.order == nullptr) return {at, adapter_of(p, at)};
  const int2 o = p.order[at];
  return {o.x, o.y};
}
// Bit i: row i of 16 is the first of its adapter.
__device__ __forceinline__ uint32_t firsts_of(const Group& g) {
  uint32_t left = (uint32_t)__ballot(g.id >= 0) & 0xFFFFu, firsts = 0;
  while (left) {
    const int i = __builtin_ctz(left);
    firsts |= 1u << i;
    left &= ~(uint32_t)__ballot(g.id == __builtin_amdgcn_readlane(g.id, i));
  }
  return firsts;
}

// The adapters and rows of up to 64 rows: the z-th adapter, and the rows that have it.
struct Few {
  int id;                                    // of row `lane`
  uint64_t rows;                             // of adapter a
  int a;                                     // -1: there is no z-th adapter
  __device__ __forceinline__ Few(const RowsArgs& p, int z) {
    const int lane = threadIdx.x & 63;
    id = lane < p.M ? adapter_of(p, lane) : -1;
    uint64_t left = __ballot(id >= 0);
    a = -1;
    rows = 0;
    for (int i = 0; left != 0 && i <= z; ++i) {
      const int b = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
      const uint64_t with = __ballot(id == b);
      left &= ~with;
      if (i == z) {
        a = b;
        rows = with;
      }
    }
  }
  // the first 16 rows of those left, which it takes away
  __device__ __forceinline__ Group next() {
    const int lane = threadIdx.x & 63, before = __popcll(rows & ((1ull << lane) - 1)), n = min(__popcll(rows), 16);
    const bool has = (rows >> lane) & 1;
    // row `lane` to lane `before`; the others to lanes behind, which nobody looks at
    const int to = has ? before : 63 - (lane - before);
    const int row = __shfl(__builtin_amdgcn_ds_permute(4 * to, lane), lane & 15, 64);
    const Group g{(lane & 15) < n ? row : -1, (lane & 15) < n ? a : -1};
    for (int i = 0; i < n; ++i) rows &= rows - 1;
    return g;
  }
};

// f as the sum of two bf16 halves: 2^-17 relative; an infinity or NaN in the first.  (Next to the largest float the
// first would round up to an infinity, and the second with it.)
__device__ __forceinline__ void split_halves(float f, uint32_t& hi, uint32_t& lo) {
  hi = codec::bf16_rne(f);
  lo = 0;
  if (!__builtin_isfinite(f)) return;
  if ((hi & 0x7FFFu) == 0x7F80u) --hi;
  lo = codec::bf16_rne(f - codec::as_f32(hi << 16));
}

// Where chunk c (16 bytes of 128) of row r of 16 lies in a wave's LDS: reads of 16 rows' chunks c meet different banks.
__device__ __forceinline__ int chunk_at(int r, int c) { return r * 8 + (c ^ (r & 7)); }
template <int TILES, bool HALVES>
constexpr bool kDownStaged = HALVES && TILES == 2;
// A workgroup's LDS: the waves' operands of 64 k (staged), afterwards their sums.
template <int TILES, bool HALVES>
constexpr int kDownLds = kDownWaves * (kDownStaged<TILES, HALVES> ? (TILES + 1) * 2048 : TILES * 1024);

// z of adapter a's rows among 16; each wave a part of the slice, 128 k at once.  Of many rows and 17 to 32 ranks 128 bytes
// a row are loaded, by eight lanes each, and go through LDS to the lanes that multiply them (staged; 4099 rows of 6
// adapters, rank 32, K 4096: 18.7 us; loaded as they are multiplied, 64 bytes of 16 rows, every line is asked for
// twice: 28.5).  Elsewhere the way through LDS costs more than it saves.  4000 rows, 4096 -> 8192, the whole call in us,
// staged / not:  of 6 adapters, ranks 16, 32, 64, 128, 256:  62 / 59   58 / 68   110 / 101   175 / 149   309 / 238
//                of 200, mixed:                               83 / 73   89 / 94   182 / 158   334 / 281   651 / 539
// (and 61 rows of 24, rank 64, 20.5 / 17.2).
template <int TILES, bool HALVES>
__device__ __forceinline__ void down_rows(const RowsArgs& p, char* smem, const Group& grp, int a, int slice, int j0) {
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int K = (int)p.s.K, k_hi = min((slice + 1) * p.kc, K), per = (p.kc / kDownWaves + 31) / 32 * 32;
  const int w_lo = slice * p.kc + wv * per, w_hi = min(w_lo + per, k_hi), rank = rank_of(p.s, a);
  const uint16_t* const A = p.s.A + (int64_t)a * p.s.r * K;
  f32x4_t acc[TILES];
#pragma unroll
  for (int t = 0; t < TILES; ++t) acc[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  int k0 = w_lo;
  if constexpr (kDownStaged<TILES, HALVES>) {
    constexpr int P = 2;                       // 64 k that are under way at a time
    // operand 0: X's rows, 1 ..: A's; this lane's rows of 128 bytes are lane / 8 and lane / 8 + 8
    const uint16_t* src[TILES + 1][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = (lane >> 3) + 8 * h;
      src[0][h] = p.X + max(__shfl(grp.row, r, 64), 0) * p.ldx + 8 * (lane & 7);
#pragma unroll
      for (int t = 0; t < TILES; ++t) src[t + 1][h] = A + (int64_t)min(j0 + 16 * t + r, p.s.r - 1) * K + 8 * (lane & 7);
    }
    uint4* const stage = reinterpret_cast<uint4*>(smem) + wv * (TILES + 1) * 128;
    // 64 k that lie in LDS
    auto multiply = [&]() {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint4 xv = stage[chunk_at(l16, 4 * u + g)];
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[t] = mfma(xv, stage[(t + 1) * 128 + chunk_at(l16, 4 * u + g)], acc[t]);
      }
    };
    for (; k0 + 64 * P <= w_hi; k0 += 64 * P) {
      uint4 v[P][TILES + 1][2];
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int o = 0; o <= TILES; ++o)
#pragma unroll
          for (int h = 0; h < 2; ++h) v[i][o][h] = *reinterpret_cast<const uint4*>(src[o][h] + k0 + 64 * i);
#pragma unroll
      for (int i = 0; i < P; ++i) {
#pragma unroll
        for (int o = 0; o <= TILES; ++o)
#pragma unroll
          for (int h = 0; h < 2; ++h) stage[o * 128 + chunk_at((lane >> 3) + 8 * h, lane & 7)] = v[i][o][h];
        multiply();
      }
    }
#pragma unroll 1
    for (; k0 < w_hi; k0 += 64) {              // the rest of the wave's part, zeros behind it
#pragma unroll
      for (int o = 0; o <= TILES; ++o)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          stage[o * 128 + chunk_at((lane >> 3) + 8 * h, lane & 7)] =
              k0 + 8 * (lane & 7) < w_hi ? *reinterpret_cast<const uint4*>(src[o][h] + k0) : make_uint4(0, 0, 0, 0);
      multiply();
    }
    __syncthreads();
  } else {
    constexpr int U = 4;
    const uint16_t* const x = p.X + max(grp.row, 0) * p.ldx;
    const uint16_t* f[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) f[t] = A + (int64_t)min(j0 + 16 * t + l16, p.s.r - 1) * K;
    for (; k0 + 32 * U <= w_hi; k0 += 32 * U) {
      uint4 xv[U], av[U][TILES];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k0 + 32 * u + 8 * g;
#pragma unroll
        for (int t = 0; t < TILES; ++t) av[u][t] = *reinterpret_cast<const uint4*>(f[t] + k);
        xv[u] = *reinterpret_cast<const uint4*>(x + k);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int t = 0; t < TILES; ++t) acc[t] = mfma(xv[u], av[u][t], acc[t]);
    }
#pragma unroll 1
    for (; k0 < w_hi; k0 += 32) {            // the rest of the wave's part
      const int k = k0 + 8 * g;
      const uint4 xv = k < w_hi ? *reinterpret_cast<const uint4*>(x + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const uint4 av = k < w_hi ? *reinterpret_cast<const uint4*>(f[t] + k) : make_uint4(0, 0, 0, 0);
        acc[t] = mfma(xv, av, acc[t]);
      }
    }
  }
  f32x4_t(*const part)[kDownWaves][64] = reinterpret_cast<f32x4_t(*)[kDownWaves][64]>(smem);
#pragma unroll
  for (int t = 0; t < TILES; ++t) part[t][wv][lane] = acc[t];
  __syncthreads();
  if (wv < TILES) {                          // tile wv: rows 4 g + k of 16, rank l16
    f32x4_t v = part[wv][0][lane];
#pragma unroll
    for (int w = 1; w < kDownWaves; ++w) v += part[wv][w][lane];
    const int j = j0 + 16 * wv + l16;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = __shfl(grp.row, 4 * g + k, 64), id = __shfl(grp.id, 4 * g + k, 64);
      if (id != a) continue;
      if constexpr (HALVES) {
        if (j >= p.s.r) continue;
        const float f = j < rank ? p.s.scale[a] * v[k] : 0.0f;
        uint32_t hi, lo;
        split_halves(f, hi, lo);
        uint16_t* const to = reinterpret_cast<uint16_t*>(p.z) + (int64_t)row * 2 * p.s.r + j;
        to[0] = (uint16_t)hi;
        to[p.s.r] = (uint16_t)lo;
      } else {
        if (j < rank) p.z[((int64_t)slice * p.M + row) * p.s.r + j] = v[k];
      }
    }
  }
  __syncthreads();
}

// Grid: (16 places and adapter, slice, 64 ranks); FEW: up to 64 rows.
template <int TILES, bool FEW>
__global__ __launch_bounds__(64 * kDownWaves) void down_kernel(RowsArgs p) {
  __shared__ __align__(16) char smem[kDownLds<TILES, !FEW>];
  const int slice = blockIdx.y, j0 = blockIdx.z * 16 * kRankTiles;
  if constexpr (FEW) {
    Few few(p, blockIdx.x);
    while (few.rows) {
      const Group g = few.next();
      down_rows<TILES, false>(p, smem, g, few.a, slice, j0);
    }
  } else {
    const int z0 = blockIdx.x % p.abreast;
    const Group g = group_at(p, (p.group0 + (int)(blockIdx.x / p.abreast)) * 16);
    int i = 0;
    for (uint32_t left = firsts_of(g); left; left &= left - 1, ++i)
      if (i % p.abreast == z0) down_rows<TILES, true>(p, smem, g, __builtin_amdgcn_readlane(g.id, __builtin_ctz(left)), slice, j0);
  }
}

// Eight values of `rank` ranks from j on; those past the rank are zeros.
__device__ __forceinline__ uint4 keep_ranks(uint4 v, int j, int rank) {
  if (j + 8 <= rank) return v;
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (j + 2 * i + 1 >= rank) w[i] &= 0xFFFFu;
    if (j + 2 * i >= rank) w[i] = 0;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Y's (base's) columns 8 by 8: 8 elements at `at`, of which `left` exist.
template <bool F32>
struct Eight {
  uint4 w[F32 ? 2 : 1];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) w[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void load(const void* p, int64_t at, int left) {
    if (F32) {
      const float* const s = static_cast<const float*>(p) + at;
      if (left >= 8) {
        w[0] = *reinterpret_cast<const uint4*>(s);
        w[F32 ? 1 : 0] = *reinterpret_cast<const uint4*>(s + 4);
      } else {
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i < left ? codec::as_u32(s[i]) : 0u;
        w[0] = make_uint4(h[0], h[1], h[2], h[3]);
        w[F32 ? 1 : 0] = make_uint4(h[4], h[5], h[6], h[7]);
      }
    } else {
      const uint16_t* const s = static_cast<const uint16_t*>(p) + at;
      if (left >= 8) {
        w[0] = *reinterpret_cast<const uint4*>(s);
      } else {
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = i < left ? s[i] : 0u;
        w[0] = codec::pack8(h);
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    const uint4 v = w[F32 ? i / 4 : 0];
    const int k = F32 ? i % 4 : i / 2;
    const uint32_t u = k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w;
    return F32 ? codec::as_f32(u) : codec::as_f32(i % 2 ? u & 0xFFFF0000u : u << 16);
  }
  __device__ __forceinline__ void store(void* p, int64_t at, int left, const float v[8]) const {
    if (F32) {
      float* const d = static_cast<float*>(p) + at;
      if (left >= 8) {
        *reinterpret_cast<float4*>(d) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(d + 4) = make_float4(v[4], v[5], v[6], v[7]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < left) d[i] = v[i];
      }
    } else {
      uint16_t* const d = static_cast<uint16_t*>(p) + at;
      // (a NaN keeps its sign and leading bits)
      const uint4 h = make_uint4(codec::bf16x2_rne_nonnan(v[0], v[1]), codec::bf16x2_rne_nonnan(v[2], v[3]),
                                 codec::bf16x2_rne_nonnan(v[4], v[5]), codec::bf16x2_rne_nonnan(v[6], v[7]));
      if (left >= 8) {
        *reinterpret_cast<uint4*>(d) = h;
      } else {
        uint32_t e[8];
        codec::unpack8(h, e);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < left) d[i] = (uint16_t)e[i];
      }
    }
  }
};

// A row of 16 by neighbouring lanes, 8 columns each: lane's rows are lane / 8 and lane / 8 + 8.
__device__ __forceinline__ int row_of(int lane, int half) { return (lane >> 3) + 8 * half; }
constexpr int kRowWords = kCols + 4;         // a row of sums in LDS: four banks further than the one before

// 64 columns from n0 on of adapter a's rows among 16 RB.  The products are taken transposed, the factor's rows n
// against the 16 rows of z, and tile t of a pair holds n = 8 (i / 4) + 4 t + i % 4 in its row i, so that a lane ends up
// with 8 neighbouring columns of row lane % 16.  Of many rows base and Y go by whole lines, 128 bytes a row, and the sums to
// their lanes through LDS (`sums`, the wave's): 4099 x 24576 95 us, 111 with 64 bytes of 16 rows at a time; of few rows
// (HALVES false) that way costs more (61 of 24 adapters 17.1 us for 16.5).
template <bool F32, int STEPS, int RB, bool HALVES>
__device__ __forceinline__ void up_rows(const RowsArgs& p, float* sums, const Group* grp, int a, int n0) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, N = (int)p.s.N, r = p.s.r;
  const int rank = rank_of(p.s, a);
  const uint16_t* const B = p.s.B + (int64_t)a * N * r;
  constexpr bool LINES = HALVES;
  Eight<F32> v[RB][2];
  f32x4_t acc[RB][4];
  auto row_mine = [&](int b, int c) { return LINES ? __shfl(grp[b].row, row_of(lane, c), 64) : grp[b].row; };
  auto id_mine = [&](int b, int c) { return LINES ? __shfl(grp[b].id, row_of(lane, c), 64) : grp[b].id; };
  auto n_mine = [&](int c) { return n0 + (LINES ? 8 * (lane & 7) : 32 * c + 8 * g); };
#pragma unroll
  for (int b = 0; b < RB; ++b) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = row_mine(b, c), id = id_mine(b, c), n = n_mine(c);
      v[b][c].zero();
      if (p.base && id == a && n < N) v[b][c].load(p.base, row * p.ldb + n, N - n);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[b][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {
    if (32 * st >= rank) break;
    const int j = 32 * st + 8 * g;
    uint4 f[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int n = n0 + 32 * (t >> 1) + 8 * (l16 >> 2) + 4 * (t & 1) + (l16 & 3);
      f[t] = make_uint4(0, 0, 0, 0);
      if (j < rank) f[t] = *reinterpret_cast<const uint4*>(B + (int64_t)min(n, N - 1) * r + j);
    }
    uint4 zh[RB], zl[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      zh[b] = zl[b] = make_uint4(0, 0, 0, 0);
      if (!(grp[b].id == a && j < rank)) continue;
      if constexpr (HALVES) {
        const uint16_t* const src = reinterpret_cast<const uint16_t*>(p.z) + (int64_t)grp[b].row * 2 * r + j;
        zh[b] = *reinterpret_cast<const uint4*>(src);
        zl[b] = *reinterpret_cast<const uint4*>(src + r);
      } else {
        const float s = p.s.scale[a];
        const float* src = p.z + (int64_t)grp[b].row * r + j;
        float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
        for (int sl = 0; sl < p.slices; ++sl) {
          const float4 lo = *reinterpret_cast<const float4*>(src), hi = *reinterpret_cast<const float4*>(src + 4);
          src += (int64_t)p.M * r;
          z[0] += lo.x; z[1] += lo.y; z[2] += lo.z; z[3] += lo.w;
          z[4] += hi.x; z[5] += hi.y; z[6] += hi.z; z[7] += hi.w;
        }
        uint32_t hi[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)          // (ranks past the last hold what lay there: not used)
          split_halves(j + i < rank ? s * z[i] : 0.0f, hi[i], lo[i]);
        zh[b] = codec::pack8(hi);
        zl[b] = codec::pack8(lo);
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint4 fr = keep_ranks(f[t], j, rank);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        acc[b][t] = mfma(fr, zh[b], acc[b][t]);
        acc[b][t] = mfma(fr, zl[b], acc[b][t]);
      }
    }
  }
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    if constexpr (LINES) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        *reinterpret_cast<f32x4_t*>(sums + l16 * kRowWords + 32 * (t >> 1) + 8 * g + 4 * (t & 1)) = acc[b][t];
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = row_mine(b, c), id = id_mine(b, c), n = n_mine(c);
      f32x4_t s0 = acc[b][2 * c], s1 = acc[b][2 * c + 1];
      if constexpr (LINES) {
        const float* const from = sums + row_of(lane, c) * kRowWords + 8 * (lane & 7);
        s0 = *reinterpret_cast<const f32x4_t*>(from);
        s1 = *reinterpret_cast<const f32x4_t*>(from + 4);
      }
      if (id != a || n >= N) continue;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = v[b][c].get(i) + (i < 4 ? s0[i & 3] : s1[i & 3]);
      v[b][c].store(p.Y, row * p.ldy + n, N - n, y);
    }
  }
}

// Rows without an adapter: row of lane % 16, -1: none.
template <bool F32>
__device__ __forceinline__ void copy_rows(const RowsArgs& p, int rows, int n0) {
  if (p.base == p.Y) return;
  const int lane = threadIdx.x & 63, N = (int)p.s.N, n = n0 + 8 * (lane & 7);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int row = __shfl(rows, row_of(lane, c), 64);
    if (row < 0 || n >= N) continue;
    Eight<F32> v;
    v.zero();
    if (p.base) v.load(p.base, row * p.ldb + n, N - n);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = v.get(i);
    v.store(p.Y, row * p.ldy + n, N - n, y);
  }
}

// Workgroups: (16 RB places and adapter, 256 columns), columns first (rows first, the workgroups at work at one
// time write to the same columns of many rows, and 4099 x 24576 took 155 us in all for 143); RB 0: up to 64 rows,
// the workgroups past their adapters the rows without one.
template <bool F32, int STEPS, int RB>
__global__ __launch_bounds__(64 * kUpWaves) void up_kernel(RowsArgs p) {
  const uint32_t bx = blockIdx.x / (uint32_t)p.cols;
  const int n0 = ((int)(blockIdx.x % (uint32_t)p.cols) * kUpWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kCols;
  __shared__ __align__(16) float all_sums[RB > 0 ? kUpWaves : 1][RB > 0 ? 16 * kRowWords : 4];
  float* const sums = all_sums[RB > 0 ? threadIdx.x >> 6 : 0];
  if (n0 >= p.s.N) return;
  if constexpr (RB == 0) {
    const int z0 = (int)bx;
    Few few(p, z0 < p.abreast ? z0 : 0);
    if (z0 < p.abreast) {
      while (few.rows) {
        const Group g = few.next();
        up_rows<F32, STEPS, 1, false>(p, sums, &g, few.a, n0);
      }
    } else {                                 // (the rows without an adapter as if they had one)
      few.rows = __ballot((int)(threadIdx.x & 63) < p.M && few.id < 0);
      while (few.rows) copy_rows<F32>(p, few.next().row, n0);
    }
  } else {
    const int place = (p.group0 + (int)bx / p.abreast) * 16 * RB, z0 = (int)bx % p.abreast;
    Group grp[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) grp[b] = group_at(p, place + 16 * b);
    if constexpr (RB > 1) {
      const int a = __builtin_amdgcn_readfirstlane(grp[0].id);
      bool one = a >= 0;
#pragma unroll
      for (int b = 0; b < RB; ++b) one = one && (grp[b].id == a || grp[b].row < 0);
      if (__all(one)) {
        up_rows<F32, STEPS, RB, true>(p, sums, grp, a, n0);
        return;
      }
    }
#pragma unroll 1
    for (int b = 0; b < RB; ++b) {
      const Group g = RB == 1 ? grp[0] : group_at(p, place + 16 * b);
      if (z0 == 0) copy_rows<F32>(p, g.id < 0 ? g.row : -1, n0);
      int i = 0;
      for (uint32_t left = firsts_of(g); left; left &= left - 1, ++i)
        if (i % p.abreast == z0) up_rows<F32, STEPS, 1, true>(p, sums, &g, __builtin_amdgcn_readlane(g.id, __builtin_ctz(left)), n0);
    }
  }
}

// ------------------------------------------------------------------------------ the launch rules
struct Plan {
  int rb;                                    // 16 rows a workgroup takes at once; 0: up to 64 rows
  int64_t groups;
  int abreast, slices, kc;
  bool sorted;
};
Plan plan_of(const AdapterSet& s, int64_t M) {
  Plan p;
  const int64_t n = std::max<int64_t>(1, std::min(M, s.n)), cus = compute_units();
  p.sorted = M > kFew && M <= kSortRows && s.n <= kSortAdapters;
  p.rb = M <= kFew ? 0 : M / n >= 64 ? 2 : 1;
  p.groups = p.rb == 0 ? 1 : (M + 16 * p.rb - 1) / (16 * p.rb);
  // adapters among 16 sorted rows, one more than there would be if every group began with a new one, side by side, unless
  // there are workgroups enough without the last, which few groups need.  Rank 16, 4096 -> 8192, us with / without it:
  // 100 rows of 10 adapters 17 / 26, 1000 of 30 25 / 33, 2048 of 6 32 / 39, of 100 37 / 42, 2900 of 6 43 / 44,
  // of 100 59 / 56, 4099 of 6 62 / 59, of 100 75 / 70.  n counts the adapters that are there, not those in use
  // (which only the device knows).
  p.abreast = p.rb == 0 ? (int)n : (int)std::min<int64_t>({16, n, 1 + (16 * n + (M < 12 * cus ? M - 1 : 0)) / M});
  const int64_t each = p.groups * p.abreast, want = (2 * cus + each - 1) / each;
  // slices of K for few rows, 1024 each (61 rows, K 4096, us by slices of 4096 / 2048 / 1024 / 512 / 256: 26.6 / 20.0 /
  // 16.3 / 17.2 / 20.8), 16 at most (one row, K 16384, 1 / 2 / 4 / 8 / 16: 69 / 40 / 26 / 20 / 19)
  const int64_t slices = p.rb ? 1 : std::min(want, std::min<int64_t>(std::max<int64_t>(1, s.K / 1024), 16));
  p.kc = (int)((std::max<int64_t>(s.K, 1) + slices - 1) / slices + 255) / 256 * 256;
  p.slices = (int)std::max<int64_t>(1, (s.K + p.kc - 1) / p.kc);
  return p;
}

size_t z_bytes(const AdapterSet& s, int64_t M, const Plan& p) { return ((size_t)p.slices * M * s.r * 4 + 255) / 256 * 256; }

template <int TILES>
void launch_down(const RowsArgs& a, int rb, dim3 grid, hipStream_t s) {
  const dim3 block(64 * kDownWaves);
  if (rb == 0) hipLaunchKernelGGL((down_kernel<TILES, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((down_kernel<TILES, false>), grid, block, 0, s, a);
}
template <bool F32, int STEPS>
void launch_up(const RowsArgs& a, int rb, dim3 grid, hipStream_t s) {
  const dim3 block(64 * kUpWaves);
  if (rb == 0) hipLaunchKernelGGL((up_kernel<F32, STEPS, 0>), grid, block, 0, s, a);
  else if (rb == 1) hipLaunchKernelGGL((up_kernel<F32, STEPS, 1>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((up_kernel<F32, STEPS, 2>), grid, block, 0, s, a);
}
template <bool F32>
void launch_up(const RowsArgs& a, int rb, dim3 grid, hipStream_t s) {
  const int steps = (a.s.r + 31) / 32;
  if (steps <= 1) launch_up<F32, 1>(a, rb, grid, s);
  else if (steps <= 2) launch_up<F32, 2>(a, rb, grid, s);
  else if (steps <= 4) launch_up<F32, 4>(a, rb, grid, s);
  else launch_up<F32, 8>(a, rb, grid, s);
}

}  // namespace

size_t lora_rows_ws_bytes(const AdapterSet& s, int64_t M) {
  const Plan p = plan_of(s, M);
  return z_bytes(s, M, p) + (p.sorted ? (size_t)M * 8 : 0);
}

hipError_t launch_lora_rows(const AdapterSet& s, const int32_t* ids, int64_t M, const uint16_t* X, int64_t ldx,
                            const void* base, int64_t ldb, void* Y, int64_t ldy, int y_f32, float* ws,
                            hipStream_t stream) {
  const Plan p = plan_of(s, M);
  const int64_t cols = (s.N + kUpWaves * kCols - 1) / (kUpWaves * kCols);
  int2* const order = p.sorted ? reinterpret_cast<int2*>(reinterpret_cast<char*>(ws) + z_bytes(s, M, p)) : nullptr;
  // (no adapters, or nothing to sum: the products are zeros)
  RowsArgs a{s, ids, (int)M, X, ldx, base, ldb, Y, ldy, ws, order, s.K > 0 ? p.slices : 0, p.kc, p.abreast, (int)cols, 0};
  if (order) {
    hipLaunchKernelGGL(order_kernel, dim3(1), dim3(1024), (size_t)(s.n + 1) * 4, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const unsigned ranks = (unsigned)((s.r + 16 * kRankTiles - 1) / (16 * kRankTiles));
  // a grid has fewer than 2^32 lanes
  const int64_t wide = std::max<int64_t>(cols, 2 * p.slices * ranks * std::max(p.rb, 1));
  const int64_t fit = std::max<int64_t>(1, ((int64_t)1 << 22) / (wide * p.abreast));
  for (int64_t g = 0; g < p.groups; g += fit) {
    const unsigned groups = (unsigned)std::min(fit, p.groups - g), x = groups * (unsigned)p.abreast;
    a.abreast = p.abreast;
    if (s.n > 0 && (s.K > 0 || p.rb > 0)) {  // (the halves of no sum are zeros)
      a.group0 = (int)(g * std::max(p.rb, 1));
      const dim3 grid(x * (unsigned)std::max(p.rb, 1), (unsigned)p.slices, ranks);
      if (s.r <= 16) launch_down<1>(a, p.rb, grid, stream);
      else if (s.r <= 32) launch_down<2>(a, p.rb, grid, stream);
      else launch_down<4>(a, p.rb, grid, stream);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    a.group0 = (int)g;
    if (p.rb == 2) a.abreast = 1;            // (groups of one adapter nearly all)
    const dim3 grid((unsigned)((p.rb == 0 ? x + 1 : groups * (unsigned)a.abreast) * cols));
    if (y_f32) launch_up<true>(a, p.rb, grid, stream);
    else launch_up<false>(a, p.rb, grid, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace qf
