// Low-rank adapters of many requests beside a shared projection: Y[m] = base[m] + s_a (x_m A_a^T) B_a^T
// with a = ids[m] (QATFactory Eq. qad-lora's factors, served without merging them).
//
// Two launches on v_mfma_f32_16x16x32_bf16: down, z = x A^T (FP32, in slices of K), and up, which adds the
// slices in order, splits s z into two bf16 halves and adds z B^T to base.  A workgroup takes 16 rows and one
// of the adapters that occur among them: rows of other adapters ride along in the products and are not
// stored, so rows may lie in any order, and an adapter is read once per 16 rows that use it.
// Bound by memory: the factors of the adapters in use (few rows), base and Y (many).
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

constexpr int kWaves = 4, kRankTiles = 4;    // 64 ranks a workgroup of the first product
constexpr int kCols = 64;                    // columns of Y a wave takes at a time

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
  float* z;                                  // [slices, M, r]
  int slices, kc;                            // slices of K, their size
  int abreast;                               // adapters of 16 rows that workgroups take side by side
  int block0;                                // the launch's first 16 rows
};

__device__ __forceinline__ f32x4_t mfma(uint4 a, uint4 b, f32x4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
#else
  return c;
#endif
}

// The adapters among 16 rows, by the rows' order: `id` of lane % 16's row (-1: none), bit i of `firsts`: row i
// is the first of its adapter.
struct Group {
  int id;
  uint32_t firsts, with;
};
__device__ __forceinline__ Group group_of(const RowsArgs& p, int block) {
  const int row = block * 16 + (threadIdx.x & 15);
  Group g;
  g.id = row < p.M ? p.ids[row] : -1;
  if (g.id < 0 || g.id >= p.s.n) g.id = -1;
  uint32_t same = 0;
#pragma unroll
  for (int i = 15; i >= 0; --i)
    if (__builtin_amdgcn_readlane(g.id, i) == g.id) same = i;
  g.with = (uint32_t)__ballot(g.id >= 0) & 0xFFFFu;
  g.firsts = (uint32_t)__ballot(g.id >= 0 && same == (threadIdx.x & 15)) & 0xFFFFu;
  return g;
}
__device__ __forceinline__ int drop_firsts(uint32_t firsts, int n) {   // without the n lowest bits
  while (n-- > 0) firsts &= firsts - 1;
  return (int)firsts;
}
__device__ __forceinline__ int rank_of(const AdapterSet& s, int a) {
  return s.ranks ? min(max(s.ranks[a], 0), s.r) : s.r;
}

// z[slice][row][j] of the rows of adapter after adapter.  Grid: (16 rows, adapter, slice, 64 ranks).
__global__ __launch_bounds__(64 * kWaves) void down_kernel(RowsArgs p) {
  __shared__ f32x4_t part[kWaves][kRankTiles][64];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, l16 = lane & 15, g = lane >> 4;
  const int block = p.block0 + blockIdx.x / p.abreast, slice = blockIdx.y, j0 = blockIdx.z * 16 * kRankTiles;
  const Group grp = group_of(p, block);
  const int row = min(block * 16 + l16, p.M - 1);
  // a wave's quarter of the slice, in steps of 32
  const int K = (int)p.s.K, k_lo = slice * p.kc, k_hi = min(k_lo + p.kc, K);
  const int per = (p.kc / kWaves + 31) / 32 * 32, w_lo = k_lo + wv * per, w_hi = min(w_lo + per, k_hi);
  const uint16_t* const x = p.X + row * p.ldx;
  for (uint32_t left = drop_firsts(grp.firsts, blockIdx.x % p.abreast); left; left = drop_firsts(left, p.abreast)) {
    const int a = __builtin_amdgcn_readlane(grp.id, __builtin_ctz(left));
    const int rank = rank_of(p.s, a), tiles = min((rank - j0 + 15) / 16, kRankTiles);
    const uint16_t* f[kRankTiles];
#pragma unroll
    for (int t = 0; t < kRankTiles; ++t) f[t] = p.s.A + ((int64_t)a * p.s.r + min(j0 + 16 * t + l16, p.s.r - 1)) * K;
    f32x4_t acc[kRankTiles];
#pragma unroll
    for (int t = 0; t < kRankTiles; ++t) acc[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = w_lo; k0 < w_hi; k0 += 32) {
      const int k = k0 + 8 * g;
      uint4 xv = make_uint4(0, 0, 0, 0);
      if (k < w_hi) xv = *reinterpret_cast<const uint4*>(x + k);
#pragma unroll
      for (int t = 0; t < kRankTiles; ++t)
        if (t < tiles) {
          uint4 av = make_uint4(0, 0, 0, 0);
          if (k < w_hi) av = *reinterpret_cast<const uint4*>(f[t] + k);
          acc[t] = mfma(xv, av, acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < kRankTiles; ++t) part[wv][t][lane] = acc[t];
    __syncthreads();
    if (wv < tiles) {                        // wave t finishes tile t: rows 4 g + i, rank l16
      const uint32_t mine = (uint32_t)__ballot(grp.id == a);
      f32x4_t v = part[0][wv][lane];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v += part[w][wv][lane];
      const int j = j0 + 16 * wv + l16;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j < rank && ((mine >> (4 * g + i)) & 1u))
          p.z[((int64_t)slice * p.M + block * 16 + 4 * g + i) * p.s.r + j] = v[i];
    }
    __syncthreads();
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

// Y's columns 8 by 8: loads and stores of 8 elements at column n (fewer at the end).
template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t at, int left, float v[8]) {
  if (F32) {
    const float* const s = static_cast<const float*>(p) + at;
    if (left >= 8) {
      const float4 a = *reinterpret_cast<const float4*>(s), b = *reinterpret_cast<const float4*>(s + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? s[i] : 0.0f;
    }
  } else {
    const uint16_t* const s = static_cast<const uint16_t*>(p) + at;
    uint32_t h[8];
    if (left >= 8) {
      codec::unpack8(*reinterpret_cast<const uint4*>(s), h);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = i < left ? s[i] : 0u;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = codec::as_f32(h[i] << 16);
  }
}
template <bool F32>
__device__ __forceinline__ void store8(void* p, int64_t at, int left, const float v[8]) {
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
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = codec::bf16_rne(v[i]);
    if (left >= 8) {
      *reinterpret_cast<uint4*>(d) = codec::pack8(h);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) d[i] = (uint16_t)h[i];
    }
  }
}

// Grid: (16 rows and adapter, 256 columns).  The products are taken transposed, the factor's rows n against
// the 16 rows of z, and tile t of a pair holds n = 8 (i / 4) + 4 t + i % 4 in its row i, so that a lane ends
// up with 8 neighbouring columns of its row.
template <bool F32, int STEPS>
__global__ __launch_bounds__(64 * kWaves) void up_kernel(RowsArgs p) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, l16 = lane & 15, g = lane >> 4;
  const int block = p.block0 + blockIdx.x / p.abreast, z0 = blockIdx.x % p.abreast;
  const Group grp = group_of(p, block);
  const int n0 = ((int)blockIdx.y * kWaves + wv) * kCols, N = (int)p.s.N, r = p.s.r;
  if (n0 >= N) return;
  const int row = block * 16 + l16;
  if (z0 == 0 && grp.id < 0 && row < p.M && p.base != p.Y) {          // rows without an adapter
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int n = n0 + 32 * c + 8 * g;
      if (n >= N) break;
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (p.base) load8<F32>(p.base, row * p.ldb + n, N - n, v);
      store8<F32>(p.Y, row * p.ldy + n, N - n, v);
    }
  }
  for (uint32_t left = drop_firsts(grp.firsts, z0); left; left = drop_firsts(left, p.abreast)) {
    const int a = __builtin_amdgcn_readlane(grp.id, __builtin_ctz(left));
    const int rank = rank_of(p.s, a);
    const float s = p.s.scale[a];
    const bool mine = grp.id == a;
    float v[2][8];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = 0.0f;
      const int n = n0 + 32 * c + 8 * g;
      if (p.base && mine && n < N) load8<F32>(p.base, row * p.ldb + n, N - n, v[c]);
    }
    f32x4_t acc[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) acc[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int st = 0; st < STEPS; ++st) {
      const int j = 32 * st + 8 * g;
      if (32 * st >= rank) break;
      float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (mine && j < rank) {
        for (int sl = 0; sl < p.slices; ++sl) {
          const float* const src = p.z + ((int64_t)sl * p.M + row) * r + j;
          const float4 lo = *reinterpret_cast<const float4*>(src), hi = *reinterpret_cast<const float4*>(src + 4);
          z[0] += lo.x; z[1] += lo.y; z[2] += lo.z; z[3] += lo.w;
          z[4] += hi.x; z[5] += hi.y; z[6] += hi.z; z[7] += hi.w;
        }
      }
      uint32_t hi[8], lo[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {          // (ranks past the last hold what lay there: not used)
        const float f = j + i < rank ? s * z[i] : 0.0f;
        hi[i] = codec::bf16_rne(f);
        const float rest = f - codec::as_f32(hi[i] << 16);
        lo[i] = __builtin_isfinite(f) ? codec::bf16_rne(rest) : 0u;
      }
      const uint4 zh = codec::pack8(hi), zl = codec::pack8(lo);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int n = n0 + 32 * (t >> 1) + 8 * (l16 >> 2) + 4 * (t & 1) + (l16 & 3);
        uint4 b = make_uint4(0, 0, 0, 0);
        if (j < rank) b = keep_ranks(*reinterpret_cast<const uint4*>(p.s.B + ((int64_t)a * N + min(n, N - 1)) * r + j), j, rank);
        acc[t] = mfma(b, zh, acc[t]);
        acc[t] = mfma(b, zl, acc[t]);
      }
    }
    if (mine) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int n = n0 + 32 * c + 8 * g;
        if (n >= N) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] += acc[2 * c + (i >> 2)][i & 3];
        store8<F32>(p.Y, row * p.ldy + n, N - n, v[c]);
      }
    }
  }
}

// ------------------------------------------------------------------------------ the launch rules
struct Plan {
  int slices, kc, abreast;
};
Plan plan_of(const AdapterSet& s, int64_t M) {
  Plan p;
  const int64_t blocks = (M + 15) / 16;
  // few rows: an adapter a workgroup; many: one after the other, where a block's rows mostly share one
  p.abreast = M <= 256 ? (int)std::min<int64_t>(16, std::max<int64_t>(1, std::min(M, s.n))) : 1;
  const int64_t want = (2 * compute_units() + blocks * p.abreast - 1) / std::max<int64_t>(1, blocks * p.abreast);
  const int64_t most = std::max<int64_t>(1, (s.K + 511) / 512);
  const int64_t slices = std::min(std::max<int64_t>(want, 1), std::min<int64_t>(most, 16));
  p.kc = (int)((std::max<int64_t>(s.K, 1) + slices - 1) / slices + 127) / 128 * 128;
  p.slices = (int)std::max<int64_t>(1, (s.K + p.kc - 1) / p.kc);
  return p;
}

template <bool F32>
void launch_up(const RowsArgs& a, dim3 grid, hipStream_t s) {
  const int steps = (a.s.r + 31) / 32;
  if (steps <= 1) hipLaunchKernelGGL((up_kernel<F32, 1>), grid, dim3(64 * kWaves), 0, s, a);
  else if (steps <= 2) hipLaunchKernelGGL((up_kernel<F32, 2>), grid, dim3(64 * kWaves), 0, s, a);
  else if (steps <= 4) hipLaunchKernelGGL((up_kernel<F32, 4>), grid, dim3(64 * kWaves), 0, s, a);
  else hipLaunchKernelGGL((up_kernel<F32, 8>), grid, dim3(64 * kWaves), 0, s, a);
}

}  // namespace

size_t lora_rows_ws_bytes(const AdapterSet& s, int64_t M) {
  return (size_t)plan_of(s, M).slices * M * s.r * 4;
}

hipError_t launch_lora_rows(const AdapterSet& s, const int32_t* ids, int64_t M, const uint16_t* X, int64_t ldx,
                            const void* base, int64_t ldb, void* Y, int64_t ldy, int y_f32, float* ws,
                            hipStream_t stream) {
  const Plan p = plan_of(s, M);
  // (no adapters, or nothing to sum: the products are zeros)
  RowsArgs a{s, ids, (int)M, X, ldx, base, ldb, Y, ldy, ws, s.K > 0 ? p.slices : 0, p.kc, p.abreast, 0};
  const int64_t blocks = (M + 15) / 16;
  const unsigned cols = (unsigned)((s.N + kWaves * kCols - 1) / (kWaves * kCols));
  const unsigned ranks = (unsigned)((s.r + 16 * kRankTiles - 1) / (16 * kRankTiles));
  // a grid has fewer than 2^32 lanes, and at most 65535 workgroups along y
  const int64_t fit = std::max<int64_t>(1, ((int64_t)1 << 23) / ((int64_t)std::max(std::min(cols, 65535u), p.slices * ranks) * p.abreast));
  for (int64_t b = 0; b < blocks; b += fit) {
    a.block0 = (int)b;
    const unsigned x = (unsigned)(std::min(fit, blocks - b) * p.abreast);
    if (s.n > 0 && s.K > 0) {
      hipLaunchKernelGGL(down_kernel, dim3(x, (unsigned)p.slices, ranks), dim3(64 * kWaves), 0, stream, a);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    if (y_f32) launch_up<true>(a, dim3(x, cols), stream);
    else launch_up<false>(a, dim3(x, cols), stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace qf
