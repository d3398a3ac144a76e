// Attention over the 4-bit cache: what its kernels share (qf_attend.hip says how they work).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qf.h"
#include "qf_codecs.h"
#include "qf_internal.h"
#include "qf_kv.h"

#define QF_LDS(T, p) ((__attribute__((address_space(3))) T*)(p))

namespace qf {
namespace attend {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int v2i_t __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4, kTile = 64;       // waves of a workgroup, tokens of a step
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kUp = 14.0f;                 // probabilities are held 2^14 times as large

struct AttendArgs {
  KvCache c;
  KvSeqs q;
  AttendCall a;
  int G, Gg, groups;                         // queries' heads to a cache head, of them in a row tile
  int tpt;                                   // tokens in a row tile
  int splits, chunk;                         // pieces a row tile's tokens may have, their size
  int most, window;                          // positions from `most` on are not looked at
  int item0;
  float* part;                               // [splits, T Hq, D], then (m, l) [splits, T Hq, 2]
};

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// The sequence of row tile `item` and the tile's index in it: tiles of sequence b are those from
// off[b] / tpt + b on, which leaves one too many at most.  Every wave finds it by itself, 64 steps at a
// time.  False if the tile does not exist.
__device__ __forceinline__ bool find_tile(const KvSeqs& q, int tpt, int item, int& b, int& tok0, int& first, int& n) {
  if (q.off == nullptr) {
    b = tok0 = item;
    first = 0;
    n = 1;
    return item < q.B;
  }
  const int lane = threadIdx.x & 63;
  auto off = [&](int i) { return (int)min(max(q.off[i], (int64_t)0), q.T); };
  int lo = 0, hi = (int)q.B;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const bool below = i < hi && off(i) / tpt + i <= item;
    const int k = __popcll(__ballot(below));
    if (k == 0) return false;
    lo += (k - 1) * step;
    hi = min(lo + step, hi);
  }
  b = __builtin_amdgcn_readfirstlane(lo);
  const int o = __builtin_amdgcn_readfirstlane(off(b));
  n = __builtin_amdgcn_readfirstlane(off(b + 1)) - o;
  first = (item - (o / tpt + b)) * tpt;
  tok0 = o + first;
  return b < q.B && first >= 0 && first < n;
}

// The positions [lo, hi) that any row of a tile sees; lo is a multiple of 16.
struct Reach {
  int lo, hi;
};
__device__ __forceinline__ Reach reach_of(const AttendArgs& p, int len, int pos0, int pos1) {
  Reach r;
  r.hi = min(min(pos1 + 1, len), p.most);
  r.lo = p.window > 0 ? max(pos0 - p.window + 1, 0) & ~15 : 0;
  return r;
}
__device__ __forceinline__ int live_pieces(const Reach& r, int chunk) {
  return r.hi > r.lo ? (r.hi - r.lo - 1) / chunk + 1 : 0;
}

// The maximum and sum of a row's piece in the workspace, behind the pieces' outputs.
__device__ __forceinline__ f32x2_t& row_sums(const AttendArgs& p, int split, int64_t row, int D) {
  const int64_t R = p.q.T * p.a.Hq;
  return *reinterpret_cast<f32x2_t*>(p.part + p.splits * R * D + (split * R + row) * 2);
}

template <int FMT>
__device__ __forceinline__ f32x4_t mfma_z(uint4 a, uint4 b, f32x4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (FMT == QF_FMT_NVFP4)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
#else
  return c;
#endif
}
__device__ __forceinline__ f32x4_t mfma_o(uint4 a, uint4 b, f32x4_t c) {
  return mfma_z<QF_FMT_NVFP4>(a, b, c);
}

// Eight codes as FP16, pairs times the scale pairs s[0..3].
__device__ __forceinline__ uint4 decode_f16(uint32_t cw, const f16x2_t s[4]) {
#if defined(__HIP_DEVICE_COMPILE__)
  const f16x2_t v0 = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(cw, 1.0f, 0)) * s[0];
  const f16x2_t v1 = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(cw, 1.0f, 1)) * s[1];
  const f16x2_t v2 = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(cw, 1.0f, 2)) * s[2];
  const f16x2_t v3 = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(cw, 1.0f, 3)) * s[3];
  return make_uint4(__builtin_bit_cast(uint32_t, v0), __builtin_bit_cast(uint32_t, v1), __builtin_bit_cast(uint32_t, v2),
                    __builtin_bit_cast(uint32_t, v3));
#else
  return make_uint4(0, 0, 0, 0);
#endif
}
// The E4M3 values of the low two bytes of w.
__device__ __forceinline__ f16x2_t e4m3_f16(uint32_t w) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_bit_cast(f16x2_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false));
#else
  return f16x2_t{};
#endif
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2_t));
}

// Scale codes of V that the products do not take.
template <int FMT>
__device__ __forceinline__ bool is_special(uint32_t e) {
  return FMT == QF_FMT_NVFP4 ? (e & 0x7Fu) == 0x7Fu : e != 0u && (e < 107u || e > 134u);
}

// What one lane holds of 64 tokens on their way in: a quarter of the bytes of 4 x 16 tokens.
template <int FMT, int D>
struct Tile {
  static constexpr int W = D / 32;           // words of codes of a token's quarter
  static constexpr int KS = FMT == QF_FMT_NVFP4 ? D / 64 : D == 256 ? 2 : 1;     // scale bytes of it
  static constexpr int VS = FMT == QF_FMT_NVFP4 ? D / 16 : D / 32;               // scale bytes of a token
  uint32_t k[4][W], ks[4], vs[4];
};

// A wave's address p and a lane's offset, left apart: the load takes one from scalar and the other from vector
// registers (as one 64-bit address a lane they cost additions and twice the registers).
typedef const __attribute__((address_space(1))) uint8_t global_byte;
__device__ __forceinline__ global_byte* lane_at(const uint8_t* p, uint32_t offset) {
  global_byte* g = (global_byte*)p;
#if defined(__HIP_DEVICE_COMPILE__)
  const uint64_t v = (uint64_t)p;
  g = (global_byte*)((uint64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v));
  asm volatile("" : "+s"(g), "+v"(offset));
#endif
  return g + offset;
}
template <class U>
__device__ __forceinline__ U load_as(global_byte* p) {
  return *(const __attribute__((address_space(1))) U*)p;
}

template <int W>
__device__ __forceinline__ void load_words(global_byte* p, uint32_t* w) {
  typedef uint32_t words __attribute__((ext_vector_type(W < 4 ? W : 4)));
#pragma unroll
  for (int i = 0; i < W; i += 4) {
    const words x = load_as<words>(p + 4 * i);
#pragma unroll
    for (int k = 0; k < (W < 4 ? W : 4); ++k) w[i + k] = x[k];
  }
}

// V's codes in LDS: row r (16 u + 4 g + i) of D / 2 bytes, its 16-byte chunk c at c ^ v_swap(r).  A transposed
// read takes 8 bytes of 16 rows, four consecutive ones of each u: with the chunks exchanged by u (and, where
// four rows pass 256 bytes, by i) they lie on different banks (D = 64: on half as many as there are).
template <int D>
__device__ __forceinline__ int v_swap(int r) {
  const int u = r >> 4;
  return D == 64 ? u & 1 : D == 128 ? u : u ^ ((r & 2) << 1);
}

// A copy from memory to LDS: the 16 bytes at p + offset of lane i go to l + 16 i (p, l and `bytes`, what may be read from p
// on, are the wave's).  (The global form, without a resource, makes the compiler wait for it before any LDS access.)
__device__ __forceinline__ void copy16(const uint8_t* p, uint32_t bytes, uint32_t offset, char* l) {
#if defined(__HIP_DEVICE_COMPILE__)
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, (int)bytes, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)l, 16, (int)offset, 0, 0, 0);
#endif
}
// V's codes of the 16 tokens at p, tokens 16 u .. of a tile, to LDS: rows back to back, chunks exchanged.
template <int D>
__device__ __forceinline__ void copy_values(const uint8_t* p, int u, int lane, char* to) {
  constexpr int C = D / 32, R = 64 / C;                 // chunks of a row, rows a copy
#pragma unroll
  for (int i = 0; i < (16 + R - 1) / R; ++i) {
    const int r = i * R + lane / C;
    if (R <= 16 || lane < 16 * C)
      copy16(p, 16 * (D / 2), r * (D / 2) + 16 * ((lane % C) ^ v_swap<D>(16 * u + r)), to + (16 * u + i * R) * (D / 2));
  }
}

// A row of Q as the products take it, lane group g's quarter of D, and the factor that brings its scores to units of
// log 2: positive and finite, so that hidden scores stay -inf.  A row with an infinity or NaN, or whose factor would be
// one, gets NaNs and the factor 1: its scores are NaN where it sees a token, and nowhere else.
template <int FMT, int D>
__device__ __forceinline__ float load_query(const AttendArgs& p, int row_at, int g, float S_k, uint4 (&q)[D / 32]) {
  constexpr int CS = D / 32;
  const uint32_t flip = (p.a.scale < 0.0f) != (S_k < 0.0f) ? 0x80008000u : 0u;
  const int t = row_at / (int)p.a.Hq, hq = row_at - t * (int)p.a.Hq;
  const uint16_t* const src = p.a.Q + t * p.a.ldq + (int64_t)hq * D + g * (D / 4);
  uint32_t top = 0;
#pragma unroll
  for (int s = 0; s < CS; ++s) {
    q[s] = *reinterpret_cast<const uint4*>(src + 8 * s);
    uint32_t w[8];
    codec::unpack8(q[s], w);
    top = max(top, codec::max_abs_bits8(w));
    q[s] = make_uint4(q[s].x ^ flip, q[s].y ^ flip, q[s].z ^ flip, q[s].w ^ flip);
  }
  top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
  const int e = (int)(top >> 7) - 127 - 14;             // (zeros and subnormals: any factor will do)
#pragma unroll
  for (int s = 0; s < CS; ++s) {
    const uint32_t w[4] = {q[s].x, q[s].y, q[s].z, q[s].w};
    uint32_t o[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float lo = __builtin_ldexpf(codec::as_f32(w[k] << 16), -e), hi = __builtin_ldexpf(codec::as_f32(w[k] & 0xFFFF0000u), -e);
      o[k] = FMT == QF_FMT_NVFP4 ? pack_f16(lo, hi) : codec::bf16x2_rne_nonnan(lo, hi);
    }
    q[s] = make_uint4(o[0], o[1], o[2], o[3]);
  }
  // (mantissas and exponents apart: scale S_k alone may be out of range or have few bits left)
#if defined(__HIP_DEVICE_COMPILE__)
  const float a = __builtin_amdgcn_frexp_mantf(p.a.scale) * __builtin_amdgcn_frexp_mantf(S_k);
  const int ea = __builtin_amdgcn_frexp_expf(p.a.scale) + __builtin_amdgcn_frexp_expf(S_k);
#else
  const float a = 0.0f;
  const int ea = 0;
#endif
  const float f = __builtin_ldexpf(__builtin_fabsf(a) * kLog2e, e + ea);
  const bool nan = top >= 0x7F80u || !__builtin_isfinite(f);
  q[0].x = nan ? (FMT == QF_FMT_NVFP4 ? 0x7E007E00u : 0x7FC07FC0u) : q[0].x;
  return nan ? 1.0f : f < 0x1p-126f ? 0x1p-126f : f;
}

// Step s of 16 tokens' keys as the A operand: codes cw, the scale bytes ks of the lane's quarter of D.
template <int FMT>
__device__ __forceinline__ uint4 decode_key(uint32_t cw, uint32_t ks, int s) {
  if constexpr (FMT == QF_FMT_NVFP4) {
    const f16x2_t v = e4m3_f16(ks >> (8 * (s >> 2 << 1)));   // scales of 32 elements
    const f16x2_t q2 = (s >> 1) & 1 ? f16x2_t{v[1], v[1]} : f16x2_t{v[0], v[0]}, q4[4] = {q2, q2, q2, q2};
    return decode_f16(cw, q4);
  } else {
    uint32_t w[4];
    codec::fp4_decode8(cw, codec::e8m0_scale((ks >> (8 * (s >> 2))) & 0xFFu), w);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// Bit r: token r of 16 has a NaN scale (MXFP4; under NVFP4 the decoded key is NaN by itself).
template <int FMT, int KS>
__device__ __forceinline__ uint32_t nan_keys(uint32_t ks) {
  if constexpr (FMT == QF_FMT_NVFP4) return 0;
  const uint64_t all = __ballot((ks & 0xFFu) == 0xFFu || (KS == 2 && (ks >> 8) == 0xFFu));
  return (uint32_t)(all | (all >> 16) | (all >> 32) | (all >> 48)) & 0xFFFFu;
}

// Scale bytes of V of a token's quarter, to FP16 in the order in which the products take them: token 16 u + 4 gg + k lies
// at 4 u + k of the lanes of group gg.  True if one of them is special (and was taken as zero).
template <int FMT, int KS>
__device__ __forceinline__ bool store_scales(uint32_t sv, int block, int u, int lane, _Float16* vscale) {
  bool special = false;
#pragma unroll
  for (int k = 0; k < KS; ++k)
    if (is_special<FMT>((sv >> (8 * k)) & 0xFFu)) {
      sv &= ~(0xFFu << (8 * k));
      special = true;
    }
  _Float16* const to = vscale + (block * 4 + (lane >> 4)) * 16 + 4 * u + ((lane >> 2) & 3);
#pragma unroll
  for (int k = 0; k < KS; k += 2) {
    uint32_t w;
    if constexpr (FMT == QF_FMT_NVFP4) {
      w = __builtin_bit_cast(uint32_t, e4m3_f16(sv >> (8 * k)));
    } else {                                            // 2^(e - 127 + 6): exponent field e - 106
      const uint32_t lo = (sv >> (8 * k)) & 0xFFu, hi = (sv >> (8 * k + 8)) & 0xFFu;
      w = (lo ? (lo - 106u) << 10 : 0u) | (hi ? (hi - 106u) << 26 : 0u);
    }
    to[k * 64] = __builtin_bit_cast(f16x2_t, w)[0];
    if (k + 1 < KS) to[k * 64 + 64] = __builtin_bit_cast(f16x2_t, w)[1];
  }
  return special;
}

// Tile d of V^T over 64 tokens, its two A operands, from their codes (rows as v_swap lays them) and scales in LDS.
template <int FMT, int D>
__device__ __forceinline__ void decode_values(const char* codes, const _Float16* vscale, int d, int lane, uint4& v0, uint4& v1) {
  const int l16 = lane & 15, g = lane >> 4, rr = 16 * (l16 >> 2) + 4 * g + (l16 & 3);
  const char* const from = codes + rr * (D / 2) + 8 * (d ^ (v_swap<D>(rr) << 1));
#if defined(__HIP_DEVICE_COMPILE__)
  const v2i_t cw = __builtin_amdgcn_ds_read_tr4_b64_v2i32(QF_LDS(v2i_t, const_cast<char*>(from)));
#else
  const v2i_t cw = {};
  (void)from;
#endif
  const uint4* const sp = reinterpret_cast<const uint4*>(vscale + ((FMT == QF_FMT_NVFP4 ? d : d >> 1) * 4 + g) * 16);
  const uint4 sa = sp[0], sb = sp[1];
  const f16x2_t s0[4] = {__builtin_bit_cast(f16x2_t, sa.x), __builtin_bit_cast(f16x2_t, sa.y),
                         __builtin_bit_cast(f16x2_t, sa.z), __builtin_bit_cast(f16x2_t, sa.w)};
  const f16x2_t s1[4] = {__builtin_bit_cast(f16x2_t, sb.x), __builtin_bit_cast(f16x2_t, sb.y),
                         __builtin_bit_cast(f16x2_t, sb.z), __builtin_bit_cast(f16x2_t, sb.w)};
  v0 = decode_f16((uint32_t)cw[0], s0);
  v1 = decode_f16((uint32_t)cw[1], s1);
}

// The largest of the four lanes that hold one row: 16 and 32 lanes apart, exchanged without LDS.
__device__ __forceinline__ float row_max(float x) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t v = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  x = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  const uint32_t w = __builtin_bit_cast(uint32_t, x);
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  x = fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
#endif
  return x;
}

// One step of the rows' running softmax over the tile's 64 tokens, of which the lane holds scores z of 16 u + 4 g + i: a
// row sees those from `from` to below `to` that have a page (whole: no lane has to look).  Probabilities go to pw in FP16.
// (All rows' maxima first, then one branch: taken one row after the other each waits for its own exchanges.)
// A row whose reference m is kFar or more from zero rounds its scores first, as the reference was, and then takes the
// difference, which is exact: 14 - m is not exact there, and the reference is off the largest score's exact product
// by more than FP16 has room for.  It goes by the row's own reference, so that equal scores count the same in every
// tile.  `far`: some row of the wave is one.  (One branch for all rows: one for each kept their exponents apart, 363 us for 350.)
constexpr float kFar = 0x1p22f;
__device__ __forceinline__ bool is_far(float m) { return __builtin_fabsf(m) >= kFar && m != neg_inf(); }
template <int DT, int NQ>
__device__ __forceinline__ void softmax_step(float (&z)[NQ][16], const float (&cz)[NQ], const int (&from)[NQ], const int (&to)[NQ],
                                             bool whole, uint32_t bad, int g, float (&m)[NQ], float (&l)[NQ], f32x4_t (&acc)[NQ][DT],
                                             uint32_t (&pw)[NQ][8], int& far) {
  bool all = whole;
#pragma unroll
  for (int j = 0; j < NQ; ++j) all = all && to[j] >= kTile && from[j] <= 0;
  if (!__all(all)) {
#pragma unroll
    for (int j = 0; j < NQ; ++j)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int t = 16 * (i >> 2) + 4 * g + (i & 3);
        if (t < from[j] || t >= to[j] || ((bad >> (i >> 2)) & 1u)) z[j][i] = neg_inf();
      }
  }
  float top[NQ];
  bool grows = false;
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    top[j] = z[j][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top[j] = fmaxf(top[j], z[j][i]);
    // The reference is a whole number, so that adding it to 14 and powers of two of it are exact.  It may lag behind the
    // largest by one (probabilities up to 2^15): fewer steps have to scale what was
    // summed (355 -> 350 us for 2048 new tokens behind 8192).
    top[j] = fmaxf(__builtin_ceilf(row_max(top[j]) * cz[j]), m[j]);
    grows = grows || top[j] - m[j] > 1.0f;              // (m + 1 may round up to m + 2)
  }
  if (__any(grows)) {
    bool any = false;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
      const float down = __builtin_amdgcn_exp2f(m[j] - (top[j] == neg_inf() ? 0.0f : top[j]));
      l[j] *= down;
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[j][d] *= down;
      m[j] = top[j];
      any = any || is_far(m[j]);
    }
    far = __builtin_amdgcn_readfirstlane(__any(any));
  }
  float by[NQ], up[NQ];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    by[j] = cz[j];
    up[j] = m[j] == neg_inf() ? 0.0f : kUp - m[j];      // (nothing seen yet: probabilities of zero)
  }
  if (__builtin_expect(far, 0)) {
#pragma unroll
    for (int j = 0; j < NQ; ++j)
      if (is_far(m[j])) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[j][i] = z[j][i] * by[j] - m[j];
        up[j] = kUp;
        by[j] = 1.0f;
      }
  }
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j][i], by[j], up[j]));
      const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j][i + 1], by[j], up[j]));
      sum[0] += a;
      sum[1] += b;
      pw[j][i / 2] = pack_f16(a, b);
    }
    l[j] += sum[0] + sum[1];
  }
}

// The special blocks of token r of the tile's 16 u .. added in FP32: scales sp and codes of the token, this lane's two
// bytes of tile d at codes + 8 (d ^ swap).
template <int FMT, int D, int NQ, class Codes>
__device__ __forceinline__ void add_special(const AttendArgs& p, const uint8_t* sp, Codes codes, int u, int r, int pos, int l16,
                                            const uint32_t (&pw)[NQ][8], const int (&row_pos)[NQ], f32x4_t (&acc)[NQ][D / 16]) {
  const int i = 4 * u + (r & 3);                        // its place among the probabilities of group r / 4
  float pr[NQ];
  bool sees[NQ];
#pragma unroll
  for (int j = 0; j < NQ; ++j) {
    uint32_t w = pw[j][0];
#pragma unroll
    for (int k = 1; k < 8; ++k) w = i >> 1 == k ? pw[j][k] : w;
    w = (uint32_t)__shfl((int)w, 16 * (r >> 2) + l16, 64);
    pr[j] = (float)__builtin_bit_cast(f16x2_t, w >> (16 * (i & 1)))[0];
    sees[j] = pos <= row_pos[j] && (p.window <= 0 || pos > row_pos[j] - p.window);
  }
#pragma unroll
  for (int d = 0; d < D / 16; ++d) {
    const uint32_t sc = sp[FMT == QF_FMT_NVFP4 ? d : d >> 1];
    if (!is_special<FMT>(sc)) continue;
    const uint32_t four = codes(d);
    float f;
    if constexpr (FMT == QF_FMT_NVFP4) f = __builtin_nanf("");
    else f = sc == 0xFFu ? __builtin_nanf("") : __builtin_ldexpf(1.0f, (int)sc - 127 + 6);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t code = (four >> (4 * k)) & 15u;
      const float v = codec::e2m1_value(code & 7u) * f;
#pragma unroll
      for (int j = 0; j < NQ; ++j)
        if (sees[j]) acc[j][d][k] = __builtin_fmaf(pr[j], code & 8u ? -v : v, acc[j][d][k]);
    }
  }
}

// A row's sums: the output, or, of several pieces, this one's part of it.
template <int FMT, int D>
__device__ __forceinline__ void emit_row(const AttendArgs& p, int split, int row_at, int h, int g, const f32x4_t (&acc)[D / 16],
                                         float m, float l) {
  if (p.splits > 1) {
    float* const to = p.part + ((int64_t)split * (p.q.T * p.a.Hq) + row_at) * D + 4 * g;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f32x4_t*>(to + 16 * d) = acc[d];
    if (g == 0) row_sums(p, split, row_at, D) = f32x2_t{m, l};
    return;
  }
  const float f = 1.0f / l, S = FMT == QF_FMT_NVFP4 ? p.c.S[1][h] : 0x1p-6f;   // (S / l may have few bits left)
  const int t = row_at / (int)p.a.Hq;
  uint16_t* const to = p.a.O + t * p.a.ldo + (int64_t)(row_at - t * (int)p.a.Hq) * D + 4 * g;
#pragma unroll
  for (int d = 0; d < D / 16; ++d) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = codec::bf16_rne(l == 0.0f ? 0.0f : acc[d][k] * f * S);
    *reinterpret_cast<uint2*>(to + 16 * d) = make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
  }
  if (p.a.lse && g == 0) p.a.lse[row_at] = l == 0.0f ? neg_inf() : (m + (__builtin_log2f(l) - kUp)) * kLn2;
}

// Sequences with many new tokens (qf_attend_rows.hip): 128 rows a workgroup.
constexpr int kManyRows = 128;
hipError_t launch_rows(const AttendArgs& a, int64_t items, hipStream_t s);

}  // namespace attend
}  // namespace qf
