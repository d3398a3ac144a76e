// Products of few rows with packed weights (QATFactory Sec. 3.4, 3.5: the weights an engine serves),
// dense or per expert: Y = X W^T with W decoded in registers on its way to the matrix cores.
//
// A workgroup takes 16 NT weight rows against up to 16 rows of X, its waves take slices of 512 k in
// turn, and their FP32 partial sums meet in LDS in wave order.  A slice's codes and X rows go straight
// from memory to LDS, each wave into a region of its own, so nothing but the final sum waits for
// another wave, and no registers are held while the copies are under way: the 16 to 24 waves that a
// compute unit's registers hold wait for 4 to 5 KB of codes each.  Copies are contiguous (256 bytes of
// four rows per instruction) where loads in the shape of the matrix operand, 16 bytes of 16 rows, kept
// the L1's address port busy four times as long (24576 x 4096 NVFP4 times one row: 18.2 us with such
// loads, 14.3 with copies, the decode as it was).  A 16-byte chunk c of row r lies at c ^ r of its row
// in LDS, so the operand reads, the same chunk of 16 rows, fall on different banks.
//
// On v_mfma_f32_16x16x32_bf16 X is the A operand (lane: row lane % 16, k 8 (lane / 16) + 0..7) and W
// the B operand (lane: weight row lane % 16, the same k); any bijection of k is fine as long as both
// sides use it: lane group g = lane / 16 takes k 128 g .. 128 g + 127 of a slice, so the scales of a
// lane's codes are consecutive bytes too (8 or 4, loaded into registers).
//   NVFP4  V s is exact in bf16 (E2M1 has 2 significant bits, E4M3 4; 2^-10 <= |V s| <= 2688), so the
//          block scale goes into the operand and the tensor scale S onto the finished sum.
//   MXFP4  V 2^p is exact in bf16.
//   Q4_K   a sub-block of 32 is one MFMA deep.  16 + q is exact in bf16 and made from a code by a shift
//          and a mask; with X1 = -16 sum x from one MFMA as the next one's addend, P = sum (16 + q) x
//          + X1 = sum q x, and a super-block adds d sum s6 P + (dmin / 16) sum m6 X1.  (Sums of s6 x and
//          m6 x on the matrix cores instead of vector operations: 13.0 -> 14.1 us, 14336 x 4096, five rows.)
//          These sums are taken 2^-18 times as large, d and dmin 2^18 times: a super-block's are at most
//          2^18 max |x| before that, so no finite x makes them infinite.  What is lost are bits below
//          2^-149 of the scaled sums, which matter where all |x| are below 2^-108.
// Bound by reading the weight once, 0.53 to 0.56 bytes an element (NVFP4, 24576 x 4096, one row: 56.7
// MB in 12.3 us = 4.6 TB/s; the copies alone take 11.2), Q4_K by its decode, which is that of 16 rows
// whatever their number (14336 x 4096, five rows: 13.1 us, 9.9 without the arithmetic; one row 12.1).  Small
// weights are bound by the launch and one trip to memory (4096 x 4096: 5.0 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "qf.h"
#include "qf_codecs.h"
#include "qf_internal.h"
#include "qf_matvec_plan.h"

#define QF_LDS(p) ((__attribute__((address_space(3))) void*)(p))
#define QF_GLOBAL(p) ((__attribute__((address_space(1))) void*)(p))

namespace qf {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4_t mfma16(uint4 a, uint4 b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                 __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// Copies from memory to LDS: lane l's 16 (4) bytes at g go to l + 16 (4) lane.  The non-temporal form
// leaves the caches to others.
__device__ __forceinline__ void copy16(const void* g, void* l) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(QF_GLOBAL(const_cast<void*>(g)), QF_LDS(l), 16, 0, 0);
#endif
}
__device__ __forceinline__ void copy16_nt(const void* g, void* l) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(QF_GLOBAL(const_cast<void*>(g)), QF_LDS(l), 16, 0, 2);
#endif
}
__device__ __forceinline__ void copy4(const void* g, void* l) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_global_load_lds(QF_GLOBAL(const_cast<void*>(g)), QF_LDS(l), 4, 0, 0);
#endif
}

// v_mfma_f32_4x4x4_16b_bf16: sixteen products of 4 x 4 x 4, block b = lane / 4.  A: row lane % 4, four k;
// B: column lane % 4, four k; C: column lane % 4, the four rows.
typedef short s16x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f32x4_t mfma4(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(s16x4_t, make_uint2(a0, a1)),
                                                __builtin_bit_cast(s16x4_t, make_uint2(b0, b1)), c, 0, 0, 0);
}

struct MatvecArgs {
  PackedOperand w;
  const uint16_t* X;
  int64_t ldx, M;
  void* Y;
  int64_t ldy, R;
  int y_f32;
  const int64_t* off;     // null: dense
  const int32_t* rows;
  int rows_div;
  int xmax;               // rows of X a workgroup takes at most (1 .. 16)
  int xrows;              // rows of X that lie in LDS at once: xmax, or 8 of 16
  int waves;              // waves that share a tile's slices
  int item0;              // experts: the launch's first row group
};

// The X row of row r of Y, -1 if there is none.
__device__ __forceinline__ int64_t x_row(const MatvecArgs& p, int64_t r) {
  int64_t x = r;
  if (p.rows) x = p.rows[r] < 0 ? -1 : p.rows[r] / p.rows_div;
  return x < p.M ? x : -1;
}

// Work item `item` of a grouped call: expert e and its rows [r0, r1), at most `chunk`; items count
// the experts' chunks in order.  Every wave finds it by itself: lane l sums the chunks of its experts
// (offsets cut to 0 .. R < 2^30), a prefix sum over the lanes finds whose the item is.  False past
// the last one; [r0, r1) lies in 0 .. R and is not empty whatever the offsets are.
__device__ __forceinline__ bool find_item(const int64_t* off, int E, int64_t R, int item, int chunk,
                                          int& e, int64_t& r0, int64_t& r1) {
  const int lane = threadIdx.x & 63, per = (E + 63) / 64, e0 = lane * per;
  auto at = [&](int i) { return (int)min(max(off[i < E ? i : E], (int64_t)0), R); };
  auto chunks = [&](int a, int b) { return b > a ? (b - a + chunk - 1) / chunk : 0; };
  int sum = 0, o0 = 0, o1 = 0, o2 = 0;
  if (per <= 2) {                                 // the usual case: three loads at once
    o0 = at(e0);
    o1 = at(e0 + 1);
    o2 = at(e0 + per);
    sum = chunks(o0, o1) + chunks(o1, o2);
  } else {
    for (int i = 0; i < per; ++i) sum += chunks(at(e0 + i), at(e0 + i + 1));
  }
  int inc = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(inc, d, 64);
    if (lane >= d) inc += o;
  }
  if (item >= __builtin_amdgcn_readlane(inc, 63)) return false;
  const int owner = __ffsll((unsigned long long)__ballot(inc > item)) - 1;
  int left = item - (inc - sum), i = 0;           // meaningful in the owner
  if (per <= 2) {
    if (left >= chunks(o0, o1)) {
      left -= chunks(o0, o1);
      i = 1;
      o0 = o1;
      o1 = o2;
    }
  } else {
    for (; i < per; ++i) {
      o0 = at(e0 + i);
      o1 = at(e0 + i + 1);
      if (left < chunks(o0, o1)) break;
      left -= chunks(o0, o1);
    }
  }
  const int lo = o0 + left * chunk;
  e = __builtin_amdgcn_readlane(e0 + i, owner);
  r0 = __builtin_amdgcn_readlane(lo, owner);
  r1 = __builtin_amdgcn_readlane(min(lo + chunk, o1), owner);
  return r0 >= 0 && r0 < r1;                      // (offsets that fall can overflow the sums)
}

// ------------------------------------------------------------------------------- the formats
// Copies of 16 code rows (row i at base + min(i, last) pitch) of slice sl into l, in whole 64-lane
// instructions; lanes with nothing to fetch fetch something that exists.  FP4: 16 rows of 256 bytes,
// chunks exchanged as above; rows 8-byte aligned (K = 16 modulo 32) go in words.  Q4_K: two
// super-blocks a row as they lie (16 rows of 288 bytes: rows 8 banks apart); `half`: only one is left.
template <int FMT, int COPY>
__device__ __forceinline__ void copy_codes(const uint8_t* base, int64_t pitch, int last, int sl,
                                           bool half, char* l) {
  const int lane = threadIdx.x & 63;
  if (FMT == QF_FMT_Q4K) {
#pragma unroll
    for (int j = 0; j < 5; ++j) {
      const int i = j * 64 + lane, row = i / 18 < 15 ? i / 18 : 15, c = half ? i % 18 % 9 : i % 18;
      const uint8_t* const g = base + (row < last ? row : last) * pitch + (int64_t)sl * 288 + 16 * c;
      if (COPY == kCopyNt) copy16_nt(g, l + j * 1024);
      else copy16(g, l + j * 1024);
    }
  } else if (COPY == kCopyWords) {
#pragma unroll 4
    for (int row = 0; row < 16; ++row)
      copy4(base + (row < last ? row : last) * pitch + (int64_t)sl * 256 + 16 * ((lane >> 2) ^ row) + 4 * (lane & 3),
            l + row * 256);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = 4 * j + (lane >> 4);
      const uint8_t* const g = base + (row < last ? row : last) * pitch + (int64_t)sl * 256 + 16 * ((lane & 15) ^ row);
      if (COPY == kCopyNt) copy16_nt(g, l + j * 1024);
      else copy16(g, l + j * 1024);
    }
  }
}

// The scale bytes of this lane's 128 codes in slice sl (NVFP4 8, MXFP4 4), at any address.
struct Bytes8 { uint8_t b[8]; };
struct Bytes4 { uint8_t b[4]; };
template <int FMT>
__device__ __forceinline__ uint2 load_scales(const uint8_t* sp, int sl) {
  if (FMT == QF_FMT_NVFP4) return __builtin_bit_cast(uint2, *reinterpret_cast<const Bytes8*>(sp + (int64_t)sl * 32));
  if (FMT == QF_FMT_MXFP4)
    return make_uint2(__builtin_bit_cast(uint32_t, *reinterpret_cast<const Bytes4*>(sp + (int64_t)sl * 16)), 0u);
  return make_uint2(0u, 0u);
}

// The B operand of 8 codes: V s (NVFP4, s FP32) or V 2^p (MXFP4, e the E8M0 code).
__device__ __forceinline__ uint4 decode_nvfp4(uint32_t cw, float s) {
  uint32_t w[4];
  codec::nvfp4_decode8_finite(cw, s, w);     // exact: nothing is rounded (a NaN scale stays NaN)
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 decode_mxfp4(uint32_t cw, uint32_t e) {
  uint32_t w[4];
  codec::mxfp4_decode8(cw, e, w);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// 32 codes under their scale bytes s (NVFP4: two, MXFP4: one; low bytes).
template <int FMT>
__device__ __forceinline__ void multiply32(const uint4& c, uint32_t s, const uint4 x[4], f32x4_t& acc) {
  const uint32_t cw[4] = {c.x, c.y, c.z, c.w};
  const auto sf = __builtin_amdgcn_cvt_pk_f32_fp8((int)s, false);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 b = FMT == QF_FMT_NVFP4 ? decode_nvfp4(cw[i], i < 2 ? sf[0] : sf[1]) : decode_mxfp4(cw[i], s & 0xFFu);
    acc = mfma16(x[i], b, acc);
  }
}

// The same for NVFP4 and at most four rows of X, on 4 x 4 x 4 blocks: a lane's columns are its own, so
// the sixteen products of a scale block come out by themselves and the scale goes onto their sum, one
// multiplication a row instead of one a weight (2.06 vector operations a weight -> 0.6 to 0.8; 24576 x
// 4096, one row: 14.2 -> 12.1 us).
__device__ __forceinline__ void multiply32_small(const uint4& c, uint32_t s, const uint4 x[4], f32x4_t& acc) {
  const uint32_t cw[4] = {c.x, c.y, c.z, c.w};
  const auto sf = __builtin_amdgcn_cvt_pk_f32_fp8((int)s, false);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4_t p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 2 * h; i < 2 * h + 2; ++i) {
      uint32_t w[4];
      codec::fp4_decode8(cw[i], 1.0f, w);
      p = mfma4(x[i].x, x[i].y, w[0], w[1], p);
      p = mfma4(x[i].z, x[i].w, w[2], w[3], p);
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) acc[m] = __builtin_fmaf(sf[h], p[m], acc[m]);
  }
}

// Two bf16 values 2^-18 (16 + q) of the codes in the low (HIGH: high) nibbles of bytes 0 and 2 of w.
template <bool HIGH>
__device__ __forceinline__ uint32_t q4k_pair(uint32_t w) {
  return ((HIGH ? w >> 1 : w << 3) & 0x00780078u) | 0x38803880u;
}
// One super-block of this lane's weight row (144 bytes at `row`) against the X row at xl (chunks of 8
// exchanged by xw, the super-block's first chunk c0).
__device__ __forceinline__ void q4k_superblock(const char* row, const char* xl, int xw, int c0, int g,
                                               f32x4_t& acc) {
  const uint4 head = *reinterpret_cast<const uint4*>(row);
  const float d = codec::f16_value(head.x & 0xFFFFu) * 0x1p18f, dm = codec::f16_value(head.x >> 16) * 0x1p14f;
  const uint32_t s6[2] = {head.y & 0x3F3F3F3Fu, (head.w & 0x0F0F0F0Fu) | ((head.y >> 2) & 0x30303030u)};
  const uint32_t m6[2] = {head.z & 0x3F3F3F3Fu, ((head.w >> 4) & 0x0F0F0F0Fu) | ((head.z >> 2) & 0x30303030u)};
  const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
  const uint4 minus16 = make_uint4(0xB880B880u, 0xB880B880u, 0xB880B880u, 0xB880B880u);
  f32x4_t ps = zero, pm = zero;
#pragma unroll
  for (int c = 0; c < 4; ++c) {                   // sub-blocks 2 c (low nibbles) and 2 c + 1
    const uint2 w = *reinterpret_cast<const uint2*>(row + 16 + 32 * c + 8 * g);
    const uint32_t t[4] = {__builtin_amdgcn_perm(0u, w.x, 0x0C010C00u), __builtin_amdgcn_perm(0u, w.x, 0x0C030C02u),
                           __builtin_amdgcn_perm(0u, w.y, 0x0C010C00u), __builtin_amdgcn_perm(0u, w.y, 0x0C030C02u)};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int j = 2 * c + h;
      const uint4 b = h == 0 ? make_uint4(q4k_pair<false>(t[0]), q4k_pair<false>(t[1]), q4k_pair<false>(t[2]), q4k_pair<false>(t[3]))
                             : make_uint4(q4k_pair<true>(t[0]), q4k_pair<true>(t[1]), q4k_pair<true>(t[2]), q4k_pair<true>(t[3]));
      const uint4 a = *reinterpret_cast<const uint4*>(xl + 16 * ((c0 + 4 * j + g) ^ xw));
      const float fs = (float)((s6[j / 4] >> (8 * (j % 4))) & 0xFFu), fm = (float)((m6[j / 4] >> (8 * (j % 4))) & 0xFFu);
      const f32x4_t x1 = mfma16(a, minus16, zero), pr = mfma16(a, b, x1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ps[i] = __builtin_fmaf(fs, pr[i], ps[i]);
        pm[i] = __builtin_fmaf(fm, x1[i], pm[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) acc[i] = __builtin_fmaf(dm, pm[i], __builtin_fmaf(d, ps[i], acc[i]));
}

// -------------------------------------------------------------------------------- the kernel
// Rows of X.  kSmall: xmax <= 4 and NVFP4 (multiply32_small); A operand rows are then lane % 4, and the
// four lane groups hold partial sums of their own k.  kTwice: up to 16 rows through LDS for 8: lanes
// 0 .. 7 of each 16 take their operands of the whole slice into registers, then the other rows are
// copied there; codes are copied and decoded once for all 16 where LDS for 16 rows would cost waves.
// (Twice the registers, 160: a variant of its own.)
template <int FMT, int NT, int COPY, int ROWS>
__global__ __launch_bounds__(64 * kMatvecMaxWaves) void matvec_kernel(MatvecArgs p) {
  extern __shared__ __align__(256) char smem[];
  constexpr int CB = matvec_code_bytes(FMT);
  constexpr bool SMALL = ROWS == kSmall;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int N = (int)p.w.N, K = (int)p.w.K;
  const int tiles = (N + 16 * NT - 1) / (16 * NT);
  const int item = (int)(blockIdx.x / tiles), n0 = (int)(blockIdx.x % tiles) * 16 * NT;
  int e = 0;
  int64_t r0 = (int64_t)item * p.xmax, r1 = min(r0 + p.xmax, p.R);
  if (p.off != nullptr && !find_item(p.off, (int)p.w.E, p.R, p.item0 + item, p.xmax, e, r0, r1)) return;
  const int xn = (int)(r1 - r0);
  // lane l16 knows X row l16 of the group; a row that does not exist reads row 0, and zeros are stored
  const int64_t xrow = l16 < xn ? x_row(p, r0 + l16) : -1;
  const int xlo = xrow < 0 ? 0 : (int)xrow;
  char* const mine = smem + wv * (NT * CB + p.xrows * 1024);
  char* const xs = mine + NT * CB;
  const int am = SMALL ? lane & 3 : l16;          // A operand row
  const int mr = am < xn ? am : xn - 1;           // rows past the last repeat it and are not stored
  const char* const xl = xs + mr * 1024;
  const int64_t pitch = FMT == QF_FMT_Q4K ? (int64_t)(K / 256) * 144 : K / 2;
  const int64_t spitch = FMT == QF_FMT_NVFP4 ? K / 16 : K / 32;
  const uint8_t* const codes = p.w.codes + ((int64_t)e * N + n0) * pitch;
  const int last = N - 1 - n0;                    // weight rows past N repeat the last, not stored
  const uint8_t* const scales = p.w.scales + ((int64_t)e * N + n0) * spitch;
  const uint8_t* sp[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int row = 16 * t + l16;
    sp[t] = scales + (row < last ? row : last) * spitch;
  }
  f32x4_t acc[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) acc[t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

  const int whole = FMT == QF_FMT_Q4K ? (K + 511) / 512 : K / 512;
  for (int sl = wv; sl < whole; sl += p.waves) {
    const bool half = FMT == QF_FMT_Q4K && K - sl * 512 < 512;
    uint2 s[NT];
    const int first = min(xn, p.xrows);
    for (int m = 0; m < first; ++m) {
      const int c = lane ^ m;
      copy16(p.X + (int64_t)__builtin_amdgcn_readlane(xlo, m) * p.ldx + sl * 512 + 8 * (half ? c & 31 : c), xs + m * 1024);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int rest = last - 16 * t;             // (below zero: the tile is past N, its rows the last one)
      copy_codes<FMT, COPY>(codes + (int64_t)(rest < 0 ? last : 16 * t) * pitch, pitch, rest < 0 ? 0 : rest, sl,
                            half, mine + t * CB);
    }
    asm volatile("" ::: "memory");                // the codes first: they are what takes long
#pragma unroll
    for (int t = 0; t < NT; ++t) s[t] = load_scales<FMT>(sp[t] + g * (FMT == QF_FMT_NVFP4 ? 8 : 4), sl);
    __builtin_amdgcn_s_waitcnt(0x0F70);           // vmcnt(0): this wave's copies are in its region
    asm volatile("" ::: "memory");
    if constexpr (FMT == QF_FMT_Q4K) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const char* const row = mine + t * CB + l16 * 288;
        q4k_superblock(row, xl, mr, 0, g, acc[t]);
        if (!half) q4k_superblock(row + 144, xl, mr, 32, g, acc[t]);
      }
    } else if (ROWS == kTwice && xn > 8) {
      uint4 x[4][4];
      const char* const xa = xs + (l16 & 7) * 1024;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        x[i >> 2][i & 3] = *reinterpret_cast<const uint4*>(xa + 16 * ((16 * g + i) ^ (l16 & 7)));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      for (int m = 8; m < xn; ++m)
        copy16(p.X + (int64_t)__builtin_amdgcn_readlane(xlo, m) * p.ldx + sl * 512 + 8 * (lane ^ (m - 8)),
               xs + (m - 8) * 1024);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0F70);
      asm volatile("" ::: "memory");
      if (l16 >= 8) {
#pragma unroll
        for (int i = 0; i < 16; ++i)             // (past row xn: what lay there, in rows that are not stored)
          x[i >> 2][i & 3] = *reinterpret_cast<const uint4*>(xa + 16 * ((16 * g + i) ^ (l16 & 7)));
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint4 c = *reinterpret_cast<const uint4*>(mine + t * CB + l16 * 256 + 16 * ((4 * g + q) ^ l16));
          const uint32_t sv = FMT == QF_FMT_NVFP4 ? (q < 2 ? s[t].x : s[t].y) >> (16 * (q & 1)) : s[t].x >> (8 * q);
          multiply32<FMT>(c, sv, x[q], acc[t]);
        }
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)               // (rows 0 .. 3 exchange chunks of four: one address for all q)
          x[i] = *reinterpret_cast<const uint4*>(SMALL ? xl + 256 * g + 16 * (i ^ mr) + 64 * q
                                                       : xl + 16 * ((16 * g + 4 * q + i) ^ mr));
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint4 c = *reinterpret_cast<const uint4*>(mine + t * CB + l16 * 256 + 16 * ((4 * g + q) ^ l16));
          const uint32_t sv = FMT == QF_FMT_NVFP4 ? (q < 2 ? s[t].x : s[t].y) >> (16 * (q & 1)) : s[t].x >> (8 * q);
          if constexpr (SMALL) multiply32_small(c, sv, x, acc[t]);
          else multiply32<FMT>(c, sv, x, acc[t]);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the next copies land
  }
  if constexpr (FMT != QF_FMT_Q4K) {
    // the k past the last whole slice, 128 at a time by the waves whose turn it is, 16 at a time per
    // lane and straight from memory: nothing past K is read
    const uint16_t* const xp = p.X + (int64_t)__shfl(xlo, mr, 64) * p.ldx;
    for (int k1 = whole * 512, turn = whole % p.waves; k1 < K; k1 += 128, turn = turn + 1 == p.waves ? 0 : turn + 1) {
      if (turn != wv) continue;
      const int k = k1 + 32 * g;
      uint4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = make_uint4(0, 0, 0, 0);
        if (k + 8 * i < K) x[i] = *reinterpret_cast<const uint4*>(xp + k + 8 * i);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int row = 16 * t + l16;
        const uint8_t* const cp = codes + (row < last ? row : last) * pitch + k / 2;
        uint4 c = make_uint4(0, 0, 0, 0);
        uint32_t s = 0;
        if (k < K) {
          const uint2 v = *reinterpret_cast<const uint2*>(cp);
          c.x = v.x;
          c.y = v.y;
          s = sp[t][FMT == QF_FMT_NVFP4 ? k / 16 : k / 32];
        }
        if (k + 16 < K) {
          const uint2 v = *reinterpret_cast<const uint2*>(cp + 8);
          c.z = v.x;
          c.w = v.y;
          if (FMT == QF_FMT_NVFP4) s |= (uint32_t)sp[t][k / 16 + 1] << 8;
        }
        if constexpr (SMALL) multiply32_small(c, s, x, acc[t]);
        else multiply32<FMT>(c, s, x, acc[t]);
      }
    }
  }

  __syncthreads();                                // the regions become the partial sums [wave][NT][4][64]
  float* const red = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[(wv * NT + t) * 256 + i * 64 + lane] = acc[t][i];
  __syncthreads();
  const float S = FMT == QF_FMT_NVFP4 ? p.w.S[e] : 1.0f;
  for (int o = tid; o < NT * (SMALL ? 64 : 256); o += p.waves * 64) {
    // SMALL: (tile, row, column), else (tile, row % 4, row / 4, column)
    const int ln = SMALL ? o & 15 : o & 63, i = (SMALL ? o >> 4 : o >> 6) & 3, t = SMALL ? o >> 6 : o >> 8;
    const int64_t r = r0 + (SMALL ? i : 4 * (ln >> 4) + i);
    const int n = n0 + 16 * t + (ln & 15);
    if (r >= r1 || n >= N) continue;
    const float* const part = red + t * 256 + i * 64 + ln;
    float v = 0.0f;
    for (int w = 0; w < p.waves; ++w) {
      v += part[w * NT * 256];
      if (SMALL) v += (part[w * NT * 256 + 16] + part[w * NT * 256 + 32]) + part[w * NT * 256 + 48];
    }
    if (FMT == QF_FMT_NVFP4) v *= S;
    if (x_row(p, r) < 0) v = 0.0f;
    if (p.y_f32) static_cast<float*>(p.Y)[r * p.ldy + n] = v;
    else static_cast<uint16_t*>(p.Y)[r * p.ldy + n] = (uint16_t)codec::bf16_rne(v);
  }
}

template <int FMT, int NT, int COPY, int ROWS>
hipError_t launch_groups(MatvecArgs a, const MatvecPlan& p, hipStream_t s) {
  const size_t lds = (size_t)p.waves * (NT * matvec_code_bytes(FMT) + p.xrows * 1024);
  for (int64_t i = 0; i < p.items; i += p.per_launch) {
    if (a.off) {
      a.item0 = (int)i;                          // (items < 2^30)
    } else if (i > 0) {                          // of a dense call the rows that are left
      const int64_t done = p.per_launch * p.xmax;
      a.X += done * a.ldx;
      a.Y = static_cast<char*>(a.Y) + done * a.ldy * (a.y_f32 ? 4 : 2);
      a.M -= done;
      a.R -= done;
    }
    const dim3 grid((unsigned)(p.tiles * std::min(p.per_launch, p.items - i)));
    hipLaunchKernelGGL((matvec_kernel<FMT, NT, COPY, ROWS>), grid, dim3(64 * p.waves), lds, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int FMT, int NT, int COPY>
hipError_t launch_rows(const MatvecArgs& a, const MatvecPlan& p, hipStream_t s) {
  if constexpr (FMT == QF_FMT_NVFP4)
    if (p.rows == kSmall) return launch_groups<FMT, NT, COPY, kSmall>(a, p, s);
  if constexpr (FMT != QF_FMT_Q4K)
    if (p.rows == kTwice) return launch_groups<FMT, NT, COPY, kTwice>(a, p, s);
  return launch_groups<FMT, NT, COPY, kAll>(a, p, s);
}

template <int FMT>
hipError_t launch_fmt(const MatvecArgs& a, const MatvecPlan& p, hipStream_t s) {
  if constexpr (FMT == QF_FMT_NVFP4)
    if (p.copy == kCopyWords) return p.nt == 1 ? launch_rows<FMT, 1, kCopyWords>(a, p, s) : launch_rows<FMT, 2, kCopyWords>(a, p, s);
  if (p.copy == kCopyNt) return p.nt == 1 ? launch_rows<FMT, 1, kCopyNt>(a, p, s) : launch_rows<FMT, 2, kCopyNt>(a, p, s);
  return p.nt == 1 ? launch_rows<FMT, 1, kCopy>(a, p, s) : launch_rows<FMT, 2, kCopy>(a, p, s);
}

}  // namespace

hipError_t launch_packed_matvec(const PackedOperand& w, const int64_t* off, int64_t R,
                                const int32_t* rows, int64_t rows_div, int64_t M, const uint16_t* X,
                                int64_t ldx, void* Y, int64_t ldy, int y_f32, hipStream_t s) {
  const int64_t K = M == 0 ? 0 : w.K;             // no X at all: zeros
  const MatvecPlan p = matvec_plan(w.fmt, off != nullptr, w.E, w.N, K, R, compute_units());
  MatvecArgs a{w, X, ldx, M, Y, ldy, R, y_f32, off, rows, (int)rows_div, p.xmax, p.xrows, p.waves, 0};
  a.w.K = K;
  switch (w.fmt) {
    case QF_FMT_NVFP4: return launch_fmt<QF_FMT_NVFP4>(a, p, s);
    case QF_FMT_MXFP4: return launch_fmt<QF_FMT_MXFP4>(a, p, s);
    default: return launch_fmt<QF_FMT_Q4K>(a, p, s);
  }
}

}  // namespace qf
