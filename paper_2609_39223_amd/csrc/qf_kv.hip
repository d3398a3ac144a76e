// The 4-bit cache of keys and values (QATFactory Sec. 3.2.3's formats applied to what attention keeps):
// new tokens' rows quantized into their sequences' pages, and rows read back.
//
// Both are the quantizers' per-chunk codecs (qf_codecs.h) with the row's address taken from the table of
// pages: a lane owns 8 consecutive elements of a token's keys or values (a block is 2 or 4 lanes), finds
// its token's sequence by binary search in the offsets, and the page.  NVFP4's tensor scale S is given
// per head, so one pass suffices.  Bound by memory: 2 bytes an element one way, 0.53 or 0.56 the other.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "qf.h"
#include "qf_codecs.h"
#include "qf_internal.h"
#include "qf_kv.h"

namespace qf {
namespace {

using namespace codec;

constexpr int kTok = 4;                  // tokens a lane takes, their loads all in flight

struct KvRows {
  KvCache c;
  KvSeqs q;
  uint16_t* x[2];                        // keys, values [T, H D]; either null when read back
  int64_t ld[2];
  int log_lanes;                         // lanes that share a token (a power of two, at most 256)
  int64_t group0;                        // the launch's first group of tokens
};

// The place of token t in the cache: first byte of a page counted in tokens (page 2^log + offset, H
// heads apart), -1 if it has none.
__device__ __forceinline__ int64_t kv_place(const KvCache& c, const KvSeqs& q, int64_t t, int& offset) {
  if (t >= q.T) return -1;
  int64_t b = t, behind = 1;             // tokens of the sequence from t on
  if (q.off) {
    int64_t lo = 0, hi = q.B;            // the first b with off[b + 1] > t
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if (q.off[mid + 1] > t) hi = mid;
      else lo = mid + 1;
    }
    b = lo;
    if (b >= q.B || q.off[b] > t) return -1;
    behind = q.off[b + 1] - t;
  }
  const int64_t pos = q.lens[b] - behind;
  if (pos < 0 || (pos >> c.page_log) >= q.cols) return -1;
  const int64_t page = q.table[b * q.cols + (pos >> c.page_log)];
  offset = (int)(pos & ((1 << c.page_log) - 1));
  return page < c.pages ? page : -1;     // (a negative entry is none either)
}

template <int FMT, bool READ>
__global__ __launch_bounds__(256) void kv_rows_kernel(KvRows p) {
  constexpr int BLOCK = FMT == QF_FMT_NVFP4 ? 16 : 32;
  const int H = p.c.H, D = p.c.D, chunks = H * D / 8;
  const int lanes = 1 << p.log_lanes;
  int col = (int)blockIdx.y * lanes + (threadIdx.x & (lanes - 1));
  if (col >= 2 * chunks) return;         // (whole groups of 8 lanes: 2 H D / 8 is a multiple of 16)
  const int v = col >= chunks;
  uint16_t* const x = p.x[v];
  if (x == nullptr) return;
  col -= v * chunks;
  const int h = col / (D / 8), d = col % (D / 8);
  const int64_t t0 = ((p.group0 + blockIdx.x) * (256 >> p.log_lanes) + (threadIdx.x >> p.log_lanes)) * kTok;
  int64_t page[kTok];
  int at[kTok];
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    at[i] = 0;
    page[i] = kv_place(p.c, p.q, t0 + i, at[i]);
  }
  const float S = FMT == QF_FMT_NVFP4 ? p.c.S[v][h] : 1.0f;
  uint16_t* const row = x + t0 * p.ld[v] + (int64_t)col * 8;
  if constexpr (READ) {
    uint32_t cw[kTok], sc[kTok];
#pragma unroll
    for (int i = 0; i < kTok; ++i) {
      cw[i] = sc[i] = 0;
      if (page[i] < 0) continue;
      cw[i] = *reinterpret_cast<const uint32_t*>(p.c.codes[v] + kv_page_at(p.c, page[i], h, D / 2) +
                                                 (int64_t)at[i] * (D / 2) + 4 * d);
      sc[i] = p.c.scales[v][kv_page_at(p.c, page[i], h, D / BLOCK) + (int64_t)at[i] * (D / BLOCK) + d * 8 / BLOCK];
    }
#pragma unroll
    for (int i = 0; i < kTok; ++i) {
      // a token of a sequence that has no place reads as zeros; rows of no sequence are left alone
      if (t0 + i >= p.q.T || (p.q.off && t0 + i >= p.q.off[p.q.B])) continue;
      uint32_t w[4] = {0, 0, 0, 0};
      if (page[i] >= 0) {
        if (FMT == QF_FMT_NVFP4) nvfp4_decode8(cw[i], S * __builtin_amdgcn_cvt_f32_fp8((int)sc[i], 0), w);
        else mxfp4_decode8(cw[i], sc[i], w);
      }
      *reinterpret_cast<uint4*>(row + i * p.ld[v]) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
    uint4 in[kTok];
#pragma unroll
    for (int i = 0; i < kTok; ++i) {
      in[i] = make_uint4(0, 0, 0, 0);
      if (page[i] >= 0) in[i] = *reinterpret_cast<const uint4*>(row + i * p.ld[v]);
    }
    const float six_s = 6.0f * S;
#pragma unroll
    for (int i = 0; i < kTok; ++i) {
      uint32_t hh[8], cw, sc, xh[8];
      unpack8(in[i], hh);
      if (FMT == QF_FMT_NVFP4) nvfp4_chunk(hh, S, six_s, cw, sc, xh);
      else mxfp4_chunk(hh, cw, sc, xh);
      // the scale bytes of 8 lanes (64 elements: four NVFP4 blocks or two MXFP4 ones) in one store
      uint32_t s8;
      if (FMT == QF_FMT_NVFP4) {
        s8 = sc | (xor2_u32(sc) << 8);
        s8 |= xor_swz_u32<4>(s8) << 16;
      } else {
        s8 = sc | (xor_swz_u32<4>(sc) << 8);
      }
      if (page[i] < 0) continue;
      *reinterpret_cast<uint32_t*>(p.c.codes[v] + kv_page_at(p.c, page[i], h, D / 2) + (int64_t)at[i] * (D / 2) + 4 * d) = cw;
      if ((d & 7) == 0) {
        uint8_t* const to = p.c.scales[v] + kv_page_at(p.c, page[i], h, D / BLOCK) + (int64_t)at[i] * (D / BLOCK) + d * 8 / BLOCK;
        if (FMT == QF_FMT_NVFP4) *reinterpret_cast<uint32_t*>(to) = s8;
        else *reinterpret_cast<uint16_t*>(to) = (uint16_t)s8;
      }
    }
  }
}

template <int FMT, bool READ>
hipError_t launch_rows(KvRows p, hipStream_t s) {
  const int cols = 2 * p.c.H * p.c.D / 8;
  p.log_lanes = 4;                       // 16 chunks at least
  while (p.log_lanes < 8 && (1 << p.log_lanes) < cols) ++p.log_lanes;
  const int64_t per = (int64_t)(256 >> p.log_lanes) * kTok, groups = (p.q.T + per - 1) / per;
  const unsigned wide = (unsigned)((cols + (1 << p.log_lanes) - 1) >> p.log_lanes);
  const int64_t most = ((int64_t)1 << 23) / wide;     // a grid has fewer than 2^32 lanes
  for (int64_t g = 0; g < groups; g += most) {
    p.group0 = g;
    hipLaunchKernelGGL((kv_rows_kernel<FMT, READ>), dim3((unsigned)std::min(most, groups - g), wide), dim3(256), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_kv_write(const KvCache& c, const KvSeqs& q, const uint16_t* K, int64_t ldk,
                           const uint16_t* V, int64_t ldv, hipStream_t s) {
  const KvRows p{c, q, {const_cast<uint16_t*>(K), const_cast<uint16_t*>(V)}, {ldk, ldv}, 0, 0};
  return c.fmt == QF_FMT_NVFP4 ? launch_rows<QF_FMT_NVFP4, false>(p, s) : launch_rows<QF_FMT_MXFP4, false>(p, s);
}

hipError_t launch_kv_read(const KvCache& c, const KvSeqs& q, uint16_t* K, int64_t ldk, uint16_t* V,
                          int64_t ldv, hipStream_t s) {
  const KvRows p{c, q, {K, V}, {ldk, ldv}, 0, 0};
  return c.fmt == QF_FMT_NVFP4 ? launch_rows<QF_FMT_NVFP4, true>(p, s) : launch_rows<QF_FMT_MXFP4, true>(p, s);
}

}  // namespace qf
