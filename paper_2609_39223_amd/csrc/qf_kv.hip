// The 4-bit cache of keys and values (QATFactory Sec. 3.2.3's formats applied to what attention keeps):
// new tokens' rows quantized into their sequences' pages, and rows read back.
//
// Both are the quantizers' per-chunk codecs (qf_codecs.h) with the row's address taken from the table of
// pages: a lane owns 8 consecutive elements of a token's keys or values (a block is 2 or 4 lanes).  A workgroup
// first finds the places of its tokens, one a thread (binary search in the offsets, length, page: four trips to
// memory one after the other), and leaves them in LDS; rows to be written are loaded meanwhile.  NVFP4's tensor
// scale S is given per head, so one pass suffices.  Bound by memory: 2 bytes an element one way, 0.53 or 0.56
// the other; few tokens by the trips.  32768 tokens x 1024 of K and of V read back (MXFP4): 41 us, 4.1 TB/s;
// 15852 x 1024 written: 27.5 us, 3.0 TB/s (NVFP4), 25.7 (MXFP4), waiting: the places' trips, the rows, the codes and the
// stores come one after the other.  The vector units are busy 35 % of it, 23 % in MXFP4.
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

struct KvRows {
  KvCache c;
  KvSeqs q;
  uint16_t* x[2];                        // keys, values [T, H D]; either null when read back
  int64_t ld[2];
  int log_lanes;                         // lanes that share a token (a power of two, at most 256)
  int64_t group0;                        // the launch's first group of tokens
};

// The place of token t in the cache: page << page_log | offset; -1 if it has none, -2 if it is nobody's.
__device__ __forceinline__ int64_t kv_place(const KvCache& c, const KvSeqs& q, int64_t t) {
  if (t >= q.T) return -2;
  int64_t b = t, behind = 1;             // tokens of the sequence from t on
  if (q.off) {
    int64_t lo = 0, hi = q.B;            // the first b with off[b + 1] > t
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if (q.off[mid + 1] > t) hi = mid;
      else lo = mid + 1;
    }
    b = lo;
    if (b >= q.B || q.off[b] > t) return -2;
    behind = q.off[b + 1] - t;
  }
  const int64_t pos = q.lens[b] - behind;
  if (pos < 0 || (pos >> c.page_log) >= q.cols) return -1;
  const int64_t page = q.table[b * q.cols + (pos >> c.page_log)];
  if (page < 0 || page >= c.pages) return -1;
  return (page << c.page_log) | (pos & ((1 << c.page_log) - 1));
}

// A block's (D, 1 / D) where it is known already.
struct Nvfp4Known {
  f32x2_t dr;
  __device__ __forceinline__ f32x2_t operator()(uint32_t) const { return dr; }
};

// Codes and scale bytes of N chunks.  NVFP4: the two lanes of a block share the scales' work, the even one takes
// chunks 0, 2 .., the odd one chunks 1, 3 .., and each hands the other its results (two divisions a block instead of
// a lane; 15852 tokens x 2048: 34 -> 32 us).
template <int FMT, int N>
__device__ __forceinline__ void encode(const uint4 in[N], float S, uint32_t cw[N], uint32_t sc[N]) {
  uint32_t h[8], xh[8];
  if constexpr (FMT == QF_FMT_NVFP4 && N % 2 == 0) {
    const float six_s = 6.0f * S;
    const bool odd = threadIdx.x & 1;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      uint32_t h1[8];
      unpack8(in[i], h);
      unpack8(in[i + 1], h1);
      const uint32_t ab0 = nvfp4_block_max(h), ab1 = nvfp4_block_max(h1);
      const uint32_t own = nvfp4_scale_code(odd ? ab1 : ab0, S, six_s);
      const f32x2_t dr = nvfp4_scale_pair(S, own), other = {xor1_f(dr.x), xor1_f(dr.y)};
      const uint32_t so = xor1_u32(own);
      sc[i] = odd ? so : own;
      sc[i + 1] = odd ? own : so;
      nvfp4_encode(h, ab0, sc[i], Nvfp4Known{{odd ? other.x : dr.x, odd ? other.y : dr.y}}, cw[i], xh);
      nvfp4_encode(h1, ab1, sc[i + 1], Nvfp4Known{{odd ? dr.x : other.x, odd ? dr.y : other.y}}, cw[i + 1], xh);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      unpack8(in[i], h);
      if (FMT == QF_FMT_NVFP4) nvfp4_chunk(h, S, 6.0f * S, cw[i], sc[i], xh);
      else mxfp4_chunk(h, cw[i], sc[i], xh);
    }
  }
}

// N tokens a lane, one after the other of a group's 256 >> log_lanes N.
template <int FMT, bool READ, int N>
__global__ __launch_bounds__(256) void kv_rows_kernel(KvRows p) {
  constexpr int BLOCK = FMT == QF_FMT_NVFP4 ? 16 : 32;
  __shared__ int64_t places[16 * N];
  const int H = p.c.H, D = p.c.D, chunks = H * D / 8, log = p.c.page_log;
  const int lanes = 1 << p.log_lanes, abreast = 256 >> p.log_lanes, mine = threadIdx.x >> p.log_lanes;
  const int64_t t0 = (p.group0 + blockIdx.x) * abreast * N;
  int col = (int)blockIdx.y * lanes + (threadIdx.x & (lanes - 1));
  const int v = col >= chunks;
  uint16_t* const x = p.x[v];
  const bool has = col < 2 * chunks && x != nullptr;   // (whole groups of 8 lanes: H D / 8 is a multiple of 8)
  col -= v * chunks;
  const int h = has ? col / (D / 8) : 0, d = col % (D / 8);
  uint16_t* const row = x + (t0 + mine) * p.ld[v] + (int64_t)col * 8;
  const int64_t step = abreast * p.ld[v];
  uint4 in[N];
  auto load = [&]() {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      in[i] = make_uint4(0, 0, 0, 0);
      if (has && t0 + mine + i * abreast < p.q.T) in[i] = *reinterpret_cast<const uint4*>(row + i * step);
    }
  };
  // (several rows behind the places: in front of them each trip waited for the rows, 15852 tokens took 32 us for 27)
  if (!READ && N == 1) load();
  if ((int)threadIdx.x < abreast * N) places[threadIdx.x] = kv_place(p.c, p.q, t0 + threadIdx.x);
  const float S = FMT == QF_FMT_NVFP4 ? p.c.S[v][h] : 1.0f;
  __syncthreads();
  if (!has) return;
  if (!READ && N > 1) load();
  // the page's first token of head h, then the token: bytes of codes and scales follow from it
  int64_t at[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t w = places[mine + i * abreast];
    at[i] = w < 0 ? w : ((((w >> log) * H + h) << log) | (w & ((1 << log) - 1)));
  }
  if constexpr (READ) {
    uint32_t cw[N], sc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      cw[i] = sc[i] = 0;
      if (at[i] < 0) continue;
      cw[i] = *reinterpret_cast<const uint32_t*>(p.c.codes[v] + at[i] * (D / 2) + 4 * d);
      sc[i] = p.c.scales[v][at[i] * (D / BLOCK) + d * 8 / BLOCK];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (at[i] == -2) continue;         // (a token without a place reads as zeros)
      uint32_t w[4] = {0, 0, 0, 0};
      if (at[i] >= 0) {
        if (FMT == QF_FMT_NVFP4) nvfp4_decode8(cw[i], S * __builtin_amdgcn_cvt_f32_fp8((int)sc[i], 0), w);
        else mxfp4_decode8(cw[i], sc[i], w);
      }
      *reinterpret_cast<uint4*>(row + i * step) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
    uint32_t cw[N], sc[N];
    encode<FMT, N>(in, S, cw, sc);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // the scale bytes of 8 lanes (64 elements: four NVFP4 blocks or two MXFP4 ones) in one store
      uint32_t s8;
      if (FMT == QF_FMT_NVFP4) {
        s8 = sc[i] | (xor2_u32(sc[i]) << 8);
        s8 |= xor_swz_u32<4>(s8) << 16;
      } else {
        s8 = sc[i] | (xor_swz_u32<4>(sc[i]) << 8);
      }
      if (at[i] < 0) continue;
      *reinterpret_cast<uint32_t*>(p.c.codes[v] + at[i] * (D / 2) + 4 * d) = cw[i];
      if ((d & 7) == 0) {
        uint8_t* const to = p.c.scales[v] + at[i] * (D / BLOCK) + d * 8 / BLOCK;
        if (FMT == QF_FMT_NVFP4) *reinterpret_cast<uint32_t*>(to) = s8;
        else *reinterpret_cast<uint16_t*>(to) = (uint16_t)s8;
      }
    }
  }
}

template <int FMT, bool READ, int N>
hipError_t launch_n(KvRows p, hipStream_t s) {
  const int cols = 2 * p.c.H * p.c.D / 8;
  p.log_lanes = 4;                       // 16 chunks at least
  while (p.log_lanes < 8 && (1 << p.log_lanes) < cols) ++p.log_lanes;
  const int64_t per = (int64_t)(256 >> p.log_lanes) * N, groups = (p.q.T + per - 1) / per;
  const unsigned wide = (unsigned)((cols + (1 << p.log_lanes) - 1) >> p.log_lanes);
  const int64_t most = ((int64_t)1 << 23) / wide;     // a grid has fewer than 2^32 lanes
  for (int64_t g = 0; g < groups; g += most) {
    p.group0 = g;
    hipLaunchKernelGGL((kv_rows_kernel<FMT, READ, N>), dim3((unsigned)std::min(most, groups - g), wide), dim3(256), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Tokens a lane takes, by lanes of one token each in units of two workgroups a compute unit (8 heads of 128; us,
// writing / reading NVFP4):  4 units (2048 tokens)  1: 12.2 / 5.9   2: 11.5 / 5.6
//   8 (4096)  1: 18.9 / 8.7   2: 14.6 / 6.7   8: 16.3 / 7.4     16 (8192)  2: 23.6 / 11.6   8: 22.7 / 10.2
// (4 a lane at 15852 tokens: 49.0 us for both directions, 16: 50.1, 8: 48.1.)
template <int FMT, bool READ>
hipError_t launch_rows(const KvRows& p, hipStream_t s) {
  const int64_t lanes = p.q.T * (2 * p.c.H * p.c.D / 8), unit = 512 * compute_units();
  return lanes >= 10 * unit ? launch_n<FMT, READ, 8>(p, s) : lanes >= 2 * unit ? launch_n<FMT, READ, 2>(p, s) : launch_n<FMT, READ, 1>(p, s);
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
