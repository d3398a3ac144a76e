// Around the grouped (mixture-of-experts) layer (QATFactory Sec. 3.3 "Mixture-of-experts
// adaptation"): the router's top-k with its gradient, the stable sort of token slots by expert with
// the rows' copy, and the weighted sum back to token order with its gradients.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "qf.h"
#include "qf_codecs.h"
#include "qf_internal.h"

namespace qf {
namespace {

using codec::as_f32;
using codec::as_u32;

// =============================================================================== the router
// A token's row is held by L lanes, 8 C consecutive-by-8 logits each (chunk c of lane l: experts
// 8 (c L + l) .. + 7).  Each of the k rounds takes the largest (logit, lowest expert) of the row
// by a maximum over ordered keys and strikes it out, so choices come out in order and equal logits
// by rising expert whatever L and C are.
constexpr int kRouteThreads = 256;

// DPP cross-lane moves inside rows of 16 lanes.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
struct MaxU {
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
struct MaxF {
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const {
    return as_u32(fmaxf(as_f32(a), as_f32(b)));
  }
};
struct AddF {
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const {
    return as_u32(as_f32(a) + as_f32(b));
  }
};
// Reduction over the L lanes of a token (16, 32 or 64), the same bits in all of them: lane ^ 1, ^ 2,
// then the mirror images inside 8 and 16 lanes (whose sources are alike within 4 and 8), ^ 16 and ^ 32
// by the swaps of 16- and 32-lane rows (which hand a register's even and odd rows to every lane).
template <int L, class Op>
__device__ __forceinline__ uint32_t group_reduce(uint32_t v, Op op) {
  v = op(v, dpp_u32<0xB1>(v));
  v = op(v, dpp_u32<0x4E>(v));
  v = op(v, dpp_u32<0x141>(v));
  v = op(v, dpp_u32<0x140>(v));
  if (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = op(r[0], r[1]);
  }
  if (L == 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = op(r[0], r[1]);
  }
  return v;
}
template <int L>
__device__ __forceinline__ float group_sum(float v) { return as_f32(group_reduce<L>(as_u32(v), AddF())); }
template <int L>
__device__ __forceinline__ float group_max(float v) { return as_f32(group_reduce<L>(as_u32(v), MaxF())); }

// FP32 bits -> an unsigned key of the same order, 0 for -inf (and nothing else); zeros alike, NaN
// above +inf.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = as_u32(v);
  if (v != v) return 0xFFFFFFFFu;
  if (u == 0xFF800000u) return 0u;
  const uint32_t p = v == 0.0f ? 0u : u;
  return (p >> 31) ? ~p : (p | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return as_f32((k >> 31) ? (k & 0x7FFFFFFFu) : ~k);
}

__device__ __forceinline__ float load_logit(const uint16_t* z, int64_t i) { return as_f32((uint32_t)z[i] << 16); }
__device__ __forceinline__ float load_logit(const float* z, int64_t i) { return z[i]; }
__device__ __forceinline__ void load_logits8(const uint16_t* p, float v[8]) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  uint32_t h[8];
  codec::unpack8(q, h);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = as_f32(h[i] << 16);
}
__device__ __forceinline__ void load_logits8(const float* p, float v[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(uint16_t* p, const float v[8]) {
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = codec::bf16_rne(v[i]);
  *reinterpret_cast<uint4*>(p) = codec::pack8(h);
}
__device__ __forceinline__ void store8(float* p, const float v[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = (uint16_t)codec::bf16_rne(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// Experts whose logits may move in whole chunks: none where rows do not start at one (rows back to back
// may have any length).
__device__ __forceinline__ int in_chunks(int E, int64_t ld) { return ld % 8 == 0 ? E : 0; }
// This lane's chunk c of a row (experts e0 .. e0 + 7; -inf past E, which is never read).
template <class Z>
__device__ __forceinline__ void load_chunk(const Z* row, int e0, int E, int Ec, float v[8]) {
  if (e0 + 8 <= Ec) {
    load_logits8(row + e0, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e0 + i < E ? load_logit(row, e0 + i) : -INFINITY;
  }
}

// log(1 / (1 + exp(-x))), finite for every finite x.
__device__ __forceinline__ float log_sigmoid(float x) {
  return fminf(x, 0.0f) - log1pf(expf(-fabsf(x)));
}

// Lane j < k of the group ends up with choice j (expert id, -1: none left; its logit v).
//
// FP32 logits, and more than 512 experts: a round finds the largest key of the row, the first lane that
// has it and that lane's first expert with it, which is struck out: two reductions and three passes over
// the lane's keys (32768 tokens, 8 choices: 128 experts 10.5 us where bf16 takes 7.2, 256 17.9 / 12.3, 1024
// 54 either way).
template <int L, int C>
__device__ __forceinline__ void choose(uint32_t key[8 * C], int lane, int k, int& id, float& v) {
  id = -1;
  v = 0.0f;
  for (int j = 0; j < k; ++j) {
    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) best = key[i] > best ? key[i] : best;
    const uint32_t top = group_reduce<L>(best, MaxU());
    if (top == 0u) break;                         // (the same in all lanes of the group)
    // of the logits equal to it the lowest expert: the largest complement
    uint32_t cand = 0;
#pragma unroll
    for (int i = 8 * C - 1; i >= 0; --i)
      if (key[i] == top) cand = 0xFFFFu - (uint32_t)(8 * ((i >> 3) * L + lane) + (i & 7));
    const uint32_t e = 0xFFFFu - group_reduce<L>(cand, MaxU());
#pragma unroll
    for (int i = 0; i < 8 * C; ++i)
      if (e == (uint32_t)(8 * ((i >> 3) * L + lane) + (i & 7))) key[i] = 0u;
    if (lane == j) {
      id = (int)e;
      v = key_value(top);
    }
  }
}

// bf16 logits leave 16 bits of a key for the expert's complement, so one maximum decides a round;
// a lane sorts its eight keys once and a round takes the best lane's first one away (32768 x 128, 8
// choices: 9.8 us without either, 7.0 so).
__device__ __forceinline__ void sort8_falling(uint32_t a[8]) {
  constexpr int net[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                              {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
  for (int i = 0; i < 19; ++i) {
    const uint32_t x = a[net[i][0]], y = a[net[i][1]];
    a[net[i][0]] = x > y ? x : y;
    a[net[i][1]] = x > y ? y : x;
  }
}
template <int L>
__device__ __forceinline__ void choose_sorted(uint32_t key[8], int lane, int k, int& id, float& v) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    key[i] = key[i] ? (key[i] & 0xFFFF0000u) | (0xFFFFu - (uint32_t)(8 * lane + i)) : 0u;
  sort8_falling(key);
  uint32_t mine = 0;
  for (int j = 0; j < k; ++j) {
    const uint32_t top = group_reduce<L>(key[0], MaxU());
    const bool taken = key[0] == top;             // one lane's, or top = 0 and nothing is left
#pragma unroll
    for (int i = 0; i < 7; ++i) key[i] = taken ? key[i + 1] : key[i];
    key[7] = taken ? 0u : key[7];
    if (lane == j) mine = top;
  }
  id = mine ? (int)(0xFFFFu - (mine & 0xFFFFu)) : -1;
  v = mine ? key_value((mine >> 31) ? mine & 0xFFFF0000u : mine | 0xFFFFu) : 0.0f;
}

template <class Z, int L, int C>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(
    const Z* __restrict__ z, int64_t T, int E, int64_t ldz, int k, int score, int norm, float scale,
    const uint8_t* __restrict__ mask, int32_t* __restrict__ ids, float* __restrict__ w) {
  const int lane = threadIdx.x % L;
  const int64_t t = (int64_t)blockIdx.x * (kRouteThreads / L) + threadIdx.x / L;
  const bool live = t < T && (mask == nullptr || mask[t] != 0);
  float x[8 * C];
  uint32_t key[8 * C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (live) {
      load_chunk(z + t * ldz, 8 * (c * L + lane), E, in_chunks(E, ldz), x + 8 * c);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[8 * c + i] = -INFINITY;
    }
  }
#pragma unroll
  for (int i = 0; i < 8 * C; ++i) key[i] = key_of(x[i]);
  int id;
  float v;
  if constexpr (sizeof(Z) == 2 && C == 1) choose_sorted<L>(key, lane, k, id, v);
  else choose<L, C>(key, lane, k, id, v);
  const bool has = id >= 0;
  float out;
  if (norm) {
    const float a = score == QF_SCORE_SIGMOID ? log_sigmoid(v) : v;
    const float m = group_max<L>(has ? a : -INFINITY);   // (a NaN is passed over here and comes back below)
    const float e = has ? expf(a - m) : 0.0f;
    out = e / group_sum<L>(e);
  } else if (score == QF_SCORE_SIGMOID) {
    out = 1.0f / (1.0f + expf(-v));
  } else {
    float m = x[0], s = 0.0f;
#pragma unroll
    for (int i = 1; i < 8 * C; ++i) m = fmaxf(m, x[i]);
    m = group_max<L>(m);
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) s += expf(x[i] - m);
    out = expf(v - m) / group_sum<L>(s);
  }
  if (t < T && lane < k) {
    ids[t * k + lane] = id;
    w[t * k + lane] = has ? scale * out : 0.0f;
  }
}

// The gradient: lane j < k of a token's group holds choice j; the chosen experts' values go through
// LDS into the row, whose lanes write it out 8 logits a chunk.
template <class Z, int L, int C>
__global__ __launch_bounds__(kRouteThreads) void route_bwd_kernel(
    const Z* __restrict__ z, int64_t T, int E, int64_t ldz, int k, int score, int norm, float scale,
    const int32_t* __restrict__ ids, const float* __restrict__ dw, Z* __restrict__ dz, int64_t lddz) {
  __shared__ __align__(16) float rows[kRouteThreads / L][8 * C * L];
  const int lane = threadIdx.x % L;
  const int64_t t = (int64_t)blockIdx.x * (kRouteThreads / L) + threadIdx.x / L;
  float* const row = rows[threadIdx.x / L];
  int id = -1;
  float g = 0.0f, v = 0.0f;
  if (t < T && lane < k) {
    id = ids[t * k + lane];
    if (id < 0 || id >= E) id = -1;
    if (id >= 0) {
      g = scale * dw[t * k + lane];
      v = load_logit(z + t * ldz, id);
    }
  }
  const bool has = id >= 0;
  const bool whole = !norm && score == QF_SCORE_SOFTMAX;   // every logit has a gradient
  float x[8 * C], m = -INFINITY, s = 0.0f;
  if (whole) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (t < T) {
        load_chunk(z + t * ldz, 8 * (c * L + lane), E, in_chunks(E, ldz), x + 8 * c);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[8 * c + i] = -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) m = fmaxf(m, x[i]);
    m = group_max<L>(m);
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) s += expf(x[i] - m);
    s = group_sum<L>(s);
  }
  float d, dot = 0.0f;
  if (norm) {
    const float a = score == QF_SCORE_SIGMOID ? log_sigmoid(v) : v;
    const float mk = group_max<L>(has ? a : -INFINITY);
    const float e = has ? expf(a - mk) : 0.0f;
    const float q = e / group_sum<L>(e);
    d = q * (g - group_sum<L>(has ? q * g : 0.0f));
    if (score == QF_SCORE_SIGMOID) d = d / (1.0f + expf(v));
  } else if (score == QF_SCORE_SIGMOID) {
    const float e = expf(-fabsf(v));
    d = g * e / ((1.0f + e) * (1.0f + e));
  } else {
    d = g;
    dot = group_sum<L>(has ? g * (expf(v - m) / s) : 0.0f);
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    float4* const p = reinterpret_cast<float4*>(row + 8 * (c * L + lane));
    p[0] = p[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
  __syncthreads();
  if (has) row[id] = d;
  __syncthreads();
  if (t >= T) return;
  // a token without choices has no gradient, whatever its logits are
  const bool none = whole && (__ballot(has) >> ((threadIdx.x & 63) / L * L) & (L == 64 ? ~0ull : (1ull << L % 64) - 1)) == 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int e0 = 8 * (c * L + lane);
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      o[i] = row[e0 + i];
      if (whole) o[i] = none ? 0.0f : expf(x[8 * c + i] - m) / s * (o[i] - dot);
    }
    Z* const out = dz + t * lddz + e0;
    if (e0 + 8 <= in_chunks(E, lddz)) {
      store8(out, o);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (e0 + i < E) store1(out + i, o[i]);
    }
  }
}

// ================================================================================= the sort
// Buckets 0 .. E - 1 are the experts, bucket E the dropped slots.
__device__ __forceinline__ int bucket_of(int id, int E) { return id >= 0 && id < E ? id : E; }

constexpr int kSortThreads = 256;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMaxChunks = 256;
constexpr int64_t kMinChunk = 1024;
// A launch that compares all pairs, or three: 256 tokens x 8 10.3 / 10.9 us, 1024 x 2 7.1 / 14.4, 512 x 8
// 18.5 / 11.4 (128 and 256 experts, rows of 512 and 2048 columns copied).
constexpr int64_t kSmallSort = 2048;
constexpr int kMaxBuckets = 1025;

// Slots of a chunk: a multiple of 256, such that at most kMaxChunks chunks cover n slots.
int64_t sort_chunk(int64_t n) {
  const int64_t c = (n + kMaxChunks - 1) / kMaxChunks;
  return std::max<int64_t>(kMinChunk, (c + 255) / 256 * 256);
}

// counts [chunk][E + 1].
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(const int32_t* __restrict__ ids,
                                                                  int64_t n, int E, int64_t chunk,
                                                                  int32_t* __restrict__ counts) {
  __shared__ int h[kMaxBuckets];
  for (int e = threadIdx.x; e <= E; e += kSortThreads) h[e] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * chunk, i1 = i0 + chunk < n ? i0 + chunk : n;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kSortThreads) atomicAdd(&h[bucket_of(ids[i], E)], 1);
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += kSortThreads) counts[(int64_t)blockIdx.x * (E + 1) + e] = h[e];
}

// In-place exclusive prefix sum of a[0 .. nb) over the workgroup (nb <= kMaxBuckets; `part`: one
// int per wave).
__device__ __forceinline__ void block_exclusive(int* a, int nb, int* part) {
  constexpr int kPer = (kMaxBuckets + kSortThreads - 1) / kSortThreads;
  const int b0 = threadIdx.x * kPer, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  int own[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    own[i] = b0 + i < nb ? a[b0 + i] : 0;
    sum += own[i];
  }
  int inc = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(inc, d, 64);
    if (lane >= d) inc += o;
  }
  if (lane == 63) part[wv] = inc;
  __syncthreads();
  int run = inc - sum;
  for (int i = 0; i < wv; ++i) run += part[i];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (b0 + i < nb) a[b0 + i] = run;
    run += own[i];
  }
  __syncthreads();
}

// Rows of one chunk's slots: the bucket's first row, plus its slots in earlier chunks (summed here
// from counts: at most 256 chunks), in earlier waves of this chunk and before it in its wave.  A
// wave walks its quarter 64 slots at a time; the slots of the same bucket in such a step find each
// other by ballots over the bucket's bits.
__global__ __launch_bounds__(kSortThreads) void sort_rank_kernel(
    const int32_t* __restrict__ ids, int64_t n, int E, int64_t chunk, const int32_t* __restrict__ counts,
    int64_t* __restrict__ offsets, int32_t* __restrict__ row_of, int32_t* __restrict__ slot_of) {
  __shared__ int first[kMaxBuckets];                 // total, then first row, of each bucket
  __shared__ int before[kMaxBuckets];                // slots of the bucket in earlier chunks
  __shared__ int next[kSortWaves][kMaxBuckets];      // next row of the bucket in each wave
  __shared__ int part[kSortWaves];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, nb = E + 1;
  const int nchunks = gridDim.x, me = blockIdx.x;
  for (int e = threadIdx.x; e < nb; e += kSortThreads) {
    first[e] = before[e] = 0;
    for (int i = 0; i < kSortWaves; ++i) next[i][e] = 0;
  }
  __syncthreads();
  // wave w sums the chunks w, w + 4, ..., a lane per bucket (a long chain of loads if one wave did)
  for (int e = lane; e < nb; e += 64) {
    int pre = 0, all = 0;
#pragma unroll 8
    for (int c = wv; c < nchunks; c += kSortWaves) {
      const int v = counts[(int64_t)c * nb + e];
      all += v;
      pre += c < me ? v : 0;
    }
    atomicAdd(&first[e], all);
    atomicAdd(&before[e], pre);
  }
  __syncthreads();
  block_exclusive(first, nb, part);
  if (me == 0)
    for (int e = threadIdx.x; e < nb; e += kSortThreads) offsets[e] = first[e];
  const int64_t quarter = chunk / kSortWaves;
  const int64_t i0 = (int64_t)me * chunk + wv * quarter;
  const int64_t end = (int64_t)me * chunk + chunk < n ? (int64_t)me * chunk + chunk : n;
  const int64_t i1 = i0 + quarter < end ? i0 + quarter : end;
  for (int64_t i = i0 + lane; i < i1; i += 64) atomicAdd(&next[wv][bucket_of(ids[i], E)], 1);
  __syncthreads();
  for (int e = threadIdx.x; e < nb; e += kSortThreads) {
    int run = first[e] + before[e];
    for (int i = 0; i < kSortWaves; ++i) {
      const int c = next[i][e];
      next[i][e] = run;
      run += c;
    }
  }
  __syncthreads();
  const int live = first[E], bits = 32 - __clz(nb);
  volatile int* const mine = next[wv];
  for (int64_t b = i0; b < i1; b += 64) {
    const int64_t i = b + lane;
    const bool in = i < i1;
    const int e = in ? bucket_of(ids[i], E) : nb;    // past the end: a bucket of their own
    uint64_t same = ~0ull;
    for (int bit = 0; bit < bits; ++bit) {
      const bool one = (e >> bit) & 1;
      const uint64_t v = __ballot(one);
      same &= one ? v : ~v;
    }
    if (in) {
      const int row = mine[e] + __popcll(same & ((1ull << lane) - 1));
      row_of[i] = e < E ? row : ~row;
      slot_of[row] = row < live ? (int32_t)i : -1;
    }
    __builtin_amdgcn_wave_barrier();
    if (in && (same >> lane) == 1ull) mine[e] += __popcll(same);   // the last of each bucket
    __builtin_amdgcn_wave_barrier();
  }
}

// Few slots, all in one launch: workgroup t counts, for each of token t's slots, the slots that come
// before it (a lower bucket, or the same one and a lower slot) by ballots over all n, and copies its
// row; the last workgroup counts the buckets.  T n comparisons instead of two more launches.
__global__ __launch_bounds__(kSortThreads) void sort_small_kernel(
    const int32_t* __restrict__ ids, int64_t T, int E, int k, int64_t* __restrict__ offsets,
    int32_t* __restrict__ row_of, int32_t* __restrict__ slot_of, const uint16_t* __restrict__ X,
    int64_t H, int64_t ldx, uint16_t* __restrict__ Xg) {
  __shared__ int h[kMaxBuckets];
  __shared__ int part[kSortWaves];
  __shared__ int count[kSortWaves][64];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, n = (int)T * k, t = blockIdx.x;
  if (t == (int)T) {
    for (int e = tid; e <= E; e += kSortThreads) h[e] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kSortThreads) atomicAdd(&h[bucket_of(ids[i], E)], 1);
    __syncthreads();
    block_exclusive(h, E + 1, part);
    for (int e = tid; e <= E; e += kSortThreads) offsets[e] = h[e];
    return;
  }
  // lane j < k of every wave: the bucket and the slots found before slot (t, j)
  const int own = lane < k ? bucket_of(ids[t * k + lane], E) : 0;
  int before = 0;
  for (int i0 = wv * 64; i0 < n; i0 += kSortThreads) {
    const int i = i0 + lane, e = i < n ? bucket_of(ids[i], E) : 0x7FFFFFFF;
    for (int j = 0; j < k; ++j) {
      const int b = __builtin_amdgcn_readlane(own, j);
      const int c = __popcll(__ballot(e < b || (e == b && i < t * k + j)));
      if (lane == j) before += c;
    }
  }
  count[wv][lane] = before;
  __syncthreads();
  int row = 0;
  if (lane < k) {
    for (int i = 0; i < kSortWaves; ++i) row += count[i][lane];
    if (wv == 0) {
      row_of[t * k + lane] = own < E ? row : ~row;
      slot_of[row] = own < E ? t * k + lane : -1;
    }
  }
  if (X == nullptr) return;
  for (int64_t c = tid * 8; c < H; c += kSortThreads * 8) {
    const uint4 v = *reinterpret_cast<const uint4*>(X + t * ldx + c);
    for (int j = 0; j < k; ++j)
      *reinterpret_cast<uint4*>(Xg + (int64_t)__builtin_amdgcn_readlane(row, j) * H + c) =
          __builtin_amdgcn_readlane(own, j) < E ? v : make_uint4(0, 0, 0, 0);
  }
}

// Expert rows are read non-temporally: a launch reads each once, and seldom again soon.  They are
// written so only past half the last-level cache of 256 MB: below, the product that follows finds them
// there (8 rows of 3072 a token, us without / with: sum of 2048 tokens 24.3 / 20.9, of 32768 351 / 328;
// sort, copy and gradient of 32768 738 / 708; gradients of 4096 91.6 / 84.2 alone, but with the sum that
// reads them next 106 / 124).
typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_nt(const uint16_t* p) {
  const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <bool NT>
__device__ __forceinline__ void store_row(uint16_t* p, uint4 q) {
  const u32x4_t u = {q.x, q.y, q.z, q.w};
  if (NT) __builtin_nontemporal_store(u, reinterpret_cast<u32x4_t*>(p));
  else *reinterpret_cast<uint4*>(p) = q;
}
bool rows_past_cache(int64_t n, int64_t H) { return n * H * 2 > (int64_t)128 << 20; }

// Xg[row] = X[t] for the rows of token t's slots, zeros for dropped ones: a wave copies 512 columns.
// Bound by writing the rows: 32768 tokens x 8 x 3072 378 us = 4.8 TB/s.
template <bool NT>
__global__ __launch_bounds__(256) void gather_kernel(const int32_t* __restrict__ row_of, int64_t T,
                                                     int k, int64_t H, int64_t ldx, int segs,
                                                     const uint16_t* __restrict__ X,
                                                     uint16_t* __restrict__ Xg) {
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t t = __builtin_amdgcn_readfirstlane((int)(item / segs));
  const int64_t c = (item % segs) * 512 + (threadIdx.x & 63) * 8;
  if (t >= T || c >= H) return;
  const uint4 v = *reinterpret_cast<const uint4*>(X + t * ldx + c);
  const int32_t* const r = row_of + t * k;
  for (int j = 0; j < k; ++j) {
    const int row = r[j];
    store_row<NT>(Xg + (int64_t)(row >= 0 ? row : ~row) * H + c, row >= 0 ? v : make_uint4(0, 0, 0, 0));
  }
}

// ============================================================================= weighted sum
// A wave's view of KB slots of token t from j0 on: lane j < KB holds slot j0 + j's entry of row_of
// (kNoRow past k) and its weight; bit j of `live`: the slot has a row.
constexpr int kNoRow = 0x7FFFFFFF;
template <int KB>
struct Slots {
  int row;
  float wt;
  uint32_t live;
  __device__ __forceinline__ Slots(const int32_t* row_of, const float* w, int64_t t, int k, int j0, int64_t n) {
    const int j = j0 + (threadIdx.x & 63);
    const bool in = (int)(threadIdx.x & 63) < KB && j < k;
    row = in ? row_of[t * k + j] : kNoRow;
    wt = in && w ? w[t * k + j] : 1.0f;
    live = (uint32_t)__ballot(row >= 0 && row < n);        // (n < 2^31, so never a kNoRow)
  }
  __device__ __forceinline__ int row_at(int j) const { return __builtin_amdgcn_readlane(row, j); }
  __device__ __forceinline__ float weight_at(int j) const {
    return as_f32((uint32_t)__builtin_amdgcn_readlane((int)as_u32(wt), j));
  }
  __device__ __forceinline__ bool has(int j) const { return (live >> j) & 1u; }
};

// Y[t] = sum over j of w_j Yg[row_j]: a wave takes 512 columns of a token and has KB rows' loads in
// flight (a slot without a row loads row 0 and leaves it: no branch between the loads).  Bound by
// reading the rows: 32768 tokens x 8 x 3072 312 us = 5.8 TB/s.
template <int KB>
__global__ __launch_bounds__(256) void combine_kernel(const int32_t* __restrict__ row_of,
                                                      const float* __restrict__ w, int64_t T, int k,
                                                      int64_t H, int segs, const uint16_t* __restrict__ Yg,
                                                      uint16_t* __restrict__ Y, int64_t ldy) {
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t t = __builtin_amdgcn_readfirstlane((int)(item / segs)), n = T * k;
  const int64_t c0 = (item % segs) * 512 + (threadIdx.x & 63) * 8, c = c0 < H ? c0 : 0;
  if (t >= T) return;
  float acc[8] = {};
  for (int j0 = 0; j0 < k; j0 += KB) {
    const Slots<KB> s(row_of, w, t, k, j0, n);
    if (s.live == 0) continue;
    uint4 v[KB];
#pragma unroll
    for (int j = 0; j < KB; ++j) v[j] = load_nt(Yg + (s.has(j) ? (int64_t)s.row_at(j) * H : 0) + c);
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      if (!s.has(j)) continue;
      uint32_t h[8];
      codec::unpack8(v[j], h);
      const float wt = s.weight_at(j);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = __builtin_fmaf(wt, as_f32(h[i] << 16), acc[i]);
    }
  }
  if (c0 < H) store8(Y + t * ldy + c, acc);
}

// dYg[row_j] = w_j dY[t] and dw_j = <dY[t], Yg[row_j]>: a workgroup of W waves takes a token, wave w
// the 512-column pieces w, w + W, ..., KB rows at a time; dw's partial sums meet in LDS in wave
// order.  Bound by the rows read and written: 32768 tokens x 8 x 3072 682 us = 5.0 TB/s.
template <int KB, int W, bool NT>
__global__ __launch_bounds__(64 * W) void combine_bwd_kernel(
    const int32_t* __restrict__ row_of, const float* __restrict__ w, int64_t T, int k, int64_t H,
    const uint16_t* __restrict__ dY, int64_t lddy, const uint16_t* __restrict__ Yg,
    uint16_t* __restrict__ dYg, float* __restrict__ dw) {
  __shared__ float part[W][KB];
  const int64_t t = blockIdx.x, n = T * k;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int j0 = 0; j0 < k; j0 += KB) {
    const Slots<KB> s(row_of, w, t, k, j0, n);
    float dot[KB];
#pragma unroll
    for (int j = 0; j < KB; ++j) dot[j] = 0.0f;
    for (int64_t c0 = wv * 512; c0 < H; c0 += 512 * W) {
      const int64_t c1 = c0 + lane * 8, c = c1 < H ? c1 : 0;
      const bool in = c1 < H;
      float d[8];
      uint4 y[KB];
      load_logits8(dY + t * lddy + c, d);
      if (dw) {
#pragma unroll
        for (int j = 0; j < KB; ++j) y[j] = load_nt(Yg + (s.has(j) ? (int64_t)s.row_at(j) * H : 0) + c);
      }
      if (dYg) {
#pragma unroll
        for (int j = 0; j < KB; ++j) {
          const int row = s.row_at(j);
          const int64_t to = row >= 0 ? row : ~row;
          const float wt = s.weight_at(j);
          uint32_t o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = s.has(j) ? codec::bf16_rne(wt * d[i]) : 0u;
          if (to < n && in) store_row<NT>(dYg + to * H + c, codec::pack8(o));
        }
      }
      if (dw) {
#pragma unroll
        for (int j = 0; j < KB; ++j) {
          uint32_t h[8];
          codec::unpack8(y[j], h);
#pragma unroll
          for (int i = 0; i < 8; ++i) dot[j] = __builtin_fmaf(in ? d[i] : 0.0f, in ? as_f32(h[i] << 16) : 0.0f, dot[j]);
        }
      }
    }
    if (!dw) continue;
#pragma unroll
    for (int j = 0; j < KB; ++j) {
#pragma unroll
      for (int m = 1; m < 64; m *= 2) dot[j] += __shfl_xor(dot[j], m, 64);
      if (lane == 0) part[wv][j] = dot[j];
    }
    __syncthreads();
    if (threadIdx.x < KB && j0 + (int)threadIdx.x < k) {
      float v = 0.0f;
      for (int i = 0; i < W; ++i) v += part[i][threadIdx.x];
      dw[t * k + j0 + threadIdx.x] = s.has((int)threadIdx.x) ? v : 0.0f;   // (a slot without a row saw row 0)
    }
    __syncthreads();
  }
}

// Waves a token: as many as its row has 512-column pieces, up to 4, which then take several each (8
// rows of 3072, 32768 tokens, us, 1 / 2 / 4 / 8 waves 1041 / 1035 / 1034 / 1032; 9000 x 4 rows of 1000:
// 58 / 55 / 58 / 76), 8 where tokens are fewer than compute units (16 tokens 20.1 / 13.7 / 11.6 / 10.7).
template <int KB, int W>
void launch_combine_bwd_waves(const int32_t* row_of, const float* w, int64_t T, int k, int64_t H,
                              const uint16_t* dY, int64_t lddy, const uint16_t* Yg, uint16_t* dYg,
                              float* dw, hipStream_t s) {
  if (rows_past_cache(T * k, H))
    hipLaunchKernelGGL((combine_bwd_kernel<KB, W, true>), dim3((unsigned)T), dim3(64 * W), 0, s, row_of, w, T, k, H,
                       dY, lddy, Yg, dYg, dw);
  else
    hipLaunchKernelGGL((combine_bwd_kernel<KB, W, false>), dim3((unsigned)T), dim3(64 * W), 0, s, row_of, w, T, k, H,
                       dY, lddy, Yg, dYg, dw);
}
template <int KB>
void launch_combine_bwd(const int32_t* row_of, const float* w, int64_t T, int k, int64_t H,
                        const uint16_t* dY, int64_t lddy, const uint16_t* Yg, uint16_t* dYg, float* dw,
                        hipStream_t s) {
  if (H <= 512) launch_combine_bwd_waves<KB, 1>(row_of, w, T, k, H, dY, lddy, Yg, dYg, dw, s);
  else if (H <= 1024) launch_combine_bwd_waves<KB, 2>(row_of, w, T, k, H, dY, lddy, Yg, dYg, dw, s);
  else if (H <= 2048 || T >= compute_units()) launch_combine_bwd_waves<KB, 4>(row_of, w, T, k, H, dY, lddy, Yg, dYg, dw, s);
  else launch_combine_bwd_waves<KB, 8>(row_of, w, T, k, H, dY, lddy, Yg, dYg, dw, s);
}

int rows_at_once(int k) { return k <= 1 ? 1 : k <= 2 ? 2 : k <= 4 ? 4 : 8; }

}  // namespace

// 8 experts a lane: 16 lanes a token (four tokens a wave) for up to 128 experts and 16 choices, 32
// for up to 256 and 32, else 64, with 16 experts a lane past 512 (32768 tokens, us: 128 experts 7.1, 256
// in 32 lanes 11.6, in 64 22.3).
#define QF_ROUTE(KERNEL, Z, L, C, ...)                                                           \
  hipLaunchKernelGGL((KERNEL<Z, L, C>), dim3((unsigned)((T + kRouteThreads / L - 1) / (kRouteThreads / L))), \
                     dim3(kRouteThreads), 0, s, __VA_ARGS__)
#define QF_ROUTE_BY_SIZE(KERNEL, Z, ...)                            \
  do {                                                              \
    if (E <= 128 && k <= 16) QF_ROUTE(KERNEL, Z, 16, 1, __VA_ARGS__); \
    else if (E <= 256 && k <= 32) QF_ROUTE(KERNEL, Z, 32, 1, __VA_ARGS__); \
    else if (E <= 512) QF_ROUTE(KERNEL, Z, 64, 1, __VA_ARGS__);     \
    else QF_ROUTE(KERNEL, Z, 64, 2, __VA_ARGS__);                   \
  } while (0)

hipError_t launch_moe_route(const void* z, int z_f32, int64_t T, int E, int64_t ldz, int k, int score,
                            int norm, float scale, const uint8_t* mask, int32_t* ids, float* w,
                            hipStream_t s) {
  if (z_f32) QF_ROUTE_BY_SIZE(route_kernel, float, static_cast<const float*>(z), T, E, ldz, k, score, norm, scale, mask, ids, w);
  else QF_ROUTE_BY_SIZE(route_kernel, uint16_t, static_cast<const uint16_t*>(z), T, E, ldz, k, score, norm, scale, mask, ids, w);
  return hipGetLastError();
}

hipError_t launch_moe_route_bwd(const void* z, int z_f32, int64_t T, int E, int64_t ldz, int k,
                                int score, int norm, float scale, const int32_t* ids,
                                const float* dw, void* dz, int64_t lddz, hipStream_t s) {
  if (z_f32) QF_ROUTE_BY_SIZE(route_bwd_kernel, float, static_cast<const float*>(z), T, E, ldz, k, score, norm, scale, ids, dw, static_cast<float*>(dz), lddz);
  else QF_ROUTE_BY_SIZE(route_bwd_kernel, uint16_t, static_cast<const uint16_t*>(z), T, E, ldz, k, score, norm, scale, ids, dw, static_cast<uint16_t*>(dz), lddz);
  return hipGetLastError();
}

size_t moe_sort_ws_bytes(int64_t n, int64_t E) {
  const int64_t c = sort_chunk(n);
  return (size_t)((n + c - 1) / c) * (size_t)(E + 1) * sizeof(int32_t);
}

hipError_t launch_moe_sort(const int32_t* ids, int64_t T, int E, int k, int64_t* offsets,
                           int32_t* row_of, int32_t* slot_of, const uint16_t* X, int64_t H,
                           int64_t ldx, uint16_t* Xg, int32_t* ws, hipStream_t s) {
  const int64_t n = T * k, chunk = sort_chunk(n);
  if (n <= kSmallSort) {
    hipLaunchKernelGGL(sort_small_kernel, dim3((unsigned)T + 1), dim3(kSortThreads), 0, s, ids, T, E, k, offsets,
                       row_of, slot_of, X, H, ldx, Xg);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)((n + chunk - 1) / chunk));
  hipLaunchKernelGGL(sort_count_kernel, grid, dim3(kSortThreads), 0, s, ids, n, E, chunk, ws);
  hipLaunchKernelGGL(sort_rank_kernel, grid, dim3(kSortThreads), 0, s, ids, n, E, chunk, ws, offsets, row_of, slot_of);
  if (X && H > 0) {
    const int segs = (int)((H + 511) / 512);
    const dim3 rows((unsigned)((T * segs + 3) / 4)), b(256);
    if (rows_past_cache(n, H)) hipLaunchKernelGGL(gather_kernel<true>, rows, b, 0, s, row_of, T, k, H, ldx, segs, X, Xg);
    else hipLaunchKernelGGL(gather_kernel<false>, rows, b, 0, s, row_of, T, k, H, ldx, segs, X, Xg);
  }
  return hipGetLastError();
}

hipError_t launch_moe_combine(const int32_t* row_of, const float* w, int64_t T, int k, int64_t H,
                              const uint16_t* Yg, uint16_t* Y, int64_t ldy, hipStream_t s) {
  const int segs = (int)((H + 511) / 512);
  const dim3 grid((unsigned)((T * segs + 3) / 4)), b(256);
  switch (rows_at_once(k)) {
    case 1: hipLaunchKernelGGL(combine_kernel<1>, grid, b, 0, s, row_of, w, T, k, H, segs, Yg, Y, ldy); break;
    case 2: hipLaunchKernelGGL(combine_kernel<2>, grid, b, 0, s, row_of, w, T, k, H, segs, Yg, Y, ldy); break;
    case 4: hipLaunchKernelGGL(combine_kernel<4>, grid, b, 0, s, row_of, w, T, k, H, segs, Yg, Y, ldy); break;
    default: hipLaunchKernelGGL(combine_kernel<8>, grid, b, 0, s, row_of, w, T, k, H, segs, Yg, Y, ldy);
  }
  return hipGetLastError();
}

hipError_t launch_moe_combine_bwd(const int32_t* row_of, const float* w, int64_t T, int k, int64_t H,
                                  const uint16_t* dY, int64_t lddy, const uint16_t* Yg,
                                  uint16_t* dYg, float* dw, hipStream_t s) {
  switch (rows_at_once(k)) {
    case 1: launch_combine_bwd<1>(row_of, w, T, k, H, dY, lddy, Yg, dYg, dw, s); break;
    case 2: launch_combine_bwd<2>(row_of, w, T, k, H, dY, lddy, Yg, dYg, dw, s); break;
    case 4: launch_combine_bwd<4>(row_of, w, T, k, H, dY, lddy, Yg, dYg, dw, s); break;
    default: launch_combine_bwd<8>(row_of, w, T, k, H, dY, lddy, Yg, dYg, dw, s);
  }
  return hipGetLastError();
}

}  // namespace qf
