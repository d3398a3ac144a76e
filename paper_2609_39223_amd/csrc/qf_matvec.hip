// Products of few rows with packed weights (QATFactory Sec. 3.4, 3.5: the weights an engine serves),
// dense or per expert: Y = X W^T with W decoded in registers on its way to the matrix cores.
//
// A workgroup takes 16 NT weight rows against up to 16 MT rows of X; its waves split K by steps and
// add their FP32 partial sums in LDS in wave order.  On v_mfma_f32_16x16x32_bf16 X is the A operand
// (lane: row lane % 16, k 8 (lane / 16) + 0..7) and W the B operand (lane: weight row lane % 16, the
// same k); any bijection of k is fine as long as both sides use it, so a lane takes 32 consecutive
// codes of its weight row (16 bytes) per step of 128 and feeds them to four MFMAs.
//   NVFP4  V s is exact in bf16 (E2M1 has 2 significant bits, E4M3 4; 2^-10 <= |V s| <= 2688), so the
//          block scale goes into the operand and the tensor scale S onto the finished sum.
//   MXFP4  V 2^p is exact in bf16.
//   Q4_K   a sub-block is one MFMA deep: P = sum (16 + q) x and X1 = sum x, 16 + q being exact in
//          bf16 and formed from a code by a shift and a mask; the sub-block adds
//          (d s6) P - (dmin m6 + 16 d s6) X1.
// Bound by reading the weight once: 0.53 to 0.56 bytes an element.
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

__device__ __forceinline__ f32x4_t mfma16(uint4 a, uint4 b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                 __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
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
};

// Work item `item` of a grouped call: expert e and rows [r0, r1) of at most `chunk`, items counted
// over the experts in order.  Every wave finds it by itself: lane l sums the chunks of its E / 64
// experts, a prefix sum over the lanes finds whose they are.  False past the last item.
__device__ __forceinline__ bool find_item(const int64_t* off, int E, int64_t R, int item, int chunk,
                                          int& e, int64_t& r0, int64_t& r1) {
  const int lane = threadIdx.x & 63, per = (E + 63) / 64, e0 = lane * per;
  int sum = 0;
  int64_t a = e0 <= E ? min(max(off[e0 <= E ? e0 : E], (int64_t)0), R) : 0;
  const int64_t first = a;
  for (int i = 0; i < per; ++i) {
    if (e0 + i >= E) break;
    const int64_t b = min(max(off[e0 + i + 1], (int64_t)0), R);
    if (b > a) sum += (int)((b - a + chunk - 1) / chunk);
    a = b;
  }
  int inc = sum;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(inc, d, 64);
    if (lane >= d) inc += o;
  }
  if (item >= __shfl(inc, 63, 64)) return false;
  const uint64_t past = __ballot(inc > item);
  const int owner = __ffsll((unsigned long long)past) - 1;
  int left = item - (inc - sum), found = 0;         // meaningful in the owner
  int64_t lo = 0, hi = 0;
  a = first;
  for (int i = 0; i < per; ++i) {
    if (e0 + i >= E) break;
    const int64_t b = min(max(off[e0 + i + 1], (int64_t)0), R);
    const int n = b > a ? (int)((b - a + chunk - 1) / chunk) : 0;
    if (left >= 0 && left < n) {
      found = e0 + i;
      lo = a + (int64_t)left * chunk;
      hi = min(lo + chunk, b);
    }
    left -= n;
    a = b;
  }
  e = __builtin_amdgcn_readfirstlane(__shfl(found, owner, 64));
  const int l = __shfl((int)lo, owner, 64), h = __shfl((int)hi, owner, 64);   // R < 2^30
  r0 = __builtin_amdgcn_readfirstlane(l);
  r1 = __builtin_amdgcn_readfirstlane(h);
  return true;
}

// ---- FP4 formats: a step is 128 deep ----------------------------------------------------------
// A lane's 32 codes and their scale bytes (NVFP4: two, MXFP4: one) for each of its NT weight rows,
// and the four A operands for each of the MT row blocks.
template <int MT, int NT>
struct Stage {
  uint4 c[NT];
  uint32_t s[NT];
  uint4 x[MT][4];
};

// ODD: K = 16 modulo 32 (NVFP4): code rows 8-byte aligned, scale rows with an odd pitch.
template <int FMT, int MT, int NT, bool ODD>
__device__ __forceinline__ void load_stage(Stage<MT, NT>& st, const uint8_t* const cp[NT],
                                           const uint8_t* const sp[NT], const uint16_t* const xp[MT],
                                           int k, int kend) {
  const bool in = k < kend, half = !ODD || k + 16 < kend;   // (kend: past every k in the full steps)
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    st.c[t] = make_uint4(0, 0, 0, 0);
    st.s[t] = 0;
    if (!in) continue;
    const uint8_t* const c = cp[t] + k / 2;
    if (ODD) {
      const uint2 a = *reinterpret_cast<const uint2*>(c);
      st.c[t].x = a.x;
      st.c[t].y = a.y;
      st.s[t] = sp[t][k / 16];
      if (half) {
        const uint2 b = *reinterpret_cast<const uint2*>(c + 8);
        st.c[t].z = b.x;
        st.c[t].w = b.y;
        st.s[t] |= (uint32_t)sp[t][k / 16 + 1] << 8;
      }
    } else {
      st.c[t] = *reinterpret_cast<const uint4*>(c);
      if (FMT == QF_FMT_NVFP4) st.s[t] = *reinterpret_cast<const uint16_t*>(sp[t] + k / 16);
      else st.s[t] = sp[t][k / 32];
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      st.x[m][i] = make_uint4(0, 0, 0, 0);
      if (in && (i < 2 || half)) st.x[m][i] = *reinterpret_cast<const uint4*>(xp[m] + k + 8 * i);
    }
}

// The B operand of 8 codes: V s (NVFP4, s FP32) or V 2^p (MXFP4, s the E8M0 code).
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

template <int FMT, int MT, int NT>
__device__ __forceinline__ void multiply_stage(const Stage<MT, NT>& st, f32x4_t acc[MT][NT]) {
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint32_t cw[4] = {st.c[t].x, st.c[t].y, st.c[t].z, st.c[t].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint4 b;
      if (FMT == QF_FMT_NVFP4) {
        const auto s = __builtin_amdgcn_cvt_pk_f32_fp8((int)st.s[t], false);
        b = decode_nvfp4(cw[i], i < 2 ? s[0] : s[1]);
      } else {
        b = decode_mxfp4(cw[i], st.s[t]);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m][t] = mfma16(st.x[m][i], b, acc[m][t]);
    }
  }
}

// ---- Q4_K: a step is one super-block of 256 ------------------------------------------------------
// Two bf16 values 16 + q of the codes at bits 4 (..) of bytes P and P + 2 of w.
template <int P, bool HIGH>
__device__ __forceinline__ uint32_t q4k_pair(uint32_t w) {
  constexpr int at = 8 * P + (HIGH ? 4 : 0);
  const uint32_t v = at < 3 ? w << (3 - at) : w >> (at - 3);
  return (v & 0x00780078u) | 0x41804180u;
}

template <int MT, int NT>
__device__ __forceinline__ void q4k_step(const uint8_t* const cp[NT], const uint16_t* const xp[MT],
                                         int sb, int g, f32x4_t acc[MT][NT]) {
  uint4 head[NT];
  uint2 c[NT][4];
  uint4 x[MT][8];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint8_t* const p = cp[t] + (int64_t)sb * 144;
    head[t] = *reinterpret_cast<const uint4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[t][i] = *reinterpret_cast<const uint2*>(p + 16 + 32 * i + 8 * g);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[m][j] = *reinterpret_cast<const uint4*>(xp[m] + sb * 256 + 32 * j + 8 * g);
  const uint4 ones = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
  const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
  float d[NT], dm[NT];
  uint32_t s6[NT][2], m6[NT][2];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    d[t] = codec::f16_value(head[t].x & 0xFFFFu);
    dm[t] = codec::f16_value(head[t].x >> 16);
    s6[t][0] = head[t].y & 0x3F3F3F3Fu;
    m6[t][0] = head[t].z & 0x3F3F3F3Fu;
    s6[t][1] = (head[t].w & 0x0F0F0F0Fu) | ((head[t].y >> 2) & 0x30303030u);
    m6[t][1] = ((head[t].w >> 4) & 0x0F0F0F0Fu) | ((head[t].z >> 2) & 0x30303030u);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint4 a[MT];
    f32x4_t x1[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {               // elements in the codes' order 0 2 | 1 3 | 4 6 | 5 7
      const uint4 v = x[m][j];
      a[m] = make_uint4(__builtin_amdgcn_perm(v.y, v.x, 0x05040100u), __builtin_amdgcn_perm(v.y, v.x, 0x07060302u),
                        __builtin_amdgcn_perm(v.w, v.z, 0x05040100u), __builtin_amdgcn_perm(v.w, v.z, 0x07060302u));
      x1[m] = mfma16(a[m], ones, zero);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint2 w = c[t][j / 2];
      const uint4 b = j % 2 == 0 ? make_uint4(q4k_pair<0, false>(w.x), q4k_pair<1, false>(w.x),
                                              q4k_pair<0, false>(w.y), q4k_pair<1, false>(w.y))
                                 : make_uint4(q4k_pair<0, true>(w.x), q4k_pair<1, true>(w.x),
                                              q4k_pair<0, true>(w.y), q4k_pair<1, true>(w.y));
      const float t1 = d[t] * (float)((s6[t][j / 4] >> (8 * (j % 4))) & 0xFFu);
      const float t2 = dm[t] * (float)((m6[t][j / 4] >> (8 * (j % 4))) & 0xFFu);
      const float u = __builtin_fmaf(16.0f, t1, t2);
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const f32x4_t p = mfma16(a[m], b, zero);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[m][t][i] += __builtin_fmaf(t1, p[i], -(u * x1[m][i]));
      }
    }
  }
}

constexpr int kMaxWaves = 8;

template <int FMT, int MT, int NT, bool ODD>
__global__ __launch_bounds__(64 * kMaxWaves) void matvec_kernel(MatvecArgs p) {
  extern __shared__ float red[];                 // [waves][MT][NT][4][64]
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, nw = blockDim.x >> 6;
  const int l16 = lane & 15, g = lane >> 4;
  const int N = (int)p.w.N, K = (int)p.w.K, tiles = (N + 16 * NT - 1) / (16 * NT);
  const int item = (int)(blockIdx.x / tiles), n0 = (int)(blockIdx.x % tiles) * 16 * NT;
  int e = 0;
  int64_t r0 = 0, r1 = p.R;
  if (p.off != nullptr && !find_item(p.off, (int)p.w.E, p.R, item, 16 * MT, e, r0, r1)) return;
  // X rows of this lane; rows that do not exist read row 0 and are not stored (or stored as zeros)
  const uint16_t* xp[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int64_t r = r0 + 16 * m + l16;
    int64_t xr = 0;
    if (r < r1) {
      xr = r;
      if (p.rows) xr = p.rows[r] < 0 ? -1 : p.rows[r] / p.rows_div;
    }
    xp[m] = p.X + (xr >= 0 && xr < p.M ? xr : 0) * p.ldx;
  }
  const int64_t rowbytes = FMT == QF_FMT_Q4K ? (int64_t)(K / 256) * 144 : K / 2;
  const int64_t rowscales = FMT == QF_FMT_NVFP4 ? K / 16 : K / 32;
  const uint8_t *cp[NT], *sp[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {                 // weight rows past N read the last one, not stored
    const int n = n0 + 16 * t + l16;
    const int64_t row = (int64_t)e * N + (n < N ? n : N - 1);
    cp[t] = p.w.codes + row * rowbytes;
    sp[t] = p.w.scales + row * rowscales;
  }
  f32x4_t acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[m][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

  if (FMT == QF_FMT_Q4K) {
    for (int sb = wv; sb < K / 256; sb += nw) q4k_step<MT, NT>(cp, xp, sb, g, acc);
  } else {
    const int full = K / 128;
    Stage<MT, NT> cur, nxt;
    int st = wv;
    if (st < full) load_stage<FMT, MT, NT, ODD>(cur, cp, sp, xp, st * 128 + 32 * g, 0x7FFFFFFF);
    while (st < full) {
      const int n = st + nw;
      if (n < full) load_stage<FMT, MT, NT, ODD>(nxt, cp, sp, xp, n * 128 + 32 * g, 0x7FFFFFFF);
      multiply_stage<FMT, MT, NT>(cur, acc);
      cur = nxt;
      st = n;
    }
    if (st == full && full * 128 < K) {          // the ragged end, by the wave whose turn it is
      load_stage<FMT, MT, NT, ODD>(cur, cp, sp, xp, full * 128 + 32 * g, K);
      multiply_stage<FMT, MT, NT>(cur, acc);
    }
  }

  const int per = MT * NT * 256;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wv * per + ((m * NT + t) * 4 + i) * 64 + lane] = acc[m][t][i];
  __syncthreads();
  const float S = FMT == QF_FMT_NVFP4 ? p.w.S[e] : 1.0f;
  for (int o = threadIdx.x; o < per; o += blockDim.x) {
    const int ln = o & 63, i = (o >> 6) & 3, mt = o >> 8, t = mt % NT, m = mt / NT;
    const int64_t r = r0 + 16 * m + 4 * (ln >> 4) + i;
    const int n = n0 + 16 * t + (ln & 15);
    if (r >= r1 || n >= N) continue;
    float s = 0.0f;
    for (int w = 0; w < nw; ++w) s += red[w * per + o];
    if (FMT == QF_FMT_NVFP4) s *= S;
    if (p.off != nullptr) {                      // an X row that does not exist counts as zeros
      const int64_t xr = p.rows ? (p.rows[r] < 0 ? -1 : p.rows[r] / p.rows_div) : r;
      if (xr < 0 || xr >= p.M) s = 0.0f;
    }
    if (p.y_f32) static_cast<float*>(p.Y)[r * p.ldy + n] = s;
    else static_cast<uint16_t*>(p.Y)[r * p.ldy + n] = (uint16_t)codec::bf16_rne(s);
  }
}

template <int FMT, int MT, int NT, bool ODD>
hipError_t launch_one(const MatvecArgs& a, int64_t items, hipStream_t s) {
  const int64_t N = a.w.N, K = a.w.K, step = FMT == QF_FMT_Q4K ? 256 : 128;
  const int nw = (int)std::max<int64_t>(1, std::min<int64_t>(kMaxWaves, (K + step - 1) / step));
  const int64_t blocks = (N + 16 * NT - 1) / (16 * NT) * items;
  if (blocks > INT32_MAX) return hipErrorInvalidValue;
  hipLaunchKernelGGL((matvec_kernel<FMT, MT, NT, ODD>), dim3((unsigned)blocks), dim3(64 * nw),
                     (size_t)nw * MT * NT * 1024, s, a);
  return hipGetLastError();
}

template <int FMT, bool ODD>
hipError_t launch_fmt(const MatvecArgs& a, int mt, int nt, int64_t items, hipStream_t s) {
  if (mt == 1 && nt == 1) return launch_one<FMT, 1, 1, ODD>(a, items, s);
  if (mt == 1) return launch_one<FMT, 1, 2, ODD>(a, items, s);
  if (mt == 2 && nt == 1) return launch_one<FMT, 2, 1, ODD>(a, items, s);
  if (mt == 2) return launch_one<FMT, 2, 2, ODD>(a, items, s);
  if (nt == 1) return launch_one<FMT, 4, 1, ODD>(a, items, s);
  return launch_one<FMT, 4, 2, ODD>(a, items, s);
}

}  // namespace

hipError_t launch_packed_matvec(const PackedOperand& w, const int64_t* off, int64_t R,
                                const int32_t* rows, int64_t rows_div, int64_t M, const uint16_t* X,
                                int64_t ldx, void* Y, int64_t ldy, int y_f32, hipStream_t s) {
  MatvecArgs a{w, X, ldx, M, Y, ldy, R, y_f32, off, rows, (int)rows_div};
  if (M == 0) a.w.K = 0;                         // no X at all: zeros
  int mt = R <= 16 ? 1 : R <= 32 ? 2 : 4;
  int64_t items = 1;
  if (off != nullptr) {
    mt = R <= 8 * w.E ? 1 : R <= 16 * w.E ? 2 : 4;
    items = std::min<int64_t>(w.E, R) + R / (16 * mt);      // sum of ceil(rows / chunk) at most
  }
  const int nt = (w.N + 31) / 32 * items >= 2 * compute_units() ? 2 : 1;
  switch (w.fmt) {
    case QF_FMT_NVFP4:
      if (w.K % 32) return launch_fmt<QF_FMT_NVFP4, true>(a, mt, nt, items, s);
      return launch_fmt<QF_FMT_NVFP4, false>(a, mt, nt, items, s);
    case QF_FMT_MXFP4: return launch_fmt<QF_FMT_MXFP4, false>(a, mt, nt, items, s);
    default: return launch_fmt<QF_FMT_Q4K, false>(a, mt, nt, items, s);
  }
}

}  // namespace qf
