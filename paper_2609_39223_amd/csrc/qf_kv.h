// The 4-bit cache of keys and values as its kernels see it (qf_kv.hip, qf_attend.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qf {

// Pages of 2^page_log tokens: codes [pages, H, tokens, D / 2], scales [pages, H, tokens, D / block],
// S [H] (NVFP4).
struct KvCache {
  uint8_t* codes[2];                     // keys, values
  uint8_t* scales[2];
  const float* S[2];
  int64_t pages;
  int H, D, page_log, fmt;
};
// The sequences of a call: lens [B] tokens in the cache, the last off[b + 1] - off[b] of them (off
// null: one) new; their pages in table [B, cols].
struct KvSeqs {
  const int64_t* off;
  const int32_t* lens;
  const int32_t* table;
  int64_t cols, B, T;
};

hipError_t launch_kv_write(const KvCache& c, const KvSeqs& q, const uint16_t* K, int64_t ldk,
                           const uint16_t* V, int64_t ldv, hipStream_t s);
hipError_t launch_kv_read(const KvCache& c, const KvSeqs& q, uint16_t* K, int64_t ldk, uint16_t* V,
                          int64_t ldv, hipStream_t s);

struct AttendCall {
  const uint16_t* Q;
  int64_t ldq;
  uint16_t* O;
  int64_t ldo;
  float* lse;                            // [T, Hq] or null
  int64_t Hq, max_len, window;           // window 0: none
  float scale;
};
// Workspace bytes of launch_kv_attention (a function of the sizes alone).
size_t kv_attention_ws_bytes(const KvCache& c, const KvSeqs& q, const AttendCall& a);
hipError_t launch_kv_attention(const KvCache& c, const KvSeqs& q, const AttendCall& a, float* ws,
                               hipStream_t s);

}  // namespace qf
