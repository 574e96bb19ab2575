// What the attention kernels over the paged FB4 cache share: the sequence and mask arithmetic and the output store.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fb4_internal.h"

namespace fb4att {

constexpr float kLn2 = 0.69314718055994531f;

struct Sequence {
  int32_t q0, n_q, kv;      // first query row, query rows, cached tokens
};

// The lengths of sequence b, clamped to what the call allows; `tell`: report a value that was outside.
__device__ __forceinline__ Sequence sequence(const Fb4Attend& a, int32_t b, bool tell) {
  const int64_t s0 = __ldg(a.q_start + b), s1 = __ldg(a.q_start + b + 1), len = __ldg(a.kv_len + b);
  const int64_t q0 = s0 < 0 ? 0 : s0 < a.total_q ? s0 : a.total_q;
  int64_t q1 = s1 < q0 ? q0 : s1 < a.total_q ? s1 : a.total_q;
  if (q1 - q0 > a.max_q) q1 = q0 + a.max_q;
  const int64_t room = (int64_t)a.max_pages << a.page_shift;
  int64_t kv = len < 0 ? 0 : len < a.max_kv ? len : a.max_kv;
  if (kv > room) kv = room;
  if (tell && (q0 != s0 || q1 != s1 || kv != len)) atomicOr(a.status, 2u);
  return Sequence{(int32_t)q0, (int32_t)(q1 - q0), (int32_t)kv};
}

struct Range {
  int32_t lo, hi;           // tokens lo <= j < hi
};

// The cached tokens that query i of a sequence sees.
__device__ __forceinline__ Range visible(const Fb4Attend& a, const Sequence& s, int32_t i) {
  const int64_t pos = (int64_t)s.kv - s.n_q + i;
  int64_t hi = s.kv, lo = 0;
  if (a.causal && pos + 1 < hi) hi = pos + 1;
  if (a.window > 0 && pos - a.window + 1 > 0) lo = pos - a.window + 1;
  if (hi < 0) hi = 0;
  if (lo > hi) lo = hi;
  return Range{(int32_t)lo, (int32_t)hi};
}

__device__ __forceinline__ void store_out(const Fb4Attend& a, int64_t at, float x) {
  if (a.out_dtype == 0) static_cast<float*>(a.out)[at] = x;
  else if (a.out_dtype == 1) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(x);
  else static_cast<__half*>(a.out)[at] = __float2half_rn(x);
}

}  // namespace fb4att
