// What the kernels over the paged caches and those of the products with FB4 weights share: sequences and masks, decoders, softmax, the output store.
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
template <typename Call>
__device__ __forceinline__ Sequence sequence(const Call& a, int32_t b, bool tell) {
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

// ---- decode of FB4 codes to packed bf16 pairs
//
// A magnitude m (0..15) enters as the byte 8 m: as the low byte of a bf16 whose high byte holds the sign alone it is the
// subnormal number m * 2^-130, and one multiplication by a power of two brings it to m * 2^(scale byte - 127) * 2^-64.
// That leaves one table permute per four elements, one permute per pair that joins magnitudes and signs, and one
// multiplication per pair on the FMA pipe; a table of bf16 magnitudes takes two permutes per four elements, a third for
// their signs and a scaled table of its own for every block.  The factor 2^-64 keeps the multiplier in range for scale
// bytes up to 188 (element scale 2^61; larger ones are read as 188) and is made good in the softmax scale and in the last
// division; a product below 2^-133, an element below 2^-69, is rounded to a multiple of that.

constexpr float kUnshift = 0x1p64f;

struct BlockScale {
  uint32_t t0, t1;          // the dialect's magnitudes, 8 m per byte
  uint32_t f;               // 2^(scale byte + 66 - 127) in both halves
};

__device__ __forceinline__ uint32_t prmt(uint32_t x, uint32_t y, uint32_t sel) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(y), "r"(sel));
  return d;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t x, uint32_t y) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(x), "r"(y));
  return d;
}

// book = shared address of the 32 dialects' magnitude bytes; use = false: every element reads as zero, whatever the
// record holds
__device__ __forceinline__ BlockScale block_scale(uint32_t meta, uint32_t book, bool use) {
  BlockScale s;
  asm("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(s.t0), "=r"(s.t1) : "r"(book + ((meta >> 5) & 0xf8u)));
  const uint32_t x = min(meta & 255u, 188u);
  s.f = use ? x * 0x00800080u + 66u * 0x00800080u : 0u;
  return s;
}

// One code word (8 channels n0..n7) -> the pairs (n0,n2) (n1,n3) (n4,n6) (n5,n7), times 2^-64
__device__ __forceinline__ void decode_word(uint32_t w, const BlockScale& s, uint32_t (&o)[4]) {
  const uint32_t sel = w & 0x77777777u;
  const uint32_t lo = prmt(s.t0, s.t1, sel), hi = prmt(s.t0, s.t1, sel >> 16);
  const uint32_t odd = w & 0x80808080u, even = (w << 4) & 0x80808080u;
  o[0] = mul_bf16x2(prmt(lo, even, 0x5240u), s.f);
  o[1] = mul_bf16x2(prmt(lo, odd, 0x5341u), s.f);
  o[2] = mul_bf16x2(prmt(hi, even, 0x7260u), s.f);
  o[3] = mul_bf16x2(prmt(hi, odd, 0x7361u), s.f);
}

// thread i of 64 writes word i of the magnitude bytes (256 bytes at book)
__device__ __forceinline__ void fill_book(uint32_t* book, const Fb4DeviceTables* t, int i) {
  book[i] = reinterpret_cast<const uint32_t*>(t->formatbook)[i] << 3;      // magnitudes are at most 15: no carry between bytes
}

// ---- decode of the 8-bit cache to packed bf16 pairs
//
// A code (0..255) as the low byte of a bf16 is the number code * 2^-133, subnormals and the first normal binade being one scale; one
// fused multiply-add takes it to (code - 128) * 2^(scale byte - 127) * 2^-64, exactly: 8 instructions per 8 elements.  Scale bytes are read as
// 58 to 185, for which every value and both constants are bf16 numbers.
struct Int8Scale {
  uint32_t f, c;            // 2^(scale byte + 69 - 127) and -128 * 2^(scale byte - 127 - 64), in both halves
};

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t x, uint32_t y, uint32_t z) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(x), "r"(y), "r"(z));
  return d;
}

// use = false: every element reads as zero
__device__ __forceinline__ Int8Scale int8_scale(uint32_t byte, bool use) {
  const uint32_t x = min(max(byte, 58u), 185u);
  return Int8Scale{use ? (x + 69u) * 0x00800080u : 0u, use ? (x - 57u) * 0x00800080u | 0x80008000u : 0u};
}

// 8 codes n0..n7 -> the pairs (n0,n2) (n1,n3) (n4,n6) (n5,n7), times 2^-64: the order of decode_word
__device__ __forceinline__ void decode_bytes(uint32_t w0, uint32_t w1, const Int8Scale& s, uint32_t (&o)[4]) {
  o[0] = fma_bf16x2(w0 & 0x00ff00ffu, s.f, s.c);
  o[1] = fma_bf16x2(prmt(w0, 0u, 0x4341u), s.f, s.c);
  o[2] = fma_bf16x2(w1 & 0x00ff00ffu, s.f, s.c);
  o[3] = fma_bf16x2(prmt(w1, 0u, 0x4341u), s.f, s.c);
}

// the warp-wide product of the kernels of few rows: 16 x 16 by 16 x 8
__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// ---- softmax
//
// Probabilities enter the second product as bf16, in both tensor-core kernels.  V needs bf16's exponent range (its block scales), and the
// two operands of a product have one type; in two bf16 pieces p would keep 16 bits, at twice the second product's instructions and twice P's
// room.  Each weight is off by at most 2^-8 of itself, as much as the rounding of a bf16 result, and the errors of a row's weights
// mostly cancel; the sum that divides is that of the unrounded ones, so lse does not see it.
// Over 8 bits the codes alone are half-precision numbers, so p could keep 11 bits with the block's power of two multiplied into it.  But these powers lie up to
// 2^127 apart, side by side, and half precision holds 2^40: with one reference for all rows, a row whose weight lies on blocks of small scales would get
// zeros.  Each row would need a second running maximum, of score plus exponent, and another multiplication for each weight for the sum that divides.
// As it is, the relative error of causal prompts in bf16 is 0.0019 against 0.0016 with weights in float32, nearly all of which is the result's rounding.
//
// The running maximum is a rounded product, score * scale; a probability takes the exact one, in one operation with the
// subtraction of the maximum.  The two differ by half a step of the maximum, which cancels between numerator and denominator as long
// as it is small: up to 2^24 it is a factor of two at most.  Beyond, the scores are multiplied first, so that the largest is the
// maximum itself (with the exact product a maximum of 2^31 gives 2^128 or 2^-128 for the very key that set it).
__device__ __forceinline__ bool beyond_fused(float m) { return fabsf(m) > 0x1p24f && m > -INFINITY; }

// Two bf16 of a query, an infinity in them turned into a NaN: every score of a query that is not finite is then NaN, and so is
// its sum (an infinity times a zero element is NaN and times others is not, and a score of -infinity would pass for a hidden one).
__device__ __forceinline__ uint32_t query_pair(uint32_t x) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %1;" : "=r"(d) : "r"(x), "r"(0u));        // x * 0 + x: x itself, or NaN
  return d;
}

// What the sum of a row's weights divides by: a row that sees nothing has sum 0 and gets zeros, one that is not finite has sum NaN.
__device__ __forceinline__ float inverse_of(float sum, float one) { return sum == 0.0f ? 0.0f : one / sum; }
__device__ __forceinline__ float lse_of(float top, float sum) { return sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2; }
// A running maximum of +infinity (a score beyond float32) has no weights: the row's sum is NaN.
__device__ __forceinline__ float finished(float sum, float m) { return m == INFINITY ? NAN : sum; }

// ---- partial results of a split call: per row (b * max_q + i) * q_heads + h and split, D sums of the second product
// (times 2^-64) and (running maximum, sum) of the softmax; the maximum in units of log2
__device__ __forceinline__ int64_t partial_row(const Fb4Attend& a, int32_t b, int32_t i, int32_t h) {
  return ((int64_t)b * a.max_q + i) * a.q_heads + h;
}
__host__ __device__ inline int64_t partial_rows(const Fb4Attend& a) { return (int64_t)a.n_seqs * a.max_q * a.q_heads; }
__device__ __forceinline__ float* partial_sums(const Fb4Attend& a, int64_t row, int32_t split, int D) {
  return a.partial + (row * a.splits + split) * D;
}
__device__ __forceinline__ float2* partial_stat(const Fb4Attend& a, int64_t row, int32_t split, int D) {
  return reinterpret_cast<float2*>(a.partial + partial_rows(a) * a.splits * D) + row * a.splits + split;
}

// griddepcontrol: a kernel launched behind this one may start; wait for the one in front to have finished
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ void store_out(const Fb4Attend& a, int64_t at, float x) {
  if (a.out_dtype == 0) static_cast<float*>(a.out)[at] = x;
  else if (a.out_dtype == 1) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(x);
  else static_cast<__half*>(a.out)[at] = __float2half_rn(x);
}

// four neighbouring channels, 16-byte (float32) or 8-byte aligned
__device__ __forceinline__ void store_out4(const Fb4Attend& a, int64_t at, const float4& v, float f) {
  if (a.out_dtype == 0) {
    *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
  } else if (a.out_dtype == 1) {
    __nv_bfloat162 p[2] = {__floats2bfloat162_rn(v.x * f, v.y * f), __floats2bfloat162_rn(v.z * f, v.w * f)};
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at) = *reinterpret_cast<uint2*>(p);
  } else {
    __half2 p[2] = {__floats2half2_rn(v.x * f, v.y * f), __floats2half2_rn(v.z * f, v.w * f)};
    *reinterpret_cast<uint2*>(static_cast<__half*>(a.out) + at) = *reinterpret_cast<uint2*>(p);
  }
}

}  // namespace fb4att
