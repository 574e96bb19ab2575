// Norm and rotation of head rows, shared by the norm-and-rotation kernel and the appends to both caches.
//
// One row = one head of one token, D channels.  A row belongs to LG lanes (a power of two >= D/16); lane j holds the two
// runs of 8 channels j and j + D/16.  So every access is 16 bytes wide and a rotation pair never leaves its lane in either
// pairing ((i, i + D/2): the two runs; (2i, 2i + 1): inside a run).
//
// Every operation is rounded once and stands in a fixed order (include/fb4.h states it), so the result is the same for every grid.
#pragma once

#include <cuda_bf16.h>

#include "fb4_block.cuh"
#include "fb4_internal.h"

namespace fb4rope {

using fb4blk::lds_v4;

struct RopeTable {
  const float2* table;      // [n_pos][P] (cos, sin); NULL = no rotation
  int64_t n_pos;
  const int32_t* pos;       // [T][n_axes]
  int32_t n_axes;
  int32_t end[4];           // end[a] = first pair behind axis a
  int32_t P;
  int32_t interleaved;
};

// A lane's share of a row: first and second members of its 8 rotation pairs.  (Scalar operations: the two-wide float32
// instructions halve the arithmetic, but they want their operands in aligned register pairs, and getting them there cost
// 106 moves per row and lane, more than they saved: 117 against 99 us on 32760 tokens of 24 heads.)
struct Share {
  float a[8], b[8];
};

// From and to the two runs of 8 channels.  INTER: pairs (2i, 2i + 1); else (i, i + D/2).
template <bool INTER>
__device__ __forceinline__ void unpack(const uint4& ua, const uint4& ub, Share& x) {
  const uint32_t w[8] = {ua.x, ua.y, ua.z, ua.w, ub.x, ub.y, ub.z, ub.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
    if (INTER) {
      x.a[i] = lo;
      x.b[i] = hi;
    } else if (i < 4) {
      x.a[2 * i] = lo;
      x.a[2 * i + 1] = hi;
    } else {
      x.b[2 * i - 8] = lo;
      x.b[2 * i - 7] = hi;
    }
  }
}
template <bool INTER, typename Join>
__device__ __forceinline__ void pack(const Share& x, Join join, uint4& ua, uint4& ub) {
  if (INTER) {
    ua = make_uint4(join(x.a[0], x.b[0]), join(x.a[1], x.b[1]), join(x.a[2], x.b[2]), join(x.a[3], x.b[3]));
    ub = make_uint4(join(x.a[4], x.b[4]), join(x.a[5], x.b[5]), join(x.a[6], x.b[6]), join(x.a[7], x.b[7]));
  } else {
    ua = make_uint4(join(x.a[0], x.a[1]), join(x.a[2], x.a[3]), join(x.a[4], x.a[5]), join(x.a[6], x.a[7]));
    ub = make_uint4(join(x.b[0], x.b[1]), join(x.b[2], x.b[3]), join(x.b[4], x.b[5]), join(x.b[6], x.b[7]));
  }
}

// (v0 + v4) + (v2 + v6) + ((v1 + v5) + (v3 + v7)) of the squares.  Not fused: the square of a bf16 has 16 bits and is exact, but only
// down to 2^-149; below that the stated order rounds it before it is added.
__device__ __forceinline__ float fold8(float v0, float v1, float v2, float v3, float v4, float v5, float v6, float v7) {
  const float a = __fadd_rn(__fmul_rn(v0, v0), __fmul_rn(v4, v4)), b = __fadd_rn(__fmul_rn(v1, v1), __fmul_rn(v5, v5));
  const float c = __fadd_rn(__fmul_rn(v2, v2), __fmul_rn(v6, v6)), d = __fadd_rn(__fmul_rn(v3, v3), __fmul_rn(v7, v7));
  return __fadd_rn(__fadd_rn(a, c), __fadd_rn(b, d));
}

// Which table column and which axis each of a lane's pairs has, two neighbouring pairs ("a couple") at a time.
struct LanePairs {
  int32_t col[4];           // pairs col, col + 1
  uint32_t axis;            // 4 bits per couple: axis of the first pair | axis of the second << 2
};

template <bool INTER>
__device__ __forceinline__ LanePairs lane_pairs(const RopeTable& r, int j, int D) {
  LanePairs lp;
  lp.axis = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lp.col[i] = INTER ? 4 * j + 2 * (i & 1) + (i < 2 ? 0 : D / 4) : 8 * j + 2 * i;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t a = 0;
#pragma unroll
      for (int q = 0; q < 3; ++q) a += (q + 1 < r.n_axes && lp.col[i] + k >= r.end[q]) ? 1u : 0u;
      lp.axis |= a << (4 * i + 2 * k);
    }
  }
  return lp;
}

struct CosSin {
  float c[8], s[8];
};

// cos / sin of the lane's 8 pairs at a token's position.  A position outside the table counts as 0 and is reported.
__device__ __forceinline__ void load_cs(const RopeTable& r, const LanePairs& lp, int64_t token, CosSin& t, bool& bad) {
  const int32_t* pos = r.pos + token * r.n_axes;
  const uint32_t n = (uint32_t)r.n_pos;
  uint32_t at[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) at[i] = (uint32_t)__ldg(pos + ((lp.axis >> (4 * i)) & 3u));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t ax = (lp.axis >> (4 * i)) & 15u;
    if (at[i] >= n) { bad = true; at[i] = 0u; }
    float4 v = __ldg(reinterpret_cast<const float4*>(r.table + (int64_t)at[i] * r.P + lp.col[i]));   // P and col are even: 16-byte aligned
    if ((ax & 3u) != ax >> 2) {                // the couple straddles two axes
      uint32_t other = (uint32_t)__ldg(pos + (ax >> 2));
      if (other >= n) { bad = true; other = 0u; }
      const float2 w = __ldg(r.table + (int64_t)other * r.P + lp.col[i] + 1);
      v.z = w.x;
      v.w = w.y;
    }
    t.c[2 * i] = v.x; t.s[2 * i] = v.y; t.c[2 * i + 1] = v.z; t.s[2 * i + 1] = v.w;
  }
}

// Norm and rotation of one row; all lanes of the warp call it (the row sum goes over the LG lanes of the row).
// norm: this side has one; gain = shared address of this lane's gains, four pieces of 16 bytes LG * 16 apart
// p: eps, inv_d (1 / D) and rope
template <int LG, bool INTER, typename Params>
__device__ __forceinline__ void norm_rotate(const uint4& ua, const uint4& ub, bool norm, uint32_t gain, const Params& p,
                                            const CosSin& t, Share& x) {
  unpack<INTER>(ua, ub, x);
  if (norm) {
    float v;
    if (INTER)
      v = __fadd_rn(fold8(x.a[0], x.b[0], x.a[1], x.b[1], x.a[2], x.b[2], x.a[3], x.b[3]), fold8(x.a[4], x.b[4], x.a[5], x.b[5], x.a[6], x.b[6], x.a[7], x.b[7]));
    else
      v = __fadd_rn(fold8(x.a[0], x.a[1], x.a[2], x.a[3], x.a[4], x.a[5], x.a[6], x.a[7]), fold8(x.b[0], x.b[1], x.b[2], x.b[3], x.b[4], x.b[5], x.b[6], x.b[7]));
#pragma unroll
    for (int off = LG / 2; off; off >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, off));
    const float r = __frcp_rn(__fsqrt_rn(__fadd_rn(__fmul_rn(v, p.inv_d), p.eps)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 g = lds_v4(gain + i * (LG * 16));
      x.a[2 * i] = __fmul_rn(__fmul_rn(x.a[2 * i], r), __uint_as_float(g.x));
      x.a[2 * i + 1] = __fmul_rn(__fmul_rn(x.a[2 * i + 1], r), __uint_as_float(g.y));
      x.b[2 * i] = __fmul_rn(__fmul_rn(x.b[2 * i], r), __uint_as_float(g.z));
      x.b[2 * i + 1] = __fmul_rn(__fmul_rn(x.b[2 * i + 1], r), __uint_as_float(g.w));
    }
  }
  if (p.rope.table) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x.a[i], b = x.b[i];
      x.a[i] = __fsub_rn(__fmul_rn(a, t.c[i]), __fmul_rn(b, t.s[i]));
      x.b[i] = __fadd_rn(__fmul_rn(b, t.c[i]), __fmul_rn(a, t.s[i]));
    }
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// The gains of q and k as float32 in shared memory, in the order the lanes read them: piece i of lane j at (4 s + i) LG + j
// p: D, q.gain and k.gain
template <int LG, bool INTER, typename Params>
__device__ __forceinline__ void stage_gains(const Params& p, uint32_t gains) {
  for (int x = threadIdx.x; x < 2 * LG; x += blockDim.x) {
    const int j = x % LG, seg = x / LG;
    const uint16_t* gain = seg ? p.k.gain : p.q.gain;
    if (!gain || j >= p.D / 16) continue;
    Share g;
    unpack<INTER>(__ldg(reinterpret_cast<const uint4*>(gain + 8 * j)), __ldg(reinterpret_cast<const uint4*>(gain + 8 * j + p.D / 2)), g);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(gains + ((4 * seg + i) * LG + j) * 16), "f"(g.a[2 * i]), "f"(g.a[2 * i + 1]), "f"(g.b[2 * i]), "f"(g.b[2 * i + 1]) : "memory");
  }
}

constexpr int kGainBytes = 2 * 4 * 16 * 16;          // LG = 16

inline int lanes_of(int D) { return D <= 32 ? 2 : D <= 64 ? 4 : D <= 128 ? 8 : 16; }

inline RopeTable rope_of(const fb4_rope* rope, int D) {
  RopeTable r{};
  if (rope) {
    r.table = reinterpret_cast<const float2*>(rope->table);
    r.n_pos = rope->n_pos;
    r.pos = rope->pos;
    r.n_axes = rope->n_axes;
    r.P = D / 2;
    r.interleaved = rope->interleaved;
    int end = 0;
    for (int a = 0; a < 4; ++a) {
      if (a < rope->n_axes) end += rope->axis_pairs[a];
      r.end[a] = end;
    }
  }
  return r;
}

struct Heads {
  const uint16_t* x;
  uint16_t* out;            // NULL: the rows go to the cache
  int64_t ld, out_ld;
  const uint16_t* gain;     // NULL = no norm
  int32_t n;
};

inline Heads heads_of(const void* x, int64_t ld, int32_t n, const void* gain, void* out, int64_t out_ld) {
  Heads h;
  h.x = static_cast<const uint16_t*>(x);
  h.out = static_cast<uint16_t*>(out);
  h.ld = ld;
  h.out_ld = out_ld;
  h.gain = n > 0 ? static_cast<const uint16_t*>(gain) : nullptr;      // ignored without heads, and then not to be read
  h.n = n;
  return h;
}

}  // namespace fb4rope
