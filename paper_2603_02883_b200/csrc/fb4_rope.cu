// Per-head RMS norm with the position rotation, and the append of keys and values to the paged FB4 cache.
//
// One row = one head of one token, D channels.  A row belongs to LG lanes (a power of two >= D/16); lane j holds the two
// runs of 8 channels j and j + D/16.  So every access is 16 bytes wide, a rotation pair never leaves its lane in either
// pairing ((i, i + D/2): the two runs; (2i, 2i + 1): inside a run), and the cosines and sines of a lane's 8 pairs stay in
// 16 registers while it walks over the heads of a token: the table is read once per token and lane instead of once per head.
//
// Every operation is rounded once and stands in a fixed order (include/fb4.h states it), so the result is the same for
// every grid; the square of a bf16 is exact in float32, which lets the first level of sums be fused multiply-adds.
//
// Both kernels stream: bytes, not instructions, bound them (about 9 instructions per element for norm and rotation against
// the 22 that fit under 4 bytes of traffic per element; the quantizer adds 9 per element on k and v).
#include <cuda_bf16.h>

#include "fb4_block.cuh"
#include "fb4_device.cuh"
#include "fb4_internal.h"

namespace {

using namespace fb4blk;

struct RopeTable {
  const float2* table;      // [n_pos][P] (cos, sin); NULL = no rotation
  int64_t n_pos;
  const int32_t* pos;       // [T][n_axes]
  int32_t n_axes;
  int32_t end[4];           // end[a] = first pair behind axis a
  int32_t P;
  int32_t interleaved;
};

struct Heads {
  const uint16_t* x;
  uint16_t* out;
  int64_t ld, out_ld;
  const uint16_t* gain;     // NULL = no norm
  int32_t n;
};

struct NormRopeParams {
  Heads seg[2];             // rows that leave as bf16: q, and k when nothing is cached
  Heads k, v;               // rows that go to the cache
  RopeTable rope;
  int64_t T;
  int32_t D;
  float eps, inv_d;
  int64_t chunk_rows[3];    // rows a warp takes at a time: seg 0, seg 1, cache rows
  const int64_t* slot;
  fb4_cache cache;
  int32_t page_shift;
  uint32_t* status;
};

// A lane's view of the rotation: which table columns it needs and on which axis each of its 8 pairs lies.
struct LanePairs {
  int32_t first[2];         // pairs first[0] .. +3 and first[1] .. +3
  uint32_t axis;            // 2 bits per pair
};

__device__ __forceinline__ LanePairs lane_pairs(const RopeTable& r, int j, int D) {
  LanePairs lp;
  lp.first[0] = r.interleaved ? 4 * j : 8 * j;
  lp.first[1] = r.interleaved ? 4 * j + D / 4 : 8 * j + 4;
  lp.axis = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int p = lp.first[i >> 2] + (i & 3);
    uint32_t a = 0;
#pragma unroll
    for (int q = 0; q < 3; ++q) a += (q + 1 < r.n_axes && p >= r.end[q]) ? 1u : 0u;
    lp.axis |= a << (2 * i);
  }
  return lp;
}

// cos / sin of the lane's 8 pairs at a token's position.  A position outside the table counts as 0 and is reported.
__device__ __forceinline__ void load_cs(const RopeTable& r, const LanePairs& lp, int64_t token, float (&c)[8], float (&s)[8],
                                        bool& bad) {
  int32_t pos[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    int32_t p = a < r.n_axes ? __ldg(r.pos + token * r.n_axes + a) : 0;
    if ((uint64_t)(int64_t)p >= (uint64_t)r.n_pos) {
      bad = true;
      p = 0;
    }
    pos[a] = p;
  }
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const uint32_t a0 = (lp.axis >> (2 * i)) & 3u, a1 = (lp.axis >> (2 * i + 2)) & 3u;
    const int32_t p0 = a0 == 0 ? pos[0] : a0 == 1 ? pos[1] : a0 == 2 ? pos[2] : pos[3];
    const int32_t p1 = a1 == 0 ? pos[0] : a1 == 1 ? pos[1] : a1 == 2 ? pos[2] : pos[3];
    const int col = lp.first[i >> 2] + (i & 3);
    const float2* row = r.table + (int64_t)p0 * r.P + col;
    if (a0 == a1) {         // P and col are even: 16-byte aligned
      const float4 v = __ldg(reinterpret_cast<const float4*>(row));
      c[i] = v.x; s[i] = v.y; c[i + 1] = v.z; s[i + 1] = v.w;
    } else {
      const float2 u = __ldg(row), w = __ldg(r.table + (int64_t)p1 * r.P + col + 1);
      c[i] = u.x; s[i] = u.y; c[i + 1] = w.x; s[i + 1] = w.y;
    }
  }
}

__device__ __forceinline__ void unpack8(const uint4& u, float* x) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

__device__ __forceinline__ float fold8(const float* x) {
  const float a = __fmaf_rn(x[4], x[4], __fmul_rn(x[0], x[0])), b = __fmaf_rn(x[5], x[5], __fmul_rn(x[1], x[1]));
  const float c = __fmaf_rn(x[6], x[6], __fmul_rn(x[2], x[2])), d = __fmaf_rn(x[7], x[7], __fmul_rn(x[3], x[3]));
  return __fadd_rn(__fadd_rn(a, c), __fadd_rn(b, d));
}

// Norm and rotation of one row; all lanes of the warp call it (the row sum goes over the LG lanes of the row).
template <int LG>
__device__ __forceinline__ void norm_rotate(const uint4& ua, const uint4& ub, bool norm, const uint4& ga, const uint4& gb,
                                            const NormRopeParams& p, const float (&c)[8], const float (&s)[8], float (&x)[16]) {
  unpack8(ua, x);
  unpack8(ub, x + 8);
  if (norm) {
    float t = __fadd_rn(fold8(x), fold8(x + 8));
#pragma unroll
    for (int off = LG / 2; off; off >>= 1) t = __fadd_rn(t, __shfl_xor_sync(0xffffffffu, t, off));
    const float r = __frcp_rn(__fsqrt_rn(__fadd_rn(__fmul_rn(t, p.inv_d), p.eps)));
    float g[16];
    unpack8(ga, g);
    unpack8(gb, g + 8);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __fmul_rn(__fmul_rn(x[i], r), g[i]);
  }
  if (p.rope.table) {
    if (p.rope.interleaved) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = x[2 * i], b = x[2 * i + 1];
        x[2 * i] = __fsub_rn(__fmul_rn(a, c[i]), __fmul_rn(b, s[i]));
        x[2 * i + 1] = __fadd_rn(__fmul_rn(b, c[i]), __fmul_rn(a, s[i]));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = x[i], b = x[8 + i];
        x[i] = __fsub_rn(__fmul_rn(a, c[i]), __fmul_rn(b, s[i]));
        x[8 + i] = __fadd_rn(__fmul_rn(b, c[i]), __fmul_rn(a, s[i]));
      }
    }
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// A position in the list of rows (token-major): advanced without divisions.
struct RowPos {
  int64_t token;
  int32_t h;
  __device__ __forceinline__ void start(int64_t row, int32_t per_token) {
    token = row / per_token;
    h = (int32_t)(row - token * per_token);
  }
  __device__ __forceinline__ void advance(int32_t rows, int32_t per_token) {
    h += rows;
    while (h >= per_token) { h -= per_token; ++token; }
  }
};

// Rows that leave as bf16.
template <int LG>
__device__ __forceinline__ void plain_rows(const NormRopeParams& p, const Heads& hs, int64_t chunk, int64_t warp, int64_t n_warps,
                                           bool& bad) {
  constexpr int RP = 32 / LG;                  // rows per pass
  const int lane = threadIdx.x & 31, j = lane % LG, g = lane / LG;
  const bool on = j < p.D / 16;
  const int64_t rows = p.T * hs.n;
  const int oa = 8 * j, ob = 8 * j + p.D / 2;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 ga = zero, gb = zero;
  if (hs.gain && on) {
    ga = __ldg(reinterpret_cast<const uint4*>(hs.gain + oa));
    gb = __ldg(reinterpret_cast<const uint4*>(hs.gain + ob));
  }
  const LanePairs lp = lane_pairs(p.rope, on ? j : 0, p.D);
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
  for (int64_t r0 = warp * chunk; r0 < rows; r0 += n_warps * chunk) {
    const int64_t r1 = r0 + chunk < rows ? r0 + chunk : rows;
    int64_t have = -1;
    RowPos at;
    at.start(r0 + g, hs.n);
    for (int64_t r = r0 + g; __any_sync(0xffffffffu, r < r1); r += 2 * RP) {
      RowPos ra = at, rb = at;
      rb.advance(RP, hs.n);
      at = rb;
      at.advance(RP, hs.n);
      const bool va = on && r < r1, vb = on && r + RP < r1;
      const uint16_t* xa = hs.x + ra.token * hs.ld + (int64_t)ra.h * p.D;
      const uint16_t* xb = hs.x + rb.token * hs.ld + (int64_t)rb.h * p.D;
      uint4 u[4] = {zero, zero, zero, zero};
      if (va) { u[0] = *reinterpret_cast<const uint4*>(xa + oa); u[1] = *reinterpret_cast<const uint4*>(xa + ob); }
      if (vb) { u[2] = *reinterpret_cast<const uint4*>(xb + oa); u[3] = *reinterpret_cast<const uint4*>(xb + ob); }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool v = k ? vb : va;
        const RowPos& rp = k ? rb : ra;
        if (p.rope.table && v && rp.token != have) {
          load_cs(p.rope, lp, rp.token, c, s, bad);
          have = rp.token;
        }
        float y[16];
        norm_rotate<LG>(u[2 * k], u[2 * k + 1], hs.gain != nullptr, ga, gb, p, c, s, y);
        if (v) {
          uint16_t* o = hs.out + rp.token * hs.out_ld + (int64_t)rp.h * p.D;
          *reinterpret_cast<uint4*>(o + oa) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
          *reinterpret_cast<uint4*>(o + ob) = make_uint4(pack_bf16(y[8], y[9]), pack_bf16(y[10], y[11]), pack_bf16(y[12], y[13]), pack_bf16(y[14], y[15]));
        }
      }
    }
  }
}

__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) {
  return prmt(__float_as_uint(lo), __float_as_uint(hi), 0x7632u);
}

// Rows that go to the cache: k heads (norm, rotation), then v heads (as they are) of every token.  The values' upper 16
// bits, all that the quantizer reads of a float32, go through shared memory (one warp's own 32 blocks at a time) from
// the 16-channels-per-lane layout to one block of 32 channels per lane.
template <int LG>
__device__ __forceinline__ void cache_rows(const NormRopeParams& p, const Tables* tb, uint32_t stage, int64_t chunk, int64_t warp,
                                           int64_t n_warps, bool& bad) {
  constexpr int RP = 32 / LG;                  // rows per pass; two passes fill the 32 lanes of the quantizer
  constexpr int NBL = LG / 2;                  // lanes of a row in the quantizer's layout
  const int lane = threadIdx.x & 31, j = lane % LG, g = lane / LG;
  const bool on = j < p.D / 16;
  const int32_t per_token = 2 * p.k.n;
  const int64_t rows = p.T * per_token;
  const int oa = 8 * j, ob = 8 * j + p.D / 2;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 ga = zero, gb = zero;
  if (p.k.gain && on) {
    ga = __ldg(reinterpret_cast<const uint4*>(p.k.gain + oa));
    gb = __ldg(reinterpret_cast<const uint4*>(p.k.gain + ob));
  }
  const LanePairs lp = lane_pairs(p.rope, on ? j : 0, p.D);
  const Lane ln = lane_state(tb);
  const int qrow = lane / NBL, qblk = lane % NBL;
  const bool qon = qblk < p.D / 32;
  const int64_t n_slots = p.cache.n_pages << p.page_shift;
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { c[i] = 1.0f; s[i] = 0.0f; }
  // run r of a row lies at 16-byte column (r & ~3) | ((r ^ r >> 2 ^ row) & 3): no bank conflicts on either side
  auto at_run = [&](int row, int run) -> uint32_t {
    return stage + (uint32_t)row * (LG * 32) + (uint32_t)(((run & ~3) | ((run ^ (run >> 2) ^ row) & 3)) * 16);
  };
  for (int64_t r0 = warp * chunk; r0 < rows; r0 += n_warps * chunk) {
    const int64_t r1 = r0 + chunk < rows ? r0 + chunk : rows;
    int64_t have = -1;
    RowPos at, qat;
    at.start(r0 + g, per_token);
    qat.start(r0 + qrow, per_token);
    for (int64_t b0 = r0; b0 < r1; b0 += 2 * RP) {
      RowPos ra = at, rb = at;
      rb.advance(RP, per_token);
      at = rb;
      at.advance(RP, per_token);
      const bool ba = b0 + g < r1, bb = b0 + g + RP < r1;
      const bool ka = ra.h < p.k.n, kb = rb.h < p.k.n;
      uint4 u[4] = {zero, zero, zero, zero};
      if (on && ba) {
        const uint16_t* x = ka ? p.k.x + ra.token * p.k.ld + (int64_t)ra.h * p.D : p.v.x + ra.token * p.v.ld + (int64_t)(ra.h - p.k.n) * p.D;
        u[0] = __ldg(reinterpret_cast<const uint4*>(x + oa));
        u[1] = __ldg(reinterpret_cast<const uint4*>(x + ob));
      }
      if (on && bb) {
        const uint16_t* x = kb ? p.k.x + rb.token * p.k.ld + (int64_t)rb.h * p.D : p.v.x + rb.token * p.v.ld + (int64_t)(rb.h - p.k.n) * p.D;
        u[2] = __ldg(reinterpret_cast<const uint4*>(x + oa));
        u[3] = __ldg(reinterpret_cast<const uint4*>(x + ob));
      }
      const bool qv = b0 + qrow < r1;
      int64_t slot = qv ? __ldg(p.slot + qat.token) : -1;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const bool key = (k ? bb : ba) && (k ? kb : ka);
        const int64_t token = k ? rb.token : ra.token;
        uint4 wa = u[2 * k], wb = u[2 * k + 1];
        if (__any_sync(0xffffffffu, key)) {    // a pass of v rows alone needs neither norm nor rotation
          if (p.rope.table && key && on && token != have) {
            load_cs(p.rope, lp, token, c, s, bad);
            have = token;
          }
          float y[16];
          norm_rotate<LG>(wa, wb, p.k.gain != nullptr, ga, gb, p, c, s, y);
          if (key) {
            wa = make_uint4(upper_halves(y[0], y[1]), upper_halves(y[2], y[3]), upper_halves(y[4], y[5]), upper_halves(y[6], y[7]));
            wb = make_uint4(upper_halves(y[8], y[9]), upper_halves(y[10], y[11]), upper_halves(y[12], y[13]), upper_halves(y[14], y[15]));
          }
        }
        if (on) {
          const int row = g + k * RP;
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at_run(row, j)), "r"(wa.x), "r"(wa.y), "r"(wa.z), "r"(wa.w) : "memory");
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at_run(row, j + p.D / 16)), "r"(wb.x), "r"(wb.y), "r"(wb.z), "r"(wb.w) : "memory");
        }
      }
      __syncwarp();
      uint32_t w[16];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint4 v = zero;
        if (qon) v = lds_v4(at_run(qrow, 4 * qblk + i));
        w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
      }
      __syncwarp();
      uint32_t cw[4], Eb[2];
      int did[2];
      quantize_packed_block<false, false, false>(w, 0xffffffffu, tb, ln.qerr_lane, ln.pair_base, 3u, 254u, cw, did, Eb);
      if (slot < -1 || slot >= n_slots) {      // reported and left out, as -1 is left out
        bad = true;
        slot = -1;
      }
      if (qon && slot >= 0) {
        const bool key = qat.h < p.k.n;
        const int head = key ? qat.h : qat.h - p.k.n;
        const int64_t row = (((slot >> p.page_shift) * p.cache.n_heads + head) << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
        uint8_t* codes = key ? p.cache.k_codes : p.cache.v_codes;
        uint16_t* meta = key ? p.cache.k_meta : p.cache.v_meta;
        *reinterpret_cast<uint4*>(codes + row * (p.D / 2) + qblk * 16) = make_uint4(cw[0], cw[1], cw[2], cw[3]);
        meta[row * (p.D / 32) + qblk] = (uint16_t)((Eb[0] - 3u) | ((uint32_t)did[0] << 8));
      }
      qat.advance(2 * RP, per_token);
    }
  }
}

constexpr int kRopeWarps = 8;
constexpr int kAppendWarps = 16;
constexpr int kStageBytes = 2048;     // two passes of 1 KB for every LG
constexpr size_t kAppendSmem = sizeof(Tables) + kAppendWarps * kStageBytes;

template <int LG>
__global__ void __launch_bounds__(kRopeWarps * 32)
fb4_norm_rope_kernel(const __grid_constant__ NormRopeParams p) {
  const int64_t warp = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5), n_warps = (int64_t)gridDim.x * kRopeWarps;
  bool bad = false;
  if (p.seg[0].n) plain_rows<LG>(p, p.seg[0], p.chunk_rows[0], warp, n_warps, bad);
  // the second segment is dealt out from the other end: a short call spreads both over different warps
  if (p.seg[1].n) plain_rows<LG>(p, p.seg[1], p.chunk_rows[1], n_warps - 1 - warp, n_warps, bad);
  if (__any_sync(0xffffffffu, bad) && (threadIdx.x & 31) == 0) atomicOr(p.status, 2u);
}

template <int LG>
__global__ void __launch_bounds__(kAppendWarps * 32)
fb4_cache_append_kernel(const __grid_constant__ NormRopeParams p, const Tables* __restrict__ g_tables) {
  extern __shared__ __align__(16) uint8_t smem[];
  Tables* tb = reinterpret_cast<Tables*>(smem);
  copy_tables(tb, g_tables);
  __syncthreads();
  const int64_t warp = (int64_t)blockIdx.x * kAppendWarps + (threadIdx.x >> 5), n_warps = (int64_t)gridDim.x * kAppendWarps;
  bool bad = false;
  cache_rows<LG>(p, tb, smem_u32(smem) + (uint32_t)sizeof(Tables) + (threadIdx.x >> 5) * kStageBytes, p.chunk_rows[2], warp, n_warps, bad);
  if (p.seg[0].n) plain_rows<LG>(p, p.seg[0], p.chunk_rows[0], n_warps - 1 - warp, n_warps, bad);
  if (__any_sync(0xffffffffu, bad) && (threadIdx.x & 31) == 0) atomicOr(p.status, 2u);
}

int lanes_of(int D) { return D <= 32 ? 2 : D <= 64 ? 4 : D <= 128 ? 8 : 16; }

// Rows a warp takes at a time: all heads of a token (the table is then read once), rounded to what a step handles,
// unless that leaves warps without work.
int64_t chunk_of(int64_t T, int32_t heads, int step, int64_t n_warps) {
  const int64_t whole = (heads + step - 1) / step * (int64_t)step;
  const int64_t fair = (T * heads + n_warps - 1) / n_warps;
  const int64_t c = (fair + step - 1) / step * step;
  return c < whole ? c : whole;
}

void fill(NormRopeParams& p, const fb4_ctx* ctx, int64_t T, int D, float eps, const fb4_rope* rope) {
  p.T = T;
  p.D = D;
  p.eps = eps;
  p.inv_d = (float)(1.0 / D);
  p.status = ctx->d_status;
  p.rope = RopeTable{};
  if (rope) {
    p.rope.table = reinterpret_cast<const float2*>(rope->table);
    p.rope.n_pos = rope->n_pos;
    p.rope.pos = rope->pos;
    p.rope.n_axes = rope->n_axes;
    p.rope.P = D / 2;
    p.rope.interleaved = rope->interleaved;
    int end = 0;
    for (int a = 0; a < 4; ++a) {
      if (a < rope->n_axes) end += rope->axis_pairs[a];
      p.rope.end[a] = end;
    }
  }
}

Heads heads_of(const void* x, int64_t ld, int32_t n, const void* gain, void* out, int64_t out_ld) {
  Heads h;
  h.x = static_cast<const uint16_t*>(x);
  h.out = static_cast<uint16_t*>(out);
  h.ld = ld;
  h.out_ld = out_ld;
  h.gain = static_cast<const uint16_t*>(gain);
  h.n = n;
  return h;
}

}  // namespace

// Opt-in to the dynamic shared memory of the append kernels on the current device.
cudaError_t fb4_rope_prepare_device() {
  cudaError_t e = cudaSuccess;
#define FB4_OPT_IN(LG) \
  if (e == cudaSuccess) e = cudaFuncSetAttribute(fb4_cache_append_kernel<LG>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kAppendSmem)
  FB4_OPT_IN(2);
  FB4_OPT_IN(4);
  FB4_OPT_IN(8);
  FB4_OPT_IN(16);
#undef FB4_OPT_IN
  return e;
}

cudaError_t fb4_launch_norm_rope(const fb4_ctx* ctx, const void* q, int32_t q_heads, int64_t q_ld, const void* k,
                                 int32_t k_heads, int64_t k_ld, int64_t T, int32_t D, const void* q_gain, const void* k_gain,
                                 float eps, const fb4_rope* rope, void* q_out, int64_t q_out_ld, void* k_out, int64_t k_out_ld,
                                 cudaStream_t stream) {
  NormRopeParams p{};
  fill(p, ctx, T, D, eps, rope);
  p.seg[0] = heads_of(q, q_ld, q_heads, q_gain, q_out, q_out_ld);
  p.seg[1] = heads_of(k, k_ld, k_heads, k_gain, k_out, k_out_ld);
  const int lg = lanes_of(D), step = 2 * (32 / lg);
  const int64_t warps = ((int64_t)T * q_heads + step - 1) / step + ((int64_t)T * k_heads + step - 1) / step;
  int64_t grid = (warps + kRopeWarps - 1) / kRopeWarps;
  const int64_t most = (int64_t)ctx->sm_count * 4;
  if (grid > most) grid = most;
  for (int i = 0; i < 2; ++i) p.chunk_rows[i] = chunk_of(T, p.seg[i].n, step, grid * kRopeWarps);
  switch (lg) {
    case 2: fb4_norm_rope_kernel<2><<<(unsigned)grid, kRopeWarps * 32, 0, stream>>>(p); break;
    case 4: fb4_norm_rope_kernel<4><<<(unsigned)grid, kRopeWarps * 32, 0, stream>>>(p); break;
    case 8: fb4_norm_rope_kernel<8><<<(unsigned)grid, kRopeWarps * 32, 0, stream>>>(p); break;
    default: fb4_norm_rope_kernel<16><<<(unsigned)grid, kRopeWarps * 32, 0, stream>>>(p); break;
  }
  return cudaGetLastError();
}

cudaError_t fb4_launch_cache_append(const fb4_ctx* ctx, const void* q, int32_t q_heads, int64_t q_ld, const void* k,
                                    int64_t k_ld, const void* v, int64_t v_ld, int64_t T, const void* q_gain,
                                    const void* k_gain, float eps, const fb4_rope* rope, const int64_t* slot,
                                    const fb4_cache* cache, void* q_out, int64_t q_out_ld, cudaStream_t stream) {
  NormRopeParams p{};
  const int D = cache->head_dim;
  fill(p, ctx, T, D, eps, rope);
  p.seg[0] = heads_of(q, q_ld, q_heads, q_gain, q_out, q_out_ld);
  p.k = heads_of(k, k_ld, cache->n_heads, k_gain, nullptr, 0);
  p.v = heads_of(v, v_ld, cache->n_heads, nullptr, nullptr, 0);
  p.slot = slot;
  p.cache = *cache;
  while ((1 << p.page_shift) < cache->page_tokens) ++p.page_shift;
  const int lg = lanes_of(D), step = 2 * (32 / lg);
  const int64_t warps = ((int64_t)T * q_heads + step - 1) / step + ((int64_t)T * 2 * cache->n_heads + step - 1) / step;
  int64_t grid = (warps + kAppendWarps - 1) / kAppendWarps;
  const int64_t most = (int64_t)ctx->sm_count * 2;
  if (grid > most) grid = most;
  p.chunk_rows[0] = chunk_of(T, q_heads, step, grid * kAppendWarps);
  p.chunk_rows[2] = chunk_of(T, 2 * cache->n_heads, step, grid * kAppendWarps);
  const Tables* tables = static_cast<const Tables*>(ctx->d_fast_tables);
#define FB4_APPEND(LG) fb4_cache_append_kernel<LG><<<(unsigned)grid, kAppendWarps * 32, kAppendSmem, stream>>>(p, tables)
  switch (lg) {
    case 2: FB4_APPEND(2); break;
    case 4: FB4_APPEND(4); break;
    case 8: FB4_APPEND(8); break;
    default: FB4_APPEND(16); break;
  }
#undef FB4_APPEND
  return cudaGetLastError();
}
