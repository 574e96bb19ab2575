// Append of keys and values to the paged 8-bit cache, and its decode.
//
// The 16 tokens of a block (16 neighbouring places of a page) share one power of two 2^e for each head, separately for K and V; a
// value is (code - 128) * 2^e.  e is the smallest with max |x| < 127.5 * 2^e, so that rounding to the nearest code never leaves
// [-127, 127].  A power of two and not the maximum over 127: a block that is filled token by token grows its scale a few times, and codes that
// are halved are off by at most one step of the last scale in all, while factors just above one would add half a step each time.
//
// Work: a CTA takes the new tokens of one block of one sequence, over all heads of K, V and Q (or a share of them, where there are few blocks).
// The tokens' cosines and sines go to shared memory once.  A warp takes the block of one head of K or V at a time (or 16 rows of Q), a few rows in
// a pass: norm and rotation, the maximum over all of them, the codes; the rows of a pass are requested during the one before.  Nobody else
// writes to a block, so there are no atomics, and the result is the same for every grid.
//
// Bound: issue and latency together (66 % of the slots, 18 warps an SM, DRAM at 40 %): 32760 tokens of 12 heads of 128 of q, k and v, 503 MB, take 139 us,
// 3.6 TB/s.  Passes one after the other, not unrolled, and the values in shared memory instead of 64 registers were 234 -> 200 us (with the
// decode of the pool, 46 us); unrolled, the three kinds of units did not stay in the instruction cache.  Groups of several blocks to a CTA cost 16 us
// of bookkeeping and saved nothing; the next unit's rows brought into L2 ahead changed nothing.
#include "fb4_attend.cuh"
#include "fb4_rope.cuh"

namespace {

using namespace fb4rope;

constexpr int kWarps = 4;
constexpr int kPlaces = 16;                // tokens of a block
constexpr int kSmem = 100 * 1024;          // of a CTA at most
constexpr int kMinByte = 58, kMaxByte = 185;

struct Append8 {
  Heads q, k, v;
  RopeTable rope;
  fb4_cache8 cache;
  int32_t D;
  float eps, inv_d;
  // which rows belong where, as in the attention
  const int32_t* page_table;
  int32_t max_pages, page_shift;
  const int32_t* kv_len;
  const int32_t* q_start;
  int32_t n_seqs, max_q, max_kv;
  int64_t total_q;
  int32_t ctas;             // > 0: CTAs per sequence; 0: the sequence is looked up (see owner)
  uint32_t* status;
};

// Sequence b owns the CTAs from q_start[b] / 16 + 2 b on: its blocks, the first of which may hold tokens already, are at most rows / 16 + 2, so
// these runs hold them, and together they are not many more than the blocks that there are.  q_start is clamped as its rows are.
__device__ __forceinline__ int64_t first_cta(const Append8& p, int32_t b) {
  const int32_t at = __ldg(p.q_start + b);
  return (at < 0 ? 0 : at < p.total_q ? at : p.total_q) / kPlaces + 2 * (int64_t)b;
}

__device__ __forceinline__ int32_t owner(const Append8& p, int64_t cta) {
  const int lane = threadIdx.x & 31;
  int32_t lo = 0, hi = p.n_seqs;           // the last b in [lo, hi) with first_cta(b) <= cta
  while (hi - lo > 1) {
    const int32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
    const uint32_t below = __ballot_sync(0xffffffffu, at < hi && first_cta(p, at) <= cta);
    const int k = below ? 31 - __clz((int)below) : 0;
    lo += k * step;
    if (lo + step < hi) hi = lo + step;
  }
  return lo;
}

// cos / sin of the block's tokens in shared memory: couple c (two pairs) of a token at this 16-byte piece of its row, so that the lanes
// that read together meet in different banks (eight lanes of one token; in heads of 64 and 32 channels the odd token's are turned by two)
__device__ __forceinline__ int cs_piece(int c) { return c ^ ((c >> 3) & 3); }
template <int LG>
__device__ __forceinline__ int cs_turn(int i) { return LG <= 4 ? (i & 1) << 1 : 0; }

__device__ __forceinline__ float top_of(const Share& x, float top) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fmaxf(fabsf(x.a[i]), fabsf(x.b[i])));
  return top;
}

// scale byte of a block whose largest magnitude is `top`: e + 127, e the smallest with top < 127.5 * 2^e
__device__ __forceinline__ int byte_of(float top) {
  const int field = (int)((__float_as_uint(top) + 0x10000u) >> 23);       // 127.5 = 255 / 128 * 2^6: the carry of the mantissa
  return min(max(field - 6, kMinByte), kMaxByte);
}

// x / 2^e as a code: the sum with 1.5 * 2^23 + 128 is rounded to an integer (ties to even), whose low byte is the code
__device__ __forceinline__ uint32_t code_bits(float x, float inv, bool clamp) {
  float y = fmaf(x, inv, 0x1.8p23f + 128.0f);
  if (clamp) y = fminf(fmaxf(y, 0x1.8p23f + 1.0f), 0x1.8p23f + 255.0f);   // beyond the largest scale only
  return __float_as_uint(y);
}

__device__ __forceinline__ uint32_t join_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// a lane's two runs of 8 channels as codes
template <bool INTER>
__device__ __forceinline__ void encode(const Share& x, float inv, bool clamp, uint2& ca, uint2& cb) {
  uint32_t a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a[i] = code_bits(x.a[i], inv, clamp);
    b[i] = code_bits(x.b[i], inv, clamp);
  }
  if (INTER) {
    ca = make_uint2(join_bytes(a[0], b[0], a[1], b[1]), join_bytes(a[2], b[2], a[3], b[3]));
    cb = make_uint2(join_bytes(a[4], b[4], a[5], b[5]), join_bytes(a[6], b[6], a[7], b[7]));
  } else {
    ca = make_uint2(join_bytes(a[0], a[1], a[2], a[3]), join_bytes(a[4], a[5], a[6], a[7]));
    cb = make_uint2(join_bytes(b[0], b[1], b[2], b[3]), join_bytes(b[4], b[5], b[6], b[7]));
  }
}

// four held codes at a scale that is 2^d times theirs
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float down) {
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = code_bits((float)(int)((w >> (8 * i)) & 255u) - 128.0f, down, false);
  return join_bytes(y[0], y[1], y[2], y[3]);
}

__device__ __forceinline__ float two_to(int byte) { return __uint_as_float((uint32_t)byte << 23); }      // 2^(byte - 127), byte >= 1

// What a warp works on at a time: the block of a head of K, V or Q, or, where fewer than 16 tokens of it are new, 16 rows of Q of several heads.
enum Kind { kK, kV, kQ, kFewQ };
struct Unit {
  int kind;
  int32_t head;
  int32_t lo, hi;           // rows of the unit that there are: places of the block, or rows lo .. hi of all (head-major: row r = head r / tokens)
};

// A lane's 16 values of a pass in shared memory, 512 bytes apart
__device__ __forceinline__ void put(uint32_t at, const Share& x) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at + i * 512), "f"(x.a[2 * i]), "f"(x.a[2 * i + 1]), "f"(x.b[2 * i]), "f"(x.b[2 * i + 1]) : "memory");
}
__device__ __forceinline__ void get(uint32_t at, Share& x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 v = fb4blk::lds_v4(at + i * 512);
    x.a[2 * i] = __uint_as_float(v.x);
    x.a[2 * i + 1] = __uint_as_float(v.y);
    x.b[2 * i] = __uint_as_float(v.z);
    x.b[2 * i + 1] = __uint_as_float(v.w);
  }
}

template <int LG, bool INTER>
__global__ void __launch_bounds__(kWarps * 32, LG == 16 ? 2 : 5) fb4_cache8_append_kernel(const __grid_constant__ Append8 p) {
  constexpr int RP = 32 / LG, NP = kPlaces / RP;      // rows of a pass, passes of a unit
  extern __shared__ __align__(16) float4 smem4[];     // the warps' values, then cosines and sines
  __shared__ __align__(16) uint8_t gain_smem[kGainBytes];
  const uint32_t gains = fb4blk::smem_u32(gain_smem);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane % LG, g = lane / LG;
  const bool on = j < p.D / 16;
  const int half = p.D / 2, couples = p.D / 4;
  const uint32_t stage = fb4blk::smem_u32(smem4) + (warp * NP * 4 * 32 + lane) * 16;      // this lane's pieces
  float4* cs_smem = smem4 + kWarps * NP * 4 * 32;

  // ---- which tokens
  int32_t b, nth;
  if (p.ctas > 0) {
    b = (int32_t)(blockIdx.x / p.ctas);
    nth = (int32_t)(blockIdx.x - (int64_t)b * p.ctas);
  } else {
    b = owner(p, blockIdx.x);
    const int64_t d = blockIdx.x - first_cta(p, b);
    nth = d < 0 || d > 0x3ffffff ? 0x3ffffff : (int32_t)d;
    // where q_start falls a sequence may have no CTA, so that the reports are dealt out by number (there are two CTAs a sequence at least)
    if (blockIdx.x < (uint32_t)p.n_seqs && blockIdx.y == 0 && threadIdx.x == 0) fb4att::sequence(p, (int32_t)blockIdx.x, true);
  }
  const fb4att::Sequence sq = fb4att::sequence(p, b, p.ctas > 0 && nth == 0 && blockIdx.y == 0 && threadIdx.x == 0);
  const int32_t first = sq.kv - sq.n_q, from = first > 0 ? first : 0;
  const int64_t base = ((int64_t)(from >> 4) + nth) << 4;                 // position of the block's first place
  if (base >= sq.kv || sq.n_q == 0) return;
  const int32_t lo = base > from ? 0 : from & 15;                         // places lo <= i < hi of the block are new
  const int32_t hi = sq.kv - base < kPlaces ? (int32_t)(sq.kv - base) : kPlaces, n_new = hi - lo;
  const int64_t row0 = sq.q0 + (base - first);                            // row of place 0 (which may be no row of the call)
  bool bad = false;

  // ---- the units of this warp
  const int32_t H = p.cache.n_heads, q_rows = n_new * p.q.n;
  const bool few = n_new < kPlaces;
  const int32_t heads = 2 * H + (few ? 0 : p.q.n);
  const int32_t units = heads + (few ? (q_rows + kPlaces - 1) / kPlaces : 0), step = gridDim.y * kWarps;
  int32_t at = blockIdx.y * kWarps + warp;
  auto unit_at = [&](int32_t u) -> Unit {             // u in [0, units)
    if (u >= heads) return Unit{kFewQ, 0, (u - heads) * kPlaces, q_rows};
    const int kind = u < H ? kK : u < 2 * H ? kV : kQ;
    return Unit{kind, u - kind * H, lo, hi};
  };
  // Is there a row for this lane in pass n?  Also its place in the block, and for kFewQ its head.
  auto row_of = [&](const Unit& u, int n, int32_t& place, int32_t& head) -> bool {
    const int32_t i = n * RP + g;
    if (u.kind != kFewQ) {
      place = i;
      return on && i >= u.lo && i < u.hi;
    }
    const bool real = on && u.lo + i < u.hi;
    head = real ? (u.lo + i) / n_new : 0;
    place = lo + (real ? u.lo + i - head * n_new : 0);
    return real;
  };
  auto any_row = [&](const Unit& u, int n) -> bool { return u.kind != kFewQ ? (n + 1) * RP > u.lo && n * RP < u.hi : u.lo + n * RP < u.hi; };
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 ra = zero, rb = zero;                         // the row of the pass to come
  const uint16_t* src = nullptr;                      // where it is, and how far the passes are apart
  int64_t src_step = 0;
  auto begin = [&](const Unit& u) {
    const Heads& hd = u.kind == kK ? p.k : u.kind == kV ? p.v : p.q;
    src = hd.x + (row0 + g) * hd.ld + (int64_t)u.head * p.D + 8 * j;
    src_step = RP * hd.ld;
  };
  auto fetch = [&](const Unit& u, int n) {
    int32_t place, head;
    ra = rb = zero;
    if (row_of(u, n, place, head)) {
      const uint16_t* x = u.kind != kFewQ ? src : p.q.x + (row0 + place) * p.q.ld + (int64_t)head * p.D + 8 * j;
      ra = *reinterpret_cast<const uint4*>(x);                            // plain loads: q_out may be q
      rb = *reinterpret_cast<const uint4*>(x + half);
    }
    src += src_step;
  };
  Unit u{};
  if (at < units) {
    u = unit_at(at);
    begin(u);
    fetch(u, 0);
  }

  stage_gains<LG, INTER>(p, gains);
  int64_t page = __ldg(p.page_table + (int64_t)b * p.max_pages + (base >> p.page_shift));
  if (page < 0 || page >= p.cache.n_pages) {
    bad = true;
    page = -1;
  }
  if (p.rope.table) {
#pragma unroll 4
    for (int x = threadIdx.x; x < n_new * couples; x += kWarps * 32) {
      const int i = lo + x / couples, c = x % couples;
      const int32_t* pos = p.rope.pos + (row0 + i) * p.rope.n_axes;
      int ax[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        ax[k] = 0;
#pragma unroll
        for (int a = 0; a < 3; ++a) ax[k] += (a + 1 < p.rope.n_axes && 2 * c + k >= p.rope.end[a]) ? 1 : 0;
      }
      uint32_t at = (uint32_t)__ldg(pos + ax[0]);
      if (at >= (uint32_t)p.rope.n_pos) { bad = true; at = 0u; }
      float4 v = __ldg(reinterpret_cast<const float4*>(p.rope.table + (int64_t)at * p.rope.P + 2 * c));
      if (ax[0] != ax[1]) {                                               // the couple straddles two axes
        at = (uint32_t)__ldg(pos + ax[1]);
        if (at >= (uint32_t)p.rope.n_pos) { bad = true; at = 0u; }
        const float2 w = __ldg(p.rope.table + (int64_t)at * p.rope.P + 2 * c + 1);
        v.z = w.x;
        v.w = w.y;
      }
      cs_smem[i * couples + (cs_piece(c) ^ cs_turn<LG>(i))] = v;
    }
  }
  __syncthreads();

  const uint32_t cs_base = fb4blk::smem_u32(cs_smem);
  uint32_t cs_at[4];                                  // this lane's couples in a token's row, counted from its start: turns exchange pieces of a row
#pragma unroll
  for (int n = 0; n < 4; ++n) cs_at[n] = cs_piece(INTER ? 2 * (on ? j : 0) + (n & 1) + (n < 2 ? 0 : p.D / 8) : 4 * (on ? j : 0) + n) * 16;
  for (; at < units; at += step) {
    uint16_t* out = nullptr;
    if (u.kind == kQ) out = p.q.out + (row0 + g) * p.q.out_ld + (int64_t)u.head * p.D + 8 * j;
    const bool more = at + step < units;
    Unit next = u;
    if (more) next = unit_at(at + step);
    float top = 0.0f;
    // One pass at a time, not unrolled: the instructions of three kinds of units would not stay in the instruction cache.  The values of K
    // and V wait in shared memory for the block's maximum.
#pragma unroll 1
    for (int n = 0; n < NP; ++n) {
      const uint4 xa = ra, xb = rb;
      if (n + 1 < NP) {
        fetch(u, n + 1);
      } else if (more) {
        begin(next);
        fetch(next, 0);
      }
      if (!any_row(u, n)) continue;
      int32_t place, head;
      const bool real = row_of(u, n, place, head);
      Share y;
      if (u.kind == kV) {
        unpack<INTER>(xa, xb, y);
      } else {
        CosSin t;
        if (p.rope.table) {
          const int32_t i = real ? place : lo;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint4 v = fb4blk::lds_v4((cs_at[k] ^ (cs_turn<LG>(i) * 16)) + (cs_base + i * couples * 16));
            t.c[2 * k] = __uint_as_float(v.x); t.s[2 * k] = __uint_as_float(v.y);
            t.c[2 * k + 1] = __uint_as_float(v.z); t.s[2 * k + 1] = __uint_as_float(v.w);
          }
        }
        norm_rotate<LG, INTER>(xa, xb, (u.kind == kK ? p.k.gain : p.q.gain) != nullptr, gains + ((u.kind == kK ? 4 * LG : 0) + j) * 16, p, t, y);
      }
      if (u.kind >= kQ) {
        uint4 qa, qb;
        pack<INTER>(y, pack_bf16, qa, qb);
        uint16_t* o = u.kind == kQ ? out + n * (RP * p.q.out_ld) : p.q.out + (row0 + place) * p.q.out_ld + (int64_t)head * p.D + 8 * j;
        if (real) {
          *reinterpret_cast<uint4*>(o) = qa;
          *reinterpret_cast<uint4*>(o + half) = qb;
        }
      } else {
        put(stage + n * 2048, y);
        if (real) top = top_of(y, top);
      }
    }
    const Unit now = u;
    u = next;
    if (now.kind >= kQ || page < 0) continue;
    // -------------------------------------------------- the block of a head of K or V: its scale and its codes
    const int64_t cell = (page * H + now.head) << p.page_shift;                                // the head's tokens in the page
    const int32_t in_page = (int32_t)(base & ((1 << p.page_shift) - 1));
    uint8_t* codes = (now.kind == kV ? p.cache.v : p.cache.k) + (cell + in_page) * p.D;
    uint8_t* scale = (now.kind == kV ? p.cache.v_scale : p.cache.k_scale) + ((cell + in_page) >> 4);
    const int held = now.lo > 0 ? min(max((int)*scale, kMinByte), kMaxByte) : kMinByte;
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    const int byte = max(byte_of(top), held);
    const float inv = two_to(254 - byte);
    const bool clamp = byte == kMaxByte;
#pragma unroll 1
    for (int n = now.lo / RP; n * RP < now.hi; ++n) {
      const int32_t i = n * RP + g;
      Share y;
      get(stage + n * 2048, y);
      uint2 ca, cb;
      encode<INTER>(y, inv, clamp, ca, cb);
      if (on && i >= now.lo && i < now.hi) {
        uint8_t* c = codes + i * p.D + 8 * j;
        *reinterpret_cast<uint2*>(c) = ca;
        *reinterpret_cast<uint2*>(c + half) = cb;
      }
    }
    if (now.lo > 0 && byte > held) {                                      // the tokens that the block holds take the new scale
      const float down = two_to(127 + held - byte);
      for (int x16 = lane; x16 < now.lo * p.D / 16; x16 += 32) {
        uint4 w = *reinterpret_cast<const uint4*>(codes + 16 * x16);
        w = make_uint4(rescaled(w.x, down), rescaled(w.y, down), rescaled(w.z, down), rescaled(w.w, down));
        *reinterpret_cast<uint4*>(codes + 16 * x16) = w;
      }
    }
    __syncwarp();
    if (lane == 0) *scale = (uint8_t)byte;
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, 2u);
}

// ---- decode: 8 codes per thread and step, K then V.  A CTA takes whole blocks, as many as 1024 pieces of 8 codes hold, so that a piece's block is
// found without a 64-bit division.  A code in the last byte of 2^23 is the number 2^23 + code, and one fused multiply-add takes it to
// (code - 128) 2^e, exactly; in bfloat16 that is the upper half of it (8 bits are enough for every code).  Bound: DRAM (32768 tokens of 12 heads of 128 to
// bfloat16: 46 us, 6.6 TB/s).
constexpr int kValuesThreads = 256, kValuesSteps = 4;

template <int DTYPE>
__global__ void __launch_bounds__(kValuesThreads) fb4_cache8_values_kernel(const uint8_t* __restrict__ k, const uint8_t* __restrict__ k_scale,
                                                                           const uint8_t* __restrict__ v, const uint8_t* __restrict__ v_scale,
                                                                           void* __restrict__ k_out, void* __restrict__ v_out, int64_t blocks,
                                                                           int32_t per_block, int32_t at_once, uint32_t inverse) {
  const bool is_v = blockIdx.y != 0;
  const int64_t block0 = (int64_t)blockIdx.x * at_once;
  const int32_t pieces = (int32_t)(blocks - block0 < at_once ? blocks - block0 : at_once) * per_block;
  const uint2* src = reinterpret_cast<const uint2*>(is_v ? v : k) + block0 * per_block;
  const uint8_t* scale = (is_v ? v_scale : k_scale) + block0;
  void* out = is_v ? v_out : k_out;
  uint2 c[kValuesSteps];
  int s[kValuesSteps];
#pragma unroll
  for (int n = 0; n < kValuesSteps; ++n) {
    const int32_t at = threadIdx.x + n * kValuesThreads;
    if (at < pieces) {
      c[n] = __ldcs(src + at);
      s[n] = __ldg(scale + __umulhi((uint32_t)at, inverse));
    }
  }
#pragma unroll
  for (int n = 0; n < kValuesSteps; ++n) {
    const int32_t at = threadIdx.x + n * kValuesThreads;
    if (at >= pieces) continue;
    const float f = two_to(min(max(s[n], kMinByte), kMaxByte)), offset = -(0x1p23f + 128.0f) * f;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(__uint_as_float(__byte_perm(i < 4 ? c[n].x : c[n].y, 0x4b000000u, 0x7650 + (i & 3))), f, offset);
    const int64_t to = block0 * per_block + at;
    if (DTYPE == 0) {
      float4* o = static_cast<float4*>(out) + 2 * to;
      o[0] = make_float4(x[0], x[1], x[2], x[3]);
      o[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (DTYPE == 1) {
          w[i] = __byte_perm(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]), 0x7632);
        } else {
          const __half2 y = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t*>(&y);
        }
      }
      static_cast<uint4*>(out)[to] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

}  // namespace

// Opt-in to the dynamic shared memory of the append kernels on the current device.
cudaError_t fb4_cache8_prepare_device() {
  cudaError_t e = cudaSuccess;
#define FB4_OPT_IN(LG) \
  if (e == cudaSuccess) e = cudaFuncSetAttribute(fb4_cache8_append_kernel<LG, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); \
  if (e == cudaSuccess) e = cudaFuncSetAttribute(fb4_cache8_append_kernel<LG, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem)
  FB4_OPT_IN(2);
  FB4_OPT_IN(4);
  FB4_OPT_IN(8);
  FB4_OPT_IN(16);
#undef FB4_OPT_IN
  return e;
}

cudaError_t fb4_launch_cache8_append(const fb4_ctx* ctx, const fb4_cache8* cache, const int32_t* page_table, int32_t max_pages,
                                     const int32_t* kv_len, const int32_t* q_start, int32_t n_seqs, int32_t max_q, const void* k,
                                     int64_t k_ld, const void* v, int64_t v_ld, int64_t T, const void* k_gain, float eps,
                                     const fb4_rope* rope, const void* q, int32_t q_heads, int64_t q_ld, const void* q_gain,
                                     void* q_out, int64_t q_out_ld, cudaStream_t stream) {
  Append8 p{};
  p.D = cache->head_dim;
  p.eps = eps;
  p.inv_d = (float)(1.0 / p.D);
  p.rope = rope_of(rope, p.D);
  p.cache = *cache;
  p.q = heads_of(q, q_ld, q_heads, q_gain, q_out, q_out_ld);
  p.k = heads_of(k, k_ld, cache->n_heads, k_gain, nullptr, 0);
  p.v = heads_of(v, v_ld, cache->n_heads, nullptr, nullptr, 0);
  p.page_table = page_table;
  p.max_pages = max_pages;
  while ((1 << p.page_shift) < cache->page_tokens) ++p.page_shift;
  p.kv_len = kv_len;
  p.q_start = q_start;
  p.n_seqs = n_seqs;
  p.max_q = max_q;
  p.max_kv = 0x7fffffff;
  p.total_q = T;
  p.status = ctx->d_status;
  const int lg = lanes_of(p.D), rows = kWarps * (kPlaces * lg / 32) * 2048, per_block = kPlaces * p.D * 4;
  const int64_t slots = (int64_t)ctx->sm_count * (lg == 16 ? 2 : 5);
  // CTAs by sequence where they are not more than by rows
  const int64_t by_seq = ((int64_t)max_q + 2 * kPlaces - 2) / kPlaces, by_rows = T / kPlaces + 2 * (int64_t)n_seqs;
  p.ctas = by_seq * n_seqs <= by_rows ? (int32_t)by_seq : 0;
  const int64_t grid = p.ctas ? by_seq * n_seqs : by_rows;
  // few blocks: their heads are shared out until every warp has one unit
  const int64_t units = 2 * cache->n_heads + q_heads, most = (units + kWarps - 1) / kWarps;
  int64_t parts = (slots + grid - 1) / grid;
  if (parts > most) parts = most;
  const dim3 dims((unsigned)grid, (unsigned)parts);
  const size_t smem = (size_t)rows + (rope ? per_block : 0);
  const bool inter = rope && rope->interleaved;
#define FB4_APPEND8(LG) \
  inter ? fb4_cache8_append_kernel<LG, true><<<dims, kWarps * 32, smem, stream>>>(p) \
        : fb4_cache8_append_kernel<LG, false><<<dims, kWarps * 32, smem, stream>>>(p)
  switch (lg) {
    case 2: FB4_APPEND8(2); break;
    case 4: FB4_APPEND8(4); break;
    case 8: FB4_APPEND8(8); break;
    default: FB4_APPEND8(16); break;
  }
#undef FB4_APPEND8
  return cudaGetLastError();
}

cudaError_t fb4_launch_cache8_values(const fb4_cache8* cache, void* k_out, void* v_out, int out_dtype, cudaStream_t stream) {
  const int64_t blocks = cache->n_pages * cache->n_heads * (cache->page_tokens / kPlaces);
  const int32_t per_block = 2 * cache->head_dim, at_once = kValuesThreads * kValuesSteps / per_block;       // 64 to 512 pieces to a block
  const dim3 grid((unsigned)((blocks + at_once - 1) / at_once), 2);
  const uint32_t inverse = (uint32_t)(0x100000000ull / per_block) + 1;         // its product's upper half is the quotient, up to 2^16
#define FB4_VALUES8(DTYPE) \
  fb4_cache8_values_kernel<DTYPE><<<grid, kValuesThreads, 0, stream>>>(cache->k, cache->k_scale, cache->v, cache->v_scale, k_out, v_out, blocks, per_block, at_once, inverse)
  if (out_dtype == 0) FB4_VALUES8(0);
  else if (out_dtype == 1) FB4_VALUES8(1);
  else FB4_VALUES8(2);
#undef FB4_VALUES8
  return cudaGetLastError();
}
