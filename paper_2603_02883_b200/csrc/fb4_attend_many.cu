// Attention of many query rows per cache head (prompts in chunks, frames, large groups) over the paged caches, FB4 and 8-bit, on the
// fifth-generation tensor cores.
//
// Work: a CTA takes one sequence, one cache head, up to 256 query rows (two tiles of 128; row r = query r / group, head
// r mod group) and one run of the cached tokens, which it walks in tiles of 128.  Its warps have fixed roles:
//   load     copies codes and metadata of K and V tiles into a ring (bulk copies, page by page)
//   decode   4 warps turn them into bf16 tiles in shared memory, 128-byte swizzled, [token][channel] for both K and V
//   scores   one warp issues S_w = Q_w K^T (both operands in shared memory, accumulator in TMEM)
//   product  one warp issues O_w += P_w V (P_w from TMEM, V read with the contracted side as the strided one)
//   softmax  4 warps per query tile, one row per thread: a row's 128 scores go from TMEM into registers at once, which
//            frees their columns; running maximum and sum in registers, P back to columns of its own
// The two query tiles take turns with one buffer of scores: while one is in its exponentials, the other's scores are
// computed, and one decoded tile serves both.  TMEM: S at column 0, P_w at 128 + 64 w, O_w at 256 + D w.  Scores and products wait
// for different things, so they are issued by different warps: one warp for both, in the best order, waited with the tensor core
// idle (359 against 342 us for the frame below; P over the scores it came from, so that a tile's next scores wait for its
// product: 376 us).  The accumulators are rescaled only when a row's maximum grows by more than 2^8.
//
// The decoder leaves channels in the order 0 2 1 3 4 6 5 7 of every eight; Q is staged in the same order (the order of the
// contracted side is free) and the result is put back in order when it is stored.
//
// Bound: the shared memory that decode and tensor core have in common.  Per 128 tokens and 256 rows (2.0 us, 3800 cycles) the
// tensor core reads 192 KB of operands from it (1536 cycles; 2048 of arithmetic), decode writes 64 KB and reads 18, P goes to
// TMEM past it: 69 % of its cycles by the counters.  The exponentials take 2048 (16 per cycle and SM), all roles issue 56 % of the
// slots.  Leaving out the decode's arithmetic (and 3/4 of its stores) gives 1.45 us, leaving out the softmax's 1.9, both 1.5.
// 1560 queries of 12 heads over 32760 tokens take 352 us a call, 890 TFLOP/s, 53 % of the measured bf16 product rate (336 to 345 us
// where a graph repeats it and the pages stay in L2).  The other pairs of figures here were each taken on one box, with the kernel as it
// stood then.
// Without gain (us for that frame and for four causal prompts of 1024 tokens, against 342 / 133): 8 decode warps, four for K and four
// for V (339 to 349 / 136); decode with the next tile's codes already in registers (375 / 141); a copy of the dialects for
// every lane of a half-warp, which ends the bank conflicts (349 / 133); the first tile's Q in TMEM and P in half the columns
// (388 / 141); two threads to a row (16 softmax warps: 507 / 171); a polynomial in place of the special function for a part of
// the columns (2.2 to 2.9 us per tile).
//
// Over 8 bits the decode is cheaper (a thread takes a token's row, its scale bytes straight from memory a tile ahead) and the same frame takes 313 us, 1005
// TFLOP/s, 62 % of the product rate; heads of 64 are bound by exponentials and the chain of a tile (four causal prompts of up to 1024 tokens, 16 heads over 4, 61
// us, 388 TFLOP/s; the longest CTA's 32 tiles are 54 of them).  A ring stage of 128 channels holds 16 KB, so there is room for two.
#include "fb4_attend.cuh"
#include "fb4_staging.cuh"
#include "fb4_tcgen05.cuh"

namespace {

using namespace fb4att;
using namespace fb4tc;
using fb4blk::smem_u32;
using fb4stage::bulk_load;
using fb4stage::mbar_expect_tx;
using fb4stage::mbar_init;

constexpr int kKeys = 128;             // tokens of a tile
constexpr int kSoftmaxWarps = 8, kDecodeWarps = 4;
constexpr int kThreads = 512;          // two warpgroups of softmax, one of decode, one whose first three warps are scores, load and product
// Registers per thread of the roles.  The block is launched with 128 for each of its 512 threads; what decode and the last
// warpgroup give back is what the softmax warps, which keep a row's 128 scores in registers, take: 2 * 200 + 72 + 40 = 4 * 128.
constexpr int kLaunchRegs = 128, kSoftmaxRegs = 200, kDecodeRegs = 72, kOtherRegs = 40;
static_assert(2 * kSoftmaxRegs + kDecodeRegs + kOtherRegs <= 4 * kLaunchRegs, "register shares of the warpgroups");
constexpr int kMaxRing = 3;
constexpr int kHave = 8;               // tiles whose page flags are kept

template <int D, bool INT8>
struct Many {
  static constexpr int kRing = INT8 && D == 128 ? 2 : kMaxRing;     // ring stages: a K or a V tile's codes and metadata each
  static constexpr int kTileBytes = kKeys * D * 2;                  // one decoded tile, or one query tile
  static constexpr int kRow = INT8 ? D : D / 2, kMetaRow = INT8 ? 0 : D / 16;   // bytes of a token's codes and metadata
  static constexpr int kCodes = kKeys * kRow, kMeta = kKeys * kMetaRow, kStage = kCodes + kMeta;
  static constexpr int kBytes = 1024 + 2 * kTileBytes + 4 * kTileBytes + kRing * kStage;
};

struct Bars {
  uint64_t ring_full[kMaxRing], ring_empty[kMaxRing];
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t q_full, s_full[2], s_free, p_half[2], p_full[2], o_done[2], drained;
};

// two float32 operations in one instruction
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(*reinterpret_cast<uint64_t*>(&d))
      : "l"(*reinterpret_cast<uint64_t*>(&x)), "l"(*reinterpret_cast<uint64_t*>(&y)), "l"(*reinterpret_cast<uint64_t*>(&z)));
  return d;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<uint64_t*>(&d))
      : "l"(*reinterpret_cast<uint64_t*>(&x)), "l"(*reinterpret_cast<uint64_t*>(&y)));
  return d;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// Byte offset of 16-byte run `run` (8 channels) of row `row` in a [128 rows][D] tile of 64-channel columns, 128-byte swizzle
__device__ __forceinline__ uint32_t swizzled(int row, int run) {
  return (uint32_t)((run >> 3) * (kKeys * 128) + row * 128 + (((run ^ row) & 7) << 4));
}

// The sequence that comes at place `place` when up to 32 of them are put in order of their caches' lengths, longest first.
__device__ __forceinline__ int32_t by_length(const Fb4Attend& a, int32_t place) {
  const int lane = threadIdx.x & 31;
  const int32_t len = lane < a.n_seqs ? __ldg(a.kv_len + lane) : 0;
  int32_t before = 0;
  for (int i = 0; i < a.n_seqs; ++i) {
    const int32_t other = __shfl_sync(0xffffffffu, len, i);
    before += other > len || (other == len && i < lane) ? 1 : 0;
  }
  return __ffs((int)__ballot_sync(0xffffffffu, lane < a.n_seqs && before == place)) - 1;
}

// Query and head (inside its cache head's group) of a row, moved forward without divisions.
struct RowAt {
  int32_t i, h;
  __device__ __forceinline__ RowAt(int32_t row, int32_t group) : i(row / group), h(row - row / group * group) {}
  __device__ __forceinline__ void advance(int32_t rows, int32_t group) {
    h += rows;
    while (h >= group) { h -= group; ++i; }
  }
};

template <int D, bool INT8>
__global__ void __launch_bounds__(kThreads, 1) fb4_attend_many_kernel(const __grid_constant__ Fb4Attend a) {
  using L = Many<D, INT8>;
  constexpr int NB = D / 32, kRing = L::kRing;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ Bars bars;
  __shared__ uint32_t book[64];
  __shared__ uint32_t have[kHave];       // per tile: bit i = its tokens 16 i .. 16 i + 15 lie in a page that exists
  __shared__ uint32_t tmem_at, dead_flag;
  const uint32_t base_smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_at = base_smem, k_at = q_at + 2 * L::kTileBytes, v_at = k_at + 2 * L::kTileBytes, ring_at = v_at + 2 * L::kTileBytes;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  volatile uint32_t* dead = &dead_flag;

  let_next_start();      // the join of the splits waits for this kernel's end by itself

  // ---- which work
  const int32_t row_tiles = (a.max_q * a.group + 255) / 256;
  int64_t id = blockIdx.x;
  const int32_t split = (int32_t)(id % a.splits);
  id /= a.splits;
  const int32_t rt = row_tiles - 1 - (int32_t)(id % row_tiles);       // under a causal mask the last rows have the most to do
  id /= row_tiles;
  const int32_t head = (int32_t)(id % a.cache.n_heads);
  int32_t b = (int32_t)(id / a.cache.n_heads);
  // CTAs start in this order, so the sequences with the longest caches come first (a few of them; many even out by themselves)
  if (a.n_seqs > 1 && a.n_seqs <= 32) b = by_length(a, b);
  const Sequence sq = sequence(a, b, threadIdx.x == 0 && split == 0 && head == 0 && rt == 0);
  const int32_t rows = sq.n_q * a.group, row0 = rt * 256;
  if (row0 >= rows) return;
  const int32_t n_rows = rows - row0 < 256 ? rows - row0 : 256;
  const Range first = visible(a, sq, row0 / a.group), last = visible(a, sq, (row0 + n_rows - 1) / a.group);
  const int32_t base = first.lo & ~(kKeys - 1);
  const int32_t all = last.hi > first.lo ? (last.hi - base + kKeys - 1) / kKeys : 0;
  const int32_t per = a.split_tiles;
  const int32_t t0 = split * per < all ? split * per : all, t1 = all - t0 < per ? all : t0 + per, n_tiles = t1 - t0;
  const int n_w = n_rows > 128 ? 2 : 1;                               // query tiles in use

  // ---- set-up
  if (threadIdx.x == 0) {
    for (int i = 0; i < kRing; ++i) { mbar_init(smem_u32(&bars.ring_full[i]), 1); mbar_init(smem_u32(&bars.ring_empty[i]), kDecodeWarps); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bars.k_full[i]), kDecodeWarps);
      mbar_init(smem_u32(&bars.k_empty[i]), 1);
      mbar_init(smem_u32(&bars.v_full[i]), kDecodeWarps);
      mbar_init(smem_u32(&bars.v_empty[i]), 1);
      mbar_init(smem_u32(&bars.s_full[i]), 1);
      mbar_init(smem_u32(&bars.p_half[i]), 4);
      mbar_init(smem_u32(&bars.p_full[i]), 4);
      mbar_init(smem_u32(&bars.o_done[i]), 1);
    }
    mbar_init(smem_u32(&bars.q_full), 4 * n_w);
    mbar_init(smem_u32(&bars.s_free), 4);
    mbar_init(smem_u32(&bars.drained), 2);
    dead_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (!INT8 && threadIdx.x >= 64 && threadIdx.x < 128) fill_book(book, a.tables, threadIdx.x - 64);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0);
  const uint32_t s_col = tmem, p_col = tmem + 128, o_col = tmem + 256;      // S at column 0, P_w at 128 + 64 w, O_w at 256 + D w

  if (warp < kSoftmaxWarps) {
    // =========================================================== softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int w = warp >> 2;
    if (w < n_w) {
      const uint32_t lanes = (uint32_t)(warp & 3) << 21;              // this warp's TMEM lanes: 32 (warp mod 4) << 16
      const uint32_t s_at = s_col + lanes, p_at = p_col + 64 * w + lanes, o_at = o_col + D * w + lanes;
      // This warp's 32 rows of Q, in the decoder's channel order, while the first tile is loaded and decoded; a negative scale is
      // taken into Q's signs (the softmax wants a positive one).  Without tiles nothing would order these writes and the other
      // warps' use of the same memory for their results.
      if (n_tiles > 0) {
        const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
        constexpr int kRuns = D / 8;
        uint4 u[kRuns];
        const int32_t r0 = row0 + 128 * w + 32 * (warp & 3) + lane / kRuns;
        RowAt at(r0 < rows ? r0 : 0, a.group);
#pragma unroll
        for (int k = 0; k < kRuns; ++k) {
          u[k] = make_uint4(0, 0, 0, 0);
          if (r0 + k * (32 / kRuns) < rows)
            u[k] = __ldg(reinterpret_cast<const uint4*>(a.q + (int64_t)(sq.q0 + at.i) * a.q_ld + (int64_t)(head * a.group + at.h) * D + lane % kRuns * 8));
          at.advance(32 / kRuns, a.group);
        }
#pragma unroll
        for (int k = 0; k < kRuns; ++k) {
          u[k] = make_uint4(query_pair(u[k].x), query_pair(u[k].y), query_pair(u[k].z), query_pair(u[k].w));
          const int x = k * 32 + lane, r32 = 32 * (warp & 3) + x / kRuns;
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(q_at + w * L::kTileBytes + swizzled(r32, x % kRuns)), "r"(prmt(u[k].x, u[k].y, 0x5410u) ^ flip),
                       "r"(prmt(u[k].x, u[k].y, 0x7632u) ^ flip), "r"(prmt(u[k].z, u[k].w, 0x5410u) ^ flip), "r"(prmt(u[k].z, u[k].w, 0x7632u) ^ flip) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.q_full));
      }
      const int32_t row = row0 + 128 * w + (warp & 3) * 32 + lane;
      const bool on = row < rows;
      const int32_t rc = on ? row : rows - 1;                         // rows behind the last are computed like it and not stored
      const Range v = visible(a, sq, rc / a.group);
      const int32_t lo_max = __reduce_max_sync(0xffffffffu, v.lo), hi_min = __reduce_min_sync(0xffffffffu, v.hi);
      // scale 0 would make 0 * -infinity of a masked score
      const float scale = fmaxf(fabsf(a.scale_log2) * kUnshift, 1e-37f);
      float m = -INFINITY;
      float2 l = make_float2(0.0f, 0.0f);                             // the sum in two halves
      bool ok = true, huge = false;                                   // huge: some row's maximum is beyond_fused
      for (int32_t t = 0; t < n_tiles; ++t) {
        ok = wait(smem_u32(&bars.s_full[w]), t & 1, dead);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        fence_after();
        const int32_t j0 = base + (t0 + t) * kKeys;
        const uint32_t here = *(volatile uint32_t*)&have[t % kHave];
        const bool whole = j0 >= lo_max && j0 + kKeys <= hi_min && here == 0xffu;
        float x[kKeys];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(s_at + 32 * c, x + 32 * c);
        tmem_wait_ld();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.s_free));            // the other tile's scores may come
        if (!whole) {
          const int32_t from = v.lo - j0, to = v.hi - j0;
#pragma unroll
          for (int i = 0; i < kKeys; ++i)
            if (i < from || i >= to || !((here >> (i >> 4)) & 1u)) x[i] = -INFINITY;
        }
        float u[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
        for (int i = 4; i < kKeys; i += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k) u[k] = i + 4 < kKeys ? fmaxf(fmaxf(u[k], x[i + k]), x[i + 4 + k]) : fmaxf(u[k], x[i + k]);
        const float top = fmaxf(fmaxf(u[0], u[1]), fmaxf(u[2], u[3])) * scale;
        if (t > 0) {                                                  // the product of tile t - 1 has read its P and left its sums
          ok = wait(smem_u32(&bars.o_done[w]), (t - 1) & 1, dead);
          if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
          fence_after();
        }
        if (__any_sync(0xffffffffu, top > m + 8.0f)) {
          const float next = fmaxf(m, top);
          const float f = next == -INFINITY ? 1.0f : exp2_approx(m - next);
          m = next;
          huge = __any_sync(0xffffffffu, beyond_fused(m));
          l.x *= f;
          l.y *= f;
          if (t > 0) {
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {                        // 16 at a time: all of the row's scores are held meanwhile
              uint32_t y[16];
              tmem_ld16(o_at + 16 * c, y);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * f);
              tmem_st16(o_at + 16 * c, y);
            }
            tmem_wait_st();
          }
        }
        if (huge) {
#pragma unroll
          for (int i = 0; i < kKeys; ++i) x[i] = __fmul_rn(x[i], scale);
        }
        const float factor = huge ? 1.0f : scale;
        const float mm = m == -INFINITY ? 0.0f : -m;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float2 e = fma2(make_float2(x[32 * c + i], x[32 * c + i + 1]), make_float2(factor, factor), make_float2(mm, mm));
            const float2 q = make_float2(exp2_approx(e.x), exp2_approx(e.y));
            l = add2(l, q);
            p[i >> 1] = pack(q.x, q.y);
          }
          tmem_st16(p_at + 16 * c, p);
          if (c == 1) {                                               // the product may start on the first 64 tokens
            tmem_wait_st();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.p_half[w]));
          }
        }
        tmem_wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.p_full[w]));
      }
      // ---- result
      const float sum = finished(l.x + l.y, m);
      if (ok && n_tiles > 0) {
        ok = wait(smem_u32(&bars.o_done[w]), (n_tiles - 1) & 1, dead);
        ok = __all_sync(0xffffffffu, ok);
        fence_after();
      }
      const float inv = inverse_of(sum, kUnshift);
      if (ok) {
        if (on) {
          const int32_t i = rc / a.group, h = head * a.group + rc % a.group;
          if (a.splits > 1) *partial_stat(a, partial_row(a, b, i, h), split, D) = make_float2(m, sum);
          else if (a.lse) a.lse[(int64_t)(sq.q0 + i) * a.q_heads + h] = lse_of(m, sum);
        }
        // The rows go through this warp's part of Q's shared memory, which nobody reads any more, so that a store covers whole rows:
        // 2 D bytes of each row at a time (all of it in 16 bits, half of it in float32).
        constexpr int kPieces = D / 8;                                // of 16 bytes
        const uint32_t stage = q_at + w * L::kTileBytes + (warp & 3) * (32 * 2 * D);
        const bool wide = a.splits > 1 || a.out_dtype == 0;
        const float f = a.splits > 1 ? 1.0f : inv;
        for (int part = 0; part < (wide ? 2 : 1); ++part) {
          const int c0 = part * (D / 2), c1 = wide ? c0 + D / 2 : D;
          for (int c = c0; c < c1; c += 32) {
            float x[32];
            if (n_tiles > 0) {
              tmem_ld32(o_at + c, x);
              tmem_wait_ld();
            } else {
#pragma unroll
              for (int k = 0; k < 32; ++k) x[k] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 32; k += 8) {                         // channel order 0 2 1 3 4 6 5 7
              const float v[8] = {x[k] * f, x[k + 2] * f, x[k + 1] * f, x[k + 3] * f, x[k + 4] * f, x[k + 6] * f, x[k + 5] * f, x[k + 7] * f};
              uint32_t o[8];
              int n16 = 1;
              if (wide) {
                n16 = 2;
#pragma unroll
                for (int q = 0; q < 8; ++q) o[q] = __float_as_uint(v[q]);
              } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) o[q] = a.out_dtype == 1 ? pack(v[2 * q], v[2 * q + 1]) : pack_half(v[2 * q], v[2 * q + 1]);
                o[4] = o[5] = o[6] = o[7] = 0u;
              }
#pragma unroll
              for (int q = 0; q < 2; ++q)
                if (q < n16) {
                  const int piece = ((c - c0 + k) / 8) * n16 + q;
                  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * (2 * D) + ((piece ^ (lane & 7)) << 4)), "r"(o[4 * q]), "r"(o[4 * q + 1]), "r"(o[4 * q + 2]), "r"(o[4 * q + 3]) : "memory");
                }
            }
          }
          __syncwarp();
          const int piece = lane % kPieces;
          int32_t r = row0 + 128 * w + 32 * (warp & 3) + lane / kPieces;
          RowAt at_row(r < rows ? r : 0, a.group);
#pragma unroll 4
          for (int it = 0; it < kPieces; ++it, r += 32 / kPieces, at_row.advance(32 / kPieces, a.group)) {
            const int r32 = it * (32 / kPieces) + lane / kPieces;
            const float rsum = __shfl_sync(0xffffffffu, sum, r32);
            const uint4 v = fb4blk::lds_v4(stage + r32 * (2 * D) + ((piece ^ (r32 & 7)) << 4));
            if (r < rows) {
              const int32_t i = at_row.i, h = head * a.group + at_row.h;
              if (a.splits > 1) {
                if (rsum != 0.0f) *reinterpret_cast<uint4*>(partial_sums(a, partial_row(a, b, i, h), split, D) + c0 + piece * 4) = v;
              } else {
                const int64_t at = (int64_t)(sq.q0 + i) * a.out_ld + (int64_t)h * D;
                if (wide) *reinterpret_cast<uint4*>(static_cast<float*>(a.out) + at + c0 + piece * 4) = v;
                else *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + at + piece * 8) = v;
              }
            }
          }
          __syncwarp();
        }
      }
    }
  } else if (warp < kSoftmaxWarps + kDecodeWarps) {
    // =========================================================== decode
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kDecodeRegs));
    const int dw = warp - kSoftmaxWarps;
    const uint32_t book_at = smem_u32(book);
    bool ok = true;
    // 8 bits: this lane's token of a tile is 32 dw + lane; its scale bytes are loaded a tile ahead, and their page two tiles ahead
    int32_t page_next = -1;
    uint32_t k_byte = 0, v_byte = 0, k_next = 0, v_next = 0;
    auto page_of = [&](int32_t t) -> int32_t {
      const int32_t j = base + (t0 + t) * kKeys + dw * 32 + (lane & 16);
      if (t >= n_tiles || j >= last.hi || j + 16 <= first.lo) return -1;      // pages in front of a window may be gone
      return __ldg(a.page_table + (int64_t)b * a.max_pages + (j >> a.page_shift));
    };
    auto scales_of = [&](int32_t t, int32_t page, uint32_t& k8, uint32_t& v8) {
      if ((uint32_t)page >= (uint64_t)a.cache.n_pages) return;                // nothing of it counts; any scale will do
      const int32_t j = base + (t0 + t) * kKeys + dw * 32 + (lane & 16);
      const int64_t at = (((int64_t)page * a.cache.n_heads + head) << (a.page_shift - 4)) + ((j & ((1 << a.page_shift) - 1)) >> 4);
      k8 = __ldg(a.k_scale + at);
      v8 = __ldg(a.v_scale + at);
    };
    if (INT8) {
      scales_of(0, page_of(0), k_next, v_next);
      page_next = page_of(1);
    }
    for (int32_t part = 0; part < 2 * n_tiles && ok; ++part) {
      const int32_t t = part >> 1;
      const bool is_v = part & 1;
      const int st = part % kRing, buf = t & 1;
      ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.ring_full[st]), (part / kRing) & 1, dead));
      if (!ok) break;
      const uint32_t codes = ring_at + st * L::kStage, meta = codes + L::kCodes;
      const uint32_t dst = (is_v ? v_at : k_at) + buf * L::kTileBytes;
      if constexpr (INT8) {
        if (!is_v) {
          k_byte = k_next;
          v_byte = v_next;
          scales_of(t + 1, page_next, k_next, v_next);
          page_next = page_of(t + 2);
        }
        // 16 channels of a row per task; which, varies with the row so that neither side has bank conflicts (a row is 128 or 64 bytes
        // of codes, and its runs of 8 channels are swizzled by the row)
        constexpr int kTasks = D / 16;
        const int row = dw * 32 + lane;
        const int mix = D == 128 ? lane & 7 : (lane & 2) | (((lane >> 1) ^ (lane >> 2)) & 1);
        uint32_t cw[kTasks][4];
#pragma unroll
        for (int k = 0; k < kTasks; ++k)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(cw[k][0]), "=r"(cw[k][1]), "=r"(cw[k][2]), "=r"(cw[k][3]) : "r"(codes + row * D + (k ^ mix) * 16));
        const Int8Scale sc = int8_scale(is_v ? v_byte : k_byte, true);          // whatever a slot that no token fills holds is finite
        if (t >= 2) ok = __all_sync(0xffffffffu, wait(smem_u32(is_v ? &bars.v_empty[buf] : &bars.k_empty[buf]), ((t >> 1) - 1) & 1, dead));
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < kTasks; ++k)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t o[4];
            decode_bytes(cw[k][2 * q], cw[k][2 * q + 1], sc, o);
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst + swizzled(row, 2 * (k ^ mix) + q)), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
          }
      } else {
      const uint32_t here = *(volatile uint32_t*)&have[t % kHave];
      const int32_t j0 = base + (t0 + t) * kKeys;
      // 32 rows and one block of each per task; the block varies with the row so that neither side has bank conflicts.  All loads
      // come first: the ring's stage is free early, and the tasks' latencies overlap.
      constexpr int kTasks = 4 * NB / kDecodeWarps;
      uint32_t cw[kTasks][4];
      uint16_t mt[kTasks];
      auto row_of = [&](int k) -> int { return ((dw + k * kDecodeWarps) & 3) * 32 + lane; };
      auto block_of = [&](int k) -> int { return NB == 4 ? (((dw + k * kDecodeWarps) >> 2) + (lane >> 1)) & 3 : (dw + k * kDecodeWarps) >> 2; };
#pragma unroll
      for (int k = 0; k < kTasks; ++k) {
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(cw[k][0]), "=r"(cw[k][1]), "=r"(cw[k][2]), "=r"(cw[k][3]) : "r"(codes + row_of(k) * (D / 2) + block_of(k) * 16));
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(mt[k]) : "r"(meta + (row_of(k) * NB + block_of(k)) * 2));
      }
      BlockScale sc[kTasks];
#pragma unroll
      for (int k = 0; k < kTasks; ++k) {
        // values behind the last token or in a page that is not there must be finite: they meet p = 0
        const bool use = !is_v || (j0 + row_of(k) < sq.kv && ((here >> (row_of(k) >> 4)) & 1u));
        sc[k] = block_scale(use ? mt[k] : 0u, book_at, use);
      }
      if (t >= 2) ok = __all_sync(0xffffffffu, wait(smem_u32(is_v ? &bars.v_empty[buf] : &bars.k_empty[buf]), ((t >> 1) - 1) & 1, dead));
      if (!ok) break;
#pragma unroll
      for (int k = 0; k < kTasks; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t o[4];
          decode_word(cw[k][q], sc[k], o);
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst + swizzled(row_of(k), 4 * block_of(k) + q)), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
        }
      }
      // The fence stands between what has been written and the tensor core's reads, and between what has been read and the next copy, which
      // takes another path than the reads
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(smem_u32(is_v ? &bars.v_full[buf] : &bars.k_full[buf]));
        mbar_arrive(smem_u32(&bars.ring_empty[st]));
      }
    }
  } else {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
  if (warp == kSoftmaxWarps + kDecodeWarps || warp == kSoftmaxWarps + kDecodeWarps + 2) {
    // =========================================================== scores, product: every lane waits, one issues
    if (n_tiles > 0) {
      constexpr uint32_t kTile16 = L::kTileBytes >> 4;
      bool ok = true;
      if (warp == kSoftmaxWarps + kDecodeWarps) {
        constexpr uint32_t id_s = instr_desc(kKeys, false);
        const uint32_t q_low = desc_low(q_at, 16), k_low = desc_low(k_at, 16);
        ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.q_full), 0, dead));
        int32_t used = 0;                                              // score tiles so far: they share a buffer
        for (int32_t t = 0; t < n_tiles && ok; ++t) {
          ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.k_full[t & 1]), (t >> 1) & 1, dead));
          for (int w = 0; w < n_w; ++w, ++used) {
            if (used > 0 && ok) ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.s_free), (used - 1) & 1, dead));
            if (!ok) break;
            fence_after();
            if (elected()) {
              const uint32_t kb = k_low + (t & 1) * kTile16, qb = q_low + w * kTile16;
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint32_t off = ((k >> 2) * (kKeys * 128) + (k & 3) * 32) >> 4;
                mma_ss(s_col, qb + off, kb + off, id_s, k > 0);
              }
              commit(smem_u32(&bars.s_full[w]));
              if (w == n_w - 1) commit(smem_u32(&bars.k_empty[t & 1]));
            }
            __syncwarp();
          }
        }
      } else {
        constexpr uint32_t id_o = instr_desc(D, true);
        const uint32_t v_low = desc_low(v_at, kKeys * 128);
        for (int32_t t = 0; t < n_tiles && ok; ++t) {
          ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.v_full[t & 1]), (t >> 1) & 1, dead));
          const uint32_t vb = v_low + (t & 1) * kTile16;
          for (int w = 0; w < n_w && ok; ++w)
#pragma unroll
            for (int part = 0; part < 2; ++part) {                     // one half of the tile's tokens each
              ok = __all_sync(0xffffffffu, wait(smem_u32(part ? &bars.p_full[w] : &bars.p_half[w]), t & 1, dead));
              if (!ok) break;
              fence_after();
              if (elected()) {
#pragma unroll
                for (int k = part * (kKeys / 32); k < (part + 1) * (kKeys / 32); ++k)
                  mma_ts(o_col + D * w, p_col + 64 * w + 8 * k, vb + k * (2048 >> 4), id_o, k > 0 || t > 0);
                if (part) {
                  commit(smem_u32(&bars.o_done[w]));
                  if (w == n_w - 1) commit(smem_u32(&bars.v_empty[t & 1]));
                }
              }
              __syncwarp();
            }
        }
      }
      // nothing of this CTA may be on the tensor core when its TMEM is given back
      if (elected()) commit(smem_u32(&bars.drained));
      uint32_t tries = 0;
      while (!mbar_try_wait(smem_u32(&bars.drained), 0) && ++tries < kSpinLimit) {}
    }
    __syncwarp();
  } else if (warp == kSoftmaxWarps + kDecodeWarps + 1) {
    // =========================================================== load
    const int pieces = a.page_shift >= 7 ? 1 : 128 >> a.page_shift;   // pages that a tile touches (its start is a multiple of 128)
    const int piece_tokens = kKeys / pieces;
    bool bad = false, ok = true;
    int32_t part = 0;
    for (int32_t t = 0; t < n_tiles && ok; ++t) {
      const int32_t j0 = base + (t0 + t) * kKeys, j = j0 + lane * piece_tokens;
      int32_t page = -1;
      if (lane < pieces && j < last.hi && j + piece_tokens > first.lo) {      // pages in front of a window may be gone
        page = __ldg(a.page_table + (int64_t)b * a.max_pages + (j >> a.page_shift));
        if ((uint32_t)page >= (uint64_t)a.cache.n_pages) { bad = true; page = -1; }
      }
      const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
      uint32_t flags = 0;
      for (int i = 0; i < 8; ++i) flags |= ((there >> (i * 16 / piece_tokens)) & 1u) << i;
      const int64_t row = (((int64_t)page * a.cache.n_heads + head) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
      for (int kv = 0; kv < 2; ++kv, ++part) {
        const int st = part % kRing;
        if (part >= kRing) ok = wait(smem_u32(&bars.ring_empty[st]), (part / kRing - 1) & 1, dead);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        const uint32_t full = smem_u32(&bars.ring_full[st]), dst = ring_at + st * L::kStage;
        if (lane == 0) {
          if (kv == 0) *(volatile uint32_t*)&have[t % kHave] = flags;
          mbar_expect_tx(full, (uint32_t)__popc(there) * piece_tokens * (L::kRow + L::kMetaRow));
        }
        __syncwarp();
        if (page >= 0) {
          bulk_load(dst + lane * piece_tokens * L::kRow, (kv ? a.cache.v_codes : a.cache.k_codes) + row * L::kRow, piece_tokens * L::kRow, full);
          if (!INT8) bulk_load(dst + L::kCodes + lane * piece_tokens * (D / 16), (kv ? a.cache.v_meta : a.cache.k_meta) + row * NB, piece_tokens * (D / 16), full);
        }
      }
    }
    if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(a.status, 2u);
    // every copy has to have landed before the CTA ends
    for (int32_t p = part > kRing ? part - kRing : 0; p < part; ++p) {
      uint32_t tries = 0;
      while (!mbar_try_wait(smem_u32(&bars.ring_full[p % kRing]), (p / kRing) & 1) && ++tries < kSpinLimit) {}
    }
  }
  }
  fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *dead) atomicOr(a.status, 1u);
  if (warp == 0) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

}  // namespace

cudaError_t fb4_attend_many_prepare_device() {
  cudaError_t e = cudaSuccess;
  // the register shares count on what the block is launched with
  auto prepare = [&](void (*kernel)(Fb4Attend), int smem) {
    cudaFuncAttributes fa{};
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&fa, kernel);
    if (e == cudaSuccess && fa.numRegs < kLaunchRegs) e = cudaErrorInvalidConfiguration;
  };
  prepare(fb4_attend_many_kernel<128, false>, Many<128, false>::kBytes);
  prepare(fb4_attend_many_kernel<64, false>, Many<64, false>::kBytes);
  prepare(fb4_attend_many_kernel<128, true>, Many<128, true>::kBytes);
  prepare(fb4_attend_many_kernel<64, true>, Many<64, true>::kBytes);
  return e;
}

cudaError_t fb4_launch_attend_many(const Fb4Attend& a, cudaStream_t stream) {
  const int64_t row_tiles = ((int64_t)a.max_q * a.group + 255) / 256;
  const int64_t grid = row_tiles * a.splits * a.cache.n_heads * a.n_seqs;
#define FB4_MANY(D, INT8) fb4_attend_many_kernel<D, INT8><<<(unsigned)grid, kThreads, Many<D, INT8>::kBytes, stream>>>(a)
  if (a.cache.head_dim == 128) {
    if (a.int8) FB4_MANY(128, true);
    else FB4_MANY(128, false);
  } else {
    if (a.int8) FB4_MANY(64, true);
    else FB4_MANY(64, false);
  }
#undef FB4_MANY
  return cudaGetLastError();
}
