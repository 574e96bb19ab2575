// Attention of few query rows per cache head (single tokens, drafted tokens, small groups) over the paged caches, FB4 and 8-bit.
//
// Work: a CTA of 4 warps takes one sequence, one cache head, up to 8 * NT query rows (query-major: row r = query r / group,
// head r mod group) and one run of the cached tokens (a "split"); its warps take that run's tiles of 32 tokens in turn.  Each warp
// has its own ring of asynchronously copied tiles (codes and metadata of K and V), its own running maximum and sum, and its
// own accumulators; the warps are joined in shared memory at the end, up to 8 splits in that of their cluster, more in a second
// small kernel.
//
// The tokens are the long side, so they are the M side of the products: S^T = K Q^T (m = 16 tokens, n = 8 queries),
// O^T = V^T P^T (m = 16 channels, n = 8 queries), mma.sync m16n8k16: with one query per head 7/8 of the N side is idle, but a
// step reads every cached value once and costs 16 mma per 16 tokens.  A lane decodes a quarter of a token's channels from one 16-byte word of
// codes with one metadata record, straight into the A fragment of the first product (which channel sits at which k is
// free, as long as Q agrees); V goes through movmatrix once, because there the tokens are the contracted side.
//
// Bound: the chain of a tile and the instructions in it, neither at its limit.  Scores, maximum, exponentials and product of a tile
// follow one another in each of the 16 warps of an SM; a warp issues 464 instructions for 16 tokens of 128 channels (K and V; 311 are the
// decode and the products), 60 % of the issue slots and of the ALU pipe's.  75600 tokens of 12 heads take 51 us, 2.55 TB/s of the cache's
// 4.5 bits per value, 39 % of the copy bandwidth.  More warps at fewer registers (20 or 24 instead of 16 per SM) came out slower, and so
// did the same work on tcgen05 (K decoded into tensor memory, V into a swizzled tile, roles by warp: 61 us).
//
// Over 8 bits a tile's codes are twice as many bytes and their decode is 8 instructions per 8 values instead of 14, without metadata in the ring (a tile has two
// scale bytes for each of K and V): 75600 tokens of 12 heads take 48 us, 4.8 TB/s, 64 sequences of 131 to 8191 tokens 101 us, 5.4 TB/s (74 and 83 % of the copy
// bandwidth; issue 44 to 49 %, 12 warps an SM at 156 registers).
#include "fb4_attend.cuh"
#include "fb4_block.cuh"

namespace {

using namespace fb4att;
constexpr int kWarpsFew = 4;
constexpr int kTile = 32;              // tokens of a warp's tile

template <int D, bool INT8>
struct Few {
  static constexpr int kStagesFew = D == 128 ? 2 : INT8 ? 3 : 4;
  static constexpr int kRow = INT8 ? D : D / 2;                            // bytes of a token's codes
  static constexpr int kCodes = kTile * kRow, kMeta = INT8 ? 0 : kTile * (D / 32) * 2;
  static constexpr int kStage = 2 * kCodes + 2 * kMeta;
  static constexpr int kRing = kWarpsFew * kStagesFew * kStage;
  // the join of the warps reuses the ring: 16 rows of D sums per warp, and once more for their sum
  static constexpr int kJoin = (kWarpsFew + 1) * 16 * D * 4;
  static constexpr int kBytes = (kRing > kJoin ? kRing : kJoin);
};

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
  return d;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// 16 bytes to shared memory past L1; there = false: zeros, and nothing is read.  (Bulk copies would want one lane's
// uniform registers for each: four of them per tile cost more instructions than the nine of these.)
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
}

// CTAs per SM: registers, or with the 8-bit cache and D = 128 the ring (64 KB a CTA)
constexpr int resident(int D, int NT, bool int8) { return NT == 1 && !(int8 && D == 128) ? 4 : 3; }

template <int D, int NT, bool CLUSTER, bool INT8>
__global__ void __launch_bounds__(kWarpsFew * 32, resident(D, NT, INT8)) fb4_attend_few_kernel(const __grid_constant__ Fb4Attend a) {
  using L = Few<D, INT8>;
  constexpr int NW = D / 32;             // code words of a lane's quarter row
  constexpr int ST = L::kStagesFew;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t book[64];
  __shared__ float2 stat[kWarpsFew][8 * NT], own[8 * NT];
  if (!CLUSTER) let_next_start();        // the join of the splits waits for this kernel's end by itself
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int32_t row_tiles = (a.max_q * a.group + 8 * NT - 1) / (8 * NT);

  int64_t id = blockIdx.x;
  const int32_t split = (int32_t)(id % a.splits);
  id /= a.splits;
  const int32_t head = (int32_t)(id % a.cache.n_heads);
  id /= a.cache.n_heads;
  const int32_t row0 = (int32_t)(id % row_tiles) * 8 * NT, b = (int32_t)(id / row_tiles);

  const Sequence sq = sequence(a, b, threadIdx.x == 0 && split == 0 && head == 0 && row0 == 0);
  const int32_t rows = sq.n_q * a.group;
  if (row0 >= rows) return;
  const int32_t n_rows = rows - row0 < 8 * NT ? rows - row0 : 8 * NT;
  // what any of these rows sees, cut into tiles from its first token's multiple of 32
  const Range first = visible(a, sq, row0 / a.group), last = visible(a, sq, (row0 + n_rows - 1) / a.group);
  const int32_t base = first.lo & ~(kTile - 1);
  const int32_t tiles = last.hi > base && last.hi > first.lo ? (last.hi - base + kTile - 1) / kTile : 0;
  // the tiles are dealt out evenly over the splits, in rounds of one tile per warp
  const int32_t rounds = (tiles + kWarpsFew - 1) / kWarpsFew;
  const int32_t tile0 = (int32_t)((int64_t)rounds * split / a.splits) * kWarpsFew;
  const int32_t end = (int32_t)((int64_t)rounds * (split + 1) / a.splits) * kWarpsFew, tile1 = end < tiles ? end : tiles;

  if (!INT8) {
    if (threadIdx.x < 64) fill_book(book, a.tables, threadIdx.x);
    __syncthreads();
  }
  const uint32_t ring = fb4blk::smem_u32(smem) + warp * ST * L::kStage;
  const uint32_t book_at = fb4blk::smem_u32(book);

  // the pages of this warp's tiles: lane l holds those of tile `batch + l` (two halves of 16 tokens; equal in pages of 32 or more)
  const int32_t n_mine = tile0 + warp >= tile1 ? 0 : (tile1 - tile0 - warp + kWarpsFew - 1) / kWarpsFew;
  const int32_t my0 = tile0 + warp;
  int32_t page_lo = -1, page_hi = -1;
  uint32_t scales = 0;                     // 8 bits: the scale bytes of K (first half, second half) and V
  bool bad = false;
  auto fetch_pages = [&](int32_t from) {
    page_lo = page_hi = -1;
    if (from + lane < n_mine) {
      const int32_t j = base + (my0 + (from + lane) * kWarpsFew) * kTile;
      const int32_t* pt = a.page_table + (int64_t)b * a.max_pages;
      // only halves that some row sees are read: pages in front of a window may be gone
      const bool lo_seen = j < last.hi && j + 16 > first.lo, hi_seen = j + 16 < last.hi && j + 32 > first.lo;
      if (lo_seen) page_lo = __ldg(pt + (j >> a.page_shift));
      if (hi_seen) page_hi = __ldg(pt + ((j + 16) >> a.page_shift));
      if (lo_seen && (uint32_t)page_lo >= (uint64_t)a.cache.n_pages) { bad = true; page_lo = -1; }
      if (hi_seen && (uint32_t)page_hi >= (uint64_t)a.cache.n_pages) { bad = true; page_hi = -1; }
      if constexpr (INT8) {
        auto byte_at = [&](int32_t page, int32_t jj) -> int64_t {
          return (((int64_t)page * a.cache.n_heads + head) << (a.page_shift - 4)) + ((jj & ((1 << a.page_shift) - 1)) >> 4);
        };
        scales = 0;
        if (page_lo >= 0) scales = (uint32_t)__ldg(a.k_scale + byte_at(page_lo, j)) | (uint32_t)__ldg(a.v_scale + byte_at(page_lo, j)) << 16;
        if (page_hi >= 0) scales |= (uint32_t)__ldg(a.k_scale + byte_at(page_hi, j + 16)) << 8 | (uint32_t)__ldg(a.v_scale + byte_at(page_hi, j + 16)) << 24;
      }
    }
  };
  // Requests tile n of this warp into ring stage `st`.  Codes: lane l copies bytes 16 l .. 16 l + 15 of every 512; metadata:
  // K in lanes 0 to 15, V behind, each half of the tile in 8 (D = 128) or 4 of them.  `have`: 2 bits per stage, the halves whose
  // pages exist.  8 bits: returns the tile's scale bytes; the 16-byte pieces of odd rows of 128 are exchanged in pairs, so that the two rows
  // that eight lanes read together lie in different banks.
  uint32_t have = 0;
  const uint32_t page_mask = (1u << a.page_shift) - 1u;
  const int mh = (lane / (D / 16)) & 1, mv = lane / (D / 8);          // half and array of this lane's piece of the metadata
  const uint8_t* meta_src = reinterpret_cast<const uint8_t*>(mv ? a.cache.v_meta : a.cache.k_meta) + (lane & (D / 16 - 1)) * 16;
  const uint32_t meta_dst = 2 * L::kCodes + mv * L::kMeta + mh * (L::kMeta / 2) + (lane & (D / 16 - 1)) * 16;
  const uint32_t lane_dst = (lane * 16) ^ (INT8 && D == 128 ? (lane & 8) << 1 : 0);
  auto request = [&](int32_t n, int st) -> uint32_t {
    uint32_t sc = 0;
    if (n < n_mine) {
      if ((n & 31) == 0) fetch_pages(n);
      const int32_t plo = __shfl_sync(0xffffffffu, page_lo, n & 31), phi = __shfl_sync(0xffffffffu, page_hi, n & 31);
      have = (have & ~(3u << (2 * st))) | ((plo >= 0 ? 1u : 0u) | (phi >= 0 ? 2u : 0u)) << (2 * st);
      const uint32_t dst = ring + st * L::kStage;
      const uint32_t j = (uint32_t)(base + (my0 + n * kWarpsFew) * kTile);
      const int64_t rlo = (((int64_t)max(plo, 0) * a.cache.n_heads + head) << a.page_shift) + (j & page_mask);
      const int64_t rhi = (((int64_t)max(phi, 0) * a.cache.n_heads + head) << a.page_shift) + ((j + 16) & page_mask);
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const uint8_t* codes = (v ? a.cache.v_codes : a.cache.k_codes) + lane * 16;
#pragma unroll
        for (int i = 0; i < L::kCodes / 2; i += 512) {
          copy16(dst + v * L::kCodes + i + lane_dst, codes + rlo * L::kRow + i, plo >= 0);
          copy16(dst + v * L::kCodes + L::kCodes / 2 + i + lane_dst, codes + rhi * L::kRow + i, phi >= 0);
        }
      }
      if (INT8) sc = __shfl_sync(0xffffffffu, scales, n & 31);
      else if (D == 128 || lane < 16) copy16(dst + meta_dst, meta_src + (mh ? rhi : rlo) * (D / 16), (mh ? phi : plo) >= 0);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");               // empty behind the last tile: the count of groups stays
    return sc;
  };
  uint32_t sc[ST];                         // 8 bits: scale bytes of the tiles from the present one on
#pragma unroll
  for (int n = 0; n < ST - 1; ++n) sc[n] = request(n, n);

  // Q as the B side of S^T = K Q^T: lane (g, t) holds query row0 + 8 nt + g, channels of quarter t
  uint32_t qf[NT][NW][4];
  int32_t lo[NT][2], hi[NT][2];            // what the two queries of this lane's accumulator columns see
  int32_t lo_max = 0, hi_min = 0x7fffffff;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int32_t r = row0 + 8 * nt + g;
    const bool on = r < rows;
    // a negative scale goes into Q's signs: the running maximum wants a positive one
    const uint32_t flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
    const uint16_t* src = a.q + (int64_t)(sq.q0 + (on ? r / a.group : 0)) * a.q_ld + (int64_t)(head * a.group + (on ? r % a.group : 0)) * D + t * (D / 4);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (on) u = __ldg(reinterpret_cast<const uint4*>(src + 8 * w));
      u = make_uint4(query_pair(u.x), query_pair(u.y), query_pair(u.z), query_pair(u.w));
      qf[nt][w][0] = prmt(u.x, u.y, 0x5410u) ^ flip;
      qf[nt][w][1] = prmt(u.x, u.y, 0x7632u) ^ flip;
      qf[nt][w][2] = prmt(u.z, u.w, 0x5410u) ^ flip;
      qf[nt][w][3] = prmt(u.z, u.w, 0x7632u) ^ flip;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {          // rows behind the last one are computed like the last one and not stored
      const int32_t rc = row0 + 8 * nt + 2 * t + k < rows ? row0 + 8 * nt + 2 * t + k : rows - 1;
      const Range v = visible(a, sq, rc / a.group);
      lo[nt][k] = v.lo;
      hi[nt][k] = v.hi;
      lo_max = max(lo_max, v.lo);
      hi_min = min(hi_min, v.hi);
    }
  }
  lo_max = __reduce_max_sync(0xffffffffu, lo_max);
  hi_min = __reduce_min_sync(0xffffffffu, hi_min);

  const float scale = fmaxf(fabsf(a.scale_log2) * kUnshift, 1e-37f);        // 0 would make 0 * -infinity of a masked score
  float o[NT][2 * NW][4];
  float m[NT][2], l[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int i = 0; i < 2 * NW; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[nt][i][k] = 0.0f;
    m[nt][0] = m[nt][1] = -INFINITY;
    l[nt][0] = l[nt][1] = 0.0f;
  }

  bool huge = false;       // some row's maximum is beyond_fused
  int st = 0, ahead = ST - 1;
  for (int32_t n = 0; n < n_mine; ++n) {
    sc[ST - 1] = request(n + ST - 1, ahead);
    asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
    __syncwarp();          // every lane's copies of this tile have landed
    const uint32_t codes = ring + st * L::kStage, meta = codes + 2 * L::kCodes;
    const int32_t j0 = base + (my0 + n * kWarpsFew) * kTile;
    const uint32_t here = (have >> (2 * st)) & 3u;
    const bool whole = j0 >= lo_max && j0 + kTile <= hi_min && here == 3u;      // nothing of the tile is masked for any row

    constexpr int WR = INT8 ? 2 * NW : NW; // words of a lane's quarter row
    auto words = [&](uint32_t array, int row, uint32_t (&w)[WR]) {
      const uint32_t at = array + row * L::kRow + t * (L::kRow / 4);
      if constexpr (WR == 8) {
        const uint32_t odd = (g & 1) * 16;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at + odd));
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "r"(at + (16 - odd)));
      } else if (WR == 4) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[WR - 2]), "=r"(w[WR - 1]) : "r"(at));
      else asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
    };
    auto record = [&](uint32_t at) -> uint32_t {
      uint16_t v;
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
      return v;
    };
    auto meta_at = [&](int row) -> uint32_t { return (uint32_t)(row * (D / 32) + t / (4 / (D / 32))) * 2u; };

    // ---- S^T = K Q^T for the tile's two halves of 16 tokens
    float s[2][NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[h][nt][k] = 0.0f;
      const int ra = 16 * h + g, rb = ra + 8;
      uint32_t wa[WR], wb[WR];
      words(codes, ra, wa);
      words(codes, rb, wb);
      BlockScale sa, sb;
      Int8Scale s8;
      if (INT8) {
        s8 = int8_scale((sc[0] >> (8 * h)) & 255u, true);
      } else {
        sa = block_scale(record(meta + meta_at(ra)), book_at, true);
        sb = block_scale(record(meta + meta_at(rb)), book_at, true);
      }
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        uint32_t ka[4], kb[4];
        if constexpr (INT8) {
          decode_bytes(wa[2 * w], wa[2 * w + 1], s8, ka);
          decode_bytes(wb[2 * w], wb[2 * w + 1], s8, kb);
        } else {
          decode_word(wa[w], sa, ka);
          decode_word(wb[w], sb, kb);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma_bf16(s[h][nt], ka[0], kb[0], ka[1], kb[1], qf[nt][w][0], qf[nt][w][1]);
          mma_bf16(s[h][nt], ka[2], kb[2], ka[3], kb[3], qf[nt][w][2], qf[nt][w][3]);
        }
      }
    }
    // ---- masks, running maximum in units of log2 (moved only when it would grow by more than 2^8: the accumulators are then
    // rescaled, which is rare after the first tiles)
    if (!whole) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int32_t j = j0 + 16 * h + g + (k & 2 ? 8 : 0);
            if (j < lo[nt][k & 1] || j >= hi[nt][k & 1] || !((here >> h) & 1u)) s[h][nt][k] = -INFINITY;
          }
    }
    bool grow = false;
    float top[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        top[nt][k] = fmaxf(fmaxf(s[0][nt][k], s[0][nt][k + 2]), fmaxf(s[1][nt][k], s[1][nt][k + 2]));
        grow |= top[nt][k] * scale > m[nt][k] + 8.0f;
      }
    if (__any_sync(0xffffffffu, grow)) {
      bool far = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float x = top[nt][k];
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
          const float next = fmaxf(m[nt][k], x * scale);
          const float f = next == -INFINITY ? 1.0f : exp2_approx(m[nt][k] - next);
          m[nt][k] = next;
          far |= beyond_fused(next);
          l[nt][k] *= f;
#pragma unroll
          for (int i = 0; i < 2 * NW; ++i) {
            o[nt][i][k] *= f;
            o[nt][i][k + 2] *= f;
          }
        }
      huge = __any_sync(0xffffffffu, far);
    }
    if (huge) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 4; ++k) s[h][nt][k] = __fmul_rn(s[h][nt][k], scale);
    }
    const float factor = huge ? 1.0f : scale;
    uint32_t pf[2][NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float m0 = m[nt][0] == -INFINITY ? 0.0f : m[nt][0], m1 = m[nt][1] == -INFINITY ? 0.0f : m[nt][1];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = exp2_approx(fmaf(s[h][nt][0], factor, -m0)), p1 = exp2_approx(fmaf(s[h][nt][1], factor, -m1));
        const float p2 = exp2_approx(fmaf(s[h][nt][2], factor, -m0)), p3 = exp2_approx(fmaf(s[h][nt][3], factor, -m1));
        l[nt][0] += p0 + p2;
        l[nt][1] += p1 + p3;
        pf[h][nt][0] = transpose8x8(pack(p0, p1));
        pf[h][nt][1] = transpose8x8(pack(p2, p3));
      }
    }
    // ---- O^T += V^T P^T
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int ra = 16 * h + g, rb = ra + 8;
      uint32_t wa[WR], wb[WR];
      words(codes + L::kCodes, ra, wa);
      words(codes + L::kCodes, rb, wb);
      BlockScale sa, sb;
      Int8Scale s8;
      if (INT8) {          // whatever a slot that no token fills holds is finite, and meets p = 0
        s8 = int8_scale((sc[0] >> (16 + 8 * h)) & 255u, true);
      } else {
        // slots that no token fills may hold anything; an infinity there would meet p = 0
        const bool ua = whole || (j0 + ra < sq.kv && ((here >> h) & 1u)), ub = whole || (j0 + rb < sq.kv && ((here >> h) & 1u));
        sa = block_scale(ua ? record(meta + L::kMeta + meta_at(ra)) : 0u, book_at, ua);
        sb = block_scale(ub ? record(meta + L::kMeta + meta_at(rb)) : 0u, book_at, ub);
      }
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        uint32_t va[4], vb[4];
        if constexpr (INT8) {
          decode_bytes(wa[2 * w], wa[2 * w + 1], s8, va);
          decode_bytes(wb[2 * w], wb[2 * w + 1], s8, vb);
        } else {
          decode_word(wa[w], sa, va);
          decode_word(wb[w], sb, vb);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          va[k] = transpose8x8(va[k]);
          vb[k] = transpose8x8(vb[k]);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma_bf16(o[nt][2 * w], va[0], va[1], vb[0], vb[1], pf[h][nt][0], pf[h][nt][1]);
          mma_bf16(o[nt][2 * w + 1], va[2], va[3], vb[2], vb[3], pf[h][nt][0], pf[h][nt][1]);
        }
      }
    }
    __syncwarp();          // the stage may be filled again
    st = st + 1 == ST ? 0 : st + 1;
    ahead = ahead + 1 == ST ? 0 : ahead + 1;
#pragma unroll
    for (int k = 0; k + 1 < ST; ++k) sc[k] = sc[k + 1];
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(a.status, 2u);

  // ---- join the warps
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) l[nt][k] += __shfl_xor_sync(0xffffffffu, l[nt][k], off);
      if (g == 0) stat[warp][8 * nt + 2 * t + k] = make_float2(m[nt][k], finished(l[nt][k], m[nt][k]));
    }
  __syncthreads();         // every warp is done with its ring
  float* join = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = 8 * nt + 2 * t + k;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarpsFew; ++w) top = fmaxf(top, stat[w][r].x);
      const float f = m[nt][k] == -INFINITY ? 0.0f : exp2_approx(m[nt][k] - top);
      // accumulator (2 w + j, half, column k): nibble {0,1,4,5}[2 j + half] + 2 (g mod 2) of word w of quarter g / 2
#pragma unroll
      for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int c = (g >> 1) * (D / 4) + 8 * w + 4 * j + half + 2 * (g & 1);
            join[(warp * 8 * NT + r) * D + c] = o[nt][2 * w + j][2 * half + k] * f;
          }
    }
  __syncthreads();
  auto joined = [&](int r, int c, float& top, float& sum) -> float4 {
    top = -INFINITY;
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarpsFew; ++w) top = fmaxf(top, stat[w][r].x);
#pragma unroll
    for (int w = 0; w < kWarpsFew; ++w) sum += stat[w][r].y == 0.0f ? 0.0f : stat[w][r].y * exp2_approx(stat[w][r].x - top);
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kWarpsFew; ++w) {
      const float4 u = *reinterpret_cast<const float4*>(join + (w * 8 * NT + r) * D + c);
      v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    return v;
  };
  auto finish = [&](int r, int c, const float4& v, float top, float sum) {
    const int32_t i = (row0 + r) / a.group, h = head * a.group + (row0 + r) % a.group;
    store_out4(a, (int64_t)(sq.q0 + i) * a.out_ld + (int64_t)h * D + c, v, inverse_of(sum, kUnshift));
    if (c == 0 && a.lse) a.lse[(int64_t)(sq.q0 + i) * a.q_heads + h] = lse_of(top, sum);
  };
  if constexpr (CLUSTER) {
    // the splits are the CTAs of a cluster: each leaves its joined rows in its shared memory (behind the warps' rows: the
    // ring has the room), then every CTA finishes a part of the rows from all of them
    float* mine = join + kWarpsFew * 8 * NT * D;
    for (int x = threadIdx.x; x < n_rows * (D / 4); x += kWarpsFew * 32) {
      const int r = x / (D / 4), c = x % (D / 4) * 4;
      float top, sum;
      *reinterpret_cast<float4*>(mine + r * D + c) = joined(r, c, top, sum);
      if (c == 0) own[r] = make_float2(top, sum);
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    for (int x = split * kWarpsFew * 32 + threadIdx.x; x < n_rows * (D / 4); x += a.splits * kWarpsFew * 32) {
      const int r = x / (D / 4), c = x % (D / 4) * 4;
      const uint32_t row_at = fb4blk::smem_u32(mine + r * D + c), own_at = fb4blk::smem_u32(own + r);
      float top = -INFINITY, sum = 0.0f;
      float2 st[8];
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        st[z] = make_float2(-INFINITY, 0.0f);
        if (z < a.splits) {
          asm volatile("{\n\t.reg .b32 q;\n\tmapa.shared::cluster.u32 q, %2, %3;\n\tld.shared::cluster.v2.f32 {%0, %1}, [q];\n\t}"
                       : "=f"(st[z].x), "=f"(st[z].y) : "r"(own_at), "r"(z));
          top = fmaxf(top, st[z].x);
        }
      }
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        if (st[z].y != 0.0f) {
          const float f = exp2_approx(st[z].x - top);
          float4 u;
          asm volatile("{\n\t.reg .b32 q;\n\tmapa.shared::cluster.u32 q, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [q];\n\t}"
                       : "=f"(u.x), "=f"(u.y), "=f"(u.z), "=f"(u.w) : "r"(row_at), "r"(z));
          v.x = fmaf(u.x, f, v.x); v.y = fmaf(u.y, f, v.y); v.z = fmaf(u.z, f, v.z); v.w = fmaf(u.w, f, v.w);
          sum = fmaf(st[z].y, f, sum);
        }
      }
      finish(r, c, v, top, sum);
    }
    // nobody's shared memory goes away while another CTA reads it
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    for (int x = threadIdx.x; x < n_rows * (D / 4); x += kWarpsFew * 32) {
      const int r = x / (D / 4), c = x % (D / 4) * 4;
      float top, sum;
      const float4 v = joined(r, c, top, sum);
      if (a.splits > 1) {
        const int32_t i = (row0 + r) / a.group, h = head * a.group + (row0 + r) % a.group;
        const int64_t pr = partial_row(a, b, i, h);
        if (sum != 0.0f) *reinterpret_cast<float4*>(partial_sums(a, pr, split, D) + c) = v;
        if (c == 0) *partial_stat(a, pr, split, D) = make_float2(top, sum);
      } else {
        finish(r, c, v, top, sum);
      }
    }  }
}

// Joins the splits: NW warps per query row and head take the splits in turn, lane l holds channels 4 l to 4 l + 3.  Splits that
// saw nothing have sum 0 and their D sums are not read.
template <int D, int NW>
__global__ void __launch_bounds__(128) fb4_attend_join_kernel(const __grid_constant__ Fb4Attend a) {
  __shared__ float4 part[4][32];
  __shared__ float2 stat[4];
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % NW;
  const int64_t row = (int64_t)blockIdx.x * (4 / NW) + warp / NW;
  const bool real = row < partial_rows(a);
  const int32_t h = (int32_t)(row % a.q_heads);
  const int64_t bi = row / a.q_heads;
  const int32_t b = real ? (int32_t)(bi / a.max_q) : 0, i = (int32_t)(bi % a.max_q);
  const Sequence sq = sequence(a, b, false);
  const bool on = real && i < sq.n_q;
  float top = -INFINITY, sum = 0.0f;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (on) {
    for (int s = sub + lane * NW; s < a.splits; s += 32 * NW) {
      const float2 st = *partial_stat(a, row, s, D);
      if (st.y > 0.0f) top = fmaxf(top, st.x);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    for (int s0 = sub; s0 < a.splits; s0 += 32 * NW) {
      float w = 0.0f;
      if (s0 + lane * NW < a.splits) {
        const float2 st = *partial_stat(a, row, s0 + lane * NW, D);
        if (st.y != 0.0f) {
          w = exp2_approx(st.x - top);
          sum += w * st.y;
        }
      }
      const int left = (a.splits - s0 + NW - 1) / NW, n = left < 32 ? left : 32;
#pragma unroll 8
      for (int s = 0; s < n; ++s) {
        const float f = __shfl_sync(0xffffffffu, w, s);
        if (f > 0.0f && lane * 4 < D) {
          const float4 u = *reinterpret_cast<const float4*>(partial_sums(a, row, s0 + s * NW, D) + lane * 4);
          v.x = fmaf(u.x, f, v.x); v.y = fmaf(u.y, f, v.y); v.z = fmaf(u.z, f, v.z); v.w = fmaf(u.w, f, v.w);
        }
      }
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  }
  if (NW > 1) {
    part[warp][lane] = v;
    if (lane == 0) stat[warp] = make_float2(top, sum);
    __syncthreads();
    if (sub != 0) return;
    float all = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) all = fmaxf(all, stat[warp + w].x);
    v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = stat[warp + w].y == 0.0f ? 0.0f : exp2_approx(stat[warp + w].x - all);
      const float4 u = part[warp + w][lane];
      v.x = fmaf(u.x, f, v.x); v.y = fmaf(u.y, f, v.y); v.z = fmaf(u.z, f, v.z); v.w = fmaf(u.w, f, v.w);
      sum = fmaf(stat[warp + w].y, f, sum);
    }
    top = all;
  }
  if (!on) return;
  if (lane * 4 < D) store_out4(a, (int64_t)(sq.q0 + i) * a.out_ld + (int64_t)h * D + lane * 4, v, inverse_of(sum, kUnshift));
  if (lane == 0 && a.lse) a.lse[(int64_t)(sq.q0 + i) * a.q_heads + h] = lse_of(top, sum);
}

template <typename... Args>
cudaError_t launch_with(void (*kernel)(Args...), int64_t grid, int threads, int smem, int cluster, bool behind, cudaStream_t stream,
                        Args... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  if (cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = (unsigned)cluster;
    attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  if (behind) {            // may be set up while the kernel in front still runs
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
  }
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int D, int NT, bool INT8>
cudaError_t launch(const Fb4Attend& a, cudaStream_t stream) {
  const int64_t row_tiles = ((int64_t)a.max_q * a.group + 8 * NT - 1) / (8 * NT);
  const int64_t grid = row_tiles * a.splits * a.cache.n_heads * a.n_seqs;
  if (a.splits > 1 && !a.partial)
    return launch_with(fb4_attend_few_kernel<D, NT, true, INT8>, grid, kWarpsFew * 32, Few<D, INT8>::kBytes, a.splits, false, stream, a);
  return launch_with(fb4_attend_few_kernel<D, NT, false, INT8>, grid, kWarpsFew * 32, Few<D, INT8>::kBytes, 1, false, stream, a);
}

template <int D>
cudaError_t launch_join(const Fb4Attend& a, cudaStream_t stream) {
  // a warp per row, or the 4 warps of a CTA where a row has many splits
  if (a.splits >= 16) return launch_with(fb4_attend_join_kernel<D, 4>, partial_rows(a), 128, 0, 1, true, stream, a);
  return launch_with(fb4_attend_join_kernel<D, 1>, (partial_rows(a) + 3) / 4, 128, 0, 1, true, stream, a);
}

}  // namespace

cudaError_t fb4_attend_prepare_device() {
  const cudaFuncAttribute attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaSuccess;
#define FB4_OPT_IN(D, NT, INT8) \
  if (e == cudaSuccess) e = cudaFuncSetAttribute(fb4_attend_few_kernel<D, NT, false, INT8>, attr, Few<D, INT8>::kBytes); \
  if (e == cudaSuccess) e = cudaFuncSetAttribute(fb4_attend_few_kernel<D, NT, true, INT8>, attr, Few<D, INT8>::kBytes)
  FB4_OPT_IN(128, 1, false);
  FB4_OPT_IN(128, 2, false);
  FB4_OPT_IN(64, 1, false);
  FB4_OPT_IN(64, 2, false);
  FB4_OPT_IN(128, 1, true);
  FB4_OPT_IN(128, 2, true);
  FB4_OPT_IN(64, 1, true);
  FB4_OPT_IN(64, 2, true);
#undef FB4_OPT_IN
  if (e == cudaSuccess) e = fb4_attend_many_prepare_device();
  return e;
}

Fb4AttendPlan fb4_attend_plan(const fb4_ctx* ctx, int int8, int32_t q_heads, int32_t n_heads, int32_t head_dim, int32_t n_seqs,
                              int32_t max_q, int32_t max_kv, int32_t window) {
  Fb4AttendPlan p{0, 1, 0x7fffffff / 64, 0};
  if ((head_dim != 64 && head_dim != 128) || ctx->force_generic || n_seqs == 0 || max_q == 0) return p;
  const int64_t rows = (int64_t)max_q * (q_heads / n_heads);
  // the longest run of tokens that a CTA's rows can see together
  const int64_t span = window > 0 && (int64_t)window + max_q < max_kv ? (int64_t)window + max_q : max_kv;
  // Up to 16 rows go together in the few-row kernel and more of them decode the same tokens again, but the many-row kernel works
  // on 128 rows however many there are, and starts slowly: 32 rows of one head over 2000 tokens take 16 against 27 us, 24 rows of 256
  // heads over 4096 tokens the same time, 32 of them 154 against 134 us.
  if (rows <= 24 || (rows <= 32 && (int64_t)n_heads * n_seqs < ctx->sm_count)) {
    p.kernel = 1;
    const int64_t nt = rows <= 8 ? 1 : 2;
    const int64_t units = (rows + 8 * nt - 1) / (8 * nt) * n_heads * n_seqs;
    // CTAs that are resident at a time; a split has at least 2 tiles for each of its warps
    const int64_t slots = (int64_t)ctx->sm_count * resident(head_dim, (int)nt, int8 != 0);
    const int64_t tiles = (span + kTile - 1) / kTile + 1;
    const int64_t most = (tiles + 2 * kWarpsFew - 1) / (2 * kWarpsFew);
    int64_t s = slots / units;                                      // one wave
    // Sequences of unlike lengths: pieces of 1024 tokens even them out, of 96 tiles in 8 bits.  us in pieces of 32, 64, 96, 128, 256 tiles, 8 heads of
    // 128 where nothing else is said: 64 sequences of 131 to 8191 tokens 141, 103, 100, 100, 107 (heads of 64: 79, 63, 59, 60, 73); 96 of 50 to 8000 183, 135, 133, 148, 148;
    // 16 of 200 to 32000 97, 97, 97, 101, 118; 128 of 100 to 2000 69, 57, 57, 56, 56; 256 of 16 to 4000, 2 heads, 63, 58, 58, 58, 58; 32 of 1000 to 16000, 4 heads of 64, 39, 40, 37,
    // 39, 39.  64 of 4096 each, where nothing is to be evened out, are 1.15 waves: 110, 105, 116, 116, 116.
    const int64_t piece = int8 ? 96 : 32, fine = tiles / piece < 8 ? tiles / piece : 8;
    if (s < fine) s = fine;
    if (s > most) s = most;
    if (s > 0x7fffffffLL / units) s = 0x7fffffffLL / units;         // a grid has at most 2^31 - 1 CTAs
    if (s < 1) s = 1;
    p.splits = (int32_t)s;
  } else {
    p.kernel = 2;
    // one CTA per SM: the number of splits that leaves the least of the last wave idle.  A split has at least 4 tiles, and its
    // start, its partial result and the join cost about as much as 8 (counted as 3: 2048 queries of 16 heads over 40000 tokens of 8
    // in 659 instead of 590 us, 5 x 100 queries over 5000 in 75.3 instead of 73.5, others the same to 1 %)
    const int64_t units = (rows + 255) / 256 * n_heads * n_seqs;
    const int64_t tiles = (span + 127) / 128 + 1;
    double best = 1e300;
    p.split_tiles = (int32_t)tiles;
    for (int64_t s = 1; s <= 32 && (s == 1 || tiles / s >= 4); ++s) {
      const int64_t per = (tiles + s - 1) / s, waves = (units * s + ctx->sm_count - 1) / ctx->sm_count;
      const double cost = (double)waves * (double)(per + (s > 1 ? 8 : 1));
      if (cost < best * 0.97) {
        best = cost;
        p.split_tiles = (int32_t)per;
      }
    }
    p.splits = (int32_t)((tiles + p.split_tiles - 1) / p.split_tiles);
  }
  // up to 8 splits of the few-row kernel are one cluster, which joins them in shared memory
  if (p.splits > 1 && !(p.kernel == 1 && p.splits <= 8)) p.workspace = (int64_t)n_seqs * max_q * q_heads * p.splits * (head_dim + 2) * 4;
  return p;
}

cudaError_t fb4_launch_attend_few(const Fb4Attend& a, cudaStream_t stream) {
  const bool wide = (int64_t)a.max_q * a.group > 8;
  if (a.int8) {
    if (a.cache.head_dim == 128) return wide ? launch<128, 2, true>(a, stream) : launch<128, 1, true>(a, stream);
    return wide ? launch<64, 2, true>(a, stream) : launch<64, 1, true>(a, stream);
  }
  if (a.cache.head_dim == 128) return wide ? launch<128, 2, false>(a, stream) : launch<128, 1, false>(a, stream);
  return wide ? launch<64, 2, false>(a, stream) : launch<64, 1, false>(a, stream);
}

cudaError_t fb4_launch_attend_join(const Fb4Attend& a, cudaStream_t stream) {
  return a.cache.head_dim == 128 ? launch_join<128>(a, stream) : launch_join<64>(a, stream);
}
