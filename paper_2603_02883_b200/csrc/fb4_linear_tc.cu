// Products of rows with FB4 weights on the fifth-generation tensor cores: y[t][n] = sum_k x[t][k] w[n][k] + bias[n].
//
// The weights are the M side: 128 rows of W are a tile, their decoded values the A operand, which lies in tensor memory, a row to a lane, so
// that a thread decodes a row of its own and nothing of the decoded weights passes through shared memory.  x, up to 96 rows at a time, is the
// B operand in shared memory; channels stand in the order 0 2 1 3 4 6 5 7 of every eight on both sides, the decoder's.
//
// Work: one CTA per SM.  A cluster takes a run of rows of W (in quarters of a tile: 32 rows, a warp's), its CTAs a run of the channels each;
// their sums are joined through distributed shared memory, always in the same order.  The warps of a CTA have fixed roles:
//   decode   4 groups of 4 warps take the items (128 rows x 256 channels) in turn, half an item at a time into a ring of 4 to 7 buffers in
//            tensor memory
//   load     codes of the items into a ring (tensor copies of 32 rows x 128 bytes, 128-byte swizzle; with rows of 64 bytes the copies alone
//            took 34 us where this takes 25)
//   product  one warp issues D_tile += A x
//   x        6 warps bring x into shared memory, in chunks where it is too large for it
//
// Bound: for large weights no part alone, but the issue slots that decode, metadata and products share (62 % of them are taken, the ALU pipe is busy 59 %
// of the time), then start and end; for small weights these two alone.  12288 x 12288 with one row takes 29.5 us, with 64 40.3 (479 TFLOP/s), 24576 x 12288 with 16
// 55.1 (3.1 TB/s), 6152 x 1568 with 61 11.7.  Copies of the kernel that leave parts out (wrong results), for the first three:
//   decode's arithmetic 26.0 / 36.1 / 46.9; the metadata's loads too 22.3 / 33.8 / 38.4; the stores to tensor memory too 20.8 / 32.7 / 35.1; the
//   products too 17.8 / 31.5 / 29.9: copies, x, start and end alone.  Metadata alone 28.8 / 36.6 / 52.1, products alone 27.5 / 38.1 / 51.1.
// The decoding warps are at work, waits among it, for 43 000 of 62 000 cycles (12288 x 12288, 16 rows); 11 000 pass until x and the first codes are there, 10 000 from
// the last decoded value to the last result: the last products, the cluster's slowest CTA, the join.  The products of half an item leave every 500 to 640 cycles,
// at most 200 of which are the tensor core's: instructions of one warp among those that decode.
// On the way (12288 x 12288), each against the kernel of its time: A through shared memory 61 us for 32 rows, 49 with a row to a thread in tensor memory; x brought
// in by 4 warps 89 for 64 rows; 4 buffers of A, one a group, 36.9 for one row, 31.9 with 7; first copies before the set-up 32.9.  x earlier gives nothing, though
// the products wait 11 000 cycles for it: in parts with a barrier each +0.5 us, its first pieces by all warps before the set-up +0.5, by asynchronous
// copies and reordered in place +3.
#include "fb4_attend.cuh"
#include "fb4_staging.cuh"
#include "fb4_tcgen05.cuh"

namespace {

using namespace fb4att;
using namespace fb4tc;
using fb4blk::smem_u32;
using fb4stage::mbar_expect_tx;
using fb4stage::mbar_init;
using fb4stage::tma_load_2d;

constexpr int kGroups = 4, kDecodeWarps = 4 * kGroups, kLoadWarp = kDecodeWarps, kProductWarp = kLoadWarp + 1, kXWarp = kProductWarp + 1, kXWarps = 6;
constexpr int kThreads = (kXWarp + kXWarps) * 32;
constexpr int kStages = 7, kQuarter = 32 * 128, kStage = 4 * kQuarter;     // bytes of 32 and of 128 rows' codes of an item
constexpr int kXBytes = 96 * 1024;                                       // of x, and the stages that a CTA of few items does not need
constexpr int kBytes = 1024 + kStages * kStage + kXBytes;
constexpr int kACols = 64, kMaxA = 7, kDCols = 512 - 4 * kACols;          // tensor memory: buffers for A, as many as D leaves, and D at its end
constexpr int kMaxRows = 96, kMaxSplits = 8;
static_assert(kXBytes / 2 >= kMaxRows * 512, "a chunk of x has at least one step");

struct Linear {
  const uint16_t* x;
  int64_t ld;
  const uint16_t* meta;
  const uint16_t* bias;
  void* out;
  int64_t out_ld;
  int64_t T, N;
  int32_t nb;               // blocks of a row
  int32_t rows;             // rows of x at a time, a multiple of 16
  int32_t splits;           // CTAs of a cluster
  int32_t quarters;         // quarters of a tile to a cluster
  int32_t stages;           // of the ring: kStages, or as many as there are items, which then do not come round
  int32_t chunk, buffers;   // steps of 256 channels whose x is held at a time, and how often
  int32_t out_dtype;
  int32_t wide_out;         // 4 neighbouring results are stored at once
  const Fb4DeviceTables* tables;
  uint32_t* status;
};

// A wait tells only whether the phase before the present one has ended, so a waiter must never be two phases ahead.  Buffers of A go round the
// groups, and a group that begins turn q (half an item) knows of the products of turns up to q - n - 7 only (n buffers: its own turn before
// was q - 7 or later, and it had a buffer).  With a barrier for the odd and one for the even uses of a buffer it waits for turn q - n where
// q - 3 n must have ended, which is so from 4 buffers on; with one barrier, q - 2 n, from 7 on.
struct Bars {
  uint64_t ring_full[kStages], ring_empty[kStages];
  uint64_t a_full[kMaxA], a_empty[2][kMaxA], x_full[2], x_empty[2], d_full, drained;
};

// The items in order: chunk by chunk of x, in it tile by tile, in it step by step.
struct Cursor {
  int32_t item, tile, s, c0, c1, chunk_no;
  __device__ __forceinline__ Cursor(int32_t begin, int32_t end, int32_t chunk) : item(0), tile(0), s(begin), c0(begin), c1(min(begin + chunk, end)), chunk_no(0) {}
  __device__ __forceinline__ void advance(int32_t by, int32_t tiles, int32_t chunk, int32_t end) {
    item += by;
    s += by;
    while (s >= c1 && c0 < end) {
      int32_t over = s - c1;
      if (++tile == tiles) {
        tile = 0;
        ++chunk_no;
        c0 = c1;
        c1 = min(c0 + chunk, end);
      }
      s = c0 + over;
    }
  }
};

__global__ void __launch_bounds__(kThreads, 1) fb4_linear_tc_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ Linear p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  __shared__ Bars bars;
  __shared__ uint32_t book[64];
  __shared__ uint32_t tmem_at, dead_flag;
  const uint32_t base_smem = (smem_u32(smem_raw) + 1023u) & ~1023u, ring_at = base_smem, x_at = base_smem + p.stages * kStage;
  float* sums = reinterpret_cast<float*>(smem_raw + (base_smem - smem_u32(smem_raw)));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  volatile uint32_t* dead = &dead_flag;

  // ---- which work
  const int32_t cluster = (int32_t)(blockIdx.x / (uint32_t)p.splits), split = (int32_t)blockIdx.x - cluster * p.splits, rows = p.rows;
  const int64_t row_base = (int64_t)cluster * p.quarters * 32, t0 = (int64_t)blockIdx.y * rows;
  const int32_t n_tok = (int32_t)(p.T - t0 < rows ? p.T - t0 : rows);
  const int64_t left = (p.N - row_base + 31) >> 5;
  const int32_t quarters = (int32_t)(left < p.quarters ? left : p.quarters), tiles = (quarters + 3) / 4;
  const int32_t steps = (p.nb + 7) / 8;
  const int32_t s_begin = steps * split / p.splits, s_end = steps * (split + 1) / p.splits;      // 2^23 steps, 8 CTAs at most
  const int32_t items = (s_end - s_begin) * tiles;

  // ---- set-up
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) { mbar_init(smem_u32(&bars.ring_full[i]), 1); mbar_init(smem_u32(&bars.ring_empty[i]), 4); }
    for (int i = 0; i < kMaxA; ++i) { mbar_init(smem_u32(&bars.a_full[i]), 4); mbar_init(smem_u32(&bars.a_empty[0][i]), 1); mbar_init(smem_u32(&bars.a_empty[1][i]), 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&bars.x_full[i]), kXWarps); mbar_init(smem_u32(&bars.x_empty[i]), 1); }
    mbar_init(smem_u32(&bars.d_full), 1);
    mbar_init(smem_u32(&bars.drained), 1);
    dead_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kProductWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_at)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (threadIdx.x >= 64 && threadIdx.x < 128) fill_book(book, p.tables, threadIdx.x - 64);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_at, 0), d_col = tmem + 512 - tiles * rows;
  const int n_a = min((512 - tiles * rows) / kACols, kMaxA);

  if (warp < kDecodeWarps) {
    // =========================================================== decode
    const int group = warp >> 2, quarter = warp & 3;
    const uint32_t lanes = (uint32_t)quarter << 21, book_at = smem_u32(book);
    const int align = p.nb % 8 == 0 ? 8 : p.nb % 4 == 0 ? 4 : 1;      // records of a row that lie together in aligned words
    auto fetch = [&](const Cursor& c) -> uint4 {
      uint32_t v[4] = {0, 0, 0, 0};
      const int64_t row = row_base + (c.tile * 4 + quarter) * 32 + lane;
      if (c.item < items && row < p.N) {
        const uint16_t* m = p.meta + row * p.nb + 8 * c.s;
        const int32_t n = p.nb - 8 * c.s;                             // records there are; those behind read as zeros, as their codes do
        if (align == 8) return __ldg(reinterpret_cast<const uint4*>(m));
        if (align == 4) {
          const uint2 lo = __ldg(reinterpret_cast<const uint2*>(m)), hi = n > 4 ? __ldg(reinterpret_cast<const uint2*>(m) + 1) : make_uint2(0, 0);
          return make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < n) v[i >> 1] |= (uint32_t)__ldg(m + i) << (16 * (i & 1));
      }
      return make_uint4(v[0], v[1], v[2], v[3]);
    };
    Cursor c(s_begin, s_end, p.chunk);
    c.advance(group, tiles, p.chunk, s_end);
    uint4 next = fetch(c);
    bool ok = true;
    // place in the ring and buffer of A of the item's first half, and how often they have been used, moved on without divisions
    int st = group, buf = 2 * group;
    uint32_t st_lap = 0, lap = 0;
    for (; buf >= n_a; buf -= n_a) ++lap;
    while (c.item < items && ok) {
      const uint32_t meta[4] = {next.x, next.y, next.z, next.w};
      const bool there = c.tile * 4 + quarter < quarters;
      c.advance(kGroups, tiles, p.chunk, s_end);
      next = fetch(c);
      ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.ring_full[st]), st_lap & 1, dead));
      if (!ok) break;
      // The whole item at once, so that its place in the ring is free for the next copy.  The fence: reads through the ordinary path are over
      // before a copy, which takes another path, may overwrite them (without it some lanes read the item after).
      uint32_t w[8][4];
      if (there) {
        const uint32_t codes = ring_at + st * kStage + quarter * kQuarter + lane * 128;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i][0]), "=r"(w[i][1]), "=r"(w[i][2]), "=r"(w[i][3]) : "r"(codes + ((i ^ (lane & 7)) << 4)));
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.ring_empty[st]));
      st += kGroups;
      if (st >= kStages) { st -= kStages; ++st_lap; }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bool waited = lap == 0;
        auto buffer_free = [&]() {           // the product that had the buffer before has read it
          if (!waited) ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.a_empty[(lap - 1) & 1][buf]), ((lap - 1) >> 1) & 1, dead));
          waited = true;
          fence_after();
        };
        if (there) {
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            uint32_t o[16];
            const uint32_t m = meta[2 * half + (h >> 1)];
            const BlockScale sc = block_scale((h & 1) ? m >> 16 : m & 0xffffu, book_at, true);
#pragma unroll
            for (int q = 0; q < 4; ++q) decode_word(w[4 * half + h][q], sc, *reinterpret_cast<uint32_t(*)[4]>(o + 4 * q));
            buffer_free();
            if (!ok) break;
            tmem_st16(tmem + buf * kACols + lanes + 16 * h, o);
          }
          tmem_wait_st();
        } else {
          buffer_free();
        }
        if (!ok) break;
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.a_full[buf]));
        buf += half ? 2 * kGroups - 1 : 1;
        for (; buf >= n_a; buf -= n_a) ++lap;
      }
    }
    // ---- the sums, [row of x][row of W], to shared memory, which nobody uses any more once the last product is done
    if (ok) ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.d_full), 0, dead));
    if (ok) {
      fence_after();
      const int32_t sums_ld = tiles * 128 + 4;
      for (int32_t tile = group; tile < tiles; tile += kGroups) {
        if (tile * 4 + quarter >= quarters) continue;
        float* at = sums + tile * 128 + quarter * 32 + lane;
        for (int32_t col = 0; col < rows; col += 16) {
          uint32_t v[16];
          tmem_ld16(d_col + tile * rows + col + lanes, v);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) at[(col + i) * sums_ld] = __uint_as_float(v[i]);
        }
      }
    }
  } else if (warp == kLoadWarp) {
    // =========================================================== load
    bool ok = true;
    Cursor c(s_begin, s_end, p.chunk);
    for (; c.item < items; c.advance(1, tiles, p.chunk, s_end)) {
      const int st = c.item % kStages;
      if (c.item >= kStages) ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.ring_empty[st]), (c.item / kStages - 1) & 1, dead));
      if (!ok) break;
      const int32_t n = min(quarters - c.tile * 4, 4);
      const uint32_t full = smem_u32(&bars.ring_full[st]);
      if (lane == 0) {
        mbar_expect_tx(full, (uint32_t)n * kQuarter);
        for (int q = 0; q < n; ++q) tma_load_2d(ring_at + st * kStage + q * kQuarter, &map, full, c.s * 128, (int)(row_base + (c.tile * 4 + q) * 32));
      }
      __syncwarp();
    }
    // every copy has to have landed before the CTA ends
    for (int32_t i = c.item > kStages ? c.item - kStages : 0; i < c.item; ++i) {
      uint32_t tries = 0;
      while (!mbar_try_wait(smem_u32(&bars.ring_full[i % kStages]), (i / kStages) & 1) && ++tries < kSpinLimit) {}
    }
  } else if (warp == kProductWarp) {
    // =========================================================== product: every lane waits, one issues
    const uint32_t idesc = instr_desc(rows, false), x_low = desc_low(x_at, 16), x_half = rows * 16, a_end = tmem + n_a * kACols;
    const uint32_t full0 = smem_u32(&bars.a_full[0]), empty0 = smem_u32(&bars.a_empty[0][0]);
    bool ok = true;
    uint32_t a = tmem, full = full0, empty = empty0, lap = 0;      // buffer of A, its barriers, and how often it has been used, mod 2
    int32_t chunk_no = 0;
    for (int32_t c0 = s_begin; c0 < s_end && ok; ++chunk_no) {
      const int32_t c1 = min(c0 + p.chunk, s_end);
      const int xb = chunk_no & (p.buffers - 1);
      ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.x_full[xb]), (chunk_no / p.buffers) & 1, dead));
      const uint32_t b0 = x_low + ((xb * (uint32_t)p.chunk * rows * 512) >> 4);
      uint32_t d = d_col;
      for (int32_t tile = 0; tile < tiles && ok; ++tile, d += rows) {
        uint32_t b = b0;
        for (int32_t half = 2 * c0; half < 2 * c1; ++half, b += x_half) {
          ok = __all_sync(0xffffffffu, wait(full, lap, dead));
          if (!ok) break;
          fence_after();
          if (elected()) {
            mma_ts(d, a, b, idesc, half > 2 * s_begin);
#pragma unroll
            for (int k = 1; k < 4; ++k) mma_ts(d, a + 8 * k, b + 2 * k, idesc, true);
#pragma unroll
            for (int k = 4; k < 8; ++k) mma_ts(d, a + 8 * k, b + (x_half >> 1) + 2 * k - 8, idesc, true);
            commit(empty);
          }
          __syncwarp();
          a += kACols;
          full += 8;
          empty += 8;
          if (a == a_end) {
            a = tmem;
            lap ^= 1u;
            full = full0;
            empty = empty0 + lap * (kMaxA * 8);
          }
        }
      }
      c0 = c1;
      if (ok && elected()) commit(smem_u32(c0 < s_end ? &bars.x_empty[xb] : &bars.d_full));
      __syncwarp();
    }
    // nothing of this CTA may be on the tensor core when its tensor memory is given back
    if (elected()) commit(smem_u32(&bars.drained));
    uint32_t tries = 0;
    while (!mbar_try_wait(smem_u32(&bars.drained), 0) && ++tries < kSpinLimit) {}
  } else {
    // =========================================================== x
    const int xw = warp - kXWarp;
    bool ok = true;
    int32_t no = 0;
    for (int32_t c0 = s_begin; c0 < s_end; c0 += p.chunk, ++no) {
      const int32_t n_steps = min(p.chunk, s_end - c0), buf = no % p.buffers;
      if (no >= p.buffers) ok = __all_sync(0xffffffffu, wait(smem_u32(&bars.x_empty[buf]), (no / p.buffers - 1) & 1, dead));
      if (!ok) break;
      const uint32_t at = x_at + (uint32_t)buf * p.chunk * rows * 512;
      // [64 channels][row] with 128-byte swizzle, rows behind the last zero; one step of 8 rows to a warp at a time
      const int32_t groups = rows >> 3;
      for (int32_t i = xw, step = xw / groups, r8 = xw - step * groups; i < n_steps * groups; i += kXWarps) {
        const int32_t run = (c0 + step) * 32 + lane;                   // 8 channels, counted from the first of all
        const bool real = (run >> 2) < p.nb;
        const uint16_t* src = p.x + (t0 + r8 * 8) * p.ld + (int64_t)run * 8;
        const uint32_t to = at + step * rows * 512 + (lane >> 3) * rows * 128 + r8 * 1024;
        uint4 u[8];
#pragma unroll
        for (int r = 0; r < 8; ++r, src += p.ld) {
          u[r] = make_uint4(0, 0, 0, 0);
          if (real && r8 * 8 + r < n_tok) u[r] = __ldg(reinterpret_cast<const uint4*>(src));
        }
#pragma unroll
        for (int r = 0; r < 8; ++r)
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to + r * 128 + (((lane ^ r) & 7) << 4)), "r"(prmt(u[r].x, u[r].y, 0x5410u)),
                       "r"(prmt(u[r].x, u[r].y, 0x7632u)), "r"(prmt(u[r].z, u[r].w, 0x5410u)), "r"(prmt(u[r].z, u[r].w, 0x7632u)) : "memory");
        for (r8 += kXWarps; r8 >= groups; r8 -= groups) ++step;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.x_full[buf]));
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  const bool whole = !*dead;
  if (threadIdx.x == 0 && !whole) atomicOr(p.status, 1u);
  if (warp == kProductWarp) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
  // ---- the CTAs of the cluster finish a part of the sums each
  if (p.splits > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  const int32_t sums_ld = tiles * 128 + 4, out_rows = quarters * 32;
  for (int32_t i = (warp * p.splits + split) * 32 + lane; i < n_tok * (out_rows / 4) && whole; i += p.splits * kThreads) {       // a warp of each CTA in turn
    const int32_t tok = i / (out_rows / 4), r = (i - tok * (out_rows / 4)) * 4;        // 4 neighbouring rows of W
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (p.splits > 1) {
      const uint32_t at = smem_u32(sums + tok * sums_ld + r);
#pragma unroll
      for (int z = 0; z < kMaxSplits; ++z)
        if (z < p.splits) {
          float4 u;
          asm volatile("{\n\t.reg .b32 q;\n\tmapa.shared::cluster.u32 q, %4, %5;\n\tld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [q];\n\t}"
                       : "=f"(u.x), "=f"(u.y), "=f"(u.z), "=f"(u.w) : "r"(at), "r"(z));
          v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
    } else {
      v = *reinterpret_cast<const float4*>(sums + tok * sums_ld + r);
    }
    const int64_t n = row_base + r, at = (t0 + tok) * p.out_ld + n;
    float y[4] = {v.x * kUnshift, v.y * kUnshift, v.z * kUnshift, v.w * kUnshift};
    if (p.bias) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (n + k < p.N) y[k] += __uint_as_float((uint32_t)__ldg(p.bias + n + k) << 16);
    }
    if (p.wide_out && n + 4 <= p.N) {
      if (p.out_dtype == 0) {
        *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = make_float4(y[0], y[1], y[2], y[3]);
      } else if (p.out_dtype == 1) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(y[0], y[1]), hi = __floats2bfloat162_rn(y[2], y[3]);
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      } else {
        const __half2 lo = __floats2half2_rn(y[0], y[1]), hi = __floats2half2_rn(y[2], y[3]);
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (n + k >= p.N) break;
        if (p.out_dtype == 0) static_cast<float*>(p.out)[at + k] = y[k];
        else if (p.out_dtype == 1) static_cast<__nv_bfloat16*>(p.out)[at + k] = __float2bfloat16_rn(y[k]);
        else static_cast<__half*>(p.out)[at + k] = __float2half_rn(y[k]);
      }
    }
  }
  // nobody's shared memory goes away while another CTA reads it
  if (p.splits > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

}  // namespace

// Opt-in to the dynamic shared memory, and the clusters that are resident at a time.
cudaError_t fb4_linear_tc_prepare_device(int32_t* clusters) {
  cudaError_t e = cudaFuncSetAttribute(fb4_linear_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
  if (e == cudaSuccess) e = fb4_clusters_at_once(reinterpret_cast<const void*>(fb4_linear_tc_kernel), kThreads, kBytes, clusters);
  return e;
}

// Rows of x in passes of equal size; of the cluster sizes that fit, the one with the fewest items for a CTA, a wave's start and join counted as 3.
Fb4LinearTcPlan fb4_linear_tc_plan(const int32_t* clusters, int64_t T, int64_t N, int64_t K) {
  Fb4LinearTcPlan p{0, 1, 1};
  const int64_t z = (T + kMaxRows - 1) / kMaxRows, each = (T + z - 1) / z;
  p.rows = (int32_t)((each + 15) / 16 * 16);
  const int64_t steps = (K / 32 + 7) / 8, most = kDCols / p.rows * 4, quarters = (N + 31) / 32;
  double best = 1e300;
  for (int c = 1; c <= kMaxSplits && (c == 1 || c <= steps); c *= 2) {
    const int64_t at_once = clusters[c];
    if (at_once == 0) continue;
    int64_t q = (quarters * z + at_once - 1) / at_once;
    if (q > most) q = most;
    const int64_t grid = (quarters + q - 1) / q * z, waves = (grid + at_once - 1) / at_once;
    const double cost = (double)waves * (double)((q + 3) / 4 * ((steps + c - 1) / c) + 3);
    if (cost < best) {
      best = cost;
      p.splits = c;
      p.quarters = (int32_t)q;
    }
  }
  return p;
}

cudaError_t fb4_launch_linear_tc(const fb4_ctx* ctx, const void* x, int64_t T, int64_t ld, const uint8_t* codes, const uint16_t* meta, int64_t N,
                                 int64_t K, const void* bias, void* out, int64_t out_ld, int out_dtype, cudaStream_t stream) {
  Linear p{};
  p.x = static_cast<const uint16_t*>(x);
  p.ld = ld;
  p.meta = meta;
  p.bias = static_cast<const uint16_t*>(bias);
  p.out = out;
  p.out_ld = out_ld;
  p.T = T;
  p.N = N;
  p.nb = (int32_t)(K / 32);
  p.out_dtype = out_dtype;
  const int64_t item_bytes = out_dtype == 0 ? 4 : 2;
  p.wide_out = reinterpret_cast<uintptr_t>(out) % (4 * item_bytes) == 0 && out_ld % 4 == 0;
  p.tables = ctx->d_tables;
  p.status = ctx->d_status;
  const Fb4LinearTcPlan plan = fb4_linear_tc_plan(ctx->linear_tc_clusters, T, N, K);
  p.rows = plan.rows;
  p.splits = plan.splits;
  p.quarters = plan.quarters;
  const int32_t steps = (p.nb + 7) / 8;
  const int64_t quarters = (N + 31) / 32, z = (T + kMaxRows - 1) / kMaxRows;
  const int32_t mine = (steps + p.splits - 1) / p.splits, step_bytes = p.rows * 512;
  const int32_t tiles = (p.quarters + 3) / 4;
  p.stages = (int64_t)mine * tiles < kStages ? mine * tiles : kStages;
  const int32_t x_bytes = kXBytes + (kStages - p.stages) * kStage;
  p.buffers = (int64_t)mine * step_bytes <= x_bytes ? 1 : 2;
  p.chunk = p.buffers == 1 ? mine : x_bytes / 2 / step_bytes;
  CUtensorMap map;
  cudaError_t e = fb4_encode_map_2d(&map, codes, (uint64_t)K / 2, (uint64_t)N, (uint64_t)K / 2, 128, 32, CU_TENSOR_MAP_SWIZZLE_128B);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  cfg.gridDim = dim3((unsigned)((quarters + p.quarters - 1) / p.quarters * p.splits), (unsigned)z);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kBytes;
  cfg.stream = stream;
  cfg.attrs = attr;
  if (p.splits > 1) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.numAttrs = 1;
  }
  return cudaLaunchKernelEx(&cfg, fb4_linear_tc_kernel, map, p);
}
