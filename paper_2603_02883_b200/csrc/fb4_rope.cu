// Per-head RMS norm with the position rotation, and the append of keys and values to the paged FB4 cache.
//
// Rows belong to lanes as fb4_rope.cuh has it; the cosines and sines of a lane's 8 pairs stay in 16 registers while it walks over the
// heads of a token: the table is read once per token and lane instead of once per head.
//
// Both kernels stream.  Norm and rotation: 288 instructions a row and lane, 66 % of the issue slots, the rest waits for loads: 32760
// tokens of 24 heads of 128 in 83 us, 4.9 TB/s, 74 % of the copy bandwidth (a plain copy of the same rows by the same loop takes 70).
// Append, where the quantizer adds about 9 instructions per element: 32760 tokens of 12 + 2 * 12 heads in 147 us, 3.1 TB/s.  Nothing
// is saturated (60 % of the issue slots, 36 % of DRAM): 128 registers leave 16 warps per SM, which wait for the rows of a unit before they
// work on it.
#include "fb4_block.cuh"
#include "fb4_device.cuh"
#include "fb4_internal.h"
#include "fb4_rope.cuh"
#include "fb4_staging.cuh"

namespace {

using namespace fb4blk;
using namespace fb4rope;

struct NormRopeParams {
  Heads q, k, v;            // k and v leave as FB4 blocks in the append, k as bf16 otherwise (v.n = 0 then)
  RopeTable rope;
  int64_t T;
  int32_t D;
  float eps, inv_d;
  // How rows are dealt out.  A warp handles RP = 32 / LG rows at a time (a pass): `per_token` of them, a power of two, belong to
  // one token, so RP / per_token tokens go together.  Two passes are a unit (what the quantizer takes at a time); a token has
  // units[0] of q and units[1] of k, or of k and v.  An item is such a group of tokens, or one of `parts` shares of its
  // units where there are few tokens; items go round the warps.
  int32_t per_token_log2, units[2], parts, part_units;
  int64_t items;
  const int64_t* slot;
  fb4_cache cache;
  int32_t page_shift;
  uint32_t* status;
};

__device__ __forceinline__ uint32_t upper_halves(float lo, float hi) {
  return prmt(__float_as_uint(lo), __float_as_uint(hi), 0x7632u);
}

// Waits, with a limit, for the copy of the quantizer's tables.
__device__ __forceinline__ void wait_tables(uint32_t bar, uint32_t* status) {
  uint32_t tries = 0;
  bool ok = fb4stage::mbar_try_wait(bar, 0u);
  while (!ok && ++tries < fb4stage::kSpinLimit) ok = fb4stage::mbar_try_wait(bar, 0u);
  if (!__all_sync(0xffffffffu, ok) && (threadIdx.x & 31) == 0) atomicOr(status, 1u);
}

// The unit's two rows of this lane group, as far as they exist.
struct Rows {
  uint4 a[2], b[2];
};

// CACHE: k and v rows are quantized and go to the cache.  Their values' upper 16 bits, all that the quantizer reads of a
// float32, go through shared memory from the 16-channels-per-lane layout to one block of 32 channels per lane.
template <int LG, bool INTER, bool CACHE>
__device__ __forceinline__ void rows_of_warp(const NormRopeParams& p, uint32_t stage, uint32_t gains, int64_t warp, int64_t n_warps,
                                             const Tables* tb, uint32_t table_bar, bool& bad) {
  constexpr int RP = 32 / LG, NBL = LG / 2;    // NBL: lanes of a row in the quantizer's layout
  const int lane = threadIdx.x & 31, j = lane % LG, g = lane / LG;
  const bool on = j < p.D / 16;
  const int half = p.D / 2;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const int lg2 = p.per_token_log2, per = 1 << lg2;
  const int sub = g >> lg2, hs = g & (per - 1);
  const LanePairs lp = lane_pairs<INTER>(p.rope, on ? j : 0, p.D);
  const int qg = (lane / NBL) % RP, qk = (lane / NBL) / RP, qblk = lane % NBL;      // the row this lane quantizes: group, pass of the two
  bool tables = false;

  for (int64_t item = warp; item < p.items; item += n_warps) {
    int64_t group = item;
    int32_t u0 = 0, u1 = p.units[0] + p.units[1];
    if (p.parts > 1) {
      group = item / p.parts;
      u0 = (int32_t)(item - group * p.parts) * p.part_units;
      u1 = min(u0 + p.part_units, u1);
    }
    const int64_t token_or_more = group * (RP >> lg2) + sub;
    const bool real = token_or_more < p.T;
    const int64_t token = real ? token_or_more : p.T - 1;
    CosSin cs;
    bool have_cs = false;
    auto want_cs = [&]() {                     // after the first rows are requested
      if (p.rope.table && !have_cs) load_cs(p.rope, lp, token, cs, bad);
      have_cs = true;
    };
#pragma unroll
    for (int seg = 0; seg < 2; ++seg) {
      const Heads& hd = seg ? p.k : p.q;
      const int32_t first = seg ? p.units[0] : 0, from = max(u0, first) - first, to = min(u1, first + p.units[seg]) - first;
      if (from >= to) continue;
      if (seg == 0 || !CACHE) {
        const uint32_t gain = gains + (seg * 4 * LG + j) * 16;
        int32_t h = from * 2 * per + hs;
        const uint16_t* x = hd.x + token * hd.ld + h * p.D + 8 * j;
        uint16_t* o = hd.out + token * hd.out_ld + h * p.D + 8 * j;
        for (int32_t u = from; u < to; ++u, h += 2 * per, x += 2 * per * p.D, o += 2 * per * p.D) {
          const bool v[2] = {real && on && h < hd.n, real && on && h + per < hd.n};
          Rows r;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            r.a[k] = r.b[k] = zero;
            if (v[k]) {
              r.a[k] = *reinterpret_cast<const uint4*>(x + k * per * p.D);
              r.b[k] = *reinterpret_cast<const uint4*>(x + k * per * p.D + half);
            }
          }
          want_cs();
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if ((2 * u + k) * per >= hd.n) break;      // the second pass may have no rows at all
            Share y;
            norm_rotate<LG, INTER>(r.a[k], r.b[k], hd.gain != nullptr, gain, p, cs, y);
            pack<INTER>(y, pack_bf16, r.a[k], r.b[k]);
            if (v[k]) {
              *reinterpret_cast<uint4*>(o + k * per * p.D) = r.a[k];
              *reinterpret_cast<uint4*>(o + k * per * p.D + half) = r.b[k];
            }
          }
        }
      } else {
        const uint32_t gain = gains + (4 * LG + j) * 16;
        // run r of row R goes to 16-byte column (r & ~3) | ((r ^ r >> 2 ^ R) & 3) of it: no bank conflicts on either side
        auto at_run = [&](int row, int run) -> uint32_t {
          return stage + (uint32_t)row * (LG * 32) + (uint32_t)(((run & ~3) | ((run ^ (run >> 2) ^ row) & 3)) * 16);
        };
        const int64_t q_token = group * (RP >> lg2) + (qg >> lg2);
        int64_t slot = q_token < p.T ? __ldg(p.slot + q_token) : -1;
        if (slot < -1 || slot >= p.cache.n_pages << p.page_shift) {      // reported and left out, as -1 is left out
          bad = true;
          slot = -1;
        }
        const int64_t slot_row = ((slot >> p.page_shift) * p.cache.n_heads << p.page_shift) + (slot & ((1 << p.page_shift) - 1));
        int32_t h = from * 2 * per + hs, qh = (from * 2 + qk) * per + (qg & (per - 1));
        const uint16_t* kx = p.k.x + token * p.k.ld + h * p.D + 8 * j;
        const uint16_t* vx = p.v.x + token * p.v.ld + (h - p.k.n) * p.D + 8 * j;
        for (int32_t u = from; u < to; ++u, h += 2 * per, qh += 2 * per, kx += 2 * per * p.D, vx += 2 * per * p.D) {
          const bool key[2] = {h < p.k.n, h + per < p.k.n};
          Rows r;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            r.a[k] = r.b[k] = zero;
            if (real && on && h + k * per < 2 * p.k.n) {
              const uint16_t* x = (key[k] ? kx : vx) + k * per * p.D;
              r.a[k] = __ldg(reinterpret_cast<const uint4*>(x));
              r.b[k] = __ldg(reinterpret_cast<const uint4*>(x + half));
            }
          }
          if (__any_sync(0xffffffffu, key[0])) want_cs();
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (__any_sync(0xffffffffu, key[k])) {      // a pass of v rows alone needs neither norm nor rotation
              Share y;
              norm_rotate<LG, INTER>(key[k] ? r.a[k] : zero, key[k] ? r.b[k] : zero, p.k.gain != nullptr, gain, p, cs, y);
              if (key[k]) pack<INTER>(y, upper_halves, r.a[k], r.b[k]);
            }
            if (on) {
              const int row = g + k * RP;
              const uint32_t wa = at_run(row, j), wb = at_run(row, j + p.D / 16);
              asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(wa), "r"(r.a[k].x), "r"(r.a[k].y), "r"(r.a[k].z), "r"(r.a[k].w) : "memory");
              asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(wb), "r"(r.b[k].x), "r"(r.b[k].y), "r"(r.b[k].z), "r"(r.b[k].w) : "memory");
            }
          }
          __syncwarp();
          if (!tables) {                       // they arrive while the first rows are loaded and rotated
            tables = true;
            wait_tables(table_bar, p.status);
          }
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint4 v = zero;
            if (qblk < p.D / 32) v = lds_v4(at_run(lane / NBL, 4 * qblk + i));
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
          }
          __syncwarp();
          uint32_t cw[4], Eb[2];
          int did[2];
          const Lane ln = lane_state(tb);
          quantize_packed_block<false, false, false>(w, 0xffffffffu, tb, ln.qerr_lane, ln.pair_base, 3u, 254u, cw, did, Eb);
          if (qblk < p.D / 32 && slot >= 0 && qh < 2 * p.k.n) {
            const bool qkey = qh < p.k.n;
            const int64_t row = slot_row + ((int64_t)(qkey ? qh : qh - p.k.n) << p.page_shift);
            uint8_t* codes = (qkey ? p.cache.k_codes : p.cache.v_codes) + row * half + qblk * 16;
            uint16_t* meta = (qkey ? p.cache.k_meta : p.cache.v_meta) + row * (p.D / 32) + qblk;
            *reinterpret_cast<uint4*>(codes) = make_uint4(cw[0], cw[1], cw[2], cw[3]);
            *meta = (uint16_t)((Eb[0] - 3u) | ((uint32_t)did[0] << 8));
          }
        }
      }
    }
  }
}

constexpr int kRopeWarps = 8, kRopeCtas = 3;         // per SM
constexpr int kAppendWarps = 16;
constexpr int kStageBytes = 2048;                    // a unit on its way to the quantizer
constexpr size_t kAppendSmem = sizeof(Tables) + kAppendWarps * kStageBytes + kGainBytes;

template <int LG, bool INTER>
__global__ void __launch_bounds__(kRopeWarps * 32, kRopeCtas) fb4_norm_rope_kernel(const __grid_constant__ NormRopeParams p) {
  __shared__ __align__(16) uint8_t gain_smem[kGainBytes];
  const uint32_t gains = smem_u32(gain_smem);
  stage_gains<LG, INTER>(p, gains);
  __syncthreads();
  bool bad = false;
  rows_of_warp<LG, INTER, false>(p, 0u, gains, (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5), (int64_t)gridDim.x * kRopeWarps, nullptr, 0u, bad);
  if (__any_sync(0xffffffffu, bad) && (threadIdx.x & 31) == 0) atomicOr(p.status, 2u);
}

template <int LG, bool INTER>
__global__ void __launch_bounds__(kAppendWarps * 32, 1)
fb4_cache_append_kernel(const __grid_constant__ NormRopeParams p, const Tables* __restrict__ g_tables) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ uint64_t table_bar;
  Tables* tb = reinterpret_cast<Tables*>(smem);
  const uint32_t bar = smem_u32(&table_bar);
  if (threadIdx.x == 0) {
    fb4stage::mbar_init(bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fb4stage::mbar_expect_tx(bar, (uint32_t)sizeof(Tables));
    fb4stage::bulk_load(smem_u32(tb), g_tables, (uint32_t)sizeof(Tables), bar);
  }
  const uint32_t warps_at = smem_u32(smem) + (uint32_t)sizeof(Tables), gains = warps_at + kAppendWarps * kStageBytes;
  stage_gains<LG, INTER>(p, gains);
  __syncthreads();
  const int64_t warp = (int64_t)blockIdx.x * kAppendWarps + (threadIdx.x >> 5), n_warps = (int64_t)gridDim.x * kAppendWarps;
  bool bad = false;
  rows_of_warp<LG, INTER, true>(p, warps_at + (threadIdx.x >> 5) * kStageBytes, gains, warp, n_warps, tb, bar, bad);
  if (__any_sync(0xffffffffu, bad) && (threadIdx.x & 31) == 0) atomicOr(p.status, 2u);
  wait_tables(bar, p.status);      // the copy must have landed before the CTA ends, in warps without cache rows too
}

// How the rows of a call are dealt out (see NormRopeParams); `warps` = all that can be resident.
void deal(NormRopeParams& p, int lg, int64_t warps) {
  const int rp = 32 / lg;
  const int32_t second = p.v.n > 0 ? 2 * p.k.n : p.k.n, most = p.q.n > second ? p.q.n : second;
  p.per_token_log2 = 0;
  while ((1 << p.per_token_log2) < rp && (1 << p.per_token_log2) < most) ++p.per_token_log2;
  const int32_t per = 1 << p.per_token_log2;
  p.units[0] = (p.q.n + 2 * per - 1) / (2 * per);
  p.units[1] = (second + 2 * per - 1) / (2 * per);
  const int64_t groups = (p.T + rp / per - 1) / (rp / per);
  const int32_t units = p.units[0] + p.units[1];
  // few tokens: a token's units are shared out until every warp has some
  p.parts = 1;
  p.part_units = units;
  if (groups < warps) {
    const int64_t parts = (warps + groups - 1) / groups;
    p.part_units = (int32_t)(parts < units ? (units + parts - 1) / parts : 1);
    p.parts = (units + p.part_units - 1) / p.part_units;
  }
  p.items = groups * p.parts;
}

void fill(NormRopeParams& p, const fb4_ctx* ctx, int64_t T, int D, float eps, const fb4_rope* rope) {
  p.T = T;
  p.D = D;
  p.eps = eps;
  p.inv_d = (float)(1.0 / D);
  p.status = ctx->d_status;
  p.rope = rope_of(rope, D);
}

}  // namespace

// Opt-in to the dynamic shared memory of the append kernels on the current device.
cudaError_t fb4_rope_prepare_device() {
  cudaError_t e = cudaSuccess;
#define FB4_OPT_IN(LG, INTER) \
  if (e == cudaSuccess) e = cudaFuncSetAttribute(fb4_cache_append_kernel<LG, INTER>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kAppendSmem)
  FB4_OPT_IN(2, false);
  FB4_OPT_IN(2, true);
  FB4_OPT_IN(4, false);
  FB4_OPT_IN(4, true);
  FB4_OPT_IN(8, false);
  FB4_OPT_IN(8, true);
  FB4_OPT_IN(16, false);
  FB4_OPT_IN(16, true);
#undef FB4_OPT_IN
  return e;
}

cudaError_t fb4_launch_norm_rope(const fb4_ctx* ctx, const void* q, int32_t q_heads, int64_t q_ld, const void* k,
                                 int32_t k_heads, int64_t k_ld, int64_t T, int32_t D, const void* q_gain, const void* k_gain,
                                 float eps, const fb4_rope* rope, void* q_out, int64_t q_out_ld, void* k_out, int64_t k_out_ld,
                                 cudaStream_t stream) {
  NormRopeParams p{};
  fill(p, ctx, T, D, eps, rope);
  p.q = heads_of(q, q_ld, q_heads, q_gain, q_out, q_out_ld);
  p.k = heads_of(k, k_ld, k_heads, k_gain, k_out, k_out_ld);
  const int lg = lanes_of(D);
  const int64_t most = (int64_t)ctx->sm_count * kRopeCtas;
  deal(p, lg, most * kRopeWarps);
  int64_t grid = (p.items + kRopeWarps - 1) / kRopeWarps;
  if (grid > most) grid = most;
  const bool inter = rope && rope->interleaved;
#define FB4_ROTATE(LG) \
  inter ? fb4_norm_rope_kernel<LG, true><<<(unsigned)grid, kRopeWarps * 32, 0, stream>>>(p) \
        : fb4_norm_rope_kernel<LG, false><<<(unsigned)grid, kRopeWarps * 32, 0, stream>>>(p)
  switch (lg) {
    case 2: FB4_ROTATE(2); break;
    case 4: FB4_ROTATE(4); break;
    case 8: FB4_ROTATE(8); break;
    default: FB4_ROTATE(16); break;
  }
#undef FB4_ROTATE
  return cudaGetLastError();
}

cudaError_t fb4_launch_cache_append(const fb4_ctx* ctx, const void* q, int32_t q_heads, int64_t q_ld, const void* k,
                                    int64_t k_ld, const void* v, int64_t v_ld, int64_t T, const void* q_gain,
                                    const void* k_gain, float eps, const fb4_rope* rope, const int64_t* slot,
                                    const fb4_cache* cache, void* q_out, int64_t q_out_ld, cudaStream_t stream) {
  NormRopeParams p{};
  const int D = cache->head_dim;
  fill(p, ctx, T, D, eps, rope);
  p.q = heads_of(q, q_ld, q_heads, q_gain, q_out, q_out_ld);
  p.k = heads_of(k, k_ld, cache->n_heads, k_gain, nullptr, 0);
  p.v = heads_of(v, v_ld, cache->n_heads, nullptr, nullptr, 0);
  p.slot = slot;
  p.cache = *cache;
  while ((1 << p.page_shift) < cache->page_tokens) ++p.page_shift;
  const int lg = lanes_of(D);
  deal(p, lg, (int64_t)ctx->sm_count * kAppendWarps);
  int64_t grid = (p.items + kAppendWarps - 1) / kAppendWarps;
  if (grid > ctx->sm_count) grid = ctx->sm_count;
  const Tables* tables = static_cast<const Tables*>(ctx->d_fast_tables);
  const bool inter = rope && rope->interleaved;
#define FB4_APPEND(LG) \
  inter ? fb4_cache_append_kernel<LG, true><<<(unsigned)grid, kAppendWarps * 32, kAppendSmem, stream>>>(p, tables) \
        : fb4_cache_append_kernel<LG, false><<<(unsigned)grid, kAppendWarps * 32, kAppendSmem, stream>>>(p, tables)
  switch (lg) {
    case 2: FB4_APPEND(2); break;
    case 4: FB4_APPEND(4); break;
    case 8: FB4_APPEND(8); break;
    default: FB4_APPEND(16); break;
  }
#undef FB4_APPEND
  return cudaGetLastError();
}
