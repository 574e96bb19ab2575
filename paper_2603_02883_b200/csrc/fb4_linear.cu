// Products of up to 16 rows with FB4 weights: y[t][n] = sum_k x[t][k] w[n][k] + bias[n].  More rows, and large weights: fb4_linear_tc.cu.
//
// The weights are the long side, so their rows are the M side of mma.sync m16n8k16 and the rows of x its N side: a warp reads a weight once
// for all of them.  A lane decodes a block of 32 channels of two rows at a time from two 16-byte words of codes, straight into
// the A fragments (which channel sits at which k is free, as long as x agrees).  x lies in shared memory in the order in which the
// lanes read it, 16 bytes for 8 channels.
//
// Work: a CTA of 8 warps takes 128 rows of W and one run of the channels; the CTAs of a row tile are a cluster, which joins their sums through
// distributed shared memory, always in the same order.
//
// Bound: the ALU pipe (decode: 10 operations per 8 weights, two thirds of all of its) while all warps are at work, CTAs that are two or three to
// an SM, and for small weights the start.  Weights out of memory, one row: 4096 x 4096 take 6.6 us, 12288 x 4096 12.9, 8192 x 8192 16.5 to 17.0 (2.2
// TB/s), 16384 x 4096 16.9, the largest; 16 rows with 6144 x 2048 8.5.  For 12288 x 4096 and 8192 x 8192, one row: 2 CTAs an SM take 16.0 and 16.4, 4 (which spill)
// 13.8 and 17.7; steps loaded one ahead 13.2 and 16.6, four ahead (spills) 14.9 and 18.8.  8192 x 8192 in clusters of 1, 2, 3, 4, 6 (the rule's choice), 8: 39.7,
// 21.9, 20.2, 15.8, 16.7, 19.3.  Of an older form, for weights that are the other kernel's now (12288 x 12288, 31.1): one CTA per SM with its rows dealt out
// evenly 39.6, 16 warps an SM with loads four steps ahead 49.8 in two waves.
#include "fb4_attend.cuh"
#include "fb4_block.cuh"

namespace {

using namespace fb4att;

constexpr int kWarps = 8;                       // a step of a warp is 128 channels: 4 blocks, one to each lane of a quad
constexpr int kAhead = 2;                        // steps that are loaded ahead
constexpr int kResident = 3;                     // CTAs per SM
constexpr int kRows = kWarps * 16;               // rows of W to a CTA
constexpr int kMaxSplits = 8;                    // portable cluster size
constexpr int kXBytes = 64 * 1024;               // most of x that a CTA holds at a time

struct Linear {
  const uint16_t* x;
  int64_t ld;
  const uint8_t* codes;
  const uint16_t* meta;
  const uint16_t* bias;
  void* out;
  int64_t out_ld;
  int64_t T, N;
  int32_t nb;               // blocks of a row
  int32_t splits;           // CTAs of a cluster
  int32_t chunk;            // steps whose x a CTA holds at a time
  int32_t wide;             // rows of x that have room in shared memory
  int32_t out_dtype;
  const Fb4DeviceTables* tables;
};

// NT: groups of 8 rows of x
template <int NT>
__global__ void __launch_bounds__(kWarps * 32, kResident) fb4_linear_kernel(const __grid_constant__ Linear p) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint32_t book[64];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t tile = blockIdx.x / (uint32_t)p.splits;
  const int32_t split = (int32_t)(blockIdx.x - (uint32_t)tile * p.splits);
  const int64_t n0 = tile * kRows + warp * 16;
  const int32_t n_tok = (int32_t)p.T;
  const int32_t steps = (p.nb + 3) / 4;
  const int32_t s_begin = steps * split / p.splits, s_end = steps * (split + 1) / p.splits;      // 2^24 steps, 8 CTAs at most
  const uint32_t x_at = fb4blk::smem_u32(smem), book_at = fb4blk::smem_u32(book);
  if (threadIdx.x < 64) fill_book(book, p.tables, threadIdx.x);

  // this lane's rows of W, from the run's first block on; rows behind the last are computed like it and not stored
  const uint8_t* codes[2];
  const uint16_t* meta[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int64_t n = n0 + 8 * r + g, at = (n < p.N ? n : p.N - 1) * p.nb + 4 * (int64_t)s_begin + t;
    codes[r] = p.codes + at * 16;
    meta[r] = p.meta + at;
  }
  float acc[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.0f;
  uint4 cw[kAhead][2];
  uint16_t mt[kAhead][2];                           // joined only when used: that would wait for the load
  const int32_t whole = p.nb / 4;                   // steps whose four blocks all exist; there is at most one more
  // loads step s, which lies i steps behind the pointers, into ring place `at`
  auto load = [&](int32_t s, int i, int at) {
    const bool there = s < whole || 4 * s + t < p.nb;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      cw[at][r] = make_uint4(0, 0, 0, 0);
      mt[at][r] = 0;                                // scale byte 0 and codes 0: zeros
      if (there) {
        cw[at][r] = __ldg(reinterpret_cast<const uint4*>(codes[r] + 64 * i));
        mt[at][r] = __ldg(meta[r] + 4 * i);
      }
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (s_begin + i < s_end) load(s_begin + i, i, i);

  // x of a chunk, piece (s, w, g, t): channels 8 w .. 8 w + 7 of block 4 s + t of row g, in the order 0 2 1 3 4 6 5 7 of the decoder; only
  // `wide` rows (a power of two) have room, and the lanes behind them read zeros
  const uint32_t x_piece = p.wide * 64;
  const bool x_there = lane < 4 * p.wide;
  for (int32_t c0 = s_begin; c0 < s_end; c0 += p.chunk) {
    const int32_t c1 = c0 + p.chunk < s_end ? c0 + p.chunk : s_end;
    __syncthreads();                                // nobody reads the x of the chunk before any more
    for (int32_t i = warp; i < p.wide * ((c1 - c0 + 1) / 2); i += kWarps) {               // 2 steps of a row to a warp
      const int32_t tok = i % p.wide, k16 = i / p.wide * 32 + lane;                     // 16-byte piece of the chunk's row
      if (k16 >= (c1 - c0) * 16) continue;
      uint4 u = make_uint4(0, 0, 0, 0);
      if (tok < n_tok && 4 * c0 + (k16 >> 2) < p.nb) u = __ldg(reinterpret_cast<const uint4*>(p.x + tok * p.ld) + (int64_t)c0 * 16 + k16);
      const uint32_t dst = x_at + tok * 64 + ((k16 >> 4) * 4 + (k16 & 3)) * x_piece + ((k16 >> 2) & 3) * 16;
      asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(prmt(u.x, u.y, 0x5410u)), "r"(prmt(u.x, u.y, 0x7632u)),
                   "r"(prmt(u.z, u.w, 0x5410u)), "r"(prmt(u.z, u.w, 0x7632u)) : "memory");
    }
    __syncthreads();
    uint32_t x_step = x_at + (NT > 1 ? lane : lane & (4 * p.wide - 1)) * 16;
    for (int32_t s0 = c0; s0 < c1; s0 += kAhead) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int32_t s = s0 + i;
        if (s >= c1) break;
        BlockScale sc[2];
        uint32_t words[2][4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          sc[r] = block_scale(mt[i][r], book_at, true);
          words[r][0] = cw[i][r].x; words[r][1] = cw[i][r].y; words[r][2] = cw[i][r].z; words[r][3] = cw[i][r].w;
        }
        if (s + kAhead < s_end) load(s + kAhead, i + kAhead, i);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t a[2][4];
          decode_word(words[0][w], sc[0], a[0]);
          decode_word(words[1][w], sc[1], a[1]);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            uint4 b = make_uint4(0, 0, 0, 0);
            if (NT > 1 || x_there) b = fb4blk::lds_v4(x_step + (i * 4 + w) * x_piece + n * 512);
            mma_bf16(acc[n], a[0][0], a[1][0], a[0][1], a[1][1], b.x, b.y);
            mma_bf16(acc[n], a[0][2], a[1][2], a[0][3], a[1][3], b.z, b.w);
          }
        }
      }
      x_step += kAhead * 4 * x_piece;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        codes[r] += 64 * kAhead;
        meta[r] += 4 * kAhead;
      }
    }
  }

  // ---- the sums, [row of x][row of W], to shared memory; then the cluster's CTAs each finish a part of them
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);
  constexpr int kLd = kRows + 4;                    // the quads' rows of x fall into different banks
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int k = 0; k < 4; ++k) sums[(8 * n + 2 * t + (k & 1)) * kLd + warp * 16 + g + 8 * (k >> 1)] = acc[n][k];
  if (p.splits > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  else __syncthreads();
  for (int32_t i = split * (kWarps * 32) + threadIdx.x; i < n_tok * kRows; i += p.splits * (kWarps * 32)) {
    const int32_t tok = i / kRows, r = i % kRows;
    const int64_t n = tile * kRows + r;
    if (n >= p.N) continue;
    float v = 0.0f;
    if (p.splits > 1) {
      const uint32_t at = fb4blk::smem_u32(sums + tok * kLd + r);
#pragma unroll
      for (int z = 0; z < kMaxSplits; ++z)
        if (z < p.splits) {
          float u;
          asm volatile("{\n\t.reg .b32 q;\n\tmapa.shared::cluster.u32 q, %1, %2;\n\tld.shared::cluster.f32 %0, [q];\n\t}" : "=f"(u) : "r"(at), "r"(z));
          v += u;
        }
    } else {
      v = sums[tok * kLd + r];
    }
    v *= kUnshift;
    if (p.bias) v += __uint_as_float((uint32_t)__ldg(p.bias + n) << 16);
    const int64_t at = tok * p.out_ld + n;
    if (p.out_dtype == 0) static_cast<float*>(p.out)[at] = v;
    else if (p.out_dtype == 1) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
    else static_cast<__half*>(p.out)[at] = __float2half_rn(v);
  }
  // nobody's shared memory goes away while another CTA reads it
  if (p.splits > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

constexpr int kJoinBytes = 8 * (kRows + 4) * 4;                 // for 8 rows of x

}  // namespace

cudaError_t fb4_clusters_at_once(const void* kernel, int threads, int smem, int32_t* clusters) {
  for (int s = 1; s <= kMaxSplits; ++s) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)s;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(s * 1024));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
    clusters[s] = e == cudaSuccess && n > 0 ? n : 0;
    if (s == 1 && clusters[s] == 0) return e != cudaSuccess ? e : cudaErrorInvalidConfiguration;
  }
  return cudaSuccess;
}

// Opt-in to the dynamic shared memory, and the clusters that are resident at a time.
cudaError_t fb4_linear_prepare_device(int32_t* clusters) {
  cudaError_t e = cudaFuncSetAttribute(fb4_linear_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, kXBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(fb4_linear_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, kXBytes);
  if (e == cudaSuccess) e = fb4_clusters_at_once(reinterpret_cast<const void*>(fb4_linear_kernel<2>), kWarps * 32, kXBytes, clusters);
  return e;
}

// The least of waves x work of a CTA, its start and its part of the join counted as 4 steps.
int32_t fb4_linear_splits(const int32_t* clusters, int64_t N, int64_t K) {
  const int64_t tiles = (N + kRows - 1) / kRows, steps = (K / 32 + 3) / 4;
  double best = 1e300;
  int32_t splits = 1;
  for (int s = 1; s <= kMaxSplits && (s == 1 || steps / s >= 2); ++s) {
    if (clusters[s] == 0) continue;
    const int64_t waves = (tiles + clusters[s] - 1) / clusters[s];
    const double cost = (double)waves * (double)((steps + s - 1) / s + 4);
    if (cost < best * 0.97) {
      best = cost;
      splits = s;
    }
  }
  return splits;
}

cudaError_t fb4_launch_linear(const fb4_ctx* ctx, const void* x, int64_t T, int64_t ld, const uint8_t* codes, const uint16_t* meta, int64_t N,
                              int64_t K, const void* bias, void* out, int64_t out_ld, int out_dtype, cudaStream_t stream) {
  // The tensor-memory kernel starts 2.5 us later, but takes less for a weight, and next to nothing for another row.  This against that one, us, weights out of
  // memory: 4096 x 4096 6.6 / 9.1 (1 row), 7.8 / 9.3 (8 rows); 12288 x 4096 12.9 / 14.9 (1), 15.1 / 15.5 (8); 16384 x 4096 16.9 / 16.8 (1), 18.1 / 16.9 (4),
  // 19.7 / 17.2 (8); 8192 x 8192 17.0 / 17.9 (1), 19.5 / 18.1 (8); 8192 x 12288 22.4 / 23.0 (1), 23.9 / 23.2 (4), 26.0 / 23.8 (8); 32768 x 4096 30.3 / 27.1 (1),
  // 36.1 / 27.7 (8).  Of 9 to 16 rows this one takes small weights only.  16 rows: 640 x 640 6.3 / 6.6, 2048 x 2048 6.4 / 8.0, 4096 x 2048 7.2 / 8.4, 8192 x 1536 8.5 /
  // 9.0, 12288 x 1024 8.4 / 9.8, 6152 x 1568 9.1 / 9.9, 6144 x 2048 8.5 / 9.5, 256 x 4096 6.4 / 7.0, 1024 x 4096 7.7 / 8.0, 3200 x 4096 9.6 / 9.6 (9 rows 9.2 / 9.4), 3200 x
  // 3200 9.4 / 9.4; beyond, 4096 x 4096 9.8 / 9.8, 14000 x 1536 12.2 / 10.1, 8192 x 4096 15.5 / 12.8, and few rows of many channels, 1536 x 6144 10.0 / 9.0, 1024 x 8192
  // 12.0 / 9.5, 512 x 12288 16.4 / 10.6.
  const double size = (double)N * (double)K;
  if (T > 16 || (T > 8 && (size > 13e6 || K > 4096)) || size * (double)(T + 4) >= 640e6) return fb4_launch_linear_tc(ctx, x, T, ld, codes, meta, N, K, bias, out, out_ld, out_dtype, stream);
  Linear p{};
  p.x = static_cast<const uint16_t*>(x);
  p.ld = ld;
  p.codes = codes;
  p.meta = meta;
  p.bias = static_cast<const uint16_t*>(bias);
  p.out = out;
  p.out_ld = out_ld;
  p.T = T;
  p.N = N;
  p.nb = (int32_t)(K / 32);
  p.out_dtype = out_dtype;
  p.tables = ctx->d_tables;
  p.splits = fb4_linear_splits(ctx->linear_clusters, N, K);
  const int64_t tiles = (N + kRows - 1) / kRows;
  const int32_t steps = (p.nb + 3) / 4;
  const int32_t mine = (steps + p.splits - 1) / p.splits;
  for (p.wide = 1; p.wide < 16 && p.wide < T; p.wide *= 2) {}
  const int per_step = 256 * p.wide;
  const int32_t most = kXBytes / per_step / kAhead * kAhead;
  p.chunk = mine < most ? (mine + kAhead - 1) / kAhead * kAhead : most;
  int smem = p.chunk * per_step;
  const int join = T > 8 ? 2 * kJoinBytes : kJoinBytes;
  if (smem < join) smem = join;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  cfg.gridDim = dim3((unsigned)(tiles * p.splits));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  if (p.splits > 1) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.splits;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.numAttrs = 1;
  }
  return T > 8 ? cudaLaunchKernelEx(&cfg, fb4_linear_kernel<2>, p) : cudaLaunchKernelEx(&cfg, fb4_linear_kernel<1>, p);
}
