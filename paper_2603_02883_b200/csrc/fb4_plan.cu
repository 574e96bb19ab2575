// Plan of a serving step: which pages every sequence holds afterwards, and sequence, position and cache slot of the step's rows.
//
// Sequence b holds len tokens in its first ceil(len / page) pages, keeps the first keep of them and asks for n more.  With prefix
// sums over the sequences, in order, of the pages that go back, of those that are asked for and of the rows, everything has its place:
// page f of those that go back is entry top - 1 - f of the free list (top: its length with all of them), and page f of those that are
// taken is entry top - 1 - f too, so a step that is planned again gives every page back to where it came from.
//
// Bound: latency.  A CTA or, for larger steps, a cluster of 8 that computes the sums in every CTA (a few loads and scans; nothing of
// them has to be passed on) and shares out the pages and the rows, with a barrier where one may read what another wrote.
#include "fb4_internal.h"

namespace {

constexpr int kMaxThreads = 1024, kCluster = 8;

struct Plan {
  int32_t* page_table;
  int32_t max_pages, page_shift;
  int32_t* kv_len;
  const int32_t* keep;      // NULL = all
  const int32_t* new_len;
  int32_t n_seqs;
  int32_t* free_pages;
  int32_t free_cap;
  int32_t* n_free;
  int64_t T;
  int32_t* q_start;
  int64_t* slot;            // NULL = not wanted
  int32_t* pos;             // NULL = not wanted
  uint32_t* status;
};

struct Step {
  int32_t keep, n;          // tokens that stay, tokens asked for (0 where the table has no room for them)
  int32_t kept, back, need; // pages that stay, that go back, that are asked for
};

__device__ __forceinline__ Step step_of(const Plan& p, int32_t b, bool& bad) {
  const int64_t room = (int64_t)p.max_pages << p.page_shift;
  const int64_t len = p.kv_len[b];             // plain loads: the kernel writes some of these arrays at its end
  const int64_t held = len < 0 ? 0 : len < room ? len : room;
  int64_t keep = held;
  if (p.keep) {
    const int64_t k = p.keep[b];
    if (k < 0) bad = true;
    keep = k < 0 ? 0 : k < held ? k : held;
  }
  int64_t n = p.new_len[b];
  if (held != len || n < 0) bad = true;
  if (n < 0 || keep + n > room) n = 0;
  const int64_t up = (1 << p.page_shift) - 1;
  Step s;
  s.keep = (int32_t)keep;
  s.n = (int32_t)n;
  s.kept = (int32_t)((keep + up) >> p.page_shift);
  s.back = (int32_t)((held + up) >> p.page_shift) - s.kept;
  s.need = (int32_t)((keep + n + up) >> p.page_shift) - s.kept;
  return s;
}

__device__ __forceinline__ void all_sync(bool cluster) {
  if (cluster) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  else __syncthreads();
}

// Inclusive sums over the threads of the CTA; the totals come back in `all`.  Two barriers.
struct Sums {
  int64_t pages, rows;
};
__device__ __forceinline__ Sums inclusive(Sums v, Sums& all, Sums* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int64_t a = __shfl_up_sync(0xffffffffu, v.pages, off), b = __shfl_up_sync(0xffffffffu, v.rows, off);
    if (lane >= off) { v.pages += a; v.rows += b; }
  }
  if (lane == 31) part[warp] = v;
  __syncthreads();
  Sums w{0, 0};
  if (lane < warps) w = part[lane];
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int64_t a = __shfl_up_sync(0xffffffffu, w.pages, off), b = __shfl_up_sync(0xffffffffu, w.rows, off);
    if (lane >= off) { w.pages += a; w.rows += b; }
  }
  all.pages = __shfl_sync(0xffffffffu, w.pages, 31);
  all.rows = __shfl_sync(0xffffffffu, w.rows, 31);
  const int before = warp ? warp - 1 : 0;
  const int64_t a = __shfl_sync(0xffffffffu, w.pages, before), b = __shfl_sync(0xffffffffu, w.rows, before);
  if (warp) { v.pages += a; v.rows += b; }
  __syncthreads();
  return v;
}

// the last i in [lo, hi) with at[i] <= x; at ascends and at[lo] <= x
__device__ __forceinline__ int32_t find(const int32_t* at, int32_t lo, int32_t hi, int64_t x) {
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (at[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kMaxThreads) fb4_plan_kernel(const __grid_constant__ Plan p) {
  extern __shared__ int32_t starts[];      // [n_seqs + 1], q_start
  __shared__ Sums part[32];
  __shared__ int32_t first[kMaxThreads], kept_of[kMaxThreads];
  const bool cluster = gridDim.x > 1;
  const int tid = threadIdx.x;
  const int32_t all = blockDim.x * gridDim.x, me = blockIdx.x * blockDim.x + tid;
  bool bad = false;

  // ---- how many pages go back
  const int32_t f0 = *p.n_free;
  int64_t free0 = f0 < 0 ? 0 : f0 < p.free_cap ? f0 : p.free_cap;
  if (free0 != f0) bad = true;
  int64_t back = 0;
  for (int32_t b0 = 0; b0 < p.n_seqs; b0 += blockDim.x) {
    Sums v{0, 0}, sum;
    if (b0 + tid < p.n_seqs) v.pages = step_of(p, b0 + tid, bad).back;
    inclusive(v, sum, part);
    back += sum.pages;
  }
  int64_t top = free0 + back;
  const int64_t over = top > p.free_cap ? top - p.free_cap : 0;      // pages that the list has no room for are lost, and reported
  if (over) bad = true;

  // ---- they go to the free list
  if (back) {
    int64_t before = 0;
    for (int32_t b0 = 0; b0 < p.n_seqs; b0 += blockDim.x) {
      Sums v{0, 0}, sum;
      Step s{};
      if (b0 + tid < p.n_seqs) s = step_of(p, b0 + tid, bad);
      v.pages = s.back;
      const Sums at = inclusive(v, sum, part);
      first[tid] = (int32_t)(at.pages - s.back);
      kept_of[tid] = s.kept;
      __syncthreads();
      for (int64_t f = me; f < sum.pages; f += all) {
        const int32_t i = find(first, 0, blockDim.x, f);
        const int64_t to = top - 1 - before - f;
        if (to < p.free_cap) p.free_pages[to] = p.page_table[(int64_t)(b0 + i) * p.max_pages + kept_of[i] + (f - first[i])];
      }
      before += sum.pages;
      __syncthreads();
    }
    all_sync(cluster);
  }
  top -= over;

  // ---- who is served, and with which pages
  Sums before{0, 0};                                                  // asked for by the sequences in front
  int64_t rows = 0, taken = 0;                                        // given to them
  for (int32_t b0 = 0; b0 < p.n_seqs; b0 += blockDim.x) {
    Sums sum;
    Step s{};
    const bool mine = b0 + tid < p.n_seqs;
    if (mine) s = step_of(p, b0 + tid, bad);
    Sums at = inclusive(Sums{s.need, s.n}, sum, part);
    at.pages += before.pages;
    at.rows += before.rows;
    const bool served = at.pages <= top && at.rows <= p.T;            // sums ascend: from the first that is not, nobody who asks for any
    const Sums mine_now = served ? Sums{s.need, s.n} : Sums{0, 0};
    Sums got = sum;
    const bool some_not = __syncthreads_or(!served && s.n > 0);
    Sums upto{at.pages - before.pages, at.rows - before.rows};
    if (some_not) upto = inclusive(mine_now, got, part);
    if (mine) {
      const int32_t start = (int32_t)(rows + upto.rows - mine_now.rows);
      starts[b0 + tid] = start;
      if (blockIdx.x == 0) p.q_start[b0 + tid] = start;
    }
    first[tid] = (int32_t)(upto.pages - mine_now.pages);
    kept_of[tid] = s.kept;
    __syncthreads();
    for (int64_t f = me; f < got.pages; f += all) {
      const int32_t i = find(first, 0, blockDim.x, f);
      p.page_table[(int64_t)(b0 + i) * p.max_pages + kept_of[i] + (f - first[i])] = p.free_pages[top - 1 - taken - f];
    }
    before.pages += sum.pages;
    before.rows += sum.rows;
    rows += got.rows;
    taken += got.pages;
    __syncthreads();
  }
  if (tid == 0) {
    starts[p.n_seqs] = (int32_t)rows;
    if (blockIdx.x == 0) p.q_start[p.n_seqs] = (int32_t)rows;
  }
  all_sync(cluster);

  // ---- the rows: a warp takes a run of them and walks over the sequences that it belongs to
  {
    const int lane = tid & 31;
    const int64_t warps = all >> 5, per = ((p.T + warps - 1) / warps + 31) & ~(int64_t)31;
    const int64_t r0 = (me >> 5) * per, r1 = r0 + per < p.T ? r0 + per : p.T;
    int32_t b = r0 < rows ? find(starts, 0, p.n_seqs, r0) : 0;
    for (int64_t r = r0 + lane; r - lane < r1; r += 32) {
      int64_t slot = -1;
      int32_t pos = 0;
      if (r - lane < rows) {                                          // some row of these 32 is a token's
        int32_t mine = b;
        if (r - lane + 31 >= starts[b + 1]) {
          mine = find(starts, b, p.n_seqs, r < rows ? r : rows - 1);
          b = __shfl_sync(0xffffffffu, mine, 31);
        }
        if (r < rows) {
          bool ignored = false;
          pos = step_of(p, mine, ignored).keep + (int32_t)(r - starts[mine]);
          const int64_t page = p.page_table[(int64_t)mine * p.max_pages + (pos >> p.page_shift)];
          slot = (page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
        }
      }
      if (r < r1) {
        if (p.slot) p.slot[r] = slot;
        if (p.pos) p.pos[r] = pos;
      }
    }
  }
  all_sync(cluster);

  // ---- lengths last: until here everybody reads what the sequences held
  for (int32_t b = me; b < p.n_seqs; b += all) {
    bool ignored = false;
    p.kv_len[b] = step_of(p, b, ignored).keep + starts[b + 1] - starts[b];
  }
  if (me == 0) *p.n_free = (int32_t)(top - taken);
  if (__syncthreads_or(bad) && me == 0) atomicOr(p.status, 2u);
}

}  // namespace

cudaError_t fb4_plan_prepare_device() {
  cudaError_t e = cudaFuncSetAttribute(fb4_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (FB4_PLAN_MAX_SEQS + 1) * 4);
  return e;
}

cudaError_t fb4_launch_cache_plan(const fb4_ctx* ctx, int32_t* page_table, int32_t max_pages, int32_t page_tokens, int32_t* kv_len,
                                  const int32_t* keep, const int32_t* new_len, int32_t n_seqs, int32_t* free_pages, int32_t free_cap,
                                  int32_t* n_free, int64_t T, int32_t* q_start, int64_t* slot, int32_t* pos, cudaStream_t stream) {
  Plan p{page_table, max_pages, 0, kv_len, keep, new_len, n_seqs, free_pages, free_cap, n_free, T, q_start, slot, pos, ctx->d_status};
  while ((1 << p.page_shift) < page_tokens) ++p.page_shift;
  const bool large = T > 2048 || n_seqs > 512;
  int threads = kMaxThreads;
  if (!large)
    for (threads = 128; threads < n_seqs; threads *= 2) {}
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  cfg.gridDim = dim3(large ? kCluster : 1);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)(n_seqs + 1) * 4;
  cfg.stream = stream;
  cfg.attrs = attr;
  if (large) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kCluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.numAttrs = 1;
  }
  return cudaLaunchKernelEx(&cfg, fb4_plan_kernel, p);
}
