// Plan of a serving step: which pages every sequence holds afterwards, and sequence, position and cache slot of the step's rows.
//
// Sequence b holds len tokens in its first ceil(len / page) pages, keeps the first keep of them and asks for n more.  With prefix
// sums over the sequences, in order, of the pages that go back, of those that are asked for and of the rows, everything has its place:
// page f of those that go back is entry top - 1 - f of the free list (top: its length with all of them), and page f of those that are
// taken is entry top - 1 - f too, so a step that is planned again gives every page back to where it came from.
//
// Bound: latency.  One CTA, or for larger steps a cluster of 8, computes the sums (in every CTA: a few loads and one scan; nothing of them
// has to be passed on) and shares out the pages, with a barrier where one may read what another wrote; many rows are left to a second
// kernel on all SMs, launched early.  Lists are dealt out in runs: a warp looks up the sequence of its first entry and walks on from it, and
// only 32 entries that belong to several sequences cost a search each.  64 sequences of one token take 5.9 us on the device (a launch alone is 3.9), 2048 of
// them with 270 000 rows and 49 000 pages that move 17.6.
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
  int32_t rows_here;        // the rows are written by the first kernel
  uint32_t* status;
};

struct Step {
  int32_t keep, n;          // tokens that stay, tokens asked for (0 where the table has no room for them)
  int32_t back, need;       // pages that go back, that are asked for
};

__device__ __forceinline__ int32_t pages_of(const Plan& p, int64_t tokens) { return (int32_t)((tokens + (1 << p.page_shift) - 1) >> p.page_shift); }

// plain loads: the kernel writes some of these arrays at its end
__device__ __forceinline__ Step step_of(const Plan& p, int32_t b, bool& bad) {
  const int64_t room = (int64_t)p.max_pages << p.page_shift;
  const int64_t len = p.kv_len[b];
  int64_t n = p.new_len[b];
  const int64_t held = len < 0 ? 0 : len < room ? len : room;
  int64_t keep = held;
  if (p.keep) {
    const int64_t k = p.keep[b];
    if (k < 0) bad = true;
    keep = k < 0 ? 0 : k < held ? k : held;
  }
  if (held != len || n < 0) bad = true;
  if (n < 0 || keep + n > room) n = 0;
  const int32_t kept = pages_of(p, keep);
  return Step{(int32_t)keep, (int32_t)n, pages_of(p, held) - kept, pages_of(p, keep + n) - kept};
}

__device__ __forceinline__ void all_sync(bool cluster) {
  if (cluster) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  else __syncthreads();
}

struct Sums {
  int32_t back, need;       // below 2^31: a page table has fewer entries
  uint32_t rows;            // counted up to T + 1 at most, so that sums stay below 2^32
};

__device__ __forceinline__ Sums add(const Sums& x, const Sums& y, uint32_t most) {
  return Sums{x.back + y.back, x.need + y.need, min(x.rows + y.rows, most)};
}
__device__ __forceinline__ Sums scanned(Sums v, uint32_t most) {      // over the lanes of a warp
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const Sums u{__shfl_up_sync(0xffffffffu, v.back, off), __shfl_up_sync(0xffffffffu, v.need, off), __shfl_up_sync(0xffffffffu, v.rows, off)};
    if (lane >= off) v = add(v, u, most);
  }
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

// This lane's entries i of from .. to - 1, of which the first at[n] belong to owners 0 .. n - 1 (owner b has entries at[b] .. at[b + 1] - 1)
// and the others to none (-1): store(i, owner, load(i, owner)), with the loads of K entries in flight.  b: owner of the run's first entry.
template <int K, typename Load, typename Store>
__device__ __forceinline__ void walk(const int32_t* at, int32_t n, int64_t from, int64_t to, int32_t b, Load load, Store store) {
  const int lane = threadIdx.x & 31;
  const int64_t owned = at[n];
  for (int64_t i0 = from; i0 < to; i0 += 32 * K) {
    int32_t owner[K];
    decltype(load(0, 0)) value[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t first = i0 + 32 * k, i = first + lane, last = first + 31 < owned ? first + 31 : owned - 1;
      owner[k] = -1;
      if (first < owned && first < to) {
        int32_t mine = b;
        if (last >= at[b + 1]) {                     // several owners, rarely more than these 32 and the next
          const int32_t near = b + 33 < n && at[b + 33] > last ? b + 33 : n;
          mine = find(at, b, near, i < owned ? i : owned - 1);
          b = __shfl_sync(0xffffffffu, mine, 31);
        }
        if (i < owned) owner[k] = mine;
      }
      if (i < to) value[k] = load(i, owner[k]);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t i = i0 + 32 * k + lane;
      if (i < to) store(i, owner[k], value[k]);
    }
  }
}

// the run of warp `warp` of `warps`: a multiple of 32 entries
__device__ __forceinline__ void run_of(int64_t count, int64_t warp, int64_t warps, int64_t& from, int64_t& to) {
  const int64_t per = ((count + warps - 1) / warps + 31) & ~(int64_t)31;
  from = warp * per < count ? warp * per : count;
  to = from + per < count ? from + per : count;
}

template <typename Load, typename Store>
__device__ __forceinline__ void shared_out(const int32_t* at, int32_t n, int64_t count, int64_t warp, int64_t warps, Load load, Store store) {
  int64_t from, to;
  run_of(count, warp, warps, from, to);
  if (from < to) walk<4>(at, n, from, to, from < at[n] ? find(at, 0, n, from) : 0, load, store);
}

// A row's position and page; `first` + r is its token's number.
__device__ __forceinline__ int2 row_at(const Plan& p, int64_t r, int32_t b, int32_t first) {
  if (b < 0) return make_int2(0, -1);
  const int32_t pos = first + (int32_t)r;
  return make_int2(pos, p.page_table[(int64_t)b * p.max_pages + (pos >> p.page_shift)]);
}
__device__ __forceinline__ void write_row(const Plan& p, int64_t r, int32_t b, int2 at) {
  if (p.slot) p.slot[r] = b < 0 ? -1 : ((int64_t)at.y << p.page_shift) + (at.x & ((1 << p.page_shift) - 1));
  if (p.pos) p.pos[r] = at.x;
}

__global__ void __launch_bounds__(kMaxThreads) fb4_plan_kernel(const __grid_constant__ Plan p) {
  extern __shared__ int32_t smem[];        // per sequence: tokens kept; and in front of it: pages that go back, pages taken, rows
  __shared__ Sums part[32];
  __shared__ int32_t served_need;
  __shared__ uint32_t served_rows;
  int32_t *keep = smem, *back = keep + p.n_seqs, *take = back + p.n_seqs + 1, *start = take + p.n_seqs + 1;
  const bool cluster = gridDim.x > 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int64_t me = (int64_t)blockIdx.x * warps + warp, all = (int64_t)gridDim.x * warps;
  const uint32_t most = (uint32_t)p.T + 1u;
  bool bad = false;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // ---- every thread a run of sequences; sums in front of each
  const int32_t per = (p.n_seqs + (int)blockDim.x - 1) / (int)blockDim.x, b0 = min(tid * per, p.n_seqs), b1 = min(b0 + per, p.n_seqs);
  const int32_t f0 = *p.n_free;
  Sums mine{0, 0, 0};
  for (int32_t b = b0; b < b1; ++b) {
    const Step s = step_of(p, b, bad);
    keep[b] = s.keep;
    back[b] = s.back;
    take[b] = s.need;
    start[b] = (int32_t)min((uint32_t)s.n, most);
    mine = add(mine, Sums{s.back, s.need, (uint32_t)start[b]}, most);
  }
  if (tid == 0) {
    served_need = 0;
    served_rows = 0;
  }
  Sums at = scanned(mine, most);
  if (lane == 31) part[warp] = at;
  __syncthreads();
  const Sums sums = scanned(lane < warps ? part[lane] : Sums{0, 0, 0}, most);
  const int before_warp = warp ? warp - 1 : 0;
  Sums base{__shfl_sync(0xffffffffu, sums.back, before_warp), __shfl_sync(0xffffffffu, sums.need, before_warp), __shfl_sync(0xffffffffu, sums.rows, before_warp)};
  if (!warp) base = Sums{0, 0, 0};
  const int32_t total_back = __shfl_sync(0xffffffffu, sums.back, 31);
  // in front of this thread's run: the inclusive sums of the thread before (sums that are cut off cannot be subtracted)
  Sums prev{__shfl_up_sync(0xffffffffu, at.back, 1), __shfl_up_sync(0xffffffffu, at.need, 1), __shfl_up_sync(0xffffffffu, at.rows, 1)};
  if (!lane) prev = Sums{0, 0, 0};
  Sums run = add(base, prev, most);
  const int64_t free0 = f0 < 0 ? 0 : f0 < p.free_cap ? f0 : p.free_cap;
  int64_t top = free0 + total_back;
  const bool over = top > p.free_cap;                                  // pages that the list has no room for are lost, and reported
  if (free0 != f0 || over) bad = true;
  const int64_t usable = over ? p.free_cap : top;
  // ---- who is served: from the first whose sums are too large on, nobody who asks for tokens
  for (int32_t b = b0; b < b1; ++b) {
    const Sums next = add(run, Sums{back[b], take[b], (uint32_t)start[b]}, most);
    const bool served = next.need <= usable && next.rows <= (uint32_t)p.T;
    back[b] = run.back;
    take[b] = served ? run.need : -1;
    start[b] = (int32_t)run.rows;
    if (served && b == b1 - 1) {
      atomicMax(&served_need, next.need);
      atomicMax(&served_rows, next.rows);
    } else if (!served && b > b0 && take[b - 1] >= 0) {               // the last served one of this run
      atomicMax(&served_need, run.need);
      atomicMax(&served_rows, run.rows);
    }
    run = next;
  }
  __syncthreads();
  const int32_t taken = served_need, rows = (int32_t)served_rows;
  for (int32_t b = b0; b < b1; ++b)
    if (take[b] < 0) {
      take[b] = taken;
      start[b] = rows;
    }
  if (tid == 0) {
    back[p.n_seqs] = total_back;
    take[p.n_seqs] = taken;
    start[p.n_seqs] = rows;
  }
  __syncthreads();

  // ---- pages to the free list, pages from it
  if (total_back) {
    shared_out(back, p.n_seqs, total_back, me, all,
               [&](int64_t f, int32_t b) { return p.page_table[(int64_t)b * p.max_pages + pages_of(p, keep[b]) + (f - back[b])]; },
               [&](int64_t f, int32_t, int32_t page) { if (top - 1 - f < p.free_cap) p.free_pages[top - 1 - f] = page; });
    all_sync(cluster);
  }
  shared_out(take, p.n_seqs, taken, me, all, [&](int64_t f, int32_t) { return p.free_pages[usable - 1 - f]; },
             [&](int64_t f, int32_t b, int32_t page) { p.page_table[(int64_t)b * p.max_pages + pages_of(p, keep[b]) + (f - take[b])] = page; });
  for (int32_t b = blockIdx.x * blockDim.x + tid; b <= p.n_seqs; b += gridDim.x * blockDim.x) p.q_start[b] = start[b];
  all_sync(cluster);

  // ---- lengths last: until here everybody reads what the sequences held
  for (int32_t b = blockIdx.x * blockDim.x + tid; b < p.n_seqs; b += gridDim.x * blockDim.x) p.kv_len[b] = keep[b] + start[b + 1] - start[b];
  if (blockIdx.x == 0 && tid == 0) *p.n_free = (int32_t)(usable - taken);
  if (p.rows_here)
    shared_out(start, p.n_seqs, p.T, me, all, [&](int64_t r, int32_t b) { return row_at(p, r, b, b < 0 ? 0 : keep[b] - start[b]); },
               [&](int64_t r, int32_t b, int2 at) { write_row(p, r, b, at); });
  if (__syncthreads_or(bad) && blockIdx.x == 0 && tid == 0) atomicOr(p.status, 2u);
}

constexpr int kRowsPerWarp = 64;

// The rows, 8 warps to a CTA.
__global__ void __launch_bounds__(256) fb4_plan_rows_kernel(const __grid_constant__ Plan p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int64_t from = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * kRowsPerWarp, to = from + kRowsPerWarp < p.T ? from + kRowsPerWarp : p.T;
  if (from >= to) return;
  int32_t lo = 0, hi = p.n_seqs;           // the sequence of the run's first row, 32 places at a time
  if (from < p.q_start[p.n_seqs]) {
    while (hi - lo > 1) {
      const int32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
      const uint32_t below = __ballot_sync(0xffffffffu, at < hi && p.q_start[at] <= from);
      const int k = below ? 31 - __clz((int)below) : 0;
      lo += k * step;
      if (lo + step < hi) hi = lo + step;
    }
  }
  walk<kRowsPerWarp / 32>(p.q_start, p.n_seqs, from, to, lo, [&](int64_t r, int32_t b) { return row_at(p, r, b, b < 0 ? 0 : p.kv_len[b] - p.q_start[b + 1]); },
                          [&](int64_t r, int32_t b, int2 at) { write_row(p, r, b, at); });
}

}  // namespace

cudaError_t fb4_plan_prepare_device() {
  return cudaFuncSetAttribute(fb4_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (4 * FB4_PLAN_MAX_SEQS + 3) * 4);
}

cudaError_t fb4_launch_cache_plan(const fb4_ctx* ctx, int32_t* page_table, int32_t max_pages, int32_t page_tokens, int32_t* kv_len,
                                  const int32_t* keep, const int32_t* new_len, int32_t n_seqs, int32_t* free_pages, int32_t free_cap,
                                  int32_t* n_free, int64_t T, int32_t* q_start, int64_t* slot, int32_t* pos, cudaStream_t stream, int* launches) {
  Plan p{page_table, max_pages, 0, kv_len, keep, new_len, n_seqs, free_pages, free_cap, n_free, T, q_start, slot, pos, T <= 8192, ctx->d_status};
  while ((1 << p.page_shift) < page_tokens) ++p.page_shift;
  const bool large = T > 2048 || n_seqs > 512;
  int threads = kMaxThreads;
  if (!large)
    for (threads = 128; threads < n_seqs || threads < T / 4; threads *= 2) {}
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[1];
  cfg.gridDim = dim3(large ? kCluster : 1);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)(4 * n_seqs + 3) * 4;
  cfg.stream = stream;
  cfg.attrs = attr;
  if (large) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kCluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.numAttrs = 1;
  }
  cudaError_t e = cudaLaunchKernelEx(&cfg, fb4_plan_kernel, p);
  *launches = 1;
  if (e != cudaSuccess || p.rows_here || (!slot && !pos)) return e;
  cfg.gridDim = dim3((unsigned)((T + 8 * kRowsPerWarp - 1) / (8 * kRowsPerWarp)));
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = 0;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // may be set up while the first kernel still runs
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 1;
  *launches = 2;
  return cudaLaunchKernelEx(&cfg, fb4_plan_rows_kernel, p);
}
