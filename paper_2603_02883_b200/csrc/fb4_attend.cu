// Attention over the paged FB4 cache: the plain kernel (any head dimension).
#include "fb4_attend.cuh"

namespace {

using namespace fb4att;

// One warp per query row and head; lane l holds channel 32 b + l of every block b.  The running maximum and sum of the softmax
// are updated key by key.  Latency-bound and only meant for head dimensions that the tensor-core kernels do not have (and to
// check them against).
template <int NB>
__global__ void __launch_bounds__(128) fb4_attend_generic_kernel(const __grid_constant__ Fb4Attend a) {
  __shared__ uint8_t book[32][8];
  if (threadIdx.x < 64) reinterpret_cast<uint32_t*>(book)[threadIdx.x] = reinterpret_cast<const uint32_t*>(a.tables->formatbook)[threadIdx.x];
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const int64_t rows = (int64_t)a.max_q * a.q_heads, per = (rows + 3) / 4;
  const int32_t b = (int32_t)(blockIdx.x / per);
  const int64_t r = (blockIdx.x % per) * 4 + (threadIdx.x >> 5);
  const Sequence sq = sequence(a, b, lane == 0 && blockIdx.x % per == 0 && threadIdx.x == 0);
  const int32_t i = (int32_t)(r / a.q_heads), h = (int32_t)(r % a.q_heads);
  if (r >= rows || i >= sq.n_q) return;
  const int64_t row = sq.q0 + i;
  const int32_t head = h / a.group, D = NB * 32;
  float q[NB], acc[NB];
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    q[k] = __uint_as_float(query_pair((uint32_t)a.q[row * a.q_ld + (int64_t)h * D + 32 * k + lane] << 16));
    acc[k] = 0.0f;
  }
  const Range v = visible(a, sq, i);
  float m = -INFINITY, l = 0.0f;
  bool bad = false;
  auto value = [&](const uint8_t* codes, const uint16_t* meta, int64_t at, int k) -> float {
    const uint32_t c = codes[at * (D / 2) + 16 * k + (lane >> 1)], mt = meta[at * NB + k];
    const uint32_t code = (lane & 1) ? c >> 4 : c & 15u;
    const float x = ldexpf((float)book[(mt >> 8) & 31u][code & 7u], (int)(mt & 255u) - 127);
    return (code & 8u) ? -x : x;
  };
  for (int32_t j = v.lo; j < v.hi; ++j) {
    const int64_t page = a.page_table[(int64_t)b * a.max_pages + (j >> a.page_shift)];
    if (page < 0 || page >= a.cache.n_pages) {
      bad = true;
      continue;
    }
    const int64_t at = ((page * a.cache.n_heads + head) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < NB; ++k) s = fmaf(q[k], value(a.cache.k_codes, a.cache.k_meta, at, k), s);
#pragma unroll
    for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    s = __fmul_rn(s, a.scale_log2);            // rounded as the maximum is, not fused with the subtraction below
    if (s == -INFINITY && m == -INFINITY) continue;      // overflowed downwards: no weight, and no maximum to stand against yet
    const float mn = fmaxf(m, s), f = exp2f(m - mn), e = exp2f(s - mn);
    l = l * f + e;
#pragma unroll
    for (int k = 0; k < NB; ++k) acc[k] = fmaf(e, value(a.cache.v_codes, a.cache.v_meta, at, k), acc[k] * f);
    m = mn;
  }
  const float inv = inverse_of(l, 1.0f);
#pragma unroll
  for (int k = 0; k < NB; ++k) store_out(a, row * a.out_ld + (int64_t)h * D + 32 * k + lane, acc[k] * inv);
  if (lane == 0) {
    if (a.lse) a.lse[row * a.q_heads + h] = lse_of(m, l);
    if (bad) atomicOr(a.status, 2u);
  }
}

}  // namespace

cudaError_t fb4_launch_attend_generic(const fb4_ctx*, const Fb4Attend& a, cudaStream_t stream) {
  const int64_t grid = ((int64_t)a.max_q * a.q_heads + 3) / 4 * a.n_seqs;
  switch (a.cache.head_dim / 32) {
    case 1: fb4_attend_generic_kernel<1><<<(unsigned)grid, 128, 0, stream>>>(a); break;
    case 2: fb4_attend_generic_kernel<2><<<(unsigned)grid, 128, 0, stream>>>(a); break;
    case 3: fb4_attend_generic_kernel<3><<<(unsigned)grid, 128, 0, stream>>>(a); break;
    case 4: fb4_attend_generic_kernel<4><<<(unsigned)grid, 128, 0, stream>>>(a); break;
    case 5: fb4_attend_generic_kernel<5><<<(unsigned)grid, 128, 0, stream>>>(a); break;
    case 6: fb4_attend_generic_kernel<6><<<(unsigned)grid, 128, 0, stream>>>(a); break;
    case 7: fb4_attend_generic_kernel<7><<<(unsigned)grid, 128, 0, stream>>>(a); break;
    default: fb4_attend_generic_kernel<8><<<(unsigned)grid, 128, 0, stream>>>(a); break;
  }
  return cudaGetLastError();
}
