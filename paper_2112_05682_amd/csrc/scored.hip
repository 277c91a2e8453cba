// Small kernels of attention with modified scores: document ranges and the last
// sums of the bias gradient.
#include "scored.hpp"

namespace mea {

// The smallest and largest id of every 32 tokens.  A block of ids is read by half
// a wave; the whole takes a launch and 4 bytes a token.
__global__ __launch_bounds__(256) void doc_range_kernel(const int* __restrict__ ids, int64_t n, int64_t units, int64_t total,
                                                        int2* __restrict__ out) {
  const int64_t u = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
  const int64_t b = u / units, i = u % units * 32 + threadIdx.x % 32;
  const bool in = u < total && i < n;
  int lo = in ? ids[b * n + i] : 0x7fffffff, hi = in ? lo : (int)0x80000000;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const int a = __shfl_xor(lo, o), c = __shfl_xor(hi, o);
    lo = a < lo ? a : lo;
    hi = c > hi ? c : hi;
  }
  if (u < total && threadIdx.x % 32 == 0) out[u] = make_int2(lo, hi);
}

hipError_t launch_doc_ranges(const int* ids, int64_t n, int64_t batches, int2* out, hipStream_t stream) {
  int64_t units = (n + 31) / 32, total = units * batches;
  void* args[] = {&ids, &n, &units, &total, &out};
  return hipLaunchKernel(reinterpret_cast<const void*>(doc_range_kernel), dim3((unsigned)((total + 7) / 8)), dim3(256), args, 0,
                         stream);
}

// d_table[t, h]: the dQ workgroups' sums, a workgroup per head; wave w adds every
// fourth part in float64, the waves in order.
__device__ __forceinline__ void store_table(const ScoredBwdParams& p, int64_t at, double x) {
  if (p.s.table_dtype == 0) static_cast<float*>(p.d_table)[at] = (float)x;
  else if (p.s.table_dtype == 1) static_cast<_Float16*>(p.d_table)[at] = (_Float16)(float)x;
  else static_cast<__bf16*>(p.d_table)[at] = (__bf16)(float)x;
}
__global__ __launch_bounds__(256) void scored_table_kernel(ScoredBwdParams p) {
  __shared__ double red[256];
  const int nb = p.s.n_edges * (p.s.two_sided ? 2 : 1);
  const int64_t parts = (int64_t)p.n_b * p.n_qtiles * p.dq_parts;
  const int head = blockIdx.x / nb, e = blockIdx.x % nb;
  double x = 0.0;
  for (int64_t i = threadIdx.x; i < parts; i += 256) x += (double)p.table_part[(head * parts + i) * nb + e];
  red[threadIdx.x] = x;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) store_table(p, (int64_t)e * p.s.heads + head, red[0]);
}

hipError_t launch_scored_table(const ScoredBwdParams& p, hipStream_t stream) {
  ScoredBwdParams a = p;
  void* args[] = {&a};
  return hipLaunchKernel(reinterpret_cast<const void*>(scored_table_kernel), dim3((unsigned)(p.s.heads * p.s.n_buckets())),
                         dim3(256), args, 0, stream);
}

}  // namespace mea
