// Sums of partial sums: out[c] = sum over parts of partial[part][c], in a fixed order: a CTA's warps take every W-th part of 32
// neighbouring columns, and their sums meet in warp order.  Bound by memory and, for few columns, by latency: as many warps as
// leave a thread some ten loads at once.
#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

constexpr int kMostOuts = 3;
struct SumArgs {
  const float* partial;
  long long columns;
  int parts;
  SumOut outs[kMostOuts];
};

template <int W>
__global__ void __launch_bounds__(32 * W) sum_parts_kernel(const SumArgs a) {
  __shared__ float red[W][32];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 32 + lane;
  float t = 0.f;
  if (c < a.columns) {
#pragma unroll 10
    for (int p = w; p < a.parts; p += W) t += a.partial[(long long)p * a.columns + c];
  }
  red[w][lane] = t;
  __syncthreads();
  if (w > 0 || c >= a.columns) return;
#pragma unroll
  for (int i = 1; i < W; ++i) t += red[i][lane];
  long long k = c;
#pragma unroll
  for (int i = 0; i < kMostOuts; ++i) {
    if (k >= 0 && k < a.outs[i].n && a.outs[i].out != nullptr) a.outs[i].out[k] = t;
    k -= a.outs[i].n;
  }
}

}  // namespace

cudaError_t launch_sum_parts(const float* partial, int parts, long long columns, std::initializer_list<SumOut> outs, cudaStream_t st) {
  SumArgs a{partial, columns, parts, {}};
  int k = 0;
  for (const SumOut& o : outs)
    if (k < kMostOuts) a.outs[k++] = o;
  const dim3 grid((unsigned)((columns + 31) / 32));
  if (parts <= 40) return launch_pdl(sum_parts_kernel<4>, grid, dim3(128), 0, st, a);
  if (parts <= 160) return launch_pdl(sum_parts_kernel<16>, grid, dim3(512), 0, st, a);
  return launch_pdl(sum_parts_kernel<32>, grid, dim3(1024), 0, st, a);
}

}  // namespace dtst
