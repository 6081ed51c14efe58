// Sums of partial sums: out[c] = sum over parts of partial[part][c], in a fixed order.  32 warps take every 32nd part of 32
// neighbouring columns, and their sums meet in warp order.  Bound by memory and, for few columns, by latency.
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

__global__ void __launch_bounds__(1024) sum_parts_kernel(const SumArgs a) {
  __shared__ float red[32][33];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long c0 = (long long)blockIdx.x * 32;
  float t = 0.f;
  if (c0 + lane < a.columns) {
#pragma unroll 8
    for (int p = w; p < a.parts; p += 32) t += a.partial[(long long)p * a.columns + c0 + lane];
  }
  red[w][lane] = t;
  __syncthreads();
  t = warp_sum(red[lane][w]);      // (turned round: warp w sums column w over the 32 warps)
  if (lane == 0 && c0 + w < a.columns) {
    long long c = c0 + w;
#pragma unroll
    for (int k = 0; k < kMostOuts; ++k) {
      if (c >= 0 && c < a.outs[k].n && a.outs[k].out != nullptr) a.outs[k].out[c] = t;
      c -= a.outs[k].n;
    }
  }
}

}  // namespace

cudaError_t launch_sum_parts(const float* partial, int parts, long long columns, std::initializer_list<SumOut> outs, cudaStream_t st) {
  SumArgs a{partial, columns, parts, {}};
  int k = 0;
  for (const SumOut& o : outs)
    if (k < kMostOuts) a.outs[k++] = o;
  return launch_pdl(sum_parts_kernel, dim3((unsigned)((columns + 31) / 32)), dim3(1024), 0, st, a);
}

}  // namespace dtst
