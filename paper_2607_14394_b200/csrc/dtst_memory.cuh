// Launchers of the recurrent-memory operators (arguments already checked by the C entry points).
#pragma once

#include <atomic>

#include "dtst_common.cuh"

namespace dtst {

// Lets a kernel have `bytes` of shared memory, once per device and kernel (`seen`: a bit per device, kept by the caller's
// static of that kernel; a racing second call sets the same value).
inline cudaError_t allow_smem(const void* kern, size_t bytes, std::atomic<uint64_t>& seen) {
  if (bytes <= 48 * 1024) return cudaSuccess;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && (seen.load(std::memory_order_relaxed) >> dev & 1u)) return cudaSuccess;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess && dev < 64) seen.fetch_or(1ull << dev, std::memory_order_relaxed);
  return e;
}

// As launch_pdl, for thread-block clusters of `cluster` CTAs (0: the kernel's own cluster size).
template <typename Kern, typename... Args>
inline cudaError_t launch_clusters(Kern kern, unsigned ctas, int cluster, int threads, size_t smem, cudaStream_t st, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  unsigned n = 0;
  if (cluster > 0) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)cluster;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (!pdl_off()) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kern, args...);
}

constexpr int kNormParts = 592;           // most CTAs (and rows of partial sums) of a norm's backward pass: 4 per SM
constexpr int kNormFieldChannels = 128;   // most channels a channels-first norm holds in registers

struct NormCall {
  int dtype;
  long long outer, channels, inner;
  float eps;
  const void *x, *residual;
  const float* weight;     // null: quantise x as it is
  void *s, *low, *y;       // low: what rounding took from s (16-bit types; may be null)
  uint8_t* q;              // non-null: 8-bit output instead of y
  float *scale, *rstd;
  long long x_ld, q_ld;    // elements between rows of x (rows only), bytes between rows of q
};
cudaError_t launch_norm_forward(const NormCall& n, cudaStream_t st);

struct NormBackCall {
  int dtype;
  long long outer, channels, inner;
  const void *grad_y, *s, *low, *grad_s;
  const float *weight, *rstd;
  void* grad_x;
  float *grad_weight, *partial;
};
cudaError_t launch_norm_backward(const NormBackCall& n, cudaStream_t st);

struct ScanCall {
  int dtype, gate;
  long long outer, length, inner;
  long long in_outer, in_step, grad_outer, grad_step;   // strides in elements; inner stride 1
  const void *v, *g, *grad_h;
  const float *h0, *grad_last;
  const int* lengths;
  void *h, *grad_v, *grad_g;
  float *h_last, *grad_h0, *checkpoints;
};
// steps between saved states for this problem (the whole length where nothing is saved)
long long scan_chunk(int dtype, long long length, long long inner);
cudaError_t scan_status(int* word, cudaStream_t st);      // reads and clears
cudaError_t launch_scan_forward(const ScanCall& c, cudaStream_t st);
cudaError_t launch_scan_backward(const ScanCall& c, cudaStream_t st);

cudaError_t launch_quantize_weight(int dtype, const void* w, long long w_ld, uint8_t* q, long long q_ld, float* scale,
                                   long long rows, long long cols, cudaStream_t st);

struct MatmulCall {
  int out_dtype;
  long long m, n, k, x_ld, w_ld, out_ld;
  const uint8_t *x, *w;
  const float *x_scale, *w_scale;
  void* out;
  int* status;
};
bool matmul_fp8_available();
cudaError_t launch_matmul_fp8(const MatmulCall& c, cudaStream_t st);

}  // namespace dtst
