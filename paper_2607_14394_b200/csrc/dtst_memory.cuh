// Launchers of the recurrent-memory operators (arguments already checked by the C entry points).
#pragma once

#include <atomic>
#include <initializer_list>

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

// CTAs of a kernel that run at once on the current device (`seen`: per device, kept by the caller's static of that kernel; a racing
// second call sets the same value).  A grid of a little more than that many, each walking over its share, would run twice as long.
struct Resident {
  std::atomic<int> n[64];
};
inline int resident_ctas(const void* kern, int threads, size_t smem, Resident& seen) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    (void)cudaGetLastError();
    return num_sms();
  }
  int n = seen.n[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    int per_sm = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kern, threads, smem) != cudaSuccess || per_sm < 1) {
      (void)cudaGetLastError();
      per_sm = 1;
    }
    n = per_sm * num_sms();
    seen.n[dev].store(n, std::memory_order_relaxed);
  }
  return n;
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

// out[k][i] = sum over `parts` rows of `partial` [parts][columns], in a fixed order; the outputs' columns follow one another, an
// output without an address is passed over.
struct SumOut {
  float* out;
  long long n;
};
cudaError_t launch_sum_parts(const float* partial, int parts, long long columns, std::initializer_list<SumOut> outs, cudaStream_t st);

struct LayerNormCall {
  int dtype;
  long long outer, channels, inner;
  float eps;
  const void *x, *residual;
  const float *weight, *bias;
  void *s, *low, *y;
  float* stats;            // mean and rstd of every position, or null
};
cudaError_t launch_layer_norm(const LayerNormCall& n, cudaStream_t st);

struct LayerNormBackCall {
  int dtype;
  long long outer, channels, inner;
  const void *grad_y, *s, *low, *grad_s;
  const float *weight, *stats;
  void* grad_x;
  float *grad_weight, *grad_bias, *partial;
};
cudaError_t launch_layer_norm_backward(const LayerNormBackCall& n, cudaStream_t st);

constexpr int kConvWidth = 4;             // widest causal convolution
struct ConvCall {
  int dtype, width, silu;
  long long batch, length, channels;
  long long x_stride[2], grad_stride[2];  // batch entry, step, in elements
  const void *x, *state, *grad_y, *grad_state_out;
  const float *weight, *bias;
  const int* lengths;
  void *y, *state_out, *grad_x, *grad_state;
  float *grad_weight, *grad_bias, *partial;
};
// most rows of partial sums of the convolution's backward pass: 16 CTAs on each of 148 SMs, over the groups of channels
inline int conv_parts(long long channels) {
  const long long n = 16 * 148 / ((channels + 127) / 128);
  return (int)(n < 1 ? 1 : n > 256 ? 256 : n);
}
cudaError_t launch_conv_forward(const ConvCall& c, cudaStream_t st);
cudaError_t launch_conv_backward(const ConvCall& c, cudaStream_t st);

constexpr int kSelectiveStates = 64;      // most states of a channel
constexpr int kSelectiveSave = 8;         // steps between the states that a forward pass saves
struct Rows {                             // a token-major tensor: its address, elements between batch entries and steps
  void* p;
  long long batch, step;
};
struct SelectiveCall {
  int dtype, softplus;
  long long batch, length, channels, states, groups;
  Rows x, dt, z, B, C;
  const void* grad_y;
  const float *A, *D, *bias, *h0, *grad_last;
  const int* lengths;
  void* y;
  float *h_last, *checkpoints;
  Rows grad_x, grad_dt, grad_z, grad_B, grad_C;
  float *grad_A, *grad_D, *grad_bias, *grad_h0;
  float* scratch;
};
long long selective_scratch_floats(const SelectiveCall& c, bool back);
cudaError_t launch_selective_forward(const SelectiveCall& c, cudaStream_t st);
cudaError_t launch_selective_backward(const SelectiveCall& c, cudaStream_t st);

struct GradEntry {
  const void* grad;
  void* out;               // null: not scaled; grad itself: in place
  long long n;
  int dtype;
};
constexpr int kGradParts = 592;           // most CTAs of one launch of the norm's sum
// launches of the sum that this many tensors take (each leaves kGradParts partial sums)
int grad_launches(long long count);
cudaError_t launch_grad_norm(const GradEntry* list, long long count, float max_norm, float eps, bool scale, float* norm,
                             double* partial, cudaStream_t st);

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
