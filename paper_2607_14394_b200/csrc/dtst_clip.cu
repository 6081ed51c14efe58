// The norm of all gradients of a program, and their clipping by it:
//     norm = sqrt(sum over tensors and elements of v^2),   c = min(1, max_norm / (norm + eps)),   v := c v
// Two launches for every kPerLaunch tensors: all the sums, then the scaling, every CTA of which adds the CTAs' sums up again, in
// order.  The list of tensors goes with the launch, so nothing is copied to
// the device and a call can be captured.  Squares are summed in 64 bits: a gradient of 1e30 does not overflow, one of
// 1e-30 is not lost, and the sum of 10^9 elements keeps its last digits; the conversions and the 64-bit adds run beside the loads.
// Bound by memory: the gradients are read twice, the second time in the opposite order, so that what the
// sum read last is still in L2 when the scaling begins.  A list that fits L2 is read from memory once.
#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

constexpr int kThreads = 256;
constexpr int kPerLaunch = 128;         // most tensors of a launch; short lists go with a shorter one (N)
constexpr int kChunkBytes = 16384;      // bytes of one tensor that a CTA takes at a time

template <int N>
struct ListArgs {
  const void* grad[N];
  void* out[N];
  long long n[N];
  int first[N + 1];                     // number of each tensor's first chunk
  unsigned char dtype[N];
  int count;
  const double* sums;                   // scaling: all launches' partial sums
  double* partial;                      // sum: this launch's
  float* norm;
  int sums_n;
  float max_norm, eps;
};

template <int N>
__device__ __forceinline__ int find(const ListArgs<N>& a, int chunk) {      // the tensor with this chunk
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

template <typename T>
__device__ __forceinline__ void sum_chunk(const T* p, long long n, double (&acc)[4]) {
  constexpr int V = 16 / (int)sizeof(T), PER = kChunkBytes / (int)sizeof(T);
  if (aligned_to_device(p, 16) && n >= PER) {
    constexpr int LOADS = kChunkBytes / 16 / kThreads;
    Pack<T, V> v[LOADS];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) v[k].load(p + ((long long)k * kThreads + threadIdx.x) * V);
#pragma unroll
    for (int k = 0; k < LOADS; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const double d = (double)v[k].get(i);
        acc[i & 3] = fma(d, d, acc[i & 3]);
      }
  } else {
    for (long long i = threadIdx.x; i < n && i < PER; i += kThreads) {
      const double d = (double)Elem<T>::get(p[i]);
      acc[0] = fma(d, d, acc[0]);
    }
  }
}

__device__ __forceinline__ double block_sum(double v, double* red) {     // the same bits in every thread
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.;
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) t += red[i];
  return t;
}

template <int N>
__global__ void __launch_bounds__(kThreads) grad_sum_kernel(const __grid_constant__ ListArgs<N> a) {
  __shared__ double red[kThreads / 32];
  pdl_trigger();
  pdl_wait();
  double acc[4] = {0., 0., 0., 0.};
  const int chunks = a.first[a.count];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int t = find(a, c);
    const long long at = (long long)(c - a.first[t]) * kChunkBytes;
    if (a.dtype[t] == DTST_F32) {
      sum_chunk(static_cast<const float*>(a.grad[t]) + at / 4, a.n[t] - at / 4, acc);
    } else if (a.dtype[t] == DTST_BF16) {
      sum_chunk(static_cast<const __nv_bfloat16*>(a.grad[t]) + at / 2, a.n[t] - at / 2, acc);
    } else {
      sum_chunk(static_cast<const __half*>(a.grad[t]) + at / 2, a.n[t] - at / 2, acc);
    }
  }
  const double sum = block_sum((acc[0] + acc[1]) + (acc[2] + acc[3]), red);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
}

// norm and coefficient from the partial sums; the coefficient as a product of two, since that of a norm beyond 2^100 is
// too small for the one
template <int N>
__device__ __forceinline__ void coefficient(const ListArgs<N>& a, double* red, float& c_hi, float& c_lo) {
  double s = 0.;
  for (int i = threadIdx.x; i < a.sums_n; i += kThreads) s += a.sums[i];
  const double norm = sqrt(block_sum(s, red));
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.norm != nullptr) *a.norm = (float)norm;
  double c = (double)a.max_norm / (norm + (double)a.eps);
  if (c > 1. || isinf(a.max_norm)) c = 1.;      // (a NaN stays where there is a bound)
  const bool tiny = c < 0x1p-60;
  c_hi = tiny ? 0x1p-60f : 1.f;
  c_lo = (float)(tiny ? c * 0x1p60 : c);
}

template <int N>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ ListArgs<N> a) {
  __shared__ double red[kThreads / 32];
  pdl_trigger();
  pdl_wait();
  float hi, lo;
  coefficient(a, red, hi, lo);
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const T* p, T* o, long long n, float hi, float lo) {
  constexpr int V = 16 / (int)sizeof(T), PER = kChunkBytes / (int)sizeof(T);
  if (aligned_to_device(p, 16) && aligned_to_device(o, 16) && n >= PER) {
    constexpr int LOADS = kChunkBytes / 16 / kThreads;
    Pack<T, V> v[LOADS];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) v[k].load(p + ((long long)k * kThreads + threadIdx.x) * V);
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      float x[V];
      v[k].unpack(x);
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = x[i] * hi * lo;
      v[k].pack(x);
      v[k].store(o + ((long long)k * kThreads + threadIdx.x) * V);
    }
  } else {
    for (long long i = threadIdx.x; i < n && i < PER; i += kThreads) o[i] = Elem<T>::put(Elem<T>::get(p[i]) * hi * lo);
  }
}

template <int N>
__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const __grid_constant__ ListArgs<N> a) {
  __shared__ double red[kThreads / 32];
  pdl_trigger();
  pdl_wait();
  float hi, lo;
  coefficient(a, red, hi, lo);
  const int chunks = a.first[a.count];
  for (int i = blockIdx.x; i < chunks; i += gridDim.x) {
    const int c = chunks - 1 - i, t = find(a, c);
    if (a.out[t] == nullptr || (a.out[t] == a.grad[t] && hi * lo == 1.f)) continue;     // in place, times one
    const long long at = (long long)(c - a.first[t]) * kChunkBytes;
    if (a.dtype[t] == DTST_F32) {
      scale_chunk(static_cast<const float*>(a.grad[t]) + at / 4, static_cast<float*>(a.out[t]) + at / 4, a.n[t] - at / 4, hi, lo);
    } else if (a.dtype[t] == DTST_BF16) {
      scale_chunk(static_cast<const __nv_bfloat16*>(a.grad[t]) + at / 2, static_cast<__nv_bfloat16*>(a.out[t]) + at / 2, a.n[t] - at / 2, hi, lo);
    } else {
      scale_chunk(static_cast<const __half*>(a.grad[t]) + at / 2, static_cast<__half*>(a.out[t]) + at / 2, a.n[t] - at / 2, hi, lo);
    }
  }
}

template <int N>
cudaError_t launch_list(const GradEntry* list, long long count, float max_norm, float eps, bool scale, float* norm, double* partial,
                        cudaStream_t st) {
  const int most = num_sms() * 4 < kGradParts ? num_sms() * 4 : kGradParts, launches = (int)((count + N - 1) / N);
  int sums = 0;
  auto fill = [&](ListArgs<N>& a, int launch) {
    const long long k0 = (long long)launch * N;
    a.count = (int)(count - k0 < N ? count - k0 : N);
    long long chunks = 0;
    for (int k = 0; k < a.count; ++k) {
      const GradEntry& e = list[k0 + k];
      a.grad[k] = e.grad, a.out[k] = e.out, a.n[k] = e.n, a.dtype[k] = (unsigned char)e.dtype, a.first[k] = (int)chunks;
      const long long per = kChunkBytes / (e.dtype == DTST_F32 ? 4 : 2);
      chunks += (e.n + per - 1) / per;
    }
    a.first[a.count] = (int)chunks;
    return (int)(chunks < most ? (chunks > 0 ? chunks : 1) : most);
  };
  ListArgs<N> a{};
  for (int l = 0; l < launches; ++l) {
    const int ctas = fill(a, l);
    a.partial = partial + sums;
    const cudaError_t e = launch_pdl(grad_sum_kernel<N>, dim3((unsigned)ctas), dim3(kThreads), 0, st, a);
    if (e != cudaSuccess) return e;
    sums += ctas;
  }
  a.sums = partial, a.sums_n = sums, a.max_norm = max_norm, a.eps = eps, a.norm = norm;
  if (!scale || launches == 0) return launch_pdl(grad_norm_kernel<N>, dim3(1), dim3(kThreads), 0, st, a);
  for (int l = launches - 1; l >= 0; --l) {
    const int ctas = launches > 1 ? fill(a, l) : (a.first[a.count] < most ? (a.first[a.count] > 0 ? a.first[a.count] : 1) : most);
    const cudaError_t e = launch_pdl(grad_scale_kernel<N>, dim3((unsigned)ctas), dim3(kThreads), 0, st, a);
    if (e != cudaSuccess) return e;
    a.norm = nullptr;
  }
  return cudaSuccess;
}

}  // namespace

int grad_launches(long long count) { return (int)((count + kPerLaunch - 1) / kPerLaunch); }

cudaError_t launch_grad_norm(const GradEntry* list, long long count, float max_norm, float eps, bool scale, float* norm,
                             double* partial, cudaStream_t st) {
  return count <= 16 ? launch_list<16>(list, count, max_norm, eps, scale, norm, partial, st)
                     : launch_list<kPerLaunch>(list, count, max_norm, eps, scale, norm, partial, st);
}

}  // namespace dtst
