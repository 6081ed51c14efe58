// Short causal convolution of every channel with its own K weights (K <= 4), token-major tensors [batch][length][channels]:
//     u = [state (K - 1 steps); x],   pre_t = b + sum_k w_k u_(t+k),   y_t = pre_t  or  pre_t sigmoid(pre_t)
// and its backward pass, with gp_t = gy_t dy/dpre:
//     grad_u_(t+k) = sum_k w_k gp_t  (+ the gradient of the new state),   grad_w_k = sum gp_t u_(t+k),   grad_b = sum gp_t
// The new state is the last K - 1 steps of u at the sequence's own length, whatever that is.
//
// Bound by memory: a thread holds a vector of neighbouring channels and walks over a run of steps with the last K inputs
// in registers, so a step is read once but for the K - 1 in front of a run (backward: also behind it).  The next steps' loads
// are under way while a step is formed.  Runs are as long as leaves enough of them to fill the GPU.  The parameters' gradients
// are summed in registers over the runs a thread visits, over a CTA's warps in shared memory, and over CTAs by a second launch,
// all in a fixed order: same bits on every run.
#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

constexpr int kWarps = 4;

struct ConvArgs {
  const void *x, *state, *gy, *gso;
  const float *weight, *bias;
  const int* lengths;
  void *y, *state_out, *gx, *gs;
  float* partial;                      // [gridDim.y][C (K + 1)]: grad_w, then grad_b
  long long B, T, C;
  long long xb, xt, gb, gt;            // strides of x and of grad_x
  int run, runs, silu;                 // steps to a run, runs to a sequence
};

__device__ __forceinline__ float sigmoid_of(float p) { return __fdividef(1.f, 1.f + __expf(-p)); }

template <typename T, int V>
__device__ __forceinline__ void load_row(float (&v)[V], const T* p, bool on, int left) {
  Pack<T, V> k;
  if (!on) k.zero();
  else if (V == 1 || left >= V) k.load(p);
  else k.load_part(p, left);
  k.unpack(v);
}
template <typename T, int V>
__device__ __forceinline__ void store_row(const float (&v)[V], T* p, int left) {
  Pack<T, V> k;
  k.pack(v);
  if (V == 1 || left >= V) k.store(p);
  else k.store_part(p, left);
}

// weights of V channels, [channel][k] in memory
template <int V, int K>
__device__ __forceinline__ void load_taps(float (&w)[K][V], float (&b)[V], const ConvArgs& a, long long c, int left) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int k = 0; k < K; ++k) w[k][i] = i < left ? __ldg(a.weight + (c + i) * K + k) : 0.f;
    b[i] = a.bias != nullptr && i < left ? __ldg(a.bias + c + i) : 0.f;
  }
}

// u of step t (t >= -(K-1)): from x, or from the state (zeros without one)
template <typename T, int V, int K>
__device__ __forceinline__ void load_u(float (&v)[V], const ConvArgs& a, long long b, long long t, long long end, long long c, int left) {
  if (t >= 0) load_row<T, V>(v, static_cast<const T*>(a.x) + b * a.xb + t * a.xt + c, t < end, left);
  else load_row<T, V>(v, static_cast<const T*>(a.state) + (b * (K - 1) + t + K - 1) * a.C + c, a.state != nullptr, left);
}

// A warp: 32 vectors of channels (blockIdx.x), one run of one sequence.
template <typename T, int V, int K>
__global__ void __launch_bounds__(32 * kWarps) conv_forward_kernel(const ConvArgs a) {
  pdl_trigger();
  pdl_wait();
  const long long c = ((long long)blockIdx.x * 32 + threadIdx.x) * V;
  const long long unit = (long long)blockIdx.y * kWarps + threadIdx.y;
  if (c >= a.C || unit >= a.B * a.runs) return;
  const int left = (int)(a.C - c < V ? a.C - c : V);
  const long long b = unit / a.runs, t0 = unit % a.runs * a.run, t1 = t0 + a.run < a.T ? t0 + a.run : a.T;
  long long n = a.T;
  if (a.lengths != nullptr) {
    n = a.lengths[b];
    n = n < 0 ? 0 : n > a.T ? a.T : n;
  }
  const long long end = t1 < n ? t1 : n;
  float w[K][V], bias[V], u[K][V];
  load_taps<V, K>(w, bias, a, c, left);
  T* y = static_cast<T*>(a.y) + b * a.T * a.C + c;
#pragma unroll
  for (int k = 0; k < K - 1; ++k) load_u<T, V, K>(u[k], a, b, t0 - (K - 1) + k, n, c, left);
  // the new state first: the old one may be in its place
  if (t0 == 0 && K > 1 && a.state_out != nullptr) {
    float s[K > 1 ? K - 1 : 1][V];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) load_u<T, V, K>(s[k], a, b, n - (K - 1) + k, n, c, left);
#pragma unroll
    for (int k = 0; k < K - 1; ++k) store_row<T, V>(s[k], static_cast<T*>(a.state_out) + (b * (K - 1) + k) * a.C + c, left);
  }
  constexpr int AHEAD = 4;
  const T* x = static_cast<const T*>(a.x) + b * a.xb + c;
  Pack<T, V> next[AHEAD];
  auto fetch = [&](int j, long long t) {
    if (t >= end) next[j].zero();
    else if (V == 1 || left >= V) next[j].load(x + t * a.xt);
    else next[j].load_part(x + t * a.xt, left);
  };
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) fetch(j, t0 + j);
  for (long long t = t0; t < end; t += AHEAD) {
    Pack<T, V> now[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) now[j] = next[j];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) fetch(j, t + AHEAD + j);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (t + j >= end) break;
      now[j].unpack(u[K - 1]);
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float p = bias[i];
#pragma unroll
        for (int k = 0; k < K; ++k) p = fmaf(w[k][i], u[k][i], p);
        o[i] = a.silu ? p * sigmoid_of(p) : p;
#pragma unroll
        for (int k = 0; k < K - 1; ++k) u[k][i] = u[k + 1][i];
      }
      store_row<T, V>(o, y + (t + j) * a.C, left);
    }
  }
  const float zero[V] = {};
  for (long long t = end > t0 ? end : t0; t < t1; ++t) store_row<T, V>(zero, y + t * a.C, left);
}

// Backward.  Step t of the loop forms gp_t; with it the gradient of u_(t) is complete and is written, as that of step
// t - (K - 1): of x, or of the state in front of a sequence's first run.
template <typename T, int V, int K>
__global__ void __launch_bounds__(32 * kWarps) conv_backward_kernel(const ConvArgs a) {
  __shared__ float red[kWarps][32][V];
  pdl_trigger();
  pdl_wait();
  const long long c = ((long long)blockIdx.x * 32 + threadIdx.x) * V;
  const bool on = c < a.C;
  const int left = (int)(a.C - c < V ? a.C - c : V);
  float gw[K][V], gb[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    gb[i] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) gw[k][i] = 0.f;
  }
  if (on) {
    float w[K][V], bias[V];
    load_taps<V, K>(w, bias, a, c, left);
    for (long long unit = (long long)blockIdx.y * kWarps + threadIdx.y; unit < a.B * a.runs; unit += (long long)gridDim.y * kWarps) {
      const long long b = unit / a.runs, t0 = unit % a.runs * a.run, t1 = t0 + a.run < a.T ? t0 + a.run : a.T;
      long long n = a.T;
      if (a.lengths != nullptr) {
        n = a.lengths[b];
        n = n < 0 ? 0 : n > a.T ? a.T : n;
      }
      const long long end = t1 < n ? t1 : n;              // first step that is not this run's
      const long long last = (end > t0 ? end : t0) + K - 1;
      const T* x = static_cast<const T*>(a.x) + b * a.xb + c;
      const T* gy = static_cast<const T*>(a.gy) + b * a.T * a.C + c;
      T* gx = static_cast<T*>(a.gx) + b * a.gb + c;
      float u[K][V], g[K][V];
#pragma unroll
      for (int k = 0; k < K - 1; ++k) {
        load_u<T, V, K>(u[k], a, b, t0 - (K - 1) + k, n, c, left);
#pragma unroll
        for (int i = 0; i < V; ++i) g[k][i] = 0.f;
      }
      // (a run without steps of its own has nothing to write but zeros; the first one has the state's gradient)
      const long long stop = end > t0 || t0 == 0 ? last : t0;
      constexpr int AHEAD = 2;
      Pack<T, V> nx[AHEAD], ng[AHEAD];
      auto fetch = [&](int j, long long t) {
        if (t >= n || t >= stop) {
          nx[j].zero(), ng[j].zero();
        } else if (V == 1 || left >= V) {
          nx[j].load(x + t * a.xt), ng[j].load(gy + t * a.C);
        } else {
          nx[j].load_part(x + t * a.xt, left), ng[j].load_part(gy + t * a.C, left);
        }
      };
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) fetch(j, t0 + j);
      for (long long t = t0; t < stop; t += AHEAD) {
        Pack<T, V> cx[AHEAD], cg[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) cx[j] = nx[j], cg[j] = ng[j];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) fetch(j, t + AHEAD + j);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          const long long s = t + j, to = s - (K - 1);
          if (s >= stop) break;
          cx[j].unpack(u[K - 1]);
          cg[j].unpack(g[K - 1]);          // (zero behind the sequence's end)
          float o[V];
#pragma unroll
          for (int i = 0; i < V; ++i) {
            if (a.silu) {
              float p = bias[i];
#pragma unroll
              for (int k = 0; k < K; ++k) p = fmaf(w[k][i], u[k][i], p);
              const float sg = sigmoid_of(p);
              g[K - 1][i] *= sg * fmaf(p, 1.f - sg, 1.f);
            }
            if (s >= n) g[K - 1][i] = 0.f;
            const float own = s < end ? g[K - 1][i] : 0.f;
            gb[i] += own;
#pragma unroll
            for (int k = 0; k < K; ++k) gw[k][i] = fmaf(own, u[k][i], gw[k][i]);
            o[i] = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) o[i] = fmaf(w[k][i], g[K - 1 - k][i], o[i]);
#pragma unroll
            for (int k = 0; k < K - 1; ++k) u[k][i] = u[k + 1][i], g[k][i] = g[k + 1][i];
          }
          if (to < t0 && (t0 > 0 || a.gs == nullptr)) continue;
          if (to >= n - (K - 1) && K > 1 && a.gso != nullptr) {
            float q[V];
            load_row<T, V>(q, static_cast<const T*>(a.gso) + (b * (K - 1) + to - (n - (K - 1))) * a.C + c, true, left);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] += q[i];
          }
          if (to >= 0) store_row<T, V>(o, gx + to * a.gt, left);
          else store_row<T, V>(o, static_cast<T*>(a.gs) + (b * (K - 1) + to + K - 1) * a.C + c, left);
        }
      }
      const float zero[V] = {};
      for (long long t = end > t0 ? end : t0; t < t1; ++t) store_row<T, V>(zero, gx + t * a.gt, left);
    }
  }
  if (a.partial == nullptr) return;
  float* out = a.partial + (long long)blockIdx.y * a.C * (K + 1);
#pragma unroll
  for (int k = 0; k <= K; ++k) {           // over the CTA's warps, in order
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) red[threadIdx.y][threadIdx.x][i] = k < K ? gw[k < K ? k : 0][i] : gb[i];
    __syncthreads();
    if (threadIdx.y == 0 && on) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float t = 0.f;
#pragma unroll
        for (int y = 0; y < kWarps; ++y) t += red[y][threadIdx.x][i];
        if (i < left) out[k < K ? (c + i) * K + k : a.C * K + c + i] = t;
      }
    }
  }
}

// steps to a run: long runs read little twice; short ones leave a few warps to every scheduler
int run_steps(long long warps_per_step, long long T, int least) {
  int run = 64;
  while (run > least && warps_per_step * ((T + run - 1) / run) < (long long)num_sms() * 32) run /= 2;
  return run;
}

template <typename T, int V, int K>
cudaError_t launch_k(ConvArgs a, bool back, int* parts, cudaStream_t st) {
  const long long groups = (a.C + 32 * V - 1) / (32 * V);
  a.run = run_steps(groups * a.B, a.T, back ? 16 : 8);
  a.runs = (int)((a.T + a.run - 1) / a.run);
  if (a.runs < 1) a.runs = 1;                                    // no steps: the state alone
  const long long units = a.B * a.runs;
  long long rows = (units + kWarps - 1) / kWarps;
  if (!back) {
    if (rows > 65535) {                                          // more runs than a grid's second dimension holds
      a.run = (int)((a.T * a.B / kWarps + 32767) / 32768 + 1);
      a.runs = (int)((a.T + a.run - 1) / a.run);
      rows = (a.B * a.runs + kWarps - 1) / kWarps;
      if (rows > 65535) return cudaErrorNotSupported;
    }
    return launch_pdl(conv_forward_kernel<T, V, K>, dim3((unsigned)groups, (unsigned)rows), dim3(32, kWarps), 0, st, a);
  }
  const int most = conv_parts(a.B, a.T, a.C);
  *parts = (int)(rows < most ? rows : most);
  return launch_pdl(conv_backward_kernel<T, V, K>, dim3((unsigned)groups, (unsigned)*parts), dim3(32, kWarps), 0, st, a);
}

template <typename T, int V>
cudaError_t launch_v(const ConvArgs& a, int width, bool back, int* parts, cudaStream_t st) {
  switch (width) {
    case 1: return launch_k<T, V, 1>(a, back, parts, st);
    case 2: return launch_k<T, V, 2>(a, back, parts, st);
    case 3: return launch_k<T, V, 3>(a, back, parts, st);
    default: return launch_k<T, V, 4>(a, back, parts, st);
  }
}

template <typename T>
cudaError_t launch_t(const ConvArgs& a, int width, bool back, int* parts, cudaStream_t st) {
  constexpr int V = 4;
  bool vec = a.C % V == 0 && a.xb % V == 0 && a.xt % V == 0 && a.gb % V == 0 && a.gt % V == 0;
  for (const void* p : {a.x, a.state, a.gy, a.gso, (const void*)a.y, (const void*)a.state_out, (const void*)a.gx, (const void*)a.gs})
    vec = vec && aligned_to(p, V * sizeof(T));
  return vec ? launch_v<T, V>(a, width, back, parts, st) : launch_v<T, 1>(a, width, back, parts, st);
}

cudaError_t launch(const ConvArgs& a, int dtype, int width, bool back, int* parts, cudaStream_t st) {
  switch (dtype) {
    case DTST_F32: return launch_t<float>(a, width, back, parts, st);
    case DTST_BF16: return launch_t<__nv_bfloat16>(a, width, back, parts, st);
    default: return launch_t<__half>(a, width, back, parts, st);
  }
}

}  // namespace

int conv_parts(long long, long long, long long channels) {
  // enough CTAs over all channel groups to fill the GPU several times
  const long long groups = (channels + 127) / 128, want = ((long long)148 * 8 + groups - 1) / groups;
  return (int)(want < 16 ? 16 : want > 256 ? 256 : want);
}

cudaError_t launch_conv_forward(const ConvCall& c, cudaStream_t st) {
  ConvArgs a{};
  a.x = c.x, a.state = c.state, a.weight = c.weight, a.bias = c.bias, a.lengths = c.lengths, a.y = c.y, a.state_out = c.state_out;
  a.B = c.batch, a.T = c.length, a.C = c.channels, a.xb = c.x_stride[0], a.xt = c.x_stride[1], a.silu = c.silu;
  int parts = 0;
  return launch(a, c.dtype, c.width, false, &parts, st);
}

cudaError_t launch_conv_backward(const ConvCall& c, cudaStream_t st) {
  ConvArgs a{};
  const bool sums = c.grad_weight != nullptr || c.grad_bias != nullptr;
  a.x = c.x, a.state = c.state, a.gy = c.grad_y, a.gso = c.grad_state_out, a.weight = c.weight, a.bias = c.bias;
  a.lengths = c.lengths, a.gx = c.grad_x, a.gs = c.grad_state, a.partial = sums ? c.partial : nullptr;
  a.B = c.batch, a.T = c.length, a.C = c.channels, a.xb = c.x_stride[0], a.xt = c.x_stride[1];
  a.gb = c.grad_stride[0], a.gt = c.grad_stride[1], a.silu = c.silu;
  int parts = 0;
  const cudaError_t e = launch(a, c.dtype, c.width, true, &parts, st);
  if (e != cudaSuccess || !sums) return e;
  return launch_sum_parts(c.partial, parts, c.channels * (c.width + 1),
                          {{c.grad_weight, c.channels * c.width}, {c.grad_bias, c.channels}}, st);
}

}  // namespace dtst
