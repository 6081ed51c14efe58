// Short causal convolution of every channel with its own K weights (K <= 4), token-major tensors [batch][length][channels]:
//     u = [state (K - 1 steps); x],   pre_t = b + sum_k w_k u_(t+k),   y_t = pre_t  or  pre_t sigmoid(pre_t)
// and its backward pass, with gp_t = gy_t dy/dpre:
//     grad_u_(t+k) = sum_k w_k gp_t  (+ the gradient of the new state),   grad_w_k = sum gp_t u_(t+k),   grad_b = sum gp_t
// The new state is the last K - 1 steps of u at the sequence's own length, whatever that is.
//
// Bound by memory: a thread holds a few neighbouring channels and walks over a run of steps with the last K inputs in registers,
// at fixed places (the loop is unrolled over a multiple of K steps), so a step is read once but for the K - 1 in front of a run
// (backward: also behind it).  The next steps are copied into shared memory of the thread's own while a step is formed; two channels
// go to an instruction.  Runs are as long as leaves enough of them to fill the GPU.  The parameters' gradients are summed in registers
// over the runs a thread visits, over a CTA's warps in shared memory, and over CTAs by a second launch, all in a fixed order: same
// bits on every run.
// Measured, [4][4096][4096], width 4, SiLU: bf16 52 us forward and 107 backward (5.1 and 3.8 TB/s), fp32 90 and 142 (6.0 and 5.7).  With
// the next four steps in registers instead: bf16 65 and 115, fp32 89 and 171; without SiLU the backward pass takes 85.  In 16 bits it is bound
// by latency: 16 warps an SM, each with chains of a dozen operations a step, issue 2 of 4 instructions a clock, with no unit and not the
// memory above half of its rate.  Four CTAs an SM (128 registers) brought 115 to 107 in 16 bits; fp32 would spill.
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

__device__ __forceinline__ float2 twice(float a) { return make_float2(a, a); }
__device__ __forceinline__ float2 sigmoid_of(float2 p) {
  const float2 q = mul_pair(p, twice(-kLog2e));
  const float2 d = add_pair(make_float2(ex2(q.x), ex2(q.y)), twice(1.f));
  return make_float2(rcp(d.x), rcp(d.y));
}

// V channels (2 or 4) as pairs, and the same in memory: in one access (VEC), or one by one
template <int V>
struct Chans {
  float2 v[V / 2];
};
template <typename T, int V, bool VEC>
struct Row {
  Pack<T, V> raw;
  __device__ __forceinline__ void load(const T* p, bool on, int left) {
    if (!on) raw.zero();
    else if (VEC) raw.load(p);
    else raw.load_part(p, left);
  }
  __device__ __forceinline__ Chans<V> get() const {
    float f[V];
    raw.unpack(f);
    Chans<V> c;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) c.v[i] = make_float2(f[2 * i], f[2 * i + 1]);
    return c;
  }
  static __device__ __forceinline__ void put(const Chans<V>& c, T* p, int left) {
    float f[V];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) f[2 * i] = c.v[i].x, f[2 * i + 1] = c.v[i].y;
    Row r;
    r.raw.pack(f);
    if (VEC) r.raw.store(p);
    else r.raw.store_part(p, left);
  }
};

// weights of V channels, [channel][k] in memory
template <int V, int K>
__device__ __forceinline__ void load_taps(Chans<V> (&w)[K], Chans<V>& b, const ConvArgs& a, long long c, int left) {
  const auto at = [&](const float* p, int i, int k, int n) { return p != nullptr && i < left ? __ldg(p + (c + i) * n + k) : 0.f; };
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
#pragma unroll
    for (int k = 0; k < K; ++k) w[k].v[i] = make_float2(at(a.weight, 2 * i, k, K), at(a.weight, 2 * i + 1, k, K));
    b.v[i] = make_float2(at(a.bias, 2 * i, 0, 1), at(a.bias, 2 * i + 1, 0, 1));
  }
}

// What a warp works on: 32 vectors of channels (blockIdx.x), one run of one sequence.
struct Run {
  long long b, t0, t1, n, end;         // steps t0 .. t1; n: the sequence's own length; end: the first step that is not this run's
  __device__ __forceinline__ Run(const ConvArgs& a, long long unit) {
    b = unit / a.runs, t0 = unit % a.runs * a.run, t1 = t0 + a.run < a.T ? t0 + a.run : a.T;
    n = a.T;
    if (a.lengths != nullptr) {
      n = a.lengths[b];
      n = n < 0 ? 0 : n > a.T ? a.T : n;
    }
    end = t1 < n ? t1 : n;
  }
};

// u of step t (t >= -(K-1)): from x, or from the state (zeros without one)
template <typename T, int V, int K, bool VEC>
__device__ __forceinline__ Row<T, V, VEC> load_u(const ConvArgs& a, const Run& r, long long t, long long c, int left) {
  Row<T, V, VEC> v;
  if (t >= 0) v.load(static_cast<const T*>(a.x) + r.b * a.xb + t * a.xt + c, t < r.n, left);
  else v.load(static_cast<const T*>(a.state) + (r.b * (K - 1) + t + K - 1) * a.C + c, a.state != nullptr, left);
  return v;
}

// steps that are unrolled: a multiple of K
template <int K>
constexpr int kUnroll = K == 3 ? 3 : 4;

// What a thread has asked for: groups of U steps of TENSORS tensors.  Vectors go to shared memory of the thread's own, copied there
// asynchronously, so that up to twelve steps are under way without a register for any (fp32: four, of twice the bytes; twelve took 104 us
// instead of 90 forward, 176 instead of 143 backward).  Only the thread itself reads them: no barrier.
template <typename T>
constexpr int kGroups = sizeof(T) == 2 ? 4 : 2;
template <typename T, int V, bool VEC, int U, int TENSORS>
struct Ring {
  static constexpr int AHEAD = kGroups<T> - 1;                 // groups under way
  static constexpr int BYTES = V * (int)sizeof(T), STRIDE = 32 * kWarps * BYTES;
  static constexpr size_t SMEM = (size_t)kGroups<T> * U * TENSORS * STRIDE;
  unsigned char* own;
  __device__ __forceinline__ explicit Ring(unsigned char* smem) : own(smem + (threadIdx.y * 32 + threadIdx.x) * BYTES) {}
  __device__ __forceinline__ unsigned char* at(int group, int j, int tensor) const {
    return own + (((group & (kGroups<T> - 1)) * U + j) * TENSORS + tensor) * STRIDE;
  }
  // p need not exist where `on` is false: nothing is read then, and zeros are put down
  __device__ __forceinline__ void ask(int group, int j, int tensor, const T* p, const T* valid, bool on, int) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(at(group, j, tensor)))),
                 "l"(on ? p : valid), "n"(BYTES), "r"(on ? BYTES : 0)
                 : "memory");
  }
  static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // until at most N groups are under way
  template <int N>
  static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
  __device__ __forceinline__ Row<T, V, VEC> get(int group, int j, int tensor) const {
    Row<T, V, VEC> r;
    r.raw = *reinterpret_cast<const Pack<T, V>*>(at(group, j, tensor));
    return r;
  }
};
// Elements one by one are no copies that the hardware makes by itself (2 bytes are too few): the next group stands in registers, one
// to an element, since what joins two of them waits for both.  [4][4096][4095], width 4: bf16 73 us forward and 136 backward, fp32 100 and
// 171; put down in shared memory as they arrive: 159 and 554, 179 and 597; two 16-bit elements to a register: 157 and 556.
template <typename T, int V, int U, int TENSORS>
struct Ring<T, V, false, U, TENSORS> {
  static constexpr int AHEAD = 1;
  static constexpr size_t SMEM = 0;
  T next[U][TENSORS][V];
  __device__ __forceinline__ explicit Ring(unsigned char*) {}
  __device__ __forceinline__ void ask(int, int j, int tensor, const T* p, const T*, bool on, int left) {
#pragma unroll
    for (int i = 0; i < V; ++i) next[j][tensor][i] = on && i < left ? p[i] : Elem<T>::put(0.f);
  }
  static __device__ __forceinline__ void commit() {}
  template <int N>
  static __device__ __forceinline__ void wait() {}
  __device__ __forceinline__ Row<T, V, false> get(int, int j, int tensor) const {
    Row<T, V, false> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.raw.v[i] = next[j][tensor][i];
    return r;
  }
};

template <typename T, int V, int K, bool VEC>
__global__ void __launch_bounds__(32 * kWarps) conv_forward_kernel(const ConvArgs a) {
  using RowT = Row<T, V, VEC>;
  constexpr int U = kUnroll<K>;
  pdl_trigger();
  pdl_wait();
  const long long c = ((long long)blockIdx.x * 32 + threadIdx.x) * V;
  const long long unit = ((long long)blockIdx.z * gridDim.y + blockIdx.y) * kWarps + threadIdx.y;
  if (c >= a.C || unit >= a.B * a.runs) return;
  const int left = (int)(a.C - c < V ? a.C - c : V);
  const Run r(a, unit);
  Chans<V> w[K], bias, u[K];           // step t's input at place (t - t0) % K
  load_taps<V, K>(w, bias, a, c, left);
#pragma unroll
  for (int k = 0; k < K - 1; ++k) u[k + 1] = load_u<T, V, K, VEC>(a, r, r.t0 - (K - 1) + k, c, left).get();
  // the new state first: the old one may be in its place
  if (r.t0 == 0 && K > 1 && a.state_out != nullptr) {
    RowT s[K > 1 ? K - 1 : 1];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) s[k] = load_u<T, V, K, VEC>(a, r, r.n - (K - 1) + k, c, left);
#pragma unroll
    for (int k = 0; k < K - 1; ++k) RowT::put(s[k].get(), static_cast<T*>(a.state_out) + (r.b * (K - 1) + k) * a.C + c, left);
  }
  const T* x = static_cast<const T*>(a.x) + r.b * a.xb + r.t0 * a.xt + c;
  T* y = static_cast<T*>(a.y) + (r.b * a.T + r.t0) * a.C + c;
  const int steps = (int)(r.end > r.t0 ? r.end - r.t0 : 0);
  extern __shared__ __align__(16) unsigned char conv_smem[];
  using RingT = Ring<T, V, VEC, U, 1>;
  RingT ring(conv_smem);
  const T* const valid = static_cast<const T*>(a.x);
  // (a group behind the end is not asked for: bf16 [4096][1][4096] 157 -> 144 us, [20000][3][512] 100 -> 93; the backward pass gains at one step, 177 -> 164,
  // and loses at three, 155 -> 194)
  const auto ask = [&](int g) {
    if (!VEC || g * U < steps) {
#pragma unroll
      for (int j = 0; j < U; ++j, x += a.xt) ring.ask(g, j, 0, x, valid, g * U + j < steps, left);
    }
    RingT::commit();
  };
  if (steps > 0) {
#pragma unroll
    for (int g = 0; g < RingT::AHEAD; ++g) ask(g);
  }
  const auto step = [&](int j, const RowT& now) {
    u[j % K] = now.get();
    Chans<V> o;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      float2 p = bias.v[i];
#pragma unroll
      for (int k = 0; k < K; ++k) p = fma_pair(w[k].v[i], u[(j + 1 + k) % K].v[i], p);
      o.v[i] = a.silu ? mul_pair(p, sigmoid_of(p)) : p;
    }
    RowT::put(o, y, left);
    y += a.C;
  };
  for (int g = 0; g * U < steps; ++g) {
    RingT::template wait<RingT::AHEAD - 1>();
    RowT now[U];
#pragma unroll
    for (int j = 0; j < U; ++j) now[j] = ring.get(g, j, 0);
    ask(g + RingT::AHEAD);                // (where the group in front of this one was)
    if ((g + 1) * U <= steps) {
#pragma unroll
      for (int j = 0; j < U; ++j) step(j, now[j]);
    } else {
#pragma unroll
      for (int j = 0; j < U - 1; ++j)
        if (g * U + j < steps) step(j, now[j]);
    }
  }
  RingT::template wait<0>();
  for (long long z = r.t0 + steps; z < r.t1; ++z, y += a.C) RowT::put(Chans<V>{}, y, left);
}

// Backward.  Step t of the loop forms gp_t; with it the gradient of u_(t) is complete and is written, as that of step
// t - (K - 1): of x, or of the state in front of a sequence's first run.
// (128 registers in 16 bits and without vectors: fp32 [4][4096][4095] 194 -> 171 us; fp32 vectors would spill.)
template <typename T, int V, int K, bool VEC>
__global__ void __launch_bounds__(32 * kWarps, sizeof(T) == 2 || !VEC ? 4 : 1) conv_backward_kernel(const ConvArgs a) {
  using RowT = Row<T, V, VEC>;
  constexpr int U = kUnroll<K>;
  __shared__ float2 red[kWarps][32][V / 2];
  pdl_trigger();
  pdl_wait();
  const long long c = ((long long)blockIdx.x * 32 + threadIdx.x) * V;
  const bool on = c < a.C;
  const int left = (int)(a.C - c < V ? a.C - c : V);
  Chans<V> gw[K + 1] = {};             // the last one: the bias'
  extern __shared__ __align__(16) unsigned char conv_smem[];
  using RingT = Ring<T, V, VEC, U, 2>;
  RingT ring(conv_smem);
  const T* const valid = static_cast<const T*>(a.x);
  if (on) {
    Chans<V> w[K], bias;
    load_taps<V, K>(w, bias, a, c, left);
    for (long long unit = (long long)blockIdx.y * kWarps + threadIdx.y; unit < a.B * a.runs; unit += (long long)gridDim.y * kWarps) {
      const Run r(a, unit);
      const T* x = static_cast<const T*>(a.x) + r.b * a.xb + r.t0 * a.xt + c;
      const T* gy = static_cast<const T*>(a.gy) + (r.b * a.T + r.t0) * a.C + c;
      T* gx = static_cast<T*>(a.gx) + r.b * a.gb + (r.t0 - (K - 1)) * a.gt + c;      // (of the step that step 0 completes)
      Chans<V> u[K], g[K] = {};        // step t's at place (t - t0) % K
#pragma unroll
      for (int k = 0; k < K - 1; ++k) u[k + 1] = load_u<T, V, K, VEC>(a, r, r.t0 - (K - 1) + k, c, left).get();
      const int own = (int)(r.end > r.t0 ? r.end - r.t0 : 0);            // steps of this run
      const int live = (int)(r.n > r.t0 ? r.n - r.t0 : 0);               // steps to the sequence's end
      // (a run without steps of its own has nothing to write but zeros; the first one has the state's gradient)
      const int stop = own > 0 || r.t0 == 0 ? own + K - 1 : 0;
      const int asked = live < stop ? live : stop;
      const auto ask = [&](int g) {
#pragma unroll
        for (int j = 0; j < U; ++j, x += a.xt, gy += a.C) {
          ring.ask(g, j, 0, x, valid, g * U + j < asked, left);
          ring.ask(g, j, 1, gy, valid, g * U + j < asked, left);
        }
        RingT::commit();
      };
      RingT::template wait<0>();         // (what the run in front of this one asked for beyond its end)
      if (asked > 0 || !VEC) {
#pragma unroll
        for (int g = 0; g < RingT::AHEAD; ++g) ask(g);
      }
      // step t = (a multiple of U) + j; INSIDE: one of this run's, which completes another one's of this run, without the new state's
      const auto step = [&](int t, int j, const RowT& cx, const RowT& cg, auto inside) {
        constexpr bool INSIDE = decltype(inside)::value;
        u[j % K] = cx.get();
        g[j % K] = cg.get();             // (zero behind the sequence's end)
        Chans<V> o;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
          float2 gp = g[j % K].v[i];
          if (a.silu) {
            float2 p = bias.v[i];
#pragma unroll
            for (int k = 0; k < K; ++k) p = fma_pair(w[k].v[i], u[(j + 1 + k) % K].v[i], p);
            const float2 sg = sigmoid_of(p);
            const float2 d = fma_pair(p, fma_pair(sg, twice(-1.f), twice(1.f)), twice(1.f));
            gp = mul_pair(gp, mul_pair(sg, d));
          }
          if (!INSIDE && t >= live) gp = twice(0.f);
          g[j % K].v[i] = gp;
          if (INSIDE || t < own) {
            gw[K].v[i] = add_pair(gw[K].v[i], gp);
#pragma unroll
            for (int k = 0; k < K; ++k) gw[k].v[i] = fma_pair(gp, u[(j + 1 + k) % K].v[i], gw[k].v[i]);
          }
          o.v[i] = mul_pair(w[0].v[i], g[j % K].v[i]);
#pragma unroll
          for (int k = 1; k < K; ++k) o.v[i] = fma_pair(w[k].v[i], g[(j + K - k) % K].v[i], o.v[i]);
        }
        if constexpr (INSIDE) {
          RowT::put(o, gx, left);
        } else {
          const long long to = r.t0 + t - (K - 1), late = to - (r.n - (K - 1));      // late: number of the new state's step
          if (to >= r.t0 || (r.t0 == 0 && a.gs != nullptr)) {
            if (K > 1 && late >= 0 && a.gso != nullptr) {
              RowT q;
              q.load(static_cast<const T*>(a.gso) + (r.b * (K - 1) + late) * a.C + c, true, left);
              const Chans<V> f = q.get();
#pragma unroll
              for (int i = 0; i < V / 2; ++i) o.v[i] = add_pair(o.v[i], f.v[i]);
            }
            if (to >= 0) RowT::put(o, gx, left);
            else RowT::put(o, static_cast<T*>(a.gs) + (r.b * (K - 1) + to + K - 1) * a.C + c, left);
          }
        }
        gx += a.gt;
      };
      for (int t = 0; t < stop; t += U) {
        const int group = t / U;
        RingT::template wait<RingT::AHEAD - 1>();
        RowT cx[U], cg[U];
#pragma unroll
        for (int j = 0; j < U; ++j) cx[j] = ring.get(group, j, 0), cg[j] = ring.get(group, j, 1);
        if (asked > 0 || !VEC) ask(group + RingT::AHEAD);      // (where the group in front of this one was; without any, what was read counts for nothing)
        // these complete the steps t - (K - 1) .. t + U - K; the new state begins at live - (K - 1)
        if (t >= K - 1 && t + U <= own && t + U <= live) {
#pragma unroll
          for (int j = 0; j < U; ++j) step(t + j, j, cx[j], cg[j], std::true_type());
        } else {
#pragma unroll
          for (int j = 0; j < U; ++j)
            if (t + j < stop) step(t + j, j, cx[j], cg[j], std::false_type());
        }
      }
      T* z = static_cast<T*>(a.gx) + r.b * a.gb + (r.t0 + own) * a.gt + c;
      for (long long t = r.t0 + own; t < r.t1; ++t, z += a.gt) RowT::put(Chans<V>{}, z, left);
    }
    RingT::template wait<0>();
  }
  if (a.partial == nullptr) return;
  float* out = a.partial + (long long)blockIdx.y * a.C * (K + 1);
#pragma unroll
  for (int k = 0; k <= K; ++k) {           // over the CTA's warps, in order
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V / 2; ++i) red[threadIdx.y][threadIdx.x][i] = gw[k].v[i];
    __syncthreads();
    if (threadIdx.y == 0 && on) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        float2 t = red[0][threadIdx.x][i];
#pragma unroll
        for (int y = 1; y < kWarps; ++y) t = add_pair(t, red[y][threadIdx.x][i]);
        const long long at = k < K ? (c + 2 * i) * K + k : a.C * K + c + 2 * i;
        if (2 * i < left) out[at] = t.x;
        if (2 * i + 1 < left) out[at + (k < K ? K : 1)] = t.y;
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

template <typename T, int V, int K, bool VEC>
cudaError_t launch_k(ConvArgs a, bool back, int* parts, cudaStream_t st) {
  const long long groups = (a.C + 32 * V - 1) / (32 * V);
  a.run = run_steps(groups * a.B, a.T, back ? 16 : 8);
  a.runs = (int)((a.T + a.run - 1) / a.run);
  if (a.runs < 1) a.runs = 1;                                    // no steps: the state alone
  const long long units = a.B * a.runs;
  const long long rows = (units + kWarps - 1) / kWarps;
  if (!back) {
    // (a grid's second dimension holds 65535: more of them go to the third)
    const long long layers = (rows + 65534) / 65535, per = (rows + layers - 1) / layers;
    return launch_pdl(conv_forward_kernel<T, V, K, VEC>, dim3((unsigned)groups, (unsigned)per, (unsigned)layers), dim3(32, kWarps),
                      Ring<T, V, VEC, kUnroll<K>, 1>::SMEM, st, a);
  }
  // as many CTAs as run at once
  static Resident seen;
  static std::atomic<uint64_t> allowed;
  auto kern = conv_backward_kernel<T, V, K, VEC>;
  constexpr size_t SMEM = Ring<T, V, VEC, kUnroll<K>, 2>::SMEM;
  const cudaError_t e = allow_smem((const void*)kern, SMEM + 4096, allowed);      // (with what the kernel declares itself)
  if (e != cudaSuccess) return e;
  long long most = resident_ctas((const void*)kern, 32 * kWarps, SMEM, seen) / groups;
  if (most < 1) most = 1;
  if (most > conv_parts(a.C)) most = conv_parts(a.C);
  *parts = (int)(rows < most ? rows : most);
  return launch_pdl(kern, dim3((unsigned)groups, (unsigned)*parts), dim3(32, kWarps), SMEM, st, a);
}

template <typename T, int V, bool VEC>
cudaError_t launch_v(const ConvArgs& a, int width, bool back, int* parts, cudaStream_t st) {
  switch (width) {
    case 1: return launch_k<T, V, 1, VEC>(a, back, parts, st);
    case 2: return launch_k<T, V, 2, VEC>(a, back, parts, st);
    case 3: return launch_k<T, V, 3, VEC>(a, back, parts, st);
    default: return launch_k<T, V, 4, VEC>(a, back, parts, st);
  }
}

// four channels a thread where every tensor's rows take such vectors, else two, else two one by one
template <typename T>
cudaError_t launch_t(const ConvArgs& a, int width, bool back, int* parts, cudaStream_t st) {
  const auto fits = [&](int v) {
    bool ok = a.C % v == 0 && a.xb % v == 0 && a.xt % v == 0 && a.gb % v == 0 && a.gt % v == 0;
    for (const void* p : {a.x, a.state, a.gy, a.gso, (const void*)a.y, (const void*)a.state_out, (const void*)a.gx, (const void*)a.gs})
      ok = ok && aligned_to(p, v * sizeof(T));
    return ok;
  };
  if (fits(4)) return launch_v<T, 4, true>(a, width, back, parts, st);
  if (fits(2)) return launch_v<T, 2, true>(a, width, back, parts, st);
  return launch_v<T, 2, false>(a, width, back, parts, st);
}

cudaError_t launch(const ConvArgs& a, int dtype, int width, bool back, int* parts, cudaStream_t st) {
  switch (dtype) {
    case DTST_F32: return launch_t<float>(a, width, back, parts, st);
    case DTST_BF16: return launch_t<__nv_bfloat16>(a, width, back, parts, st);
    default: return launch_t<__half>(a, width, back, parts, st);
  }
}

}  // namespace

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
