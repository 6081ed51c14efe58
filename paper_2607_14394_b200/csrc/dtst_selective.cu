// Selective scan: a diagonal state space for every channel whose step, input map and output map come with each token:
//     d_t = softplus(dt_t + bias)  (or dt_t + bias as it is),   a_t = exp(d_t A),   h_t = a_t h_(t-1) + d_t x_t B_t,
//     y_t = (C_t . h_t + D x_t)  [z_t sigmoid(z_t)]
// on token-major tensors [batch][length][channels], N states to a channel, B and C [batch][length][groups][N] shared by the
// channels of a group; and its backward pass, with gy' = gy z sigmoid(z):
//     e_t = gy'_t C_t + a_(t+1) e_(t+1),   q = e_t a_t h_(t-1),
//     grad_x = d (e . B) + gy' D,   grad_d = q . A + x (e . B),   grad_dt = grad_d sigmoid(dt + bias),   grad_A = sum q d,
//     grad_B = sum_c e d x,   grad_C = sum_c gy' h,   grad_z = gy (C . h + D x) d(z sigmoid z)/dz,   grad_h0 = a_0 e_0
// Everything is in 32 bits.  a_t is ex2.approx of d A log2(e): 2 units in the last place.
//
// Layout.  A thread holds four states of one channel, P = N / 4 neighbouring lanes a channel, so the sums over states are
// shuffles among P lanes; a CTA holds DC channels of one group and R runs of consecutive steps, one run to a set of DC P
// threads, so that a long sequence of few channels still fills the GPU.  A tile of R runs is staged in shared memory (the
// step, the input and the maps in 32 bits, formed once an element), while the next tile's loads are under way.
//   forward, R > 1: a run's decays stay in registers; it runs from a zero state, the runs' ends and products are joined in
//     order, and it runs again from its true state: one exponential a state and step.
//   backward: the forward pass leaves the states of every 8th step; a run of 8 steps is recomputed from there, its states and
//     decays stay in registers, and it runs back, twice where R > 1 (from zero to join the runs, then with the true gradient).
// Bound: N exponentials an element on the 16 lanes of an SM's special function unit are one clock an element at N = 16, three
// times what its bytes take; backward by the issue slots of about 15 operations a state and step.
// All sums are formed in a fixed order: same bits on every run.
#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float sigmoid_of(float p) { return __fdividef(1.f, 1.f + __expf(-p)); }
// log(1 + e^v) to the last bits on both sides: the larger of v and 0, and what is left of it
__device__ __forceinline__ float softplus_of(float v) { return fmaxf(v, 0.f) + log1pf(__expf(-fabsf(v))); }

struct F4 {
  float v[4];
};
__device__ __forceinline__ F4 as4(float4 q) { return F4{{q.x, q.y, q.z, q.w}}; }
__device__ __forceinline__ float4 quad(const F4& q) { return make_float4(q.v[0], q.v[1], q.v[2], q.v[3]); }

struct SelArgs {
  Rows x, dt, z, B, C;
  const float *A, *D, *bias, *h0, *grad_last;
  const int* lengths;
  void* y;
  const void* gy;
  float *h_last, *ck;
  Rows gx, gdt, gz;
  float *gA, *gD, *gbias, *gh0;        // gA, gD, gbias: a row of [C N], [C], [C] per batch entry
  float* gmaps;                        // [blocks of a group][batch][length][groups][2][N4]
  long long batch, length, channels;
  int states, groups, per_group, blocks;      // channels of a group, blocks of channels to a group
  int softplus, vec;                   // vec: rows of every token-major tensor take vector accesses
  int n4;                              // states rounded up to four
};

// what a CTA works on
struct Place {
  long long b;
  int group, c0, left;                 // first channel, channels of this block
  long long len;                       // steps that exist
};
template <int DC>
__device__ __forceinline__ Place place_of(const SelArgs& a) {
  Place p;
  p.b = blockIdx.y;
  p.group = blockIdx.x / a.blocks;
  const int k = (blockIdx.x % a.blocks) * DC;
  p.c0 = p.group * a.per_group + k;
  p.left = min(DC, a.per_group - k);
  p.len = a.length;
  if (a.lengths != nullptr) {
    const long long n = a.lengths[p.b];
    p.len = n < 0 ? 0 : n > a.length ? a.length : n;
  }
  return p;
}

// V neighbouring channels of a step, as they lie in memory
template <typename T, int V>
__device__ __forceinline__ void fetch_row(Pack<T, V>& k, const Rows& r, long long b, long long t, int c, bool on, int left, bool vec) {
  if (!on || left <= 0) {
    k.zero();
    return;
  }
  const T* p = static_cast<const T*>(r.p) + b * r.batch + t * r.step + c;
  if (V == 1 || (vec && left >= V)) k.load(p);
  else k.load_part(p, left);
}
template <typename T, int V>
__device__ __forceinline__ void put_row(const float (&v)[V], T* p, int left, bool vec) {
  Pack<T, V> k;
  k.pack(v);
  if (left <= 0) return;
  if (V == 1 || (vec && left >= V)) k.store(p);
  else k.store_part(p, left);
}

// four numbers of a row of `n` from `i` on
__device__ __forceinline__ F4 four(const float* p, int i, int n) {
  F4 q;
#pragma unroll
  for (int j = 0; j < 4; ++j) q.v[j] = i + j < n ? p[i + j] : 0.f;
  return q;
}

// Sums of M values over LANES neighbouring lanes: every exchange halves the values while there are several, so that M values
// cost about M exchanges; v[0 .. max(1, M / LANES)) remain, value (lane's bits, highest first) of the M.
template <int M, int LANES, int STRIDE>
__device__ __forceinline__ void lane_sums(float (&v)[M], int lane) {
  int m = M;
#pragma unroll
  for (int o = LANES / 2; o > 0; o /= 2) {
    if (m > 1) {
      m /= 2;
      const bool up = lane & (o * STRIDE);
#pragma unroll
      for (int i = 0; i < M / 2; ++i) {
        if (i >= m) break;
        const float send = up ? v[i] : v[i + m], keep = up ? v[i + m] : v[i];
        v[i] = keep + __shfl_xor_sync(0xffffffffu, send, o * STRIDE);
      }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], o * STRIDE);
    }
  }
}

// ------------------------------------------------------------------------------------------------ forward
template <int P, int R>
struct FwdCfg {
  static constexpr int THREADS = 256, S = 16, DC = THREADS / (P * R), TS = S * R, NP = 4 * P;
  static constexpr int PER = TS * DC / THREADS;               // elements a thread stages
  static constexpr int V = PER < 4 ? PER : 4, ITEMS = PER / V;
  static constexpr int MAPS = TS * NP * 2, MAP_ITEMS = (MAPS + THREADS - 1) / THREADS;
  static constexpr int YLD = DC + (DC % 32 == 0 ? 4 : 0);
  static constexpr size_t SMEM = sizeof(float) * ((size_t)2 * TS * DC * 2 + 2 * MAPS + (R > 1 ? 1 : 2) * TS * YLD + (R > 1 ? 8 * THREADS : 0));
};

template <typename T, int P, int R>
__global__ void __launch_bounds__(FwdCfg<P, R>::THREADS, 2) selective_forward_kernel(const SelArgs a) {
  using Cfg = FwdCfg<P, R>;
  constexpr int DC = Cfg::DC, TS = Cfg::TS, S = Cfg::S, NP = Cfg::NP, V = Cfg::V, ITEMS = Cfg::ITEMS, THREADS = Cfg::THREADS;
  extern __shared__ __align__(16) float sel_smem[];
  float2* dd = reinterpret_cast<float2*>(sel_smem);                     // [2][TS][DC]: step, step times input
  float* maps = sel_smem + (size_t)2 * TS * DC * 2;                     // [2][TS][2][NP]
  // sums over states [TS][YLD]; two in turn where one barrier a tile is all there is (R = 1)
  float* const ybuf = maps + 2 * Cfg::MAPS;
  float4* ends = reinterpret_cast<float4*>(ybuf + (R > 1 ? 1 : 2) * TS * Cfg::YLD);         // [R][DC P]: state at a run's end from zero
  float4* prods = ends + THREADS;                                       // [R][DC P]: product of a run's decays
  pdl_trigger();
  pdl_wait();
  const Place at = place_of<DC>(a);
  const int tid = threadIdx.x, p = tid % P, ch = tid / P % DC, run = tid / (P * DC), cp = tid % (P * DC);
  const bool mine = ch < at.left;
  const int c = at.c0 + ch;
  F4 A2 = {}, h = {};
  if (mine) {
    A2 = four(a.A + (long long)c * a.states, 4 * p, a.states);
    if (a.h0 != nullptr) h = four(a.h0 + (at.b * a.channels + c) * a.states, 4 * p, a.states);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) A2.v[j] *= kLog2e;
  const bool vec = a.vec != 0;
  // staging: this thread's vectors of a tile, the same channels every time
  const int sc = tid % (DC / V) * V, srow = tid / (DC / V);
  constexpr int ROWS = THREADS / (DC / V);
  Pack<T, V> px[ITEMS], pd[ITEMS], pz[ITEMS], cx[ITEMS];
  float bias[V], skip[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const bool on = sc + i < at.left;
    bias[i] = on && a.bias != nullptr ? a.bias[at.c0 + sc + i] : 0.f;
    skip[i] = on && a.D != nullptr ? a.D[at.c0 + sc + i] : 0.f;
  }
  T pm[Cfg::MAP_ITEMS];
  auto fetch = [&](long long t0) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const long long t = t0 + srow + k * ROWS;
      fetch_row<T, V>(px[k], a.x, at.b, t, at.c0 + sc, t < at.len, at.left - sc, vec);
      fetch_row<T, V>(pd[k], a.dt, at.b, t, at.c0 + sc, t < at.len, at.left - sc, vec);
    }
#pragma unroll
    for (int k = 0; k < Cfg::MAP_ITEMS; ++k) {
      const int e = tid + k * THREADS, n = e % NP, which = e / NP % 2;
      const long long t = t0 + e / (2 * NP);
      pm[k] = Elem<T>::put(0.f);
      if (e < Cfg::MAPS && n < a.states && t < at.len) {
        const Rows& m = which ? a.C : a.B;
        pm[k] = static_cast<const T*>(m.p)[at.b * m.batch + t * m.step + at.group * a.states + n];
      }
    }
  };
  auto stage = [&](long long t0, int buf) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int row = srow + k * ROWS;
      float x[V], d[V];
      px[k].unpack(x);
      pd[k].unpack(d);
      const bool on = t0 + row < at.len;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        d[i] += bias[i];
        if (a.softplus) d[i] = softplus_of(d[i]);
        if (!on) d[i] = 0.f;
        dd[(buf * TS + row) * DC + sc + i] = make_float2(d[i], d[i] * x[i]);
      }
      cx[k] = px[k];
    }
#pragma unroll
    for (int k = 0; k < Cfg::MAP_ITEMS; ++k) {
      const int e = tid + k * THREADS;
      if (e < Cfg::MAPS) maps[buf * Cfg::MAPS + e] = Elem<T>::get(pm[k]);
    }
  };
  if (at.len > 0) {
    fetch(0);
    stage(0, 0);
  }
  __syncthreads();
  int buf = 0;
  for (long long t0 = 0; t0 < at.len; t0 += TS, buf ^= 1) {
    float* const ys = ybuf + (R > 1 ? 0 : buf) * TS * Cfg::YLD;
    Pack<T, V> ex[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) ex[k] = cx[k];
    const bool more = t0 + TS < at.len;
    if (more) fetch(t0 + TS);
    if (a.z.p != nullptr) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const long long t = t0 + srow + k * ROWS;
        fetch_row<T, V>(pz[k], a.z, at.b, t, at.c0 + sc, t < at.len, at.left - sc, vec);
      }
    }
    const float2* dr = dd + (buf * TS + run * S) * DC + ch;
    const float4* mr = reinterpret_cast<const float4*>(maps + buf * Cfg::MAPS + run * S * 2 * NP) + p;
    F4 decay[R > 1 ? S : 1];
    if constexpr (R > 1) {
      F4 end = {};
      float sum = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const float2 d = dr[s * DC];
        const F4 B = as4(mr[s * 2 * P]);
        sum += d.x;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          decay[s].v[j] = ex2(d.x * A2.v[j]);
          end.v[j] = fmaf(decay[s].v[j], end.v[j], d.y * B.v[j]);
        }
      }
      F4 prod;
#pragma unroll
      for (int j = 0; j < 4; ++j) prod.v[j] = ex2(sum * A2.v[j]);
      ends[run * (DC * P) + cp] = quad(end);
      prods[run * (DC * P) + cp] = quad(prod);
      __syncthreads();
      // the state in front of this run, and (kept for the next tile) behind the tile
      F4 now = h;
#pragma unroll
      for (int q = 0; q < R; ++q) {
        const F4 e = as4(ends[q * (DC * P) + cp]), f = as4(prods[q * (DC * P) + cp]);
        if (q == run) now = h;
#pragma unroll
        for (int j = 0; j < 4; ++j) h.v[j] = h.v[j] == 0.f ? e.v[j] : fmaf(f.v[j], h.v[j], e.v[j]);
      }
      F4 carry = h;
      h = now;
      now = carry;
#define DTST_CARRY now
      const long long tr = t0 + run * S;
#pragma unroll
      for (int s = 0; s < S; s += 4) {
        if (s % kSelectiveSave == 0 && a.ck != nullptr && mine && 4 * p < a.n4 && tr + s < at.len)
          *reinterpret_cast<float4*>(a.ck + (((at.b * ((a.length + kSelectiveSave - 1) / kSelectiveSave) + (tr + s) / kSelectiveSave) * a.channels) + c) * a.n4 + 4 * p) = quad(h);
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 d = dr[(s + k) * DC];
          const F4 B = as4(mr[(s + k) * 2 * P]), C = as4(mr[(s + k) * 2 * P + P]);
          float t = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            h.v[j] = fmaf(decay[s + k].v[j], h.v[j], d.y * B.v[j]);
            t = fmaf(C.v[j], h.v[j], t);
          }
          y[k] = t;
        }
        lane_sums<4, P, 1>(y, tid);
        // lane p has the sums of 4 / P steps from 4 p / P on (P <= 4), or of step p / (P / 4)
        if constexpr (P <= 4) {
#pragma unroll
          for (int k = 0; k < 4 / P; ++k) ys[(run * S + s + p * (4 / P) + k) * Cfg::YLD + ch] = y[k];
        } else {
          if (p % (P / 4) == 0) ys[(run * S + s + p / (P / 4)) * Cfg::YLD + ch] = y[0];
        }
      }
      h = DTST_CARRY;
#undef DTST_CARRY
    } else {
      const int steps = (int)min((long long)TS, at.len - t0);
      for (int s = 0; s < steps; s += 4) {
        if (s % kSelectiveSave == 0 && a.ck != nullptr && mine && 4 * p < a.n4)
          *reinterpret_cast<float4*>(a.ck + (((at.b * ((a.length + kSelectiveSave - 1) / kSelectiveSave) + (t0 + s) / kSelectiveSave) * a.channels) + c) * a.n4 + 4 * p) = quad(h);
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 d = dr[(s + k) * DC];
          const F4 B = as4(mr[(s + k) * 2 * P]), C = as4(mr[(s + k) * 2 * P + P]);
          float t = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            h.v[j] = fmaf(ex2(d.x * A2.v[j]), h.v[j], d.y * B.v[j]);
            t = fmaf(C.v[j], h.v[j], t);
          }
          y[k] = t;
        }
        lane_sums<4, P, 1>(y, tid);
        if constexpr (P <= 4) {
#pragma unroll
          for (int k = 0; k < 4 / P; ++k) ys[(s + p * (4 / P) + k) * Cfg::YLD + ch] = y[k];
        } else {
          if (p % (P / 4) == 0) ys[(s + p / (P / 4)) * Cfg::YLD + ch] = y[0];
        }
      }
    }
    if (more) stage(t0 + TS, buf ^ 1);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int row = srow + k * ROWS;
      const long long t = t0 + row;
      if (t >= a.length) continue;
      float o[V], x[V], z[V];
      ex[k].unpack(x);
      if (a.z.p != nullptr) pz[k].unpack(z);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        o[i] = fmaf(skip[i], x[i], ys[row * Cfg::YLD + sc + i]);
        if (a.z.p != nullptr) o[i] *= z[i] * sigmoid_of(z[i]);
        if (t >= at.len) o[i] = 0.f;
      }
      put_row<T, V>(o, static_cast<T*>(a.y) + (at.b * a.length + t) * a.channels + at.c0 + sc, at.left - sc, vec);
    }
  }
  // behind the sequence's last tile
  const float zero[V] = {};
  for (long long t = (at.len + TS - 1) / TS * TS + srow; t < a.length; t += ROWS)
    put_row<T, V>(zero, static_cast<T*>(a.y) + (at.b * a.length + t) * a.channels + at.c0 + sc, at.left - sc, vec);
  if (a.h_last != nullptr && run == 0 && mine) {
    float* o = a.h_last + (at.b * a.channels + c) * a.states;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * p + j < a.states) o[4 * p + j] = h.v[j];
  }
}

// ------------------------------------------------------------------------------------------------ backward
template <int P, int R>
struct BackCfg {
  static constexpr int THREADS = 256, S = kSelectiveSave, DC = THREADS / (P * R), TS = S * R, NP = 4 * P;
  static constexpr int PER = TS * DC / THREADS;               // 8 / P
  static constexpr int V = PER < 1 ? 1 : PER < 4 ? PER : 4, ITEMS = PER < 1 ? 1 : PER / V;
  static constexpr int MAPS = TS * NP * 2, MAP_ITEMS = (MAPS + THREADS - 1) / THREADS;
  static constexpr int LD = DC + (DC % 32 == 0 ? 4 : 0);
  static constexpr int WARPS = THREADS / 32, RUN_WARPS = WARPS / R > 0 ? WARPS / R : 1;
  // step and step times input, gy', both maps (two buffers each); three sums over states; the warps' sums over channels;
  // the runs' ends
  static constexpr size_t SMEM = sizeof(float) * ((size_t)2 * TS * DC * 3 + 2 * MAPS + 3 * TS * LD + WARPS * S * 2 * NP + (R > 1 ? 8 * THREADS : 0));
};

template <typename T, int P, int R>
__global__ void __launch_bounds__(BackCfg<P, R>::THREADS, 2) selective_backward_kernel(const SelArgs a) {
  using Cfg = BackCfg<P, R>;
  constexpr int DC = Cfg::DC, TS = Cfg::TS, S = Cfg::S, NP = Cfg::NP, V = Cfg::V, ITEMS = Cfg::ITEMS, THREADS = Cfg::THREADS, LD = Cfg::LD;
  static_assert(Cfg::WARPS % R == 0, "a warp belongs to one run");
  extern __shared__ __align__(16) float sel_smem[];
  float2* dd = reinterpret_cast<float2*>(sel_smem);                     // [2][TS][DC]
  float* gys = sel_smem + (size_t)2 * TS * DC * 2;                      // [2][TS][DC]
  float* maps = gys + (size_t)2 * TS * DC;                              // [2][TS][2][NP]
  float* sums = maps + 2 * Cfg::MAPS;                                   // [3][TS][LD]: e . B, q . A2, C . h
  float* chan = sums + 3 * TS * LD;                                     // [WARPS][S][2][NP]: sums over a warp's channels
  float4* ends = reinterpret_cast<float4*>(chan + Cfg::WARPS * S * 2 * NP);
  float4* prods = ends + THREADS;
  pdl_trigger();
  pdl_wait();
  const Place at = place_of<DC>(a);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, p = tid % P, ch = tid / P % DC, run = tid / (P * DC), cp = tid % (P * DC);
  const bool mine = ch < at.left;
  const int c = at.c0 + ch;
  F4 A2 = {}, carry = {}, gA = {};
  if (mine) {
    A2 = four(a.A + (long long)c * a.states, 4 * p, a.states);
    if (a.grad_last != nullptr) carry = four(a.grad_last + (at.b * a.channels + c) * a.states, 4 * p, a.states);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) A2.v[j] *= kLog2e;
  const bool vec = a.vec != 0, gated = a.z.p != nullptr;
  const int sc = tid % (DC / V) * V, srow = tid / (DC / V);
  constexpr int ROWS = THREADS / (DC / V);
  const bool stager = srow < TS;                                        // (more threads than elements where P is large)
  Pack<T, V> px[ITEMS], pd[ITEMS], pz[ITEMS], pg[ITEMS];
  float bias[V], skip[V], gD[V], gbias[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const bool on = sc + i < at.left;
    bias[i] = on && a.bias != nullptr ? a.bias[at.c0 + sc + i] : 0.f;
    skip[i] = on && a.D != nullptr ? a.D[at.c0 + sc + i] : 0.f;
    gD[i] = gbias[i] = 0.f;
  }
  const Rows gyr{const_cast<void*>(a.gy), a.length * a.channels, a.channels};
  T pm[Cfg::MAP_ITEMS];
  F4 start = {};
  const long long saves = (a.length + S - 1) / S;
  auto fetch = [&](long long t0) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const long long t = t0 + srow + k * ROWS;
      const bool on = stager && t < at.len;
      fetch_row<T, V>(px[k], a.x, at.b, t, at.c0 + sc, on, at.left - sc, vec);
      fetch_row<T, V>(pd[k], a.dt, at.b, t, at.c0 + sc, on, at.left - sc, vec);
      fetch_row<T, V>(pg[k], gyr, at.b, t, at.c0 + sc, on, at.left - sc, vec);
      if (gated) fetch_row<T, V>(pz[k], a.z, at.b, t, at.c0 + sc, on, at.left - sc, vec);
    }
#pragma unroll
    for (int k = 0; k < Cfg::MAP_ITEMS; ++k) {
      const int e = tid + k * THREADS, n = e % NP, which = e / NP % 2;
      const long long t = t0 + e / (2 * NP);
      pm[k] = Elem<T>::put(0.f);
      if (e < Cfg::MAPS && n < a.states && t < at.len) {
        const Rows& m = which ? a.C : a.B;
        pm[k] = static_cast<const T*>(m.p)[at.b * m.batch + t * m.step + at.group * a.states + n];
      }
    }
    const long long tr = t0 + run * S;
    start = F4{};
    if (mine && 4 * p < a.n4 && tr < at.len)
      start = as4(*reinterpret_cast<const float4*>(a.ck + ((at.b * saves + tr / S) * a.channels + c) * a.n4 + 4 * p));
  };
  // what the end of a tile needs of its elements
  float kx[ITEMS][V], kd[ITEMS][V], kslope[ITEMS][V], kg[ITEMS][V], kz[ITEMS][V];
  auto stage = [&](long long t0, int buf) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int row = srow + k * ROWS;
      float z[V];
      px[k].unpack(kx[k]);
      pd[k].unpack(kd[k]);
      pg[k].unpack(kg[k]);
      if (gated) pz[k].unpack(z);
      const bool on = t0 + row < at.len;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float raw = kd[k][i] + bias[i];
        float d = raw, slope = 1.f;
        if (a.softplus) d = softplus_of(raw), slope = sigmoid_of(raw);
        if (!on) d = 0.f;
        kd[k][i] = d, kslope[k][i] = slope;
        kz[k][i] = 0.f;
        if (gated) {
          const float s = sigmoid_of(z[i]);
          kz[k][i] = kg[k][i] * s * fmaf(z[i], 1.f - s, 1.f);
          kg[k][i] *= z[i] * s;
        }
        if (stager) {
          dd[(buf * TS + row) * DC + sc + i] = make_float2(d, d * kx[k][i]);
          gys[(buf * TS + row) * DC + sc + i] = kg[k][i];
        }
      }
    }
#pragma unroll
    for (int k = 0; k < Cfg::MAP_ITEMS; ++k) {
      const int e = tid + k * THREADS;
      if (e < Cfg::MAPS) maps[buf * Cfg::MAPS + e] = Elem<T>::get(pm[k]);
    }
  };
  const long long tiles = (at.len + TS - 1) / TS;
  // behind the sequence's last tile
  if (stager) {
    const float zero[V] = {};
    for (long long t = tiles * TS + srow; t < a.length; t += ROWS < TS ? ROWS : TS) {
      put_row<T, V>(zero, static_cast<T*>(a.gx.p) + at.b * a.gx.batch + t * a.gx.step + at.c0 + sc, at.left - sc, vec);
      put_row<T, V>(zero, static_cast<T*>(a.gdt.p) + at.b * a.gdt.batch + t * a.gdt.step + at.c0 + sc, at.left - sc, vec);
      if (gated) put_row<T, V>(zero, static_cast<T*>(a.gz.p) + at.b * a.gz.batch + t * a.gz.step + at.c0 + sc, at.left - sc, vec);
    }
  }
  if (tiles > 0) {
    fetch((tiles - 1) * TS);
    stage((tiles - 1) * TS, 0);
  }
  __syncthreads();
  int buf = 0;
  for (long long tile = tiles - 1; tile >= 0; --tile, buf ^= 1) {
    const long long t0 = tile * TS;
    const F4 first = start;
    if (tile > 0) fetch(t0 - TS);
    const float2* dr = dd + (buf * TS + run * S) * DC + ch;
    const float* gr = gys + (buf * TS + run * S) * DC + ch;
    const float4* mr = reinterpret_cast<const float4*>(maps + buf * Cfg::MAPS + run * S * 2 * NP) + p;
    // forward again from the state that was saved
    F4 decay[S], hs[S];
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const float2 d = dr[s * DC];
      const F4 B = as4(mr[s * 2 * P]);
      sum += d.x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        decay[s].v[j] = ex2(d.x * A2.v[j]);
        hs[s].v[j] = fmaf(decay[s].v[j], s > 0 ? hs[s > 0 ? s - 1 : 0].v[j] : first.v[j], d.y * B.v[j]);
      }
    }
    if constexpr (R > 1) {
      F4 e = {}, prod;
#pragma unroll
      for (int s = S - 1; s >= 0; --s) {
        const float g = gr[s * DC];
        const F4 C = as4(mr[s * 2 * P + P]);
#pragma unroll
        for (int j = 0; j < 4; ++j) e.v[j] = decay[s].v[j] * fmaf(g, C.v[j], e.v[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) prod.v[j] = ex2(sum * A2.v[j]);
      ends[run * (DC * P) + cp] = quad(e);
      prods[run * (DC * P) + cp] = quad(prod);
      __syncthreads();
    }
    F4 m = carry;                          // what the step behind this run passes back
    if constexpr (R > 1) {
#pragma unroll
      for (int q = R - 1; q >= 0; --q) {
        const F4 e = as4(ends[q * (DC * P) + cp]), f = as4(prods[q * (DC * P) + cp]);
        if (q == run) m = carry;
#pragma unroll
        for (int j = 0; j < 4; ++j) carry.v[j] = carry.v[j] == 0.f ? e.v[j] : fmaf(f.v[j], carry.v[j], e.v[j]);
      }
    }
    // back
#pragma unroll
    for (int s4 = S - 4; s4 >= 0; s4 -= 4) {
      float eb[4], qa[4], cy[4];
#pragma unroll
      for (int k = 3; k >= 0; --k) {
        const int s = s4 + k;
        const float2 d = dr[s * DC];
        const float g = gr[s * DC];
        const F4 B = as4(mr[s * 2 * P]), C = as4(mr[s * 2 * P + P]);
        float v[8];
        eb[k] = qa[k] = cy[k] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float e = fmaf(g, C.v[j], m.v[j]);
          v[j] = e * d.y;
          v[4 + j] = g * hs[s].v[j];
          eb[k] = fmaf(e, B.v[j], eb[k]);
          if (gated) cy[k] = fmaf(C.v[j], hs[s].v[j], cy[k]);
          m.v[j] = e * decay[s].v[j];
          const float q = m.v[j] * (s > 0 ? hs[s > 0 ? s - 1 : 0].v[j] : first.v[j]);
          qa[k] = fmaf(q, A2.v[j], qa[k]);
          gA.v[j] = fmaf(q, d.x, gA.v[j]);
        }
        // over the warp's 32 / P channels; the highest lane bits choose among the values first
        constexpr int LANES = 32 / P, LEFT = LANES >= 8 ? 1 : 8 / LANES;
        lane_sums<8, LANES, P>(v, lane);
        const int order = lane / P;                   // value order / (LANES / 8), or from order * LEFT on
        float* out = chan + (warp * S + s) * 2 * NP;
        if constexpr (LANES >= 8) {
          if (order % (LANES / 8) == 0) {
            const int i = order / (LANES / 8);
            out[(i / 4) * NP + 4 * p + i % 4] = v[0];
          }
        } else {
#pragma unroll
          for (int k2 = 0; k2 < LEFT; ++k2) {
            const int i = order * LEFT + k2;
            out[(i / 4) * NP + 4 * p + i % 4] = v[k2];
          }
        }
      }
      lane_sums<4, P, 1>(eb, lane);
      lane_sums<4, P, 1>(qa, lane);
      if (gated) lane_sums<4, P, 1>(cy, lane);
      constexpr int KEPT = P <= 4 ? 4 / P : 1;
      const int from = run * S + s4 + (P <= 4 ? p * KEPT : p / (P <= 4 ? 1 : P / 4));
      if (P <= 4 || p % (P <= 4 ? 1 : P / 4) == 0) {
#pragma unroll
        for (int k = 0; k < KEPT; ++k) {
          sums[(from + k) * LD + ch] = eb[k];
          sums[(TS + from + k) * LD + ch] = qa[k];
          if (gated) sums[(2 * TS + from + k) * LD + ch] = cy[k];
        }
      }
    }
    if constexpr (R == 1) carry = m;
    __syncthreads();
    // the maps' gradients: over the warps of a run, in order
    for (int i = tid; i < Cfg::MAPS; i += THREADS) {
      const int n = i % NP, which = i / NP % 2, row = i / (2 * NP);
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < Cfg::RUN_WARPS; ++w) t += chan[((row / S * Cfg::RUN_WARPS + w) * S + row % S) * 2 * NP + which * NP + n];
      if (n < a.n4 && t0 + row < at.len)
        a.gmaps[((((long long)(blockIdx.x % a.blocks) * a.batch + at.b) * a.length + t0 + row) * a.groups + at.group) * 2 * a.n4 + which * a.n4 + n] = t;
    }
    if (stager) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int row = srow + k * ROWS;
        const long long t = t0 + row;
        if (t >= a.length) continue;
        const bool on = t < at.len;
        float ox[V], od[V], oz[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float eb = sums[row * LD + sc + i], qa = sums[(TS + row) * LD + sc + i] * kLn2;
          ox[i] = on ? fmaf(kd[k][i], eb, kg[k][i] * skip[i]) : 0.f;
          od[i] = on ? fmaf(kx[k][i], eb, qa) * kslope[k][i] : 0.f;
          if (on) {
            gD[i] = fmaf(kg[k][i], kx[k][i], gD[i]);
            gbias[i] += od[i];
          }
          if (gated) oz[i] = on ? kz[k][i] * fmaf(skip[i], kx[k][i], sums[(2 * TS + row) * LD + sc + i]) : 0.f;
        }
        put_row<T, V>(ox, static_cast<T*>(a.gx.p) + at.b * a.gx.batch + t * a.gx.step + at.c0 + sc, at.left - sc, vec);
        put_row<T, V>(od, static_cast<T*>(a.gdt.p) + at.b * a.gdt.batch + t * a.gdt.step + at.c0 + sc, at.left - sc, vec);
        if (gated) put_row<T, V>(oz, static_cast<T*>(a.gz.p) + at.b * a.gz.batch + t * a.gz.step + at.c0 + sc, at.left - sc, vec);
      }
    }
    if (tile > 0) stage(t0 - TS, buf ^ 1);
    __syncthreads();
  }
  if (run == 0 && mine && a.gh0 != nullptr) {
    float* o = a.gh0 + (at.b * a.channels + c) * a.states;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * p + j < a.states) o[4 * p + j] = carry.v[j];
  }
  // grad_A over the runs, grad_D and grad_bias over the rows of threads, in order
  float4* park = reinterpret_cast<float4*>(sel_smem);
  park[tid] = quad(gA);
  __syncthreads();
  if (run == 0 && mine && a.gA != nullptr) {
    F4 t = {};
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const F4 e = as4(park[q * (DC * P) + cp]);
#pragma unroll
      for (int j = 0; j < 4; ++j) t.v[j] += e.v[j];
    }
    float* o = a.gA + (at.b * a.channels + c) * a.states;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * p + j < a.states) o[4 * p + j] = t.v[j];
  }
  __syncthreads();
  float* rows = sel_smem;                  // [2][ROWS][DC]
#pragma unroll
  for (int i = 0; i < V; ++i) rows[srow * DC + sc + i] = gD[i], rows[(ROWS + srow) * DC + sc + i] = gbias[i];
  __syncthreads();
  for (int i = tid; i < at.left; i += THREADS) {
    float t = 0.f, u = 0.f;
    for (int r = 0; r < ROWS; ++r) t += rows[r * DC + i], u += rows[(ROWS + r) * DC + i];
    if (a.gD != nullptr) a.gD[at.b * a.channels + at.c0 + i] = t;
    if (a.gbias != nullptr) a.gbias[at.b * a.channels + at.c0 + i] = u;
  }
}

// the maps' gradients over the blocks of a group's channels, in order; zero behind a sequence's end
struct MapArgs {
  const float* part;
  Rows gB, gC;
  const int* lengths;
  long long batch, length;
  int groups, states, n4, blocks;
};
template <typename T>
__global__ void __launch_bounds__(256) selective_maps_kernel(const MapArgs a) {
  pdl_trigger();
  pdl_wait();
  const long long row = (long long)a.groups * 2 * a.n4, total = a.batch * a.length * row;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long token = i / row, b = token / a.length, t = token % a.length;
    const int e = (int)(i % row), n = e % a.n4, which = e / a.n4 % 2, g = e / (2 * a.n4);
    if (n >= a.states) continue;
    float s = 0.f;
    if (a.lengths == nullptr || t < a.lengths[b])
#pragma unroll 8
      for (int k = 0; k < a.blocks; ++k) s += a.part[k * total + i];
    const Rows& o = which ? a.gC : a.gB;
    static_cast<T*>(o.p)[b * o.batch + t * o.step + g * a.states + n] = Elem<T>::put(s);
  }
}

int lanes_of(long long states) {
  int p = 1;
  while (4 * p < states) p *= 2;
  return p;
}

// runs to a tile: as few as fill the GPU with two CTAs an SM
int runs_of(const SelectiveCall& c, int threads, int least_dc, int most, int steps) {
  const int P = lanes_of(c.states);
  int R = 1;
  while (R < most && threads / (P * R * 2) >= least_dc && c.length > R * steps) {
    const long long dc = threads / (P * R), per = c.channels / c.groups;
    if (((per + dc - 1) / dc) * c.groups * c.batch >= (long long)num_sms() * 2) break;
    R *= 2;
  }
  return R;
}

SelArgs args_of(const SelectiveCall& c, int dc, int esize, bool back) {
  SelArgs a{};
  a.x = c.x, a.dt = c.dt, a.z = c.z, a.B = c.B, a.C = c.C, a.A = c.A, a.D = c.D, a.bias = c.bias, a.h0 = c.h0;
  a.grad_last = c.grad_last, a.lengths = c.lengths, a.y = c.y, a.gy = c.grad_y, a.h_last = c.h_last, a.ck = c.checkpoints;
  a.gx = c.grad_x, a.gdt = c.grad_dt, a.gz = c.grad_z, a.gh0 = c.grad_h0;
  a.batch = c.batch, a.length = c.length, a.channels = c.channels;
  a.states = (int)c.states, a.groups = (int)c.groups, a.per_group = (int)(c.channels / c.groups);
  a.blocks = (a.per_group + dc - 1) / dc, a.softplus = c.softplus, a.n4 = (int)((c.states + 3) / 4 * 4);
  bool vec = a.per_group % 4 == 0;
  auto ok = [&](const void* p, long long b, long long s) {
    vec = vec && (p == nullptr || (aligned_to(p, 4 * esize) && b % 4 == 0 && s % 4 == 0));
  };
  for (const Rows* r : {&c.x, &c.dt, &c.z}) ok(r->p, r->batch, r->step);
  if (back) {
    for (const Rows* r : {&c.grad_x, &c.grad_dt, &c.grad_z}) ok(r->p, r->batch, r->step);
    ok(c.grad_y, 0, 0);
  } else {
    ok(c.y, 0, 0);
  }
  a.vec = vec;
  return a;
}

template <typename T, int P, int R>
cudaError_t launch_forward_k(const SelectiveCall& c, cudaStream_t st) {
  using Cfg = FwdCfg<P, R>;
  const SelArgs a = args_of(c, Cfg::DC, sizeof(T), false);
  static std::atomic<uint64_t> seen{0};
  auto kern = selective_forward_kernel<T, P, R>;
  const cudaError_t e = allow_smem((const void*)kern, Cfg::SMEM, seen);
  if (e != cudaSuccess) return e;
  return launch_pdl(kern, dim3((unsigned)(a.blocks * a.groups), (unsigned)c.batch), dim3(Cfg::THREADS), Cfg::SMEM, st, a);
}
template <typename T, int P, int R>
cudaError_t launch_backward_k(const SelectiveCall& c, cudaStream_t st) {
  using Cfg = BackCfg<P, R>;
  SelArgs a = args_of(c, Cfg::DC, sizeof(T), true);
  // scratch: a row of the parameters' gradients for each batch entry, then the maps' by blocks of channels
  const long long row = c.channels * (c.states + 2);
  float* rows = c.scratch;
  a.gA = rows, a.gD = rows + c.batch * c.channels * c.states, a.gbias = a.gD + c.batch * c.channels;
  a.gmaps = rows + c.batch * row;
  static std::atomic<uint64_t> seen{0};
  auto kern = selective_backward_kernel<T, P, R>;
  cudaError_t e = allow_smem((const void*)kern, Cfg::SMEM, seen);
  if (e == cudaSuccess)
    e = launch_pdl(kern, dim3((unsigned)(a.blocks * a.groups), (unsigned)c.batch), dim3(Cfg::THREADS), Cfg::SMEM, st, a);
  if (e != cudaSuccess) return e;
  if (c.length > 0) {
    const MapArgs m{a.gmaps, c.grad_B, c.grad_C, c.lengths, c.batch, c.length, a.groups, a.states, a.n4, a.blocks};
    const long long total = c.batch * c.length * a.groups * 2 * a.n4, ctas = (total + 255) / 256, most = (long long)num_sms() * 8;
    e = launch_pdl(selective_maps_kernel<T>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(256), 0, st, m);
    if (e != cudaSuccess) return e;
  }
  const struct { const float* from; float* to; long long n; } sums[3] = {
      {a.gA, c.grad_A, c.channels * c.states}, {a.gD, c.grad_D, c.channels}, {a.gbias, c.grad_bias, c.channels}};
  for (const auto& s : sums) {
    if (s.to == nullptr) continue;
    e = launch_sum_parts(s.from, (int)c.batch, s.n, {{s.to, s.n}}, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

constexpr int kBackThreads = 256, kFwdThreads = 256;

template <typename T, int P>
cudaError_t forward_p(const SelectiveCall& c, cudaStream_t st) {
  constexpr int MOST = P <= 4 ? 8 : 16 / P * 2;      // at least eight channels (P = 16: eight of R = 2)
  const int R = runs_of(c, kFwdThreads, 8, MOST, 16);
  if (R == 1) return launch_forward_k<T, P, 1>(c, st);
  if constexpr (MOST >= 4)
    if (R >= 4) return MOST >= 8 && R >= 8 ? launch_forward_k<T, P, MOST >= 8 ? 8 : 4>(c, st) : launch_forward_k<T, P, 4>(c, st);
  return launch_forward_k<T, P, 2>(c, st);
}
template <typename T, int P>
cudaError_t backward_p(const SelectiveCall& c, cudaStream_t st) {
  constexpr int MOST = P <= 4 ? 8 : 16 / P * 2;
  const int R = runs_of(c, kBackThreads, 8, MOST, kSelectiveSave);
  if (R == 1) return launch_backward_k<T, P, 1>(c, st);
  if constexpr (MOST >= 4)
    if (R >= 4) return MOST >= 8 && R >= 8 ? launch_backward_k<T, P, MOST >= 8 ? 8 : 4>(c, st) : launch_backward_k<T, P, 4>(c, st);
  return launch_backward_k<T, P, 2>(c, st);
}

template <typename T>
cudaError_t dispatch(const SelectiveCall& c, bool back, cudaStream_t st) {
  switch (lanes_of(c.states)) {
    case 1: return back ? backward_p<T, 1>(c, st) : forward_p<T, 1>(c, st);
    case 2: return back ? backward_p<T, 2>(c, st) : forward_p<T, 2>(c, st);
    case 4: return back ? backward_p<T, 4>(c, st) : forward_p<T, 4>(c, st);
    case 8: return back ? backward_p<T, 8>(c, st) : forward_p<T, 8>(c, st);
    default: return back ? backward_p<T, 16>(c, st) : forward_p<T, 16>(c, st);
  }
}

}  // namespace

long long selective_scratch_floats(const SelectiveCall& c) {
  const int P = lanes_of(c.states), R = runs_of(c, kBackThreads, 8, P <= 4 ? 8 : 16 / P * 2, kSelectiveSave);
  const long long dc = kBackThreads / (P * R), per = c.channels / c.groups, blocks = (per + dc - 1) / dc;
  return c.batch * c.channels * (c.states + 2) + blocks * c.batch * c.length * c.groups * 2 * ((c.states + 3) / 4 * 4);
}

cudaError_t launch_selective_forward(const SelectiveCall& c, cudaStream_t st) {
  switch (c.dtype) {
    case DTST_F32: return dispatch<float>(c, false, st);
    case DTST_BF16: return dispatch<__nv_bfloat16>(c, false, st);
    default: return dispatch<__half>(c, false, st);
  }
}
cudaError_t launch_selective_backward(const SelectiveCall& c, cudaStream_t st) {
  switch (c.dtype) {
    case DTST_F32: return dispatch<float>(c, true, st);
    case DTST_BF16: return dispatch<__nv_bfloat16>(c, true, st);
    default: return dispatch<__half>(c, true, st);
  }
}

}  // namespace dtst
