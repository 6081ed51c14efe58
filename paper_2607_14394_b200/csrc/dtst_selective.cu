// Selective scan: a diagonal state space for every channel whose step, input map and output map come with each token:
//     d_t = softplus(dt_t + bias)  (or dt_t + bias as it is),   a_t = exp(d_t A),   h_t = a_t h_(t-1) + d_t x_t B_t,
//     y_t = (C_t . h_t + D x_t)  [z_t sigmoid(z_t)]
// on token-major tensors [batch][length][channels], N states to a channel, B and C [batch][length][groups][N] shared by the
// channels of a group; and its backward pass, with gy' = gy z sigmoid(z):
//     e_t = gy'_t C_t + a_(t+1) e_(t+1),   q = e_t a_t h_(t-1),
//     grad_x = d (e . B) + gy' D,   grad_d = q . A + x (e . B),   grad_dt = grad_d sigmoid(dt + bias),   grad_A = sum q d,
//     grad_B = sum_c e d x,   grad_C = sum_c gy' h,   grad_z = gy (C . h + D x) d(z sigmoid z)/dz,   grad_h0 = a_0 e_0
// Everything is in 32 bits.  a_t is ex2.approx (2 units in the last place) of d A log2(e), whose two roundings are |d A| 2^-23 of a_t: off by
// (2 + |d A|) 2^-23 a_t at most, which is never more than 2^-22 of the state in front.  Joining segments does so once more with the sum of a
// segment's steps.
//
// Layout.  A thread holds four states of two neighbouring channels, P = N / 4 neighbouring lanes a pair of channels, so the sums
// over states are shuffles among P lanes and every word of a map that is read from shared memory serves two channels.  A CTA
// holds 256 / P channels of one group: four warps run the recurrence, four more bring its operands into shared memory (the step, its
// product with the input and the maps in 32 bits, formed once an element), a tile of steps ahead, and take the results out, a
// tile behind; so neither the loads' latency nor that of the element-wise functions holds up the recurrence.
// Few channels: a sequence is cut into segments.  A first pass runs every segment from a zero state and leaves its end and the
// sum of its steps (the product of its decays is exp(A sum)); the second joins the ends of the segments in front of its own, in order,
// and runs from there.  That is a second exponential for each state, so a sequence is cut only where it has to be.
// Backward: the forward pass leaves the states of every 8th step; a run of 8 steps is recomputed from there, its states stay in
// registers, and it runs back.  Segments likewise, from their ends.
// Bound: N exponentials an element on the 16 lanes of an SM's special function unit take a clock an element at N = 16, three times
// what its bytes take.  Shared memory delivers a word a lane and clock however many lanes share it, so the two channels a thread
// that share the maps' words bring those reads down to the same.
// All sums are formed in a fixed order: same bits on every run.
#include <cfloat>

#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

// Threads that run the recurrence, and as many again that bring its operands in and take its results out, so that neither
// the loads' nor the element-wise functions' latency holds up the recurrence.
constexpr int kThreads = 128;
constexpr int kSave = kSelectiveSave;

// Named barriers (one side arrives, the other waits): a tile's operands are there; its sums are.  Two of each, for the two
// buffers in turn.
__device__ __forceinline__ void wait_for(int id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(2 * kThreads) : "memory"); }
__device__ __forceinline__ void tell(int id) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(2 * kThreads) : "memory"); }
constexpr int kFull = 1, kDone = 3;

// The backward pass's two halves share a CTA's registers unevenly: 104 + 152 of 2 x 128.
constexpr int kFewRegisters = 104, kMoreRegisters = 152;
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters)); }
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kMoreRegisters)); }

// log(1 + e^v), and e = e^-|v|: the larger of v and 0, and log(1 + e) = 2 atanh(e / (2 + e)) as a polynomial in the square of
// that argument, fitted over its range of 0 to 1/9 to 8e-9 of the value: no digits are lost where e is small
__device__ __forceinline__ float softplus_of(float v, float& e) {
  e = ex2(-fabsf(v) * kLog2e);
  const float s = e * rcp(2.f + e), q = s * s;
  float p = fmaf(q, 0.14089166f, 0.13980302f);
  p = fmaf(q, p, 0.20012455f);
  p = fmaf(q, p, 0.33333158f);
  p = fmaf(q, p, 1.f);
  return fmaf(2.f * s, p, fmaxf(v, 0.f));
}
__device__ __forceinline__ float sigmoid_of(float v) { return rcp(1.f + ex2(-v * kLog2e)); }

// four states as two pairs, for the instructions that work on two
struct F4 {
  float2 v[2];
};
__device__ __forceinline__ F4 as4(float4 q) { return F4{{make_float2(q.x, q.y), make_float2(q.z, q.w)}}; }
__device__ __forceinline__ float4 quad(const F4& q) { return make_float4(q.v[0].x, q.v[0].y, q.v[1].x, q.v[1].y); }
__device__ __forceinline__ float2 twice(float a) { return make_float2(a, a); }
__device__ __forceinline__ float2 decay_of(float2 d, float2 A2) {
  const float2 p = mul_pair(d, A2);
  return make_float2(ex2(p.x), ex2(p.y));
}
// f h + e, where a state of zero passes a product of decays that is beyond the range
__device__ __forceinline__ float2 carry_on(float2 f, float2 h, float2 e) {
  return make_float2(h.x == 0.f ? e.x : fmaf(f.x, h.x, e.x), h.y == 0.f ? e.y : fmaf(f.y, h.y, e.y));
}

// Stores of the recurrence's sums.  They go to parts of shared memory that these warps never read, and the barrier behind them is
// volatile too: without a word on memory the compiler may move the next step's reads up in front of them.
__device__ __forceinline__ void put_shared(float* p, float v) {
  asm volatile("st.shared.f32 [%0], %1;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "f"(v));
}
__device__ __forceinline__ void put_shared(float* p, float2 v) {
  asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "f"(v.x), "f"(v.y));
}

struct SelArgs {
  Rows x, dt, z, B, C;
  const float *A, *D, *bias, *h0, *grad_last;
  const int* lengths;
  void* y;
  const void* gy;
  float *h_last, *ck;
  Rows gx, gdt, gz;
  float *gparams, *gh0;                // gparams: a row of [C N], [C], [C] per batch entry and segment: of A, D, dt_bias
  float* gmaps;                        // [blocks of a group][batch][length][groups][2][N4]
  // [segments][batch][C][N4], [segments][batch][C]: what a segment leaves, sums of its steps.  The place of the segment whose end nobody
  // joins holds h0 (backward: grad_last) as it was: h_last may take its place while other segments still read it.
  float *ends, *spans;
  long long batch, length, channels;
  int states, groups, per_group, blocks;      // channels of a group, blocks of channels to a group
  int segments, seg;                   // seg: steps to a segment
  int softplus, vec, vec_maps;         // vec: rows of every token-major tensor take vector accesses; vec_maps: and of the maps
  int n4;                              // states rounded up to four
};

// what a CTA works on
struct Place {
  long long b;
  int group, c0, left;                 // first channel, channels of this block
  int part, begin, end, stop;          // segment; its first step, the first step behind it that exists, that there is room for
};
template <int DC>
__device__ __forceinline__ Place place_of(const SelArgs& a, int part) {
  Place p;
  p.b = blockIdx.y;
  p.group = blockIdx.x / a.blocks;
  const int k = (blockIdx.x % a.blocks) * DC;
  p.c0 = p.group * a.per_group + k;
  p.left = min(DC, a.per_group - k);
  const int length = (int)a.length, len = a.lengths != nullptr ? max(0, min(a.lengths[p.b], length)) : length;
  p.part = part;
  p.begin = part * a.seg;
  p.stop = min(length, p.begin + a.seg);
  p.end = max(p.begin, min(len, p.stop));
  return p;
}

// a thread's vector of V channels of a row in a tile, of one token-major tensor
template <typename T, int V>
struct Lane {
  T* p;
  long long tile, item;                // elements between tiles' rows and between a thread's rows of a tile
  __device__ __forceinline__ Lane(const Rows& r, long long b, long long row, int c, int tile_rows, int item_rows)
      : p(static_cast<T*>(r.p) + b * r.batch + row * r.step + c), tile(tile_rows * r.step), item(item_rows * r.step) {}
  __device__ __forceinline__ void fetch(Pack<T, V>& k, int i, bool on, int left, bool full) const {
    if (!on || left <= 0) k.zero();
    else if (V == 1 || full) k.load(p + i * item);
    else k.load_part(p + i * item, left);
  }
  // what the next fetch will ask for, on its way into L2
  __device__ __forceinline__ void ahead(int i, bool on, int left) const {
    if (on && left > 0) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + i * item));
  }
  __device__ __forceinline__ void put(const float (&v)[V], int i, int left, bool full) const {
    Pack<T, V> k;
    k.pack(v);
    if (left <= 0) return;
    if (V == 1 || full) k.store(p + i * item);
    else k.store_part(p + i * item, left);
  }
};

// Sums of four values over P >= 4 neighbouring lanes, for two channels at a time: the first two exchanges halve the values.  Lane p
// ends with value p / (P / 4).
template <int P>
__device__ __forceinline__ float2 state_sums(float2 (&v)[4], int p) {
  const auto from = [](float2 a, int o) { return make_float2(__shfl_xor_sync(0xffffffffu, a.x, o), __shfl_xor_sync(0xffffffffu, a.y, o)); };
  const bool high = p & (P / 2), odd = p & (P / 4);
  const float2 a = add_pair(high ? v[2] : v[0], from(high ? v[0] : v[2], P / 2)), b = add_pair(high ? v[3] : v[1], from(high ? v[1] : v[3], P / 2));
  float2 t = add_pair(odd ? b : a, from(odd ? a : b, P / 4));
#pragma unroll
  for (int o = P / 8; o > 0; o /= 2) t = add_pair(t, from(t, o));
  return t;
}
// ... into rows 0 .. 3 of a [rows][LD] array
template <int P, int LD>
__device__ __forceinline__ void put_sums(float2 (&v)[4], float* rows, int p, int c) {
  const float2 t = state_sums<P>(v, p);
  if (P == 4 || p % (P / 4) == 0) put_shared(rows + p / (P / 4) * LD + c, t);
}

// a tile's maps on their way to shared memory: an item is four states of one map at one step
template <typename T, int P, int TS, int COUNT, int PERMS>
struct Maps {
  static constexpr int ALL = TS * COUNT * P, ITEMS = (ALL + kThreads - 1) / kThreads, WORDS = ALL * PERMS;      // (float4s in a buffer)
  Pack<T, 4> raw[ITEMS];
  // COUNT 2: both maps; 1: m0
  __device__ __forceinline__ void fetch(const SelArgs& a, const Place& at, const Rows& m0, const Rows& m1, int t0, int tid) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = tid + k * kThreads, n = 4 * (e % P), which = e / P % COUNT, t = t0 + e / (COUNT * P);
      raw[k].zero();
      if (e < ALL && t < at.end && n < a.states) {
        const Rows& m = which ? m1 : m0;
        const T* p = static_cast<const T*>(m.p) + at.b * m.batch + t * m.step + (long long)at.group * a.states + n;
        if (a.vec_maps) raw[k].load(p);
        else raw[k].load_part(p, min(4, a.states - n));
      }
    }
  }
  // PERMS copies: copy k has state j ^ k (k * 2 where there are two) in place j
  __device__ __forceinline__ void stage(float4* maps, int tid) const {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = tid + k * kThreads;
      if (e >= ALL) continue;
      float v[4];
      raw[k].unpack(v);
      float4* out = maps + (e / P) * PERMS * P + e % P;
      out[0] = make_float4(v[0], v[1], v[2], v[3]);
      if constexpr (PERMS == 2) out[P] = make_float4(v[2], v[3], v[0], v[1]);
      if constexpr (PERMS == 4) {
        out[P] = make_float4(v[1], v[0], v[3], v[2]);
        out[2 * P] = make_float4(v[2], v[3], v[0], v[1]);
        out[3 * P] = make_float4(v[3], v[2], v[1], v[0]);
      }
    }
  }
};

// four numbers of a row of `n` from `i` on, number j ^ perm in place j
__device__ __forceinline__ F4 four(const float* p, int i, int n, int perm) {
  float q[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) q[j] = i + (j ^ perm) < n ? p[i + (j ^ perm)] : 0.f;
  return F4{{make_float2(q[0], q[1]), make_float2(q[2], q[3])}};
}
__device__ __forceinline__ F4 in_order(float4 q, int perm) {        // number j ^ perm in place j
  if (perm & 1) q = make_float4(q.y, q.x, q.w, q.z);
  if (perm & 2) q = make_float4(q.z, q.w, q.x, q.y);
  return as4(q);
}
__device__ __forceinline__ void put_four(const F4& v, float* p, int i, int n, int perm) {
  const float q[4] = {v.v[0].x, v.v[0].y, v.v[1].x, v.v[1].y};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + (j ^ perm) < n) p[i + (j ^ perm)] = q[j];
}

// V neighbouring numbers of a row in shared memory
template <int V>
__device__ __forceinline__ void read_row(float (&v)[V], const float* p) {
  if constexpr (V == 4) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
  } else if constexpr (V == 2) {
    const float2 q = *reinterpret_cast<const float2*>(p);
    v[0] = q.x, v[1] = q.y;
  } else {
    v[0] = p[0];
  }
}

template <int P, int TS>
struct SelCfg {
  [[maybe_unused]] static constexpr int DC = 2 * kThreads / P, NP = 4 * P;
  [[maybe_unused]] static constexpr int PER = TS * DC / kThreads;              // elements a thread stages
  [[maybe_unused]] static constexpr int V = PER < 4 ? PER : 4, ITEMS = PER / V, VECS = DC / V, ROWS = kThreads / VECS;
  [[maybe_unused]] static constexpr int LD = DC + (DC % 32 == 0 ? 4 : 0);
  [[maybe_unused]] static constexpr int LANES = 32 / P;                        // pairs of channels in a warp
  [[maybe_unused]] static constexpr int PERMS = LANES >= 4 ? 4 : LANES;
  [[maybe_unused]] static constexpr size_t FWD = sizeof(float) * ((size_t)2 * TS * DC * 2 + 2 * TS * 2 * NP + 2 * TS * LD);
  [[maybe_unused]] static constexpr size_t ENDS = sizeof(float) * ((size_t)2 * TS * DC * 2 + 2 * TS * NP);
  [[maybe_unused]] static constexpr size_t BACK = sizeof(float) * ((size_t)2 * TS * DC * 3 + 2 * TS * 2 * NP * PERMS + 6 * TS * LD + 2 * kThreads / 32 * TS * 2 * NP);
};
// Steps to a tile forward: 4 x 2048 x 4096, 16 states, takes 276 us with 16, 396 with 8 (what a tile costs both halves of a CTA however
// long it is), 353 with 32 (its operands need registers twice as long); backward 8, the steps between saved states (16: 884 us against 804,
// spills).
constexpr int kFwdSteps = 16;

// A of a thread's states, times log2(e).  Kept finite: a step of zero, which stands behind a sequence's end, decays nothing, and the
// gradient of a decay to zero is zero; with an infinity both would be a NaN.
__device__ __forceinline__ float finite_below(float v) { return v < -FLT_MAX ? -FLT_MAX : v; }
__device__ __forceinline__ void load_A(F4 (&A2)[2], const SelArgs& a, int c, int ch, int left, int p, int perm) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    A2[k] = F4{};
    if (ch + k >= left) continue;
    A2[k] = four(a.A + (long long)(c + k) * a.states, 4 * p, a.states, perm);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float2 q = mul_pair(A2[k].v[j], twice(kLog2e));
      A2[k].v[j] = make_float2(finite_below(q.x), finite_below(q.y));
    }
  }
}
// The state in front of (the gradient behind) the whole sequence, then what a segment finds, joined over the segments in front of
// (behind) it in order.
template <bool BACK>
__device__ __forceinline__ void load_outer(F4 (&h)[2], const SelArgs& a, const Place& at, int c, int ch, int p, int perm) {
  const float* from = BACK ? a.grad_last : a.h0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    h[k] = F4{};
    if (ch + k < at.left && from != nullptr) h[k] = four(from + (at.b * a.channels + c + k) * a.states, 4 * p, a.states, perm);
  }
}
template <bool BACK>
__device__ __forceinline__ void join_segments(F4 (&h)[2], const F4 (&A2)[2], const SelArgs& a, const Place& at, int c, int ch, int p, int perm) {
  if (a.segments == 1) {
    load_outer<BACK>(h, a, at, c, ch, p, perm);
    return;
  }
  h[0] = h[1] = F4{};
  const int n = BACK ? a.segments - 1 - at.part : at.part;
  if (4 * p >= a.n4 || ch >= at.left) return;
  const int two = ch + 1 < at.left ? 1 : 0;               // (the block's last channel alone: twice the same)
  const long long seg = a.batch * a.channels, from = at.b * a.channels + c + (BACK ? (a.segments - 1) * seg : 0);
  const long long outer = at.b * a.channels + c + (BACK ? 0 : (a.segments - 1) * seg);
#pragma unroll
  for (int k = 0; k < 2; ++k) h[k] = in_order(*reinterpret_cast<const float4*>(a.ends + (outer + k * two) * a.n4 + 4 * p), perm);
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    const long long q = from + (BACK ? -i : i) * seg;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float span = a.spans[q + k * two];
      const F4 e = in_order(*reinterpret_cast<const float4*>(a.ends + (q + k * two) * a.n4 + 4 * p), perm);
#pragma unroll
      for (int j = 0; j < 2; ++j) h[k].v[j] = carry_on(decay_of(twice(span), A2[k].v[j]), h[k].v[j], e.v[j]);
    }
  }
}

// one step of two channels of a thread: f = exp(d A), h = f h + in B
__device__ __forceinline__ void step_on(F4 (&h)[2], const F4 (&A2)[2], const float4& d, const F4& B) {
  const float step[2] = {d.x, d.z}, in[2] = {d.y, d.w};
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int j = 0; j < 2; ++j) h[k].v[j] = fma_pair(decay_of(twice(step[k]), A2[k].v[j]), h[k].v[j], mul_pair(twice(in[k]), B.v[j]));
}
// ... and backwards: e = g C + m, m = f e
__device__ __forceinline__ void step_back(F4 (&m)[2], const F4 (&A2)[2], const float4& d, const F4& C) {
  const float step[2] = {d.x, d.z}, g[2] = {d.y, d.w};
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int j = 0; j < 2; ++j) m[k].v[j] = mul_pair(decay_of(twice(step[k]), A2[k].v[j]), fma_pair(twice(g[k]), C.v[j], m[k].v[j]));
}

// ------------------------------------------------------------------------------------------------ segments
// Every segment from nothing: the state that it leaves behind (BACK: the gradient that it passes to what is in front of it), and the
// sum of its steps.
template <typename T, int P, bool BACK>
__global__ void __launch_bounds__(2 * kThreads, 2) selective_ends_kernel(const SelArgs a) {
  constexpr int TS = kFwdSteps;
  using Cfg = SelCfg<P, TS>;
  constexpr int DC = Cfg::DC, CP = DC / 2, V = Cfg::V, ITEMS = Cfg::ITEMS, ROWS = Cfg::ROWS;
  using MapsT = Maps<T, P, TS, 1, 1>;
  extern __shared__ __align__(16) float sel_smem[];
  float2* dd = reinterpret_cast<float2*>(sel_smem);                     // [2][TS][DC]: step, its product with the input (BACK: gy')
  float4* maps = reinterpret_cast<float4*>(sel_smem + (size_t)2 * TS * DC * 2);      // [2][TS][P]: B (BACK: C)
  pdl_trigger();
  pdl_wait();
  const Place at = place_of<DC>(a, BACK ? blockIdx.z + 1 : blockIdx.z);
  const int tid = threadIdx.x % kThreads, tiles = (at.end - at.begin + TS - 1) / TS;
  const auto start_of = [&](int i) { return at.begin + (BACK ? tiles - 1 - i : i) * TS; };
  if (threadIdx.x >= kThreads) {
    const int sc = tid % Cfg::VECS * V, srow = tid / Cfg::VECS, left = at.left - sc, dir = BACK ? -TS : TS;
    const bool full = a.vec && left >= V, gated = a.z.p != nullptr;
    const long long row0 = (long long)start_of(0) + srow;
    const Rows other = BACK ? Rows{const_cast<void*>(a.gy), a.length * a.channels, a.channels} : a.x;
    Lane<T, V> ld(a.dt, at.b, row0, at.c0 + sc, dir, ROWS), lo(other, at.b, row0, at.c0 + sc, dir, ROWS), lz(a.z, at.b, row0, at.c0 + sc, dir, ROWS);
    Pack<T, V> pd[ITEMS], po[ITEMS], pz[ITEMS];
    float bias[V];
#pragma unroll
    for (int i = 0; i < V; ++i) bias[i] = i < left && a.bias != nullptr ? a.bias[at.c0 + sc + i] : 0.f;
    MapsT pm;
    auto fetch = [&](int t0) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const bool on = t0 + srow + k * ROWS < at.end;
        ld.fetch(pd[k], k, on, left, full);
        lo.fetch(po[k], k, on, left, full);
        if (BACK && gated) lz.fetch(pz[k], k, on, left, full);
      }
      ld.p += ld.tile, lo.p += lo.tile, lz.p += lz.tile;
      const int next = BACK ? t0 - TS : t0 + TS;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const bool on = next >= at.begin && next + srow + k * ROWS < at.end;
        ld.ahead(k, on, left);
        lo.ahead(k, on, left);
        if (BACK && gated) lz.ahead(k, on, left);
      }
      pm.fetch(a, at, BACK ? a.C : a.B, a.C, t0, tid);
    };
    if (tiles > 0) fetch(start_of(0));
    for (int i = 0; i < tiles; ++i) {
      const int buf = i & 1, t0 = start_of(i);
      if (i > 1) wait_for(kDone + buf);
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int row = srow + k * ROWS;
        float d[V], o[V], z[V];
        pd[k].unpack(d);
        po[k].unpack(o);
        if (BACK && gated) pz[k].unpack(z);
        const bool on = t0 + row < at.end;
#pragma unroll
        for (int n = 0; n < V; ++n) {
          float e;
          d[n] += bias[n];
          if (a.softplus) d[n] = softplus_of(d[n], e);
          if (!on) d[n] = 0.f;
          if (!BACK) o[n] *= d[n];
          else if (gated) o[n] *= z[n] * sigmoid_of(z[n]);
        }
        float2* out = dd + (buf * TS + row) * DC + sc;
        if constexpr (V == 1) {
          out[0] = make_float2(d[0], o[0]);
        } else {
#pragma unroll
          for (int n = 0; n < V; n += 2) *reinterpret_cast<float4*>(out + n) = make_float4(d[n], o[n], d[n + 1], o[n + 1]);
        }
      }
      pm.stage(maps + buf * MapsT::WORDS, tid);
      tell(kFull + buf);
      if (i + 1 < tiles) fetch(start_of(i + 1));
    }
    // (the barriers' last rounds, which the recurrence's threads have arrived at)
    for (int i = max(0, tiles - 2); i < tiles; ++i) wait_for(kDone + (i & 1));
    return;
  }
  const int p = tid % P, ch = 2 * (tid / P), c = at.c0 + ch;
  F4 A2[2], h[2] = {};
  load_A(A2, a, c, ch, at.left, p, 0);
  float sum[2] = {0.f, 0.f};
  for (int i = 0; i < tiles; ++i) {
    const int buf = i & 1;
    const float4* dr = reinterpret_cast<const float4*>(dd + buf * TS * DC) + ch / 2;
    const float4* mr = maps + buf * MapsT::WORDS + p;
    wait_for(kFull + buf);
#pragma unroll 8      // (sixteen would spill)
    for (int n = 0; n < TS; ++n) {
      const int s = BACK ? TS - 1 - n : n;
      const float4 d = dr[s * CP];
      const F4 m = as4(mr[s * P]);
      sum[0] += d.x, sum[1] += d.z;
      if (BACK) step_back(h, A2, d, m);
      else step_on(h, A2, d, m);
    }
    tell(kDone + buf);
  }
  const long long q = at.part * a.batch + at.b, outer = (BACK ? 0 : a.segments - 1) * a.batch + at.b;
  const bool first = at.part == (BACK ? a.segments - 1 : 0);
  F4 o[2] = {};
  if (first) load_outer<BACK>(o, a, at, c, ch, p, 0);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (ch + k >= at.left) continue;
    if (4 * p < a.n4) *reinterpret_cast<float4*>(a.ends + (q * a.channels + c + k) * a.n4 + 4 * p) = quad(h[k]);
    if (first && 4 * p < a.n4) *reinterpret_cast<float4*>(a.ends + (outer * a.channels + c + k) * a.n4 + 4 * p) = quad(o[k]);
    if (p == 0) a.spans[q * a.channels + c + k] = sum[k];
  }
}

// ------------------------------------------------------------------------------------------------ forward
__device__ __forceinline__ void store_if(bool on, float* p, const float4& v) {      // (without a branch between the steps)
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %0, 0;\n\t@p st.global.v4.f32 [%1], {%2, %3, %4, %5};\n\t}" ::"r"((int)on), "l"(p), "f"(v.x),
               "f"(v.y), "f"(v.z), "f"(v.w));
}

template <typename T, int P>
__global__ void __launch_bounds__(2 * kThreads, 2) selective_forward_kernel(const SelArgs a) {
  constexpr int TS = kFwdSteps;
  using Cfg = SelCfg<P, TS>;
  constexpr int DC = Cfg::DC, CP = DC / 2, V = Cfg::V, ITEMS = Cfg::ITEMS, ROWS = Cfg::ROWS, LD = Cfg::LD;
  using MapsT = Maps<T, P, TS, 2, 1>;
  extern __shared__ __align__(16) float sel_smem[];
  float2* dd = reinterpret_cast<float2*>(sel_smem);                     // [2][TS][DC]: step, step times input
  float4* maps = reinterpret_cast<float4*>(sel_smem + (size_t)2 * TS * DC * 2);      // [2][TS][2][P]
  float* sums = reinterpret_cast<float*>(maps + 2 * MapsT::WORDS);      // [2][TS][LD]: sums over states
  pdl_trigger();
  pdl_wait();
  const Place at = place_of<DC>(a, blockIdx.z);
  const int tid = threadIdx.x % kThreads;
  if (threadIdx.x >= kThreads) {
    // ---- in and out: this thread's vectors of a tile, the same channels every time
    const int sc = tid % Cfg::VECS * V, srow = tid / Cfg::VECS, left = at.left - sc;
    const bool full = a.vec && left >= V, gated = a.z.p != nullptr;
    const long long row0 = (long long)at.begin + srow;
    Lane<T, V> lx(a.x, at.b, row0, at.c0 + sc, TS, ROWS), ld(a.dt, at.b, row0, at.c0 + sc, TS, ROWS), lz(a.z, at.b, row0, at.c0 + sc, TS, ROWS),
        ly(Rows{a.y, a.length * a.channels, a.channels}, at.b, row0, at.c0 + sc, TS, ROWS);
    Pack<T, V> px[ITEMS], pd[ITEMS], pz[ITEMS], kx[ITEMS], kz[ITEMS];
    float bias[V], skip[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      bias[i] = i < left && a.bias != nullptr ? a.bias[at.c0 + sc + i] : 0.f;
      skip[i] = i < left && a.D != nullptr ? a.D[at.c0 + sc + i] : 0.f;
    }
    MapsT pm;
    auto fetch = [&](int t0) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const bool on = t0 + srow + k * ROWS < at.end;
        lx.fetch(px[k], k, on, left, full);
        ld.fetch(pd[k], k, on, left, full);
        if (gated) lz.fetch(pz[k], k, on, left, full);
      }
      lx.p += lx.tile, ld.p += ld.tile, lz.p += lz.tile;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const bool on = t0 + TS + srow + k * ROWS < at.end;
        lx.ahead(k, on, left);
        ld.ahead(k, on, left);
        if (gated) lz.ahead(k, on, left);
      }
      pm.fetch(a, at, a.B, a.C, t0, tid);
    };
    auto finish = [&](int t0, int buf) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int row = srow + k * ROWS, t = t0 + row;
        if (t >= at.stop) continue;
        float o[V], x[V], z[V];
        kx[k].unpack(x);
        if (gated) kz[k].unpack(z);
        read_row<V>(o, sums + (buf * TS + row) * LD + sc);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          o[i] = fmaf(skip[i], x[i], o[i]);
          if (gated) o[i] *= z[i] * sigmoid_of(z[i]);
          if (t >= at.end) o[i] = 0.f;
        }
        ly.put(o, k, left, full);
      }
      ly.p += ly.tile;
    };
    if (at.begin < at.end) fetch(at.begin);
    int buf = 0;
    for (int t0 = at.begin; t0 < at.end; t0 += TS, buf ^= 1) {
      Pack<T, V> cx[ITEMS], cz[ITEMS];
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int row = srow + k * ROWS;
        float x[V], d[V];
        px[k].unpack(x);
        pd[k].unpack(d);
        cx[k] = px[k];
        if (gated) cz[k] = pz[k];
        const bool on = t0 + row < at.end;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float e;
          d[i] += bias[i];
          if (a.softplus) d[i] = softplus_of(d[i], e);
          if (!on) d[i] = 0.f;
        }
        float2* out = dd + (buf * TS + row) * DC + sc;
        if constexpr (V == 1) {
          out[0] = make_float2(d[0], d[0] * x[0]);
        } else {
#pragma unroll
          for (int i = 0; i < V; i += 2) *reinterpret_cast<float4*>(out + i) = make_float4(d[i], d[i] * x[i], d[i + 1], d[i + 1] * x[i + 1]);
        }
      }
      pm.stage(maps + buf * MapsT::WORDS, tid);
      tell(kFull + buf);
      if (t0 + TS < at.end) fetch(t0 + TS);
      if (t0 > at.begin) {
        wait_for(kDone + (buf ^ 1));
        finish(t0 - TS, buf ^ 1);
      }
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) kx[k] = cx[k], kz[k] = cz[k];
    }
    const int behind = at.begin + (at.end - at.begin + TS - 1) / TS * TS;
    if (at.begin < at.end) {
      buf ^= 1;
      wait_for(kDone + buf);
      finish(behind - TS, buf);
    }
    // behind the sequence's last tile
    const float zero[V] = {};
    for (int t0 = behind; t0 < at.stop; t0 += TS) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
        if (t0 + srow + k * ROWS < at.stop) ly.put(zero, k, left, full);
      ly.p += ly.tile;
    }
    return;
  }
  // ---- the recurrence
  const int p = tid % P, ch = 2 * (tid / P), c = at.c0 + ch;
  F4 A2[2], h[2];
  load_A(A2, a, c, ch, at.left, p, 0);
  join_segments<false>(h, A2, a, at, c, ch, p, 0);
  const long long saves = (a.length + kSave - 1) / kSave, save_ld = a.channels * a.n4;
  float* ck = a.ck + (at.b * saves + at.begin / kSave) * save_ld + (long long)c * a.n4 + 4 * p;
  bool save[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) save[k] = a.ck != nullptr && 4 * p < a.n4 && ch + k < at.left;
  int buf = 0;
  for (int t0 = at.begin; t0 < at.end; t0 += TS, buf ^= 1, ck += TS / kSave * save_ld) {
    float* const ys = sums + buf * TS * LD;
    const float4* dr = reinterpret_cast<const float4*>(dd + buf * TS * DC) + ch / 2;
    const float4* mr = maps + buf * MapsT::WORDS + p;
    wait_for(kFull + buf);
    // N steps, and then their sums: nothing is stored to shared memory in between, behind which the compiler could not move the
    // next steps' reads up
    const auto steps = [&](int s, auto count) {
      constexpr int N = decltype(count)::value;
      if (s % kSave == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) store_if(save[k], ck + (s / kSave) * save_ld + k * a.n4, quad(h[k]));
      }
      float2 y[N / 4][4];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const F4 B = as4(mr[(s + i) * 2 * P]), C = as4(mr[(s + i) * 2 * P + P]);
        step_on(h, A2, dr[(s + i) * CP], B);
        const float2 o0 = fma_pair(C.v[1], h[0].v[1], mul_pair(C.v[0], h[0].v[0])), o1 = fma_pair(C.v[1], h[1].v[1], mul_pair(C.v[0], h[1].v[0]));
        y[i / 4][i % 4] = make_float2(o0.x + o0.y, o1.x + o1.y);
      }
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        put_sums<P, LD>(y[i], ys + (s + 4 * i) * LD, p, ch);
      }
    };
    if (t0 + TS <= at.end) {
#pragma unroll
      for (int s = 0; s < TS; s += kSave) steps(s, std::integral_constant<int, kSave>());
    } else {             // a single step, or the last few of a sequence
      for (int s = 0; s < at.end - t0; s += 4) steps(s, std::integral_constant<int, 4>());
    }
    tell(kDone + buf);
  }
  if (a.h_last == nullptr || at.part != a.segments - 1) return;
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (ch + k < at.left) put_four(h[k], a.h_last + (at.b * a.channels + c + k) * a.states, 4 * p, a.states, 0);
}

// ------------------------------------------------------------------------------------------------ backward
// Sums over the warp's pairs of channels of four values of each map's gradient.  A lane holds state j ^ perm in place j, so that what
// it keeps and what it sends stand in the same places in every lane; the third exchange chooses between the maps.
template <int P, int LANES>
__device__ __forceinline__ void channel_sums(F4& b, F4& c, int pl, float* out, int n0, int perm, int np) {
  auto swap = [](float v, int o) { return __shfl_xor_sync(0xffffffffu, v, o * P); };
  constexpr int FIRST = LANES >= 4 ? 2 : 1;
  const float2 b2 = add_pair(b.v[0], make_float2(swap(b.v[1].x, FIRST), swap(b.v[1].y, FIRST)));
  const float2 c2 = add_pair(c.v[0], make_float2(swap(c.v[1].x, FIRST), swap(c.v[1].y, FIRST)));
  if constexpr (LANES >= 4) {
    const float2 one = add_pair(make_float2(b2.x, c2.x), make_float2(swap(b2.y, 1), swap(c2.y, 1)));
    if constexpr (LANES == 8) {
      const bool up = pl & 4;
      put_shared(out + (up ? np : 0) + n0 + perm, (up ? one.y : one.x) + swap(up ? one.x : one.y, 4));
    } else {
      put_shared(out + n0 + perm, one.x), put_shared(out + np + n0 + perm, one.y);
    }
  } else {
    put_shared(out + n0 + perm, b2.x), put_shared(out + n0 + (1 ^ perm), b2.y);
    put_shared(out + np + n0 + perm, c2.x), put_shared(out + np + n0 + (1 ^ perm), c2.y);
  }
}

template <typename T, int P>
__global__ void __launch_bounds__(2 * kThreads, 2) selective_backward_kernel(const SelArgs a) {
  constexpr int TS = kSave;
  using Cfg = SelCfg<P, TS>;
  constexpr int DC = Cfg::DC, CP = DC / 2, NP = Cfg::NP, V = Cfg::V, ITEMS = Cfg::ITEMS, ROWS = Cfg::ROWS, LD = Cfg::LD;
  constexpr int LANES = Cfg::LANES, PERMS = Cfg::PERMS, WARPS = kThreads / 32;
  using MapsT = Maps<T, P, TS, 2, PERMS>;
  constexpr int SUMS = 3 * TS * LD, CHAN = WARPS * TS * 2 * NP;
  extern __shared__ __align__(16) float sel_smem[];
  float2* dd = reinterpret_cast<float2*>(sel_smem);                     // [2][TS][DC]
  float* gys = sel_smem + (size_t)2 * TS * DC * 2;                      // [2][TS][DC]
  float4* maps = reinterpret_cast<float4*>(gys + (size_t)2 * TS * DC);  // [2][TS][2][PERMS][P]
  float* sums = reinterpret_cast<float*>(maps + 2 * MapsT::WORDS);      // [2][3][TS][LD]: e . B, q . A2, C . h
  float* chan = sums + 2 * SUMS;                                        // [2][WARPS][TS][2][NP]: sums over a warp's channels
  pdl_trigger();
  pdl_wait();
  const Place at = place_of<DC>(a, blockIdx.z);
  const int tid = threadIdx.x % kThreads, tiles = (at.end - at.begin + TS - 1) / TS;
  float* const params = a.gparams + (at.b * a.segments + at.part) * a.channels * (a.states + 2);
  if (threadIdx.x >= kThreads) {
    // ---- in and out
    fewer_registers();
    const int sc = tid % Cfg::VECS * V, srow = tid / Cfg::VECS, left = at.left - sc;
    const bool full = a.vec && left >= V, gated = a.z.p != nullptr;
    const long long row0 = (long long)at.begin + (tiles - 1) * TS + srow;           // (before the first fetch nothing is read there)
    const Rows gyr{const_cast<void*>(a.gy), a.length * a.channels, a.channels};
    Lane<T, V> lx(a.x, at.b, row0, at.c0 + sc, -TS, ROWS), ld(a.dt, at.b, row0, at.c0 + sc, -TS, ROWS), lz(a.z, at.b, row0, at.c0 + sc, -TS, ROWS),
        lg(gyr, at.b, row0, at.c0 + sc, -TS, ROWS), ox(a.gx, at.b, row0, at.c0 + sc, -TS, ROWS), od(a.gdt, at.b, row0, at.c0 + sc, -TS, ROWS),
        oz(a.gz, at.b, row0, at.c0 + sc, -TS, ROWS);
    // behind the sequence's last tile
    {
      const float zero[V] = {};
      Lane<T, V> wx = ox, wd = od, wz = oz;
      for (int t0 = at.begin + tiles * TS; t0 < at.stop; t0 += TS) {
        wx.p -= wx.tile, wd.p -= wd.tile, wz.p -= wz.tile;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
          if (t0 + srow + k * ROWS >= at.stop) continue;
          wx.put(zero, k, left, full);
          wd.put(zero, k, left, full);
          if (gated) wz.put(zero, k, left, full);
        }
      }
    }
    Pack<T, V> px[ITEMS], pd[ITEMS], pz[ITEMS], pg[ITEMS], kx[ITEMS];
    float bias[V], skip[V], gD[V], gbias[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      bias[i] = i < left && a.bias != nullptr ? a.bias[at.c0 + sc + i] : 0.f;
      skip[i] = i < left && a.D != nullptr ? a.D[at.c0 + sc + i] : 0.f;
      gD[i] = gbias[i] = 0.f;
    }
    MapsT pm;
    auto fetch = [&](int t0) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const bool on = t0 + srow + k * ROWS < at.end;
        lx.fetch(px[k], k, on, left, full);
        ld.fetch(pd[k], k, on, left, full);
        lg.fetch(pg[k], k, on, left, full);
        if (gated) lz.fetch(pz[k], k, on, left, full);
      }
      lx.p += lx.tile, ld.p += ld.tile, lg.p += lg.tile, lz.p += lz.tile;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const bool on = t0 > at.begin;
        lx.ahead(k, on, left);
        ld.ahead(k, on, left);
        lg.ahead(k, on, left);
        if (gated) lz.ahead(k, on, left);
      }
      pm.fetch(a, at, a.B, a.C, t0, tid);
    };
    float slope[ITEMS][V], kz[ITEMS][V];      // what the end of a tile needs of its elements
    float* const maps_out = a.gmaps + (((long long)(blockIdx.x % a.blocks) * a.batch + at.b) * a.length * a.groups + at.group) * 2 * a.n4;
    auto finish = [&](int t0, int buf) {
      // the maps' gradients: over the warps, in order
      const float4* part = reinterpret_cast<const float4*>(chan + buf * CHAN);
#pragma unroll
      for (int i0 = 0; i0 < TS * 2 * P; i0 += kThreads) {
        const int i = i0 + tid, q = i % P, which = i / P % 2, row = i / (2 * P);
        if (i >= TS * 2 * P || 4 * q >= a.n4 || t0 + row >= at.end) continue;
        F4 t = as4(part[i]);
#pragma unroll
        for (int w = 1; w < WARPS; ++w) {
          const F4 u = as4(part[w * TS * 2 * P + i]);
          t.v[0] = add_pair(t.v[0], u.v[0]), t.v[1] = add_pair(t.v[1], u.v[1]);
        }
        *reinterpret_cast<float4*>(maps_out + (long long)(t0 + row) * a.groups * 2 * a.n4 + which * a.n4 + 4 * q) = quad(t);
      }
      const bool ragged = t0 + TS > at.end;
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int row = srow + k * ROWS, t = t0 + row;
        if (t >= at.stop) continue;
        const float* s = sums + buf * SUMS + row * LD + sc;
        float x[V], vx[V], vd[V], vz[V], eb[V], g[V];
        kx[k].unpack(x);
        read_row<V>(eb, s);
        read_row<V>(vd, s + TS * LD);
        if (gated) read_row<V>(vz, s + 2 * TS * LD);
        read_row<V>(g, gys + (buf * TS + row) * DC + sc);
#pragma unroll
        for (int i = 0; i < V; ++i) vx[i] = dd[(buf * TS + row) * DC + sc + i].x;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          vx[i] = fmaf(vx[i], eb[i], g[i] * skip[i]);
          vd[i] = fmaf(x[i], eb[i], vd[i] * kLn2) * slope[k][i];
          if (gated) vz[i] = kz[k][i] * fmaf(skip[i], x[i], vz[i]);
        }
        if (ragged && t >= at.end) {
#pragma unroll
          for (int i = 0; i < V; ++i) vx[i] = vd[i] = vz[i] = g[i] = x[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) gD[i] = fmaf(g[i], x[i], gD[i]), gbias[i] += vd[i];
        ox.put(vx, k, left, full);
        od.put(vd, k, left, full);
        if (gated) oz.put(vz, k, left, full);
      }
      ox.p += ox.tile, od.p += od.tile, oz.p += oz.tile;
    };
    if (tiles > 0) fetch(at.begin + (tiles - 1) * TS);
    int buf = 0;
    for (int tile = tiles - 1; tile >= 0; --tile, buf ^= 1) {
      const int t0 = at.begin + tile * TS;
      Pack<T, V> cx[ITEMS];
      float cslope[ITEMS][V], cz[ITEMS][V];
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        const int row = srow + k * ROWS;
        float x[V], d[V], g[V], z[V];
        px[k].unpack(x);
        pd[k].unpack(d);
        pg[k].unpack(g);
        if (gated) pz[k].unpack(z);
        cx[k] = px[k];
        const bool on = t0 + row < at.end;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float raw = d[i] + bias[i];
          float e;
          d[i] = raw, cslope[k][i] = 1.f, cz[k][i] = 0.f;
          if (a.softplus) {
            d[i] = softplus_of(raw, e);
            const float r = rcp(1.f + e);
            cslope[k][i] = raw >= 0.f ? r : e * r;
          }
          if (!on) d[i] = 0.f;
          if (gated) {
            const float s = sigmoid_of(z[i]);
            cz[k][i] = g[i] * s * fmaf(z[i], 1.f - s, 1.f);
            g[i] *= z[i] * s;
          }
        }
        float2* out = dd + (buf * TS + row) * DC + sc;
        float* og = gys + (buf * TS + row) * DC + sc;
        if constexpr (V == 1) {
          out[0] = make_float2(d[0], d[0] * x[0]), og[0] = g[0];
        } else {
#pragma unroll
          for (int i = 0; i < V; i += 2) {
            *reinterpret_cast<float4*>(out + i) = make_float4(d[i], d[i] * x[i], d[i + 1], d[i + 1] * x[i + 1]);
            *reinterpret_cast<float2*>(og + i) = make_float2(g[i], g[i + 1]);
          }
        }
      }
      pm.stage(maps + buf * MapsT::WORDS, tid);
      tell(kFull + buf);
      if (tile > 0) fetch(t0 - TS);
      if (tile < tiles - 1) {
        wait_for(kDone + (buf ^ 1));
        finish(t0 + TS, buf ^ 1);
      }
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        kx[k] = cx[k];
#pragma unroll
        for (int i = 0; i < V; ++i) slope[k][i] = cslope[k][i], kz[k][i] = cz[k][i];
      }
    }
    if (tiles > 0) {
      wait_for(kDone + (buf ^ 1));
      finish(at.begin, buf ^ 1);
    }
    // grad_D and grad_bias over the rows of threads, in order
    __syncthreads();
    float* rows = sel_smem;                  // [2][ROWS][DC]
#pragma unroll
    for (int i = 0; i < V; ++i) rows[srow * DC + sc + i] = gD[i], rows[(ROWS + srow) * DC + sc + i] = gbias[i];
    __syncthreads();
    for (int i = tid; i < at.left; i += kThreads) {
      float t = 0.f, u = 0.f;
      for (int r = 0; r < ROWS; ++r) t += rows[r * DC + i], u += rows[(ROWS + r) * DC + i];
      params[a.channels * a.states + at.c0 + i] = t;
      params[a.channels * (a.states + 1) + at.c0 + i] = u;
    }
    return;
  }
  // ---- the recurrence
  more_registers();
  const int p = tid % P, pair = tid / P, ch = 2 * pair, c = at.c0 + ch;
  const int pl = pair % LANES, perm = LANES >= 4 ? pl & 3 : (pl & 1) * 2;
  const bool gated = a.z.p != nullptr;
  F4 A2[2], m[2], gA[2] = {};              // m: what the step behind passes back
  load_A(A2, a, c, ch, at.left, p, perm);
  join_segments<true>(m, A2, a, at, c, ch, p, perm);
  const long long saves = (a.length + TS - 1) / TS, save_ld = a.channels * a.n4;
  const float* ck = a.ck + (at.b * saves + at.begin / TS + tiles - 1) * save_ld + (long long)c * a.n4 + 4 * p;
  float4 start[2];
  auto fetch = [&]() {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      start[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (ch + k < at.left && 4 * p < a.n4 ) start[k] = *reinterpret_cast<const float4*>(ck + k * a.n4);
    }
    ck -= save_ld;
  };
  if (tiles > 0) fetch();
  int buf = 0;
  for (int tile = tiles - 1; tile >= 0; --tile, buf ^= 1) {
    F4 first[2];
    first[0] = in_order(start[0], perm), first[1] = in_order(start[1], perm);
    if (tile > 0) fetch();
    const float4* dr = reinterpret_cast<const float4*>(dd + buf * TS * DC) + pair;
    const float2* gr = reinterpret_cast<const float2*>(gys + buf * TS * DC) + pair;
    const float4* mr = maps + buf * MapsT::WORDS + (PERMS == 2 ? perm / 2 : perm) * P + p;
    wait_for(kFull + buf);
    // forward again from the state that was saved
    F4 hs[TS][2];
#pragma unroll
    for (int s = 0; s < TS; ++s) {
      hs[s][0] = s > 0 ? hs[s > 0 ? s - 1 : 0][0] : first[0], hs[s][1] = s > 0 ? hs[s > 0 ? s - 1 : 0][1] : first[1];
      step_on(hs[s], A2, dr[s * CP], as4(mr[s * 2 * PERMS * P]));
    }
    // back
    float* const rs = sums + buf * SUMS;
    float* const cs = chan + buf * CHAN + pair / LANES * TS * 2 * NP;
#pragma unroll
    for (int s4 = TS - 4; s4 >= 0; s4 -= 4) {
      float2 eb[4], qa[4], cy[4];
#pragma unroll
      for (int i = 3; i >= 0; --i) {
        const int s = s4 + i;
        const float4 d = dr[s * CP];
        const float2 g2 = gr[s * CP];
        const F4 B = as4(mr[s * 2 * PERMS * P]), C = as4(mr[(s * 2 + 1) * PERMS * P]);
        const float step[2] = {d.x, d.z}, in[2] = {d.y, d.w}, g[2] = {g2.x, g2.y};
        F4 gb, gc;
        float ebk[2], qak[2], cyk[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float2 eb2, qa2, cy2;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 e = fma_pair(twice(g[k]), C.v[j], m[k].v[j]);
            gb.v[j] = k == 0 ? mul_pair(e, twice(in[k])) : fma_pair(e, twice(in[k]), gb.v[j]);
            gc.v[j] = k == 0 ? mul_pair(twice(g[k]), hs[s][k].v[j]) : fma_pair(twice(g[k]), hs[s][k].v[j], gc.v[j]);
            eb2 = j == 0 ? mul_pair(e, B.v[j]) : fma_pair(e, B.v[j], eb2);
            if (gated) cy2 = j == 0 ? mul_pair(C.v[j], hs[s][k].v[j]) : fma_pair(C.v[j], hs[s][k].v[j], cy2);
            m[k].v[j] = mul_pair(e, decay_of(twice(step[k]), A2[k].v[j]));
            const float2 q = mul_pair(m[k].v[j], s > 0 ? hs[s > 0 ? s - 1 : 0][k].v[j] : first[k].v[j]);
            qa2 = j == 0 ? mul_pair(q, A2[k].v[j]) : fma_pair(q, A2[k].v[j], qa2);
            gA[k].v[j] = fma_pair(q, twice(step[k]), gA[k].v[j]);
          }
          ebk[k] = eb2.x + eb2.y, qak[k] = qa2.x + qa2.y;
          cyk[k] = gated ? cy2.x + cy2.y : 0.f;
        }
        eb[i] = make_float2(ebk[0], ebk[1]), qa[i] = make_float2(qak[0], qak[1]), cy[i] = make_float2(cyk[0], cyk[1]);
        channel_sums<P, LANES>(gb, gc, pl, cs + s * 2 * NP, 4 * p, perm, NP);
      }
      put_sums<P, LD>(eb, rs + s4 * LD, p, ch);
      put_sums<P, LD>(qa, rs + (TS + s4) * LD, p, ch);
      if (gated) {
        put_sums<P, LD>(cy, rs + (2 * TS + s4) * LD, p, ch);
      }
    }
    tell(kDone + buf);
  }
  if (a.gh0 != nullptr && at.part == 0) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (ch + k < at.left) put_four(m[k], a.gh0 + (at.b * a.channels + c + k) * a.states, 4 * p, a.states, perm);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (ch + k < at.left) put_four(gA[k], params + (long long)(c + k) * a.states, 4 * p, a.states, perm);
  __syncthreads();       // (the other half's two)
  __syncthreads();
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
#pragma unroll 16
      for (int k = 0; k < a.blocks; ++k) s += a.part[k * total + i];
    const Rows& o = which ? a.gC : a.gB;
    static_cast<T*>(o.p)[b * o.batch + t * o.step + g * a.states + n] = Elem<T>::put(s);
  }
}

// Lanes to a pair of channels.  Four for fewer than 13 states too, some of them idle: more channels to a CTA instead left too few CTAs and
// too much to stage for each (4 x 2048 x 4096 forward: four states 567 us on one lane, eight 458 on two, 273 on four).
int lanes_of(long long states) { return states <= 16 ? 4 : states <= 32 ? 8 : 16; }
long long blocks_of(const SelectiveCall& c) {          // blocks of channels of a group
  const long long dc = 2 * kThreads / lanes_of(c.states), per = c.channels / c.groups;
  return (per + dc - 1) / dc;
}

// Segments of a sequence: one where there are nearly as many CTAs as SMs without (4 x 4096 channels x 2048 steps: 279 us in one, 384 in
// two; 2 x 4096 x 2048: 228, 226), otherwise enough for eight CTAs an SM (16384 steps of 4096 channels: 1638 us in one, 929 in four,
// 835 in 16, 819 in 32), but no more than the joining of the ends in front leaves useful (16384 steps of 64 channels: 1291 us in
// one, 165 in 16, 70 in 64, 182 in 256).
struct Cut {
  int segments, seg;
};
Cut cut_of(const SelectiveCall& c) {
  const long long ctas = blocks_of(c) * c.groups * c.batch, sms = num_sms();
  long long k = 1;
  if (ctas > 0 && ctas * 5 < sms * 4) {
    k = (8 * sms + ctas - 1) / ctas;
    long long root = 1;
    while (root * root < c.length) root *= 2;
    if (k > root / 2) k = root / 2;
  }
  const long long most = c.length / 64;                // steps to a segment: at least four tiles
  if (k > most) k = most;
  if (k > 256) k = 256;
  if (k < 1) k = 1;
  long long seg = (c.length + k - 1) / k;
  seg = (seg + kFwdSteps - 1) / kFwdSteps * kFwdSteps;
  if (seg < kFwdSteps) seg = kFwdSteps;
  return Cut{(int)(c.length > seg ? (c.length + seg - 1) / seg : 1), (int)seg};
}
// floats that the segments' ends and spans take
long long cut_floats(const SelectiveCall& c) {
  const Cut k = cut_of(c);
  return k.segments > 1 ? k.segments * c.batch * c.channels * ((c.states + 3) / 4 * 4 + 4) : 0;
}

// floats of the parameters' gradients of every batch entry and segment (what follows them begins on 16 bytes)
long long param_floats(const SelectiveCall& c) { return (c.batch * cut_of(c).segments * c.channels * (c.states + 2) + 3) / 4 * 4; }

SelArgs args_of(const SelectiveCall& c, int esize, bool back) {
  SelArgs a{};
  const Cut k = cut_of(c);
  a.x = c.x, a.dt = c.dt, a.z = c.z, a.B = c.B, a.C = c.C, a.A = c.A, a.D = c.D, a.bias = c.bias, a.h0 = c.h0;
  a.grad_last = c.grad_last, a.lengths = c.lengths, a.y = c.y, a.gy = c.grad_y, a.h_last = c.h_last, a.ck = c.checkpoints;
  a.gx = c.grad_x, a.gdt = c.grad_dt, a.gz = c.grad_z, a.gh0 = c.grad_h0;
  a.batch = c.batch, a.length = c.length, a.channels = c.channels;
  a.states = (int)c.states, a.groups = (int)c.groups, a.per_group = (int)(c.channels / c.groups);
  a.blocks = (int)blocks_of(c), a.softplus = c.softplus, a.n4 = (int)((c.states + 3) / 4 * 4);
  a.segments = k.segments, a.seg = k.seg;
  a.ends = c.scratch, a.spans = c.scratch + k.segments * c.batch * c.channels * a.n4;
  auto ok = [&](const void* p, long long b, long long s) { return p == nullptr || (aligned_to(p, 4 * esize) && b % 4 == 0 && s % 4 == 0); };
  bool vec = a.per_group % 4 == 0, maps = c.states % 4 == 0;
  for (const Rows* r : {&c.x, &c.dt, &c.z}) vec = vec && ok(r->p, r->batch, r->step);
  if (back) {
    for (const Rows* r : {&c.grad_x, &c.grad_dt, &c.grad_z}) vec = vec && ok(r->p, r->batch, r->step);
    vec = vec && ok(c.grad_y, 0, 0);
  } else {
    vec = vec && ok(c.y, 0, 0);
  }
  for (const Rows* r : {&c.B, &c.C}) maps = maps && ok(r->p, r->batch, r->step);
  a.vec = vec, a.vec_maps = maps;
  return a;
}

// The uneven split of registers takes 2 x 128 a thread pair from what the CTA was launched with: without them it would wait for ever.
template <typename Kern>
cudaError_t registers_there(Kern kern, std::atomic<uint64_t>& seen) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && (seen.load(std::memory_order_relaxed) >> dev & 1u))) return e;
  cudaFuncAttributes f;
  e = cudaFuncGetAttributes(&f, (const void*)kern);
  if (e != cudaSuccess) return e;
  if (f.numRegs * 2 < kFewRegisters + kMoreRegisters) return cudaErrorNotSupported;
  if (dev < 64) seen.fetch_or(1ull << dev, std::memory_order_relaxed);
  return cudaSuccess;
}

template <typename Kern>
cudaError_t launch(Kern kern, const SelArgs& a, int segments, size_t smem, std::atomic<uint64_t>& seen, cudaStream_t st) {
  const cudaError_t e = allow_smem((const void*)kern, smem, seen);
  if (e != cudaSuccess) return e;
  return launch_pdl(kern, dim3((unsigned)(a.blocks * a.groups), (unsigned)a.batch, (unsigned)segments), dim3(2 * kThreads), smem, st, a);
}

template <typename T, int P>
cudaError_t forward_p(const SelectiveCall& c, cudaStream_t st) {
  using Cfg = SelCfg<P, kFwdSteps>;
  const SelArgs a = args_of(c, sizeof(T), false);
  static std::atomic<uint64_t> seen[2];
  if (a.segments > 1) {
    const cudaError_t e = launch(selective_ends_kernel<T, P, false>, a, a.segments - 1, Cfg::ENDS, seen[0], st);
    if (e != cudaSuccess) return e;
  }
  return launch(selective_forward_kernel<T, P>, a, a.segments, Cfg::FWD, seen[1], st);
}
template <typename T, int P>
cudaError_t backward_p(const SelectiveCall& c, cudaStream_t st) {
  SelArgs a = args_of(c, sizeof(T), true);
  // scratch: the segments' ends, a row of the parameters' gradients for each batch entry and segment, the maps' by blocks of channels
  const long long entries = c.batch * a.segments;
  a.gparams = c.scratch + cut_floats(c);
  a.gmaps = a.gparams + param_floats(c);
  static std::atomic<uint64_t> seen[3];
  cudaError_t e = registers_there(selective_backward_kernel<T, P>, seen[2]);
  if (e == cudaSuccess && a.segments > 1) e = launch(selective_ends_kernel<T, P, true>, a, a.segments - 1, SelCfg<P, kFwdSteps>::ENDS, seen[0], st);
  if (e == cudaSuccess) e = launch(selective_backward_kernel<T, P>, a, a.segments, SelCfg<P, kSave>::BACK, seen[1], st);
  if (e != cudaSuccess) return e;
  if (c.length > 0) {
    const MapArgs m{a.gmaps, c.grad_B, c.grad_C, c.lengths, c.batch, c.length, a.groups, a.states, a.n4, a.blocks};
    const long long total = c.batch * c.length * a.groups * 2 * a.n4, ctas = (total + 255) / 256, most = (long long)num_sms() * 8;
    e = launch_pdl(selective_maps_kernel<T>, dim3((unsigned)(ctas < most ? ctas : most)), dim3(256), 0, st, m);
    if (e != cudaSuccess) return e;
  }
  if (c.grad_A == nullptr && c.grad_D == nullptr && c.grad_bias == nullptr) return cudaSuccess;
  return launch_sum_parts(a.gparams, (int)entries, c.channels * (c.states + 2),
                          {{c.grad_A, c.channels * c.states}, {c.grad_D, c.channels}, {c.grad_bias, c.channels}}, st);
}

template <typename T>
cudaError_t dispatch(const SelectiveCall& c, bool back, cudaStream_t st) {
  switch (lanes_of(c.states)) {
    case 4: return back ? backward_p<T, 4>(c, st) : forward_p<T, 4>(c, st);
    case 8: return back ? backward_p<T, 8>(c, st) : forward_p<T, 8>(c, st);
    default: return back ? backward_p<T, 16>(c, st) : forward_p<T, 16>(c, st);
  }
}

}  // namespace

long long selective_scratch_floats(const SelectiveCall& c, bool back) {
  const long long n4 = (c.states + 3) / 4 * 4;
  return cut_floats(c) + (back ? param_floats(c) + blocks_of(c) * c.batch * c.length * c.groups * 2 * n4 : 0);
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
