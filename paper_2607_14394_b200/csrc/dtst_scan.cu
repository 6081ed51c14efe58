// Gated linear recurrence along one dimension and its backward pass:
//     h_t = a_t h_{t-1} + u_t,     sigmoid gate: a = 1 / (1 + e^-g), u = (1 - a) v;     decay: a = g, u = v
//     delta_t = gh_t + a_{t+1} delta_{t+1}          (grad_last enters behind the last step)
//     sigmoid: gv = delta (1 - a), gg = delta (h_{t-1} - v) a (1 - a);   decay: gv = delta, gg = delta h_{t-1}
//     grad_h0 = a_0 delta_0
// A step is the affine map s -> a s + u; maps compose to (A, H) = (A2 A1, A2 H1 + H2), so a run of steps is summarised
// by two numbers and runs can be joined in any grouping.  A thread holds R consecutive steps in registers, composes
// them, learns the state in front of its run from the summaries of the runs before it, and then walks its steps once
// more.  Steps at and beyond a sequence's own length are the identity map, whatever stands there (the column kernels do not
// read them, the row kernels read and replace them).  States are fp32.
//
// Measured (forward, backward; sigmoid gate where none is named): fp32 [2621440][30] along contiguous steps 196 us, 272 us (4.8,
// 5.8 TB/s); fp32 [32][256][2079] 45, 89 (4.5, 3.8 TB/s), decay 46, 74 (4.4, 4.6); bf16 [1][65536][1024] 125, 264 (3.2, 2.5
// TB/s), bound by the rounds one behind the other; bf16 [6][4097][1000] 56, 105.
// Memory-bound: forward 2 tensors in, 1 out; backward 3 in, 2 out.  The backward pass does not read h: it rebuilds
// h_{t-1} inside each chunk, in fp32, from the state saved at the chunk's start.
#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_sm100.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

// Where there are few sequences, a thread-block cluster shares one: its CTAs take chunks side by side, exchange the chunks'
// summaries through distributed shared memory once per round, and each applies those of the chunks in front of its own to
// the state that all of them carry - in chunk order, so the bits are the same on every run and for every cluster size.
template <typename T>
struct ScanArgs {
  const T *v, *g, *gh;
  const float *h0, *g_last;
  const int* lengths;
  T *h, *gv, *gg;
  float *h_last, *gh0, *ckpt;
  long long outer, L, inner, groups, total;     // groups of VEC channels per outer entry, outer * groups
  long long in_o, in_t, gr_o, gr_t;
  long long chains;            // tiles side by side, `chunks` of them one behind the other
  int rounds;                  // ... taken a cluster's worth at a time
  unsigned per_outer;          // chains of an outer entry
  int chunks, sigmoid;
};

// a = 1 / (1 + e^-g) and b = 1 - a = e^-g / (1 + e^-g), both without cancellation.  The exponent is kept below 2^126 (a NaN
// stays one); the approximate exponential is good to about 2^-22, the rounding of g log2 e adds |g| 2^-24 or so to the smaller of
// the two (1e-6 at 20, 5e-6 at 80), and what it flushes to zero (g > 87) is below the smallest normal number.  a itself is
// right to 2^-25 where the gate is open (a Newton step of 1 / (1 + e): with gates around 8 the last of 5000 states is off
// by 1.6e-6, without it 1.0e-4; the forward pass over bf16 [65536][1024] takes 125 us, without it 122).  Two steps at once.
template <bool SIGMOID>
__device__ __forceinline__ void terms_pair(float2 g, float2& a, float2& b) {
  if (!SIGMOID) {
    a = g, b = make_float2(1.f, 1.f);
    return;
  }
  const float2 x = mul_pair(g, make_float2(-1.44269504f, -1.44269504f));      // -log2 e
  float2 e;           // 2^min(x, 126)
  asm("{\n\t.reg .f32 x;\n\tmin.NaN.f32 x, %1, 0f42FC0000;\n\tex2.approx.ftz.f32 %0, x;\n\t}" : "=f"(e.x) : "f"(x.x));
  asm("{\n\t.reg .f32 x;\n\tmin.NaN.f32 x, %1, 0f42FC0000;\n\tex2.approx.ftz.f32 %0, x;\n\t}" : "=f"(e.y) : "f"(x.y));
  const float2 d = add_pair(e, make_float2(1.f, 1.f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.x) : "f"(d.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.y) : "f"(d.y));
  b = mul_pair(e, a);
  // a + a (1 - a - b): the reciprocal's own error is of one sign, and a memory of thousands of steps would add it up
  const float2 minus = make_float2(-1.f, -1.f);
  a = fma_pair(a, fma_pair(b, minus, fma_pair(a, minus, make_float2(1.f, 1.f))), a);
}
// The state (or gradient) s behind a run of steps, A the product of their gates and H what they make of zero.  A decay may be
// larger than 1 and A infinite, which is no concern of a state of zero; a gate under a sigmoid is 1 at most.
template <bool SIGMOID>
__device__ __forceinline__ float through(float A, float s, float H) {
  const float r = fmaf(A, s, H);
  return !SIGMOID && s == 0.f ? H : r;
}
// d = a b and a b + c of N neighbouring channels (two at once took the forward pass over bf16 [65536][1024] from 126 us to 122 at
// the time: it is short of issue slots; the backward passes, which are not, gained nothing)
template <int N>
__device__ __forceinline__ void mul_n(float (&d)[N], const float (&a)[N], const float (&b)[N]) {
  if constexpr (N == 1) d[0] = a[0] * b[0];
#pragma unroll
  for (int j = 0; j + 1 < N; j += 2) {
    const float2 r = mul_pair(make_float2(a[j], a[j + 1]), make_float2(b[j], b[j + 1]));
    d[j] = r.x, d[j + 1] = r.y;
  }
}
template <int N>
__device__ __forceinline__ void fma_n(float (&d)[N], const float (&a)[N], const float (&b)[N], const float (&c)[N]) {
  if constexpr (N == 1) d[0] = fmaf(a[0], b[0], c[0]);
#pragma unroll
  for (int j = 0; j + 1 < N; j += 2) {
    const float2 r = fma_pair(make_float2(a[j], a[j + 1]), make_float2(b[j], b[j + 1]), make_float2(c[j], c[j + 1]));
    d[j] = r.x, d[j + 1] = r.y;
  }
}
// the gates of R x VEC steps in place: g becomes a, b is written
template <bool SIGMOID, int R, int VEC>
__device__ __forceinline__ void gates(float (&g)[R][VEC], float (&b)[R][VEC]) {
#pragma unroll
  for (int e = 0; e < R * VEC; e += 2) {
    float2 a2, b2;
    terms_pair<SIGMOID>(make_float2(g[e / VEC][e % VEC], g[(e + 1) / VEC][(e + 1) % VEC]), a2, b2);
    g[e / VEC][e % VEC] = a2.x, g[(e + 1) / VEC][(e + 1) % VEC] = a2.y;
    b[e / VEC][e % VEC] = b2.x, b[(e + 1) / VEC][(e + 1) % VEC] = b2.y;
  }
}
// the gate of a step that leaves the state alone (with v = 0): a = 1
template <typename T>
__device__ __forceinline__ T neutral_gate(int sigmoid) {
  return Elem<T>::put(sigmoid ? __int_as_float(0x7f800000) : 1.f);
}

__device__ __forceinline__ long long clamp_len(const int* lengths, long long o, long long L) {
  if (lengths == nullptr) return L;
  const long long n = lengths[o];
  return n < 0 ? 0 : (n < L ? n : L);
}

// ------------------------------------------------------------------------------------------------ columns
// [outer][L][inner], inner contiguous.  A tile is TX groups of VEC channels times SLOTS runs of R steps, a run per thread.
// Long sequences: the tiles of one outer entry lie side by side over its channels; a CTA (or a cluster) walks along L.
// Short ones (one tile holds them): groups run on across outer entries, so that few channels fill a CTA too.
// SIG and DEC: CTAs that share an SM, by gate.
template <int VEC_, int R_, int SLOTS_, int SIG = 2, int DEC = SIG>
struct ColShape {
  static constexpr int VEC = VEC_, R = R_, SLOTS = SLOTS_, THREADS = 256;
  static constexpr int ctas(bool sigmoid) { return sigmoid ? SIG : DEC; }
  static constexpr int TX = THREADS / SLOTS, W = TX * VEC, LC = SLOTS * R;
  // while runs are joined a warp has CPW channels, DG lanes each, and a lane has JOIN neighbouring runs of its channel
  static constexpr int WARPS = THREADS / 32, CPW = W / WARPS < 32 ? W / WARPS : 32, DG = 32 / CPW;
  static constexpr int JOIN = SLOTS >= DG ? SLOTS / DG : 1;
};
constexpr int kColTile = 256;     // steps of a long sequence's tile, and between saved states
enum ColMode { kOneTile = 0, kLong = 1 };

// joins (A, H) over the DG lanes of a channel, in lane order (UP) or against it; returns the summary of all of them and
// leaves in (A, H) that of the lanes before this one
template <int CPW, bool UP, bool SIGMOID>
__device__ __forceinline__ float2 join_lanes(float& A, float& H) {
  const int d = (threadIdx.x & 31) / CPW;
  constexpr int DG = 32 / CPW;
#pragma unroll
  for (int o = 1; o < DG; o *= 2) {
    const float A1 = UP ? __shfl_up_sync(0xffffffffu, A, o * CPW) : __shfl_down_sync(0xffffffffu, A, o * CPW);
    const float H1 = UP ? __shfl_up_sync(0xffffffffu, H, o * CPW) : __shfl_down_sync(0xffffffffu, H, o * CPW);
    if (UP ? d >= o : d + o < DG) H = through<SIGMOID>(A, H1, H), A *= A1;
  }
  const int ch = (threadIdx.x & 31) % CPW, last = UP ? (DG - 1) * CPW + ch : ch;
  const float2 all = make_float2(__shfl_sync(0xffffffffu, A, last), __shfl_sync(0xffffffffu, H, last));
  if constexpr (DG > 1) {
    A = UP ? __shfl_up_sync(0xffffffffu, A, CPW) : __shfl_down_sync(0xffffffffu, A, CPW);
    H = UP ? __shfl_up_sync(0xffffffffu, H, CPW) : __shfl_down_sync(0xffffffffu, H, CPW);
  }
  if (UP ? d == 0 : d == DG - 1) A = 1.f, H = 0.f;
  return all;
}

// The coming tile on its way through shared memory: a thread copies and reads its own steps, element group by element group, so
// no barrier stands between the copies and their use.  (Rows of the tile as 16-byte copies shared among the threads, two tiles
// under way, took 0.6 % less for a forward pass over bf16 [1][65536][1024] and 2 to 6 % more in every other pass measured:
// bf16 [6][4097][1000], when these took 53.2 us forward and 99 backward, 56.4 and 105.)
template <typename T, class S, int TENSORS>
struct ColSlots {
  static constexpr int VEC = S::VEC, R = S::R, BYTES = VEC * (int)sizeof(T);
  static constexpr bool ASYNC = BYTES >= 4;      // (cp.async moves 4, 8 or 16 bytes)
  static constexpr size_t TENSOR = (size_t)R * S::THREADS * BYTES, SMEM = TENSORS * TENSOR;
  using P = Pack<T, VEC>;
  unsigned char* base;
  __device__ __forceinline__ P* slot(int tensor, int r) const {
    return reinterpret_cast<P*>(base + tensor * TENSOR + ((size_t)r * S::THREADS + threadIdx.x) * BYTES);
  }
  static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
  // this thread's own steps from src on; `none` where there are fewer than R
  __device__ __forceinline__ void fetch(int tensor, const T* src, long long stride, int have, T none) const {
#pragma unroll
    for (int r = 0; r < R; ++r, src += stride) {
      P* d = slot(tensor, r);
      if (r >= have) {
        P n;
        n.fill(none);
        *d = n;
      } else if constexpr (ASYNC) {
        const uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(d));
        if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(src) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(src), "n"(BYTES) : "memory");
      } else {
        d->load(src);
      }
    }
  }
};

// A group of a tile: its outer entry, first channel and steps (0: no such group)
struct ColGroup {
  long long o;
  int i0, end;
  bool live;
};
// group x of tile `tile`
template <typename T, class S, int MODE>
__device__ __forceinline__ ColGroup col_group(const ScanArgs<T>& p, unsigned tile, int x) {
  ColGroup g;
  if (MODE == kOneTile) {
    const long long gid = (long long)tile * S::TX + x;
    g.live = gid < p.total;
    g.o = g.live ? (p.total <= 0xffffffffll ? (long long)((unsigned)gid / (unsigned)p.groups) : gid / p.groups) : 0;
    g.i0 = g.live ? (int)(gid - g.o * p.groups) * S::VEC : 0;
  } else {
    g.o = tile / p.per_outer;
    const long long at = (long long)(tile - (unsigned)g.o * p.per_outer) * S::TX + x;
    g.live = at < p.groups;
    g.i0 = g.live ? (int)at * S::VEC : 0;
  }
  g.end = g.live ? (int)clamp_len(p.lengths, g.o, p.L) : 0;
  return g;
}

// the tile's rows from `dst` on, as far as there are any, become zero
template <typename T, class S>
__device__ __forceinline__ void zero_rows(T* dst, long long stride, int left, int slot) {
  Pack<T, S::VEC> z;
  z.zero();
  dst += (long long)slot * S::R * stride;
#pragma unroll
  for (int r = 0; r < S::R; ++r, dst += stride)
    if (slot * S::R + r < left) z.store(dst);
}

// set if a wait for another CTA's summaries ever runs out (dtst_gated_scan_status)
__device__ int scan_status_word;
constexpr uint32_t kRoundPolls = 1u << 20;

// Where the CTAs of a cluster leave their chunks' summaries for each other: a box for every CTA, two sets used in turn (a CTA
// sends its next round's only when it has everybody's of this one, so the set of the round before is free again).
template <class S>
struct RoundBoxes {
  float2 box[2][8][S::W];
  uint64_t bar[2];
};

// What the runs of a tile leave for each other, a number per run and channel.  A thread writes and reads VEC neighbouring
// channels of its run at once.  While runs are joined a lane goes through the JOIN runs of its depth group; a gap of SKEW
// floats behind each such set of rows puts the lanes of different depth groups in different banks (without the gaps and with
// 8-byte pairs, half of all wavefronts of the passes over bf16 [65536][1024] were conflicts).
template <class S>
struct RunRows {
  static constexpr int SKEW = S::CPW < S::VEC ? S::VEC : S::CPW;
  __align__(16) float f[S::SLOTS > 1 ? S::SLOTS * S::W + S::SLOTS / S::JOIN * SKEW : 1];
  __device__ __forceinline__ float* at(int run, int ch) { return f + run * S::W + run / S::JOIN * SKEW + ch; }
  __device__ __forceinline__ void put(int run, int ch, const float (&v)[S::VEC]) {
    if constexpr (S::VEC == 4) *reinterpret_cast<float4*>(at(run, ch)) = make_float4(v[0], v[1], v[2], v[3]);
    else *at(run, ch) = v[0];
  }
  __device__ __forceinline__ void get(int run, int ch, float (&v)[S::VEC]) {
    if constexpr (S::VEC == 4) {
      const float4 q = *reinterpret_cast<const float4*>(at(run, ch));
      v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
      v[0] = *at(run, ch);
    }
  }
};

// One round: every CTA sends its chunk's summary `all` to the others (st.async: the bytes are counted by the receiver's
// mbarrier; no cluster barrier, no fence).  Its latency is what a round cannot hide: when the pass over bf16 [65536][1024], 32
// rounds of it, took 136 us, a copy of the kernel without the exchange took 100.  Returns the state in front of this CTA's chunk and moves `state` past
// the round.  A lane of depth group d sends to and reads the box of CTA d.
template <class S, bool SIGMOID>
__device__ __forceinline__ float join_round(const float2 all, float& state, RoundBoxes<S>& b, int round, int size, int rank, int jx,
                                            bool& dead) {
  static_assert(S::DG >= 8, "a depth group per CTA of the largest cluster");
  if (size == 1) {
    const float start = state;
    state = through<SIGMOID>(all.x, state, all.y);
    return start;
  }
  const int lane = threadIdx.x & 31, d = lane / S::CPW, ch = lane % S::CPW, set = round & 1;
  if (threadIdx.x == 0 && !dead) sm100::mbar_arrive_expect_tx(&b.bar[set], (uint32_t)(size - 1) * S::W * 8u);
  if (d < size && d != rank) {
    uint32_t to, bar;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(sm100::smem_u32(&b.box[set][rank][jx])), "r"(d));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(sm100::smem_u32(&b.bar[set])), "r"(d));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(to), "f"(all.x),
                 "f"(all.y), "r"(bar)
                 : "memory");
  }
  bool here = dead;
  for (uint32_t poll = 0; poll < kRoundPolls && !here; ++poll) here = sm100::mbar_try_wait(&b.bar[set], (uint32_t)(round >> 1) & 1u);
  if (!here) {
    dead = true;             // the results are undefined; later rounds do not wait again
    atomicExch(&scan_status_word, 1);
  }
  __syncwarp();
  float2 m = make_float2(1.f, 0.f);
  if (d == rank) m = all;
  else if (d < size) m = b.box[set][d][jx];
  float start = 0.f;
  for (int k = 0; k < size; ++k) {
    if (k == rank) start = state;
    state = through<SIGMOID>(__shfl_sync(0xffffffffu, m.x, k * S::CPW + ch), state, __shfl_sync(0xffffffffu, m.y, k * S::CPW + ch));
  }
  return start;
}

// No CTA leaves while summaries may be on their way to it.  A CTA whose waits all ended well has everybody's; one that gave up
// stays until the others have sent theirs, and for a bounded while until they have arrived.
template <class S>
__device__ __forceinline__ void leave_rounds(RoundBoxes<S>& b, int rounds, bool dead) {
  __syncwarp();
  // (relaxed: nothing is handed over, and a release would wait for the last round's stores, 2 us)
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
  const int last = rounds - 1;
  for (uint32_t poll = 0; dead && poll < 4096u && !sm100::mbar_try_wait(&b.bar[last & 1], (uint32_t)(last >> 1) & 1u); ++poll) {
  }
}

template <typename T, class S, int MODE, bool SIGMOID>
__global__ void __launch_bounds__(S::THREADS, S::ctas(SIGMOID)) scan_cols_kernel(const ScanArgs<T> p) {
  constexpr int VEC = S::VEC, R = S::R, SLOTS = S::SLOTS, W = S::W, LC = S::LC;
  using Slots = ColSlots<T, S, 2>;
  __shared__ RunRows<S> runs_a, runs_h;     // (A, H) of every run; then, in runs_a, the state in front of it
  __shared__ RoundBoxes<S> boxes;
  bool dead = false;
  extern __shared__ __align__(16) unsigned char raw[];
  Slots slots{raw};
  pdl_trigger();
  pdl_wait();
  const int size = MODE == kLong ? cluster_size() : 1, rank = MODE == kLong ? cluster_rank() : 0;
  const unsigned tile = blockIdx.x / size;
  const int slot = threadIdx.x / S::TX, x = threadIdx.x % S::TX;
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(SIGMOID);
  const long long states = p.outer * p.inner;
  const int lane = threadIdx.x & 31;
  const int jx = (threadIdx.x / 32) * S::CPW + lane % S::CPW, jq = lane / S::CPW * S::JOIN;   // while joining: channel, first run
  const bool first = lane < S::CPW;
  const ColGroup at = col_group<T, S, MODE>(p, tile, x), jg = col_group<T, S, MODE>(p, tile, jx / VEC);
  const long long ch = jg.o * p.inner + jg.i0 + jx % VEC;
  // the steps of a long sequence
  const int e_tile = MODE == kLong ? (int)clamp_len(p.lengths, at.o, p.L) : 0;
  auto fetch = [&](int c) {
    const int t0 = c * LC + slot * R;
    const long long from = at.o * p.in_o + at.i0 + t0 * p.in_t;
    slots.fetch(0, p.v + from, p.in_t, at.end - t0, none_v);
    slots.fetch(1, p.g + from, p.in_t, at.end - t0, none_g);
    Slots::commit();
  };
  fetch(rank);
  float state = SLOTS > 1 && jg.live && p.h0 != nullptr ? p.h0[ch] : 0.f;
  if (size > 1) {
    if (threadIdx.x == 0) {
      sm100::mbar_init(&boxes.bar[0], 1);
      sm100::mbar_init(&boxes.bar[1], 1);
      sm100::fence_barrier_init();
    }
    cluster_sync();        // also: every CTA has read its h0, whose place h_last may take
  }

#pragma unroll 1
  for (int round = 0; round < p.rounds; ++round) {
    const int c = round * size + rank;
    auto refill = [&]() {      // the values of the next chunk are on their way from here on
      if (round + 1 < p.rounds) fetch(c + size);
    };
    if constexpr (MODE == kLong) if (c * LC >= e_tile) {       // no step of the sequence here: the state passes, h is zero
      float start = state;
      start = join_round<S, SIGMOID>(make_float2(1.f, 0.f), state, boxes, round, size, rank, jx, dead);
      if (c == 0 && first && jg.live && p.h_last != nullptr) p.h_last[ch] = start;
      zero_rows<T, S>(p.h + (at.o * p.L + c * LC) * p.inner + at.i0, p.inner, at.live ? (int)p.L - c * LC : 0, slot);
      refill();
      continue;
    }
    float a[R][VEC], u[R][VEC], s[VEC];
    Slots::wait();
    Pack<T, VEC> pv[R], pg[R];
#pragma unroll
    for (int r = 0; r < R; ++r) pv[r] = *slots.slot(0, r), pg[r] = *slots.slot(1, r);
    if (MODE == kLong) refill();
#pragma unroll
    for (int r = 0; r < R; ++r) pg[r].unpack(a[r]);
    gates<SIGMOID, R, VEC>(a, u);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float v[VEC];
      pv[r].unpack(v);
      mul_n<VEC>(u[r], u[r], v);
    }
    if constexpr (SLOTS == 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = at.live && p.h0 != nullptr ? p.h0[at.o * p.inner + at.i0 + j] : 0.f;
    } else {
      float ra[VEC], rh[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) ra[j] = a[0][j], rh[j] = SIGMOID ? u[0][j] : fmaf(a[0][j], 0.f, u[0][j]);   // (a gate of NaN counts)
#pragma unroll
      for (int r = 1; r < R; ++r) {
        mul_n<VEC>(ra, ra, a[r]);
        fma_n<VEC>(rh, a[r], rh, u[r]);
      }
      runs_a.put(slot, x * VEC, ra);
      runs_h.put(slot, x * VEC, rh);
      __syncthreads();
      float A = 1.f, H = 0.f;
      float2 m[S::JOIN];
#pragma unroll
      for (int q = 0; q < S::JOIN; ++q) {
        m[q] = make_float2(*runs_a.at(jq + q, jx), *runs_h.at(jq + q, jx));
        A *= m[q].x;
        H = through<SIGMOID>(m[q].x, H, m[q].y);
      }
      const float2 all = join_lanes<S::CPW, true, SIGMOID>(A, H);
      float start = state;
      if constexpr (MODE == kLong) start = join_round<S, SIGMOID>(all, state, boxes, round, size, rank, jx, dead);
      else state = through<SIGMOID>(all.x, state, all.y);
      float run = through<SIGMOID>(A, start, H);
      // (a chunk in which a sequence has no step leaves its state alone)
      const bool active = c * LC < jg.end, more = (c + 1) * (long long)LC < jg.end;
      if (first && jg.live && (active || c == 0)) {
        if (MODE == kLong && p.ckpt != nullptr) p.ckpt[c * states + ch] = start;
        if (!more && p.h_last != nullptr) p.h_last[ch] = through<SIGMOID>(all.x, start, all.y);
      }
#pragma unroll
      for (int q = 0; q < S::JOIN; ++q) {
        *runs_a.at(jq + q, jx) = run;
        run = through<SIGMOID>(m[q].x, run, m[q].y);
      }
      __syncthreads();
      runs_a.get(slot, x * VEC, s);
    }
    const int t0 = c * LC + slot * R, left = at.live ? (int)p.L - t0 : 0;
    T* h = p.h + (at.o * p.L + t0) * p.inner + at.i0;
#pragma unroll
    for (int r = 0; r < R; ++r, h += p.inner) {
      fma_n<VEC>(s, a[r], s, u[r]);
      Pack<T, VEC> out;
      out.pack(s);
      if (t0 + r >= at.end) out.zero();
      if (r < left) out.store(h);
    }
    if constexpr (SLOTS == 1) {
      if (at.live && p.h_last != nullptr) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.h_last[at.o * p.inner + at.i0 + j] = s[j];
      }
    }
    if (MODE == kOneTile) return;
    __syncthreads();       // the runs' states are read before the next chunk's summaries replace them
  }
  if (size > 1) leave_rounds<S>(boxes, p.rounds, dead);
}

template <typename T, class S, int MODE, bool SIGMOID>
__global__ void __launch_bounds__(S::THREADS, S::ctas(SIGMOID)) scan_cols_backward_kernel(const ScanArgs<T> p) {
  constexpr int VEC = S::VEC, R = S::R, SLOTS = S::SLOTS, W = S::W, LC = S::LC;
  using Slots = ColSlots<T, S, 3>;
  // (A, H) and D of every run; then the state in front of it (runs_a) and the gradient that comes to it from behind (backs)
  __shared__ RunRows<S> runs_a, runs_h, backs;
  __shared__ RoundBoxes<S> boxes;
  bool dead = false;
  extern __shared__ __align__(16) unsigned char raw[];
  Slots slots{raw};
  pdl_trigger();
  pdl_wait();
  const int size = MODE == kLong ? cluster_size() : 1, rank = MODE == kLong ? cluster_rank() : 0;
  const unsigned tile = blockIdx.x / size;
  if (size > 1) {
    if (threadIdx.x == 0) {
      sm100::mbar_init(&boxes.bar[0], 1);
      sm100::mbar_init(&boxes.bar[1], 1);
      sm100::fence_barrier_init();
    }
    cluster_sync();
  }
  const int slot = threadIdx.x / S::TX, x = threadIdx.x % S::TX;
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(SIGMOID);
  const long long states = p.outer * p.inner;
  const int lane = threadIdx.x & 31;
  const int jx = (threadIdx.x / 32) * S::CPW + lane % S::CPW, jq = lane / S::CPW * S::JOIN;   // while joining: channel, first run
  const bool first = lane < S::CPW;
  const ColGroup at = col_group<T, S, MODE>(p, tile, x), jg = col_group<T, S, MODE>(p, tile, jx / VEC);
  const long long ch = jg.o * p.inner + jg.i0 + jx % VEC;
  // the steps of a long sequence
  const int e_tile = MODE == kLong ? (int)clamp_len(p.lengths, at.o, p.L) : 0;
  // chunks from the last to the first; a chunk before the first has no steps
  auto fetch = [&](int c) {
    const int t0 = c * LC + slot * R, end = c < 0 ? t0 : at.end;
    const long long from = at.o * p.in_o + at.i0 + t0 * p.in_t;
    slots.fetch(0, p.v + from, p.in_t, end - t0, none_v);
    slots.fetch(1, p.g + from, p.in_t, end - t0, none_g);
    slots.fetch(2, p.gh + (at.o * p.L + t0) * p.inner + at.i0, p.inner, end - t0, none_v);
    Slots::commit();
  };
  fetch(p.chunks - 1 - rank);
  float grad = SLOTS > 1 && jg.live && p.g_last != nullptr ? p.g_last[ch] : 0.f;

#pragma unroll 1
  for (int round = 0; round < p.rounds; ++round) {
    const int c = p.chunks - 1 - (round * size + rank);
    auto refill = [&]() {      // the values of the next chunk are on their way from here on
      if (round + 1 < p.rounds) fetch(c - size);
    };
    if constexpr (MODE == kLong) if (c < 0 || c * LC >= e_tile) {       // no step of the sequence here
      const float behind = join_round<S, SIGMOID>(make_float2(1.f, 0.f), grad, boxes, round, size, rank, jx, dead);
      if (c == 0 && jg.live && first && p.gh0 != nullptr) p.gh0[ch] = behind;
      if (c >= 0) {
        const long long from = at.o * p.gr_o + at.i0 + (long long)c * LC * p.gr_t;
        zero_rows<T, S>(p.gv + from, p.gr_t, at.live ? (int)p.L - c * LC : 0, slot);
        zero_rows<T, S>(p.gg + from, p.gr_t, at.live ? (int)p.L - c * LC : 0, slot);
      }
      Slots::wait();         // (there is nothing in it)
      refill();
      continue;
    }
    float before = 0.f;      // the state in front of the chunk: saved, or the sequence's own beginning
    if (SLOTS > 1 && jg.live && c >= 0 && (c * LC < jg.end || c == 0)) {
      if (MODE == kLong && p.ckpt != nullptr) before = p.ckpt[c * states + ch];
      else if (p.h0 != nullptr) before = p.h0[ch];
    }
    Slots::wait();
    // a and b = 1 - a, both kept: either formed from the other would lose its bits where it is small
    float a[R][VEC], b[R][VEC], v[R][VEC], s[VEC], d[VEC];
    Pack<T, VEC> pd[R];
    Pack<T, VEC> pv[R], pg[R];
#pragma unroll
    for (int r = 0; r < R; ++r) pv[r] = *slots.slot(0, r), pg[r] = *slots.slot(1, r), pd[r] = *slots.slot(2, r);
    if (MODE == kLong) refill();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      pg[r].unpack(a[r]);
      pv[r].unpack(v[r]);
    }
    gates<SIGMOID, R, VEC>(a, b);
    if constexpr (SLOTS == 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        s[j] = at.live && p.h0 != nullptr ? p.h0[at.o * p.inner + at.i0 + j] : 0.f;
        d[j] = at.live && p.g_last != nullptr ? p.g_last[at.o * p.inner + at.i0 + j] : 0.f;
      }
    } else {
      float ra[VEC], rh[VEC], D[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        ra[j] = 1.f, rh[j] = D[j] = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          ra[j] *= a[r][j];
          rh[j] = fmaf(a[r][j], rh[j], b[r][j] * v[r][j]);
        }
      }
      runs_a.put(slot, x * VEC, ra);
      runs_h.put(slot, x * VEC, rh);
#pragma unroll
      for (int r = R - 1; r >= 0; --r) {
        float gh[VEC];
        pd[r].unpack(gh);
#pragma unroll
        for (int j = 0; j < VEC; ++j) D[j] = a[r][j] * (D[j] + gh[j]);
      }
      backs.put(slot, x * VEC, D);
      __syncthreads();
      float A = 1.f, H = 0.f, B = 1.f, E = 0.f;
      float2 m[S::JOIN];
      float md[S::JOIN];
#pragma unroll
      for (int k = 0; k < S::JOIN; ++k) {
        m[k] = make_float2(*runs_a.at(jq + k, jx), *runs_h.at(jq + k, jx));
        md[k] = *backs.at(jq + k, jx);
        A *= m[k].x;
        H = through<SIGMOID>(m[k].x, H, m[k].y);
      }
#pragma unroll
      for (int k = S::JOIN - 1; k >= 0; --k) E = through<SIGMOID>(m[k].x, E, md[k]);
      B = A;
      join_lanes<S::CPW, true, SIGMOID>(A, H);
      const float2 all = join_lanes<S::CPW, false, SIGMOID>(B, E);
      float behind = grad;
      if constexpr (MODE == kLong) behind = join_round<S, SIGMOID>(all, grad, boxes, round, size, rank, jx, dead);
      if (c == 0 && jg.live && first && p.gh0 != nullptr) p.gh0[ch] = through<SIGMOID>(all.x, behind, all.y);
      float run = through<SIGMOID>(A, before, H);
#pragma unroll
      for (int k = 0; k < S::JOIN; ++k) {
        *runs_a.at(jq + k, jx) = run;
        run = through<SIGMOID>(m[k].x, run, m[k].y);
      }
      run = through<SIGMOID>(B, behind, E);
#pragma unroll
      for (int k = S::JOIN - 1; k >= 0; --k) {
        *backs.at(jq + k, jx) = run;
        run = through<SIGMOID>(m[k].x, run, md[k]);
      }
      __syncthreads();
      runs_a.get(slot, x * VEC, s);
      backs.get(slot, x * VEC, d);
    }
    // forward once more: v is replaced by what delta is multiplied with for the gate's gradient
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float u = b[r][j] * v[r][j];
        v[r][j] = SIGMOID ? (s[j] - v[r][j]) * (a[r][j] * b[r][j]) : s[j];
        s[j] = fmaf(a[r][j], s[j], u);
      }
    const int t0 = c * LC + slot * R, left = at.live && c >= 0 ? (int)p.L - t0 : 0;
    const long long back = at.o * p.gr_o + at.i0 + (t0 + R - 1) * p.gr_t;
    T *gv = p.gv + back, *gg = p.gg + back;
#pragma unroll
    for (int r = R - 1; r >= 0; --r, gv -= p.gr_t, gg -= p.gr_t) {
      float x1[VEC], x2[VEC];
      pd[r].unpack(x1);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float delta = d[j] + x1[j];
        x1[j] = delta * b[r][j];
        x2[j] = delta * v[r][j];
        d[j] = a[r][j] * delta;
      }
      Pack<T, VEC> ov, og;
      ov.pack(x1);
      og.pack(x2);
      if (t0 + r >= at.end) ov.zero(), og.zero();
      if (r < left) {
        ov.store(gv);
        og.store(gg);
      }
    }
    if constexpr (SLOTS == 1) {
      if (at.live && p.gh0 != nullptr) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.gh0[at.o * p.inner + at.i0 + j] = d[j];
      }
    }
    if (MODE == kOneTile) return;
    __syncthreads();
  }
  if (size > 1) leave_rounds<S>(boxes, p.rounds, dead);
}

// ------------------------------------------------------------------------------------------------ rows
// [outer][L], the steps contiguous, L >= 8.  A warp takes a unit of at most 512 neighbouring elements - whole rows, or a
// chunk of a long one - in vectors of 8 (32 or 16 bytes) straight from global memory: K vectors a lane, the k-th at
// (32 k + lane) 8.  Each vector is composed in its lane, the lanes are joined by a warp scan that does not reach across a row's first step
// (forward) or last step (backward), and the K scans are joined one after the other.  No shared memory, no barriers.
// Where rows begin off a vector the unit starts at the vector before; the elements in front are left alone.
// fp32 [2097152][32]: 154 us forward, 213 backward; in tensors that begin off a vector, element by element, 328 and 867 (whole
// rows by elements do not fit 128 registers and spill: up to 208 bytes forward, 716 backward).  fp32 [1900000][7], which the
// columns' kernels take: 44 and 107 us; [1900000][8] here 37 and 51.
constexpr int kUnit = 512, kRowWarps = 8;

// steps of a chunk (a chunk of odd rows leaves room for a shifted beginning)
__host__ __device__ constexpr int row_chunk(long long L) { return L % 8 == 0 ? kUnit : kUnit - 8; }

enum RowMode { kWholeRows = 0, kWalk = 1, kTeam = 2 };

// Vector k of a unit: its first element's index (below 0 in front of the unit) and step, and the element that is a row's
// first step (V: none; at most one, since L >= V).
template <int V>
struct RowVec {
  int rel, t, spos;
};

template <typename T, bool WIDE, int MODE, bool RAGGED>
struct RowUnit {
  static constexpr int V = 8, K = kUnit / 32 / V;
  using Vec = RowVec<V>;
  long long row0;       // first row
  int n, t0, shift;     // elements; step of the first one; elements of its vector in front of it
  int L, span;          // lanes that a row may reach across
  uint32_t magic;       // division by L (whole rows: L <= 512, elements < 1024)
  __device__ __forceinline__ Vec vec(int k, int& row) const {
    Vec v;
    v.rel = (k * 32 + (int)(threadIdx.x & 31)) * V - shift;
    v.spos = V;
    v.t = t0 + v.rel;
    row = 0;
    if (MODE == kWholeRows) {
      row = v.rel > 0 ? (int)__umulhi((uint32_t)v.rel, magic) : 0;
      v.t = v.rel - row * L;
      const int s = v.t <= 0 ? -v.t : L - v.t;     // (it may lie behind the unit; nothing in the unit comes after it then)
      if (s < V) v.spos = s;
    }
    return v;
  }
  // whether the last step of the vector's first row lies in the vector and in the unit
  __device__ __forceinline__ bool ends(const Vec& v) const {
    return MODE == kWholeRows && v.t >= 0 && L - v.t <= V && v.rel + (L - v.t) <= n;
  }
  __device__ __forceinline__ bool starts(const Vec& v) const { return MODE == kWholeRows && v.spos < V && v.rel + v.spos < n; }
  __device__ __forceinline__ bool full(const Vec& v) const { return v.rel >= 0 && v.rel + V <= n; }
  __device__ __forceinline__ bool on(const Vec& v, int i) const { return v.rel + i >= 0 && v.rel + i < n; }
  // the vector's elements of a tensor whose unit begins at `base`; elements outside the unit become `none`.  Not WIDE: rows
  // lie `stride` apart and vectors are loaded one by one.
  __device__ __forceinline__ void load(Pack<T, V>& r, const Vec& v, int row, const T* base, long long stride, T none) const {
    if (WIDE && full(v)) {
      r.load(base + v.rel);
      return;
    }
    r.fill(none);
    if (v.rel >= n) return;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (on(v, i)) r.v[i] = base[WIDE ? v.rel + i : offset(v, row, i, stride)];
  }
  __device__ __forceinline__ void store(const Pack<T, V>& r, const Vec& v, int row, T* base, long long stride) const {
    if (WIDE && full(v)) {
      r.store(base + v.rel);
      return;
    }
    if (v.rel >= n) return;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (on(v, i)) base[WIDE ? v.rel + i : offset(v, row, i, stride)] = r.v[i];
  }
  __device__ __forceinline__ long long offset(const Vec& v, int row, int i, long long stride) const {
    if (MODE != kWholeRows) return v.rel + i;
    const bool next = v.t + i >= L;
    return (row + (next ? 1 : 0)) * stride + (v.t + i - (next ? L : 0));
  }
  // RAGGED: which elements are steps of their sequences, as bits
  __device__ __forceinline__ uint32_t steps(const Vec& v, int row, const int* lengths, long long end) const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) m |= on(v, i) ? 1u << i : 0u;
    if (m == 0) return 0;
    long long e0 = end, e1 = 0;
    if (MODE == kWholeRows) e0 = lengths[row0 + row], e1 = v.t > 0 && starts(v) ? lengths[row0 + row + 1] : 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool next = MODE == kWholeRows && v.t + i >= L;
      if (next ? v.t + i - L >= e1 : v.t + i >= e0) m &= ~(1u << i);
    }
    return m;
  }
};

// Joins the lanes of one scan in which lanes of `marks` hold a summary that starts afresh: (A, H) of a lane becomes that of
// all lanes from the nearest mark up to it.  No summary reaches across `span` lanes or more.
template <bool UP, bool SIGMOID>
__device__ __forceinline__ bool segmented_scan(float& A, float& H, unsigned marks, int span) {
  const int lane = threadIdx.x & 31;
  const unsigned seen = UP ? marks & (0xffffffffu >> (31 - lane)) : marks & (0xffffffffu << lane);
  const bool fresh = seen != 0;
  const int room = UP ? (fresh ? lane - 31 + __clz(seen) : lane) : (fresh ? __ffs(seen) - 1 - lane : 31 - lane);
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    if (o >= span) break;
    const float A1 = UP ? __shfl_up_sync(0xffffffffu, A, o) : __shfl_down_sync(0xffffffffu, A, o);
    const float H1 = UP ? __shfl_up_sync(0xffffffffu, H, o) : __shfl_down_sync(0xffffffffu, H, o);
    if (o <= room) H = through<SIGMOID>(A, H1, H), A *= A1;
  }
  return fresh;
}

// the first unit of this warp; false if there is none.  A team (the warps of a cluster) shares a row: `me` of `members`.
template <class U, typename T, int MODE>
__device__ __forceinline__ bool first_unit(const ScanArgs<T>& p, U& u, int& me, int& members) {
  const int warp = threadIdx.x >> 5;
  const long long id = (long long)blockIdx.x * kRowWarps + warp;
  u.L = (int)p.L;
  u.magic = 0xffffffffu / (uint32_t)p.L + 1u;
  u.span = MODE == kWholeRows ? (u.L + U::V - 2) / U::V + 1 : 32;
  me = 0, members = 1;
  if (MODE == kWholeRows) {
    u.row0 = id * p.groups;                       // groups: rows of a unit
    if (u.row0 >= p.outer) return false;
    u.n = (int)((p.outer - u.row0 < p.groups ? p.outer - u.row0 : p.groups) * p.L);
    u.t0 = 0;
  } else if (MODE == kWalk) {
    if (id >= p.outer) return false;
    u.row0 = id;
  } else {
    const int size = cluster_size();
    me = cluster_rank() * kRowWarps + warp, members = size * kRowWarps;
    u.row0 = blockIdx.x / size;
  }
  return true;
}
// One round of a team: as join_round, a lane per member (at most 32).
template <bool SIGMOID>
__device__ __forceinline__ float join_team(const float2 all, float& state, float2 (*box)[kRowWarps], int round, int me, int members) {
  const int lane = threadIdx.x & 31;
  float2* mine = box[round & 1];
  if (lane == 0) mine[threadIdx.x >> 5] = all;
  if (members > kRowWarps) cluster_sync(); else __syncthreads();
  float A = 1.f, H = 0.f;
  if (lane < members) {
    const float2 m = members > kRowWarps ? cluster_read(mine + lane % kRowWarps, lane / kRowWarps) : mine[lane];
    A = m.x, H = m.y;
  }
  segmented_scan<true, SIGMOID>(A, H, 0u, 32);
  const float s = through<SIGMOID>(A, state, H);   // behind member `lane`
  const float start = me == 0 ? state : __shfl_sync(0xffffffffu, s, me > 0 ? me - 1 : 0);
  state = __shfl_sync(0xffffffffu, s, 31);
  return start;
}
template <class U, typename T, int MODE>
__device__ __forceinline__ void place_unit(const ScanArgs<T>& p, U& u, int c) {
  if (MODE != kWholeRows) {
    const int step = row_chunk(p.L);
    u.t0 = c * step;
    u.n = c < 0 || u.t0 >= p.L ? 0 : (int)(p.L - u.t0 < step ? p.L - u.t0 : step);     // (no chunk there: no elements)
    if (u.n == 0) u.t0 = 0;
  }
  // rows that begin off a vector: only contiguous tensors are read wide then, all with the same shift
  u.shift = p.L % U::V == 0 ? 0 : (int)((u.row0 * p.L + u.t0) % U::V);
}
template <typename T, bool WIDE, int MODE, bool RAGGED, bool SIGMOID>
__global__ void __launch_bounds__(32 * kRowWarps, 2) scan_rows_kernel(const ScanArgs<T> p) {
  using U = RowUnit<T, WIDE, MODE, RAGGED>;
  constexpr int V = U::V, K = U::K;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  __shared__ float2 box[2][kRowWarps];
  U u;
  int me, members;
  if (!first_unit<U, T, MODE>(p, u, me, members)) return;
  const long long end = MODE == kWholeRows ? p.L : clamp_len(p.lengths, u.row0, p.L);
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(SIGMOID);
  float carry = 0.f;
  if (MODE != kWholeRows && p.h0 != nullptr) carry = p.h0[u.row0];
#pragma unroll 1
  for (int round = 0; round < p.rounds; ++round) {
    const int c = round * members + me;
    place_unit<U, T, MODE>(p, u, c);
    typename U::Vec x[K];
    int row[K];
    Pack<T, V> pv[K], pg[K];
    float h0v[K];
    uint32_t live[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      x[k] = u.vec(k, row[k]);
      u.load(pv[k], x[k], row[k], p.v + u.row0 * p.in_o + u.t0, p.in_o, none_v);
      u.load(pg[k], x[k], row[k], p.g + u.row0 * p.in_o + u.t0, p.in_o, none_g);
      h0v[k] = 0.f;
      if (u.starts(x[k]) && p.h0 != nullptr) h0v[k] = p.h0[u.row0 + row[k] + (x[k].t > 0 ? 1 : 0)];
      if (RAGGED) live[k] = u.steps(x[k], row[k], p.lengths, end);
    }
    float a[K][V], b[K][V], A[K], H[K];
    bool fresh[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      A[k] = 1.f, H[k] = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (RAGGED && !(live[k] >> i & 1u)) pv[k].v[i] = none_v, pg[k].v[i] = none_g;
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        float2 a2, b2;
        terms_pair<SIGMOID>(make_float2(pg[k].get(i), pg[k].get(i + 1)), a2, b2);
        b2 = mul_pair(b2, make_float2(pv[k].get(i), pv[k].get(i + 1)));
        a[k][i] = a2.x, a[k][i + 1] = a2.y, b[k][i] = b2.x, b[k][i + 1] = b2.y;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (MODE == kWholeRows && i == x[k].spos) H[k] = h0v[k];
        A[k] *= a[k][i];
        H[k] = fmaf(a[k][i], H[k], b[k][i]);
      }
      fresh[k] = segmented_scan<true, SIGMOID>(A[k], H[k], MODE == kWholeRows ? __ballot_sync(0xffffffffu, x[k].spos < V) : 0u, u.span);
    }
    const bool active = MODE == kWholeRows || (u.n > 0 && u.t0 < end), more = MODE != kWholeRows && u.t0 + u.n < end;
    const long long at = (long long)c * p.outer + u.row0;
    float after = 0.f;            // the state that the team carries on
    if (MODE == kTeam) {          // the whole chunk's summary, the vectors joined in order
      float tA = 1.f, tH = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const float A1 = __shfl_sync(0xffffffffu, A[k], 31), H1 = __shfl_sync(0xffffffffu, H[k], 31);
        tH = through<SIGMOID>(A1, tH, H1), tA *= A1;
      }
      after = carry;
      carry = join_team<SIGMOID>(make_float2(tA, tH), after, box, round, me, members);
    }
    if (MODE != kWholeRows && p.ckpt != nullptr && lane == 0 && (active || c == 0)) p.ckpt[at] = carry;
    float in[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const float s = fresh[k] ? H[k] : through<SIGMOID>(A[k], carry, H[k]);
      in[k] = __shfl_up_sync(0xffffffffu, s, 1);
      if (lane == 0) in[k] = carry;
      carry = __shfl_sync(0xffffffffu, s, 31);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float s = in[k], last = 0.f;
      Pack<T, V> out;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (MODE == kWholeRows && i == x[k].spos) last = s, s = h0v[k];
        s = fmaf(a[k][i], s, b[k][i]);
        out.put(i, !RAGGED || (live[k] >> i & 1u) ? s : 0.f);
      }
      u.store(out, x[k], row[k], p.h + u.row0 * p.L + u.t0, p.L);
      if (p.h_last != nullptr && u.ends(x[k])) p.h_last[u.row0 + row[k]] = u.L - x[k].t == V ? s : last;
    }
    if (MODE != kWholeRows && lane == 0 && p.h_last != nullptr && ((active && !more) || (c == 0 && end == 0))) p.h_last[u.row0] = carry;
    if (MODE == kTeam) carry = after;
  }
  if (MODE == kTeam && members > kRowWarps) cluster_sync();       // nobody leaves while its box may be read
}

template <typename T, bool WIDE, int MODE, bool RAGGED, bool SIGMOID>
__global__ void __launch_bounds__(32 * kRowWarps, 2) scan_rows_backward_kernel(const ScanArgs<T> p) {
  using U = RowUnit<T, WIDE, MODE, RAGGED>;
  constexpr int V = U::V, K = U::K;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  __shared__ float2 box[2][kRowWarps];
  U u;
  int me, members;
  if (!first_unit<U, T, MODE>(p, u, me, members)) return;
  const long long end = MODE == kWholeRows ? p.L : clamp_len(p.lengths, u.row0, p.L);
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(SIGMOID);
  float carry = 0.f;
  if (MODE != kWholeRows && p.g_last != nullptr) carry = p.g_last[u.row0];
#pragma unroll 1
  for (int round = 0; round < p.rounds; ++round) {
    const int c = p.chunks - 1 - (round * members + me);
    place_unit<U, T, MODE>(p, u, c);
    typename U::Vec x[K];
    int row[K];
    Pack<T, V> pv[K], pg[K], pd[K];
    float h0v[K], glv[K];
    uint32_t live[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      x[k] = u.vec(k, row[k]);
      u.load(pv[k], x[k], row[k], p.v + u.row0 * p.in_o + u.t0, p.in_o, none_v);
      u.load(pg[k], x[k], row[k], p.g + u.row0 * p.in_o + u.t0, p.in_o, none_g);
      u.load(pd[k], x[k], row[k], p.gh + u.row0 * p.L + u.t0, p.L, none_v);
      h0v[k] = glv[k] = 0.f;
      if (u.starts(x[k]) && p.h0 != nullptr) h0v[k] = p.h0[u.row0 + row[k] + (x[k].t > 0 ? 1 : 0)];
      if (u.ends(x[k]) && p.g_last != nullptr) glv[k] = p.g_last[u.row0 + row[k]];
      if (RAGGED) live[k] = u.steps(x[k], row[k], p.lengths, end);
    }
    const bool active = MODE == kWholeRows || (u.n > 0 && u.t0 < end);
    const long long at = (long long)c * p.outer + u.row0;
    float start = 0.f;            // the state in front of the chunk: saved, or the row's own beginning
    if (MODE != kWholeRows && (active || c == 0)) start = p.ckpt != nullptr ? p.ckpt[at] : p.h0 != nullptr ? p.h0[u.row0] : 0.f;
    float a[K][V], b[K][V], A[K], H[K], B[K], D[K];
    bool fresh_up[K], fresh_down[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      A[k] = 1.f, H[k] = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (RAGGED && !(live[k] >> i & 1u)) pv[k].v[i] = none_v, pg[k].v[i] = none_g, pd[k].v[i] = none_v;
#pragma unroll
      for (int i = 0; i < V; i += 2) {
        float2 a2, b2;
        terms_pair<SIGMOID>(make_float2(pg[k].get(i), pg[k].get(i + 1)), a2, b2);
        a[k][i] = a2.x, a[k][i + 1] = a2.y, b[k][i] = b2.x, b[k][i + 1] = b2.y;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (MODE == kWholeRows && i == x[k].spos) H[k] = h0v[k];
        A[k] *= a[k][i];
        H[k] = fmaf(a[k][i], H[k], b[k][i] * pv[k].get(i));
      }
      D[k] = glv[k];             // (0, or a row's end at the vector's)
#pragma unroll
      for (int i = V - 1; i >= 0; --i) {
        D[k] = a[k][i] * (D[k] + pd[k].get(i));
        if (MODE == kWholeRows && i == x[k].spos) D[k] = glv[k];
      }
      B[k] = A[k];
      fresh_up[k] = segmented_scan<true, SIGMOID>(A[k], H[k], MODE == kWholeRows ? __ballot_sync(0xffffffffu, x[k].spos < V) : 0u, u.span);
      fresh_down[k] = segmented_scan<false, SIGMOID>(B[k], D[k], MODE == kWholeRows ? __ballot_sync(0xffffffffu, u.ends(x[k])) : 0u, u.span);
    }
    float after = 0.f;
    if (MODE == kTeam) {
      float tA = 1.f, tD = 0.f;
#pragma unroll
      for (int k = K - 1; k >= 0; --k) {
        const float B1 = __shfl_sync(0xffffffffu, B[k], 0), D1 = __shfl_sync(0xffffffffu, D[k], 0);
        tD = through<SIGMOID>(B1, tD, D1), tA *= B1;
      }
      after = carry;
      carry = join_team<SIGMOID>(make_float2(tA, tD), after, box, round, me, members);
    }
    float in[K], din[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const float s = fresh_up[k] ? H[k] : through<SIGMOID>(A[k], start, H[k]);
      in[k] = __shfl_up_sync(0xffffffffu, s, 1);
      if (lane == 0) in[k] = start;
      start = __shfl_sync(0xffffffffu, s, 31);
    }
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      const float d = fresh_down[k] ? D[k] : through<SIGMOID>(B[k], carry, D[k]);
      din[k] = __shfl_down_sync(0xffffffffu, d, 1);
      if (lane == 31) din[k] = carry;
      carry = __shfl_sync(0xffffffffu, d, 0);
    }
    if (MODE != kWholeRows && c == 0 && lane == 0 && p.gh0 != nullptr) p.gh0[u.row0] = carry;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float w[V], s = in[k], g0 = 0.f;
      float d = u.ends(x[k]) && u.L - x[k].t == V ? glv[k] : din[k];
#pragma unroll
      for (int i = 0; i < V; ++i) {       // what delta is multiplied with for the gate's gradient
        if (MODE == kWholeRows && i == x[k].spos) s = h0v[k];
        const float v = pv[k].get(i);
        w[i] = SIGMOID ? (s - v) * (a[k][i] * b[k][i]) : s;
        s = fmaf(a[k][i], s, b[k][i] * v);
      }
      Pack<T, V> ov, og;
#pragma unroll
      for (int i = V - 1; i >= 0; --i) {
        const bool step = !RAGGED || (live[k] >> i & 1u);
        const float delta = d + pd[k].get(i);
        ov.put(i, step ? delta * b[k][i] : 0.f);
        og.put(i, step ? delta * w[i] : 0.f);
        d = a[k][i] * delta;
        if (MODE == kWholeRows && i == x[k].spos) g0 = d, d = glv[k];
      }
      u.store(ov, x[k], row[k], p.gv + u.row0 * p.gr_o + u.t0, p.gr_o);
      u.store(og, x[k], row[k], p.gg + u.row0 * p.gr_o + u.t0, p.gr_o);
      if (u.starts(x[k]) && p.gh0 != nullptr) p.gh0[u.row0 + row[k] + (x[k].t > 0 ? 1 : 0)] = g0;
    }
    if (MODE == kTeam) carry = after;
  }
  if (MODE == kTeam && members > kRowWarps) cluster_sync();
}

// length 0: the state passes through
__global__ void __launch_bounds__(256) scan_copy_kernel(const float* __restrict__ in, float* __restrict__ out, long long n) {
  pdl_trigger();
  pdl_wait();
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256)
    out[i] = in != nullptr ? in[i] : 0.f;
}

// CTAs of a cluster that shares a sequence of `chunks` chunks: the size with the fewest rounds one after the other, over all
// the waves in which `tiles` clusters run (`slots` CTAs at once); the smallest of equals.
int cluster_for(long long tiles, long long chunks, long long slots, int most) {
  int best = 1;
  long long least = -1;
  for (int n = 1; n <= most && (n == 1 || n < 2 * chunks); n *= 2) {
    const long long rounds = (tiles * n + slots - 1) / slots * ((chunks + n - 1) / n);
    if (least < 0 || rounds < least) best = n, least = rounds;
  }
  return best;
}

template <typename T, class S, int MODE, bool BACK>
cudaError_t launch_cols_kernel(const ScanArgs<T>& p, int cluster, cudaStream_t st) {
  void (*kern)(const ScanArgs<T>);
  constexpr size_t smem = ColSlots<T, S, BACK ? 3 : 2>::SMEM;
  if constexpr (BACK) kern = p.sigmoid ? scan_cols_backward_kernel<T, S, MODE, true> : scan_cols_backward_kernel<T, S, MODE, false>;
  else kern = p.sigmoid ? scan_cols_kernel<T, S, MODE, true> : scan_cols_kernel<T, S, MODE, false>;
  static std::atomic<uint64_t> allowed[2]{};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kern), smem + 8192 + sizeof(float) * 3 * S::SLOTS * S::W, allowed[p.sigmoid != 0]);
  if (e != cudaSuccess) return e;
  if (MODE == kOneTile) return launch_pdl(kern, dim3((unsigned)p.chains), dim3(S::THREADS), smem, st, p);
  if (p.chains * cluster > 0x7fffffff) return cudaErrorNotSupported;
  return launch_clusters(kern, (unsigned)(p.chains * cluster), cluster, S::THREADS, smem, st, p);
}

// sequences that fit one tile
template <typename T, class S, bool BACK>
cudaError_t launch_short_cols(ScanArgs<T> p, cudaStream_t st) {
  p.total = p.outer * p.groups;
  p.chains = (p.total + S::TX - 1) / S::TX;
  p.chunks = p.rounds = 1;
  if (p.chains > 0x7fffffff) return cudaErrorNotSupported;
  return launch_cols_kernel<T, S, kOneTile, BACK>(p, 1, st);
}
template <typename T, class S, bool BACK>
cudaError_t launch_long_cols(ScanArgs<T> p, cudaStream_t st) {
  static_assert(S::LC == kColTile, "tiles end where states are saved");
  const long long per_outer = (p.groups + S::TX - 1) / S::TX;
  p.per_outer = (unsigned)per_outer;
  p.chains = p.outer * per_outer;
  p.chunks = (int)((p.L + S::LC - 1) / S::LC);
  const int cluster = cluster_for(p.chains, p.chunks, S::ctas(p.sigmoid != 0) * (long long)num_sms(), 8);
  p.rounds = (p.chunks + cluster - 1) / cluster;
  return launch_cols_kernel<T, S, kLong, BACK>(p, cluster, st);
}

template <typename T, bool WIDE, int MODE, bool BACK>
cudaError_t launch_rows_kernel(const ScanArgs<T>& p, long long tiles, int cluster, cudaStream_t st) {
  void (*kern)(const ScanArgs<T>);
  const bool ragged = p.lengths != nullptr, sigmoid = p.sigmoid != 0;
  if constexpr (BACK)
    kern = ragged ? (sigmoid ? scan_rows_backward_kernel<T, WIDE, MODE, true, true> : scan_rows_backward_kernel<T, WIDE, MODE, true, false>)
                  : (sigmoid ? scan_rows_backward_kernel<T, WIDE, MODE, false, true> : scan_rows_backward_kernel<T, WIDE, MODE, false, false>);
  else
    kern = ragged ? (sigmoid ? scan_rows_kernel<T, WIDE, MODE, true, true> : scan_rows_kernel<T, WIDE, MODE, true, false>)
                  : (sigmoid ? scan_rows_kernel<T, WIDE, MODE, false, true> : scan_rows_kernel<T, WIDE, MODE, false, false>);
  if (MODE == kTeam) return launch_clusters(kern, (unsigned)(tiles * cluster), cluster, 32 * kRowWarps, 0, st, p);
  const long long ctas = (tiles + kRowWarps - 1) / kRowWarps;       // a unit per warp
  if (ctas > 0x7fffffff) return cudaErrorNotSupported;
  return launch_pdl(kern, dim3((unsigned)ctas), dim3(32 * kRowWarps), 0, st, p);
}

template <typename T, bool BACK>
cudaError_t launch_rows(ScanArgs<T> p, const ScanCall& c, cudaStream_t st) {
  constexpr int V = 8;
  const int step = row_chunk(p.L);
  p.chunks = (int)((p.L + step - 1) / step);
  // one vector grid for all tensors: contiguous rows, or (a chunk is part of one row) rows that begin on vectors
  auto wide = [&](const void* base, long long stride) {
    return base == nullptr || (aligned_to(base, V * sizeof(T)) && (stride == p.L || (p.chunks > 1 && p.L % V == 0 && stride % V == 0)));
  };
  const bool w = wide(c.v, c.in_outer) && wide(c.g, c.in_outer) && wide(c.h, p.L) && wide(c.grad_h, p.L) &&
                 wide(c.grad_v, c.grad_outer) && wide(c.grad_g, c.grad_outer);
  if (p.chunks == 1) {
    // rows of a unit: as many as fit, and units that begin and end on vectors where that many are a multiple
    p.groups = (p.L % 8 == 0 ? kUnit : kUnit - 8) / p.L;
    for (long long m = V; m > 1; m /= 2)
      if (p.groups >= m && p.L % m != 0) {
        p.groups -= p.groups % m;
        break;
      }
    const long long units = (p.outer + p.groups - 1) / p.groups;
    p.rounds = 1;
    return w ? launch_rows_kernel<T, true, kWholeRows, BACK>(p, units, 1, st) : launch_rows_kernel<T, false, kWholeRows, BACK>(p, units, 1, st);
  }
  // a warp per row where that fills the GPU's 16 warps per SM, else the warps of a CTA or cluster share it (on both sides of
  // the limit, fp32 rows of 8192: 2367 shared 46 us forward, 64 backward; 2368 apart 45, 68)
  if (p.outer >= 16 * (long long)num_sms()) {
    p.rounds = p.chunks;
    return w ? launch_rows_kernel<T, true, kWalk, BACK>(p, p.outer, 1, st) : launch_rows_kernel<T, false, kWalk, BACK>(p, p.outer, 1, st);
  }
  const int cluster = cluster_for(p.outer, (p.chunks + kRowWarps - 1) / kRowWarps, 2 * (long long)num_sms(), 32 / kRowWarps), team = cluster * kRowWarps;
  p.rounds = (p.chunks + team - 1) / team;
  return w ? launch_rows_kernel<T, true, kTeam, BACK>(p, p.outer, cluster, st) : launch_rows_kernel<T, false, kTeam, BACK>(p, p.outer, cluster, st);
}

template <typename T, bool BACK>
cudaError_t scan_t(const ScanCall& c, cudaStream_t st) {
  ScanArgs<T> p{};
  p.v = static_cast<const T*>(c.v), p.g = static_cast<const T*>(c.g), p.gh = static_cast<const T*>(c.grad_h);
  p.h0 = c.h0, p.g_last = c.grad_last, p.lengths = c.lengths;
  p.h = static_cast<T*>(c.h), p.gv = static_cast<T*>(c.grad_v), p.gg = static_cast<T*>(c.grad_g);
  p.h_last = c.h_last, p.gh0 = c.grad_h0, p.ckpt = c.checkpoints;
  p.outer = c.outer, p.L = c.length, p.inner = c.inner;
  p.in_o = c.in_outer, p.in_t = c.in_step, p.gr_o = c.grad_outer, p.gr_t = c.grad_step;
  p.sigmoid = c.gate == DTST_GATE_SIGMOID;
  if (c.inner == 1 && c.length >= 8) return launch_rows<T, BACK>(p, c, st);
  const size_t need = 4 * sizeof(T);
  bool vec = c.inner % 4 == 0 && c.in_outer % 4 == 0 && c.in_step % 4 == 0 && aligned_to(c.v, need) && aligned_to(c.g, need);
  if (BACK) vec = vec && c.grad_outer % 4 == 0 && c.grad_step % 4 == 0 && aligned_to(c.grad_h, need) && aligned_to(c.grad_v, need) && aligned_to(c.grad_g, need);
  else vec = vec && aligned_to(c.h, need);
  p.groups = vec ? c.inner / 4 : c.inner;
  // The shortest tile that holds the sequences, so that few of its steps are empty: fp32 [65536][9][64] takes 100 us (forward) in
  // the tile of 16 steps, 325 in that of 64; [8192][65][64] 93 in 128 steps, 203 in the long sequences' 256.  A tile that
  // holds all steps needs no staging for a next one: [2048][256][64] takes 63 us (backward 119), 75 (155) as a long sequence.
  // The backward pass has more to keep for a step and holds half as many a thread.  One channel a thread, the price of
  // channel counts that are no multiple of four: 88 us for [2048][256][65].  Of its backward tile of 16 steps a thread two CTAs
  // share an SM under a sigmoid gate, whose a and b do not fit the 80 registers of three (fp32 [32][256][2079] 89 us against
  // 95, bf16 [8][2500][1025] 97 against 154), and three under a decay, which has no b (73 against 86, 104 against 95).  Three
  // as well in the tile of 16 steps under a decay (fp32 [65536][9][64] 126 us against 156 of two; under a sigmoid it needs 128 registers).
  constexpr int R = BACK ? 4 : 8, N = BACK ? 2 : 1;
  if (vec) {
    if (c.length <= 8) return launch_short_cols<T, ColShape<4, 8, 1>, BACK>(p, st);
    if (c.length <= 16) return launch_short_cols<T, ColShape<4, 4, 4, 2, BACK ? 3 : 2>, BACK>(p, st);
    if (c.length <= 32) return launch_short_cols<T, ColShape<4, R, 4 * N>, BACK>(p, st);
    if (c.length <= 64) return launch_short_cols<T, ColShape<4, R, 8 * N>, BACK>(p, st);
    if (c.length <= 128) return launch_short_cols<T, ColShape<4, R, 16 * N>, BACK>(p, st);
    if (c.length <= 256) return launch_short_cols<T, ColShape<4, R, 32 * N>, BACK>(p, st);
    return launch_long_cols<T, ColShape<4, R, 32 * N>, BACK>(p, st);
  }
  if (c.length <= 8) return launch_short_cols<T, ColShape<1, 8, 1>, BACK>(p, st);
  if (c.length <= 16) return launch_short_cols<T, ColShape<1, 8, 2>, BACK>(p, st);
  if (c.length <= 32) return launch_short_cols<T, ColShape<1, 8, 4>, BACK>(p, st);
  if (c.length <= 64) return launch_short_cols<T, ColShape<1, 8, 8>, BACK>(p, st);
  if (c.length <= 128) return launch_short_cols<T, ColShape<1, 8, 16>, BACK>(p, st);
  if (c.length <= 256) return launch_short_cols<T, ColShape<1, 16, 16, BACK ? 2 : 4, BACK ? 3 : 4>, BACK>(p, st);
  return launch_long_cols<T, ColShape<1, 16, 16, BACK ? 2 : 4, BACK ? 3 : 4>, BACK>(p, st);
}

}  // namespace

// States are saved every 256 steps of [outer][L][inner] sequences, every 512 (or 504) of contiguous ones - or once, in
// front of a sequence that fits one tile.
long long scan_chunk(int, long long length, long long inner) {
  const long long lc = inner == 1 ? row_chunk(length) : kColTile;
  return length <= lc ? (length < 1 ? 1 : length) : lc;
}

cudaError_t scan_status(int* word, cudaStream_t st) {
  const int none = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(word, scan_status_word, sizeof(int), 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && *word != 0) e = cudaMemcpyToSymbolAsync(scan_status_word, &none, sizeof(int), 0, cudaMemcpyHostToDevice, st);
  return e == cudaSuccess && *word != 0 ? cudaStreamSynchronize(st) : e;
}

cudaError_t launch_scan_forward(const ScanCall& c, cudaStream_t st) {
  if (c.length == 0) {
    if (c.h_last == nullptr) return cudaSuccess;
    const long long n = c.outer * c.inner, ctas = (n + 255) / 256;
    return launch_pdl(scan_copy_kernel, dim3((unsigned)(ctas < 1024 ? ctas : 1024)), dim3(256), 0, st, c.h0, c.h_last, n);
  }
  switch (c.dtype) {
    case DTST_F32: return scan_t<float, false>(c, st);
    case DTST_BF16: return scan_t<__nv_bfloat16, false>(c, st);
    default: return scan_t<__half, false>(c, st);
  }
}

cudaError_t launch_scan_backward(const ScanCall& c, cudaStream_t st) {
  if (c.length == 0) {
    if (c.grad_h0 == nullptr) return cudaSuccess;
    const long long n = c.outer * c.inner, ctas = (n + 255) / 256;
    return launch_pdl(scan_copy_kernel, dim3((unsigned)(ctas < 1024 ? ctas : 1024)), dim3(256), 0, st, c.grad_last, c.grad_h0, n);
  }
  switch (c.dtype) {
    case DTST_F32: return scan_t<float, true>(c, st);
    case DTST_BF16: return scan_t<__nv_bfloat16, true>(c, st);
    default: return scan_t<__half, true>(c, st);
  }
}

}  // namespace dtst
