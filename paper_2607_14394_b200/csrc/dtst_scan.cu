// Gated linear recurrence along one dimension and its backward pass:
//     h_t = a_t h_{t-1} + u_t,     sigmoid gate: a = 1 / (1 + e^-g), u = (1 - a) v;     decay: a = g, u = v
//     delta_t = gh_t + a_{t+1} delta_{t+1}          (grad_last enters behind the last step)
//     sigmoid: gv = delta (1 - a), gg = delta (h_{t-1} - v) a (1 - a);   decay: gv = delta, gg = delta h_{t-1}
//     grad_h0 = a_0 delta_0
// A step is the affine map s -> a s + u; maps compose to (A, H) = (A2 A1, A2 H1 + H2), so a run of steps is summarised
// by two numbers and runs can be joined in any grouping.  A thread holds R consecutive steps in registers, composes
// them, learns the state in front of its run from the summaries of the runs before it, and then walks its steps once
// more.  Steps at and beyond a sequence's own length are the identity map and are not read.  States are fp32.
//
// Memory-bound: forward 2 tensors in, 1 out; backward 3 in, 2 out.  The backward pass does not read h: it rebuilds
// h_{t-1} inside each chunk, in fp32, from the state saved at the chunk's start.
#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

constexpr int kScanThreads = 256;

// Chained tiles.  Where there are few sequences, the chunks of one sequence are tiles of their own, handed out in
// time order by a ticket counter.  A tile publishes the summary (A, H) of its chunk, looks back for the nearest chunk
// whose end state is known, applies the summaries in between to it - one after the other, so the result has the same
// bits whichever state it started from - and publishes its own end state.  Every 32-bit value travels in one 64-bit
// word with the call's number, so no fence and no clearing is needed; the last CTA advances the number.  A tile waits only
// for tiles with earlier tickets, which are running or done; the wait is bounded all the same.
struct ChainCtrl {
  unsigned ticket, done, epoch;
};
constexpr uint32_t kChainPolls = 1u << 20;

__device__ __forceinline__ unsigned long long tagged(float v, unsigned tag) {
  return (unsigned long long)tag << 32 | __float_as_uint(v);
}
__device__ __forceinline__ void put_sum(ulonglong2* at, float A, float H, unsigned tag) {
  asm volatile("st.relaxed.gpu.global.v2.b64 [%0], {%1, %2};" ::"l"(at), "l"(tagged(A, tag)), "l"(tagged(H, tag)) : "memory");
}
__device__ __forceinline__ void put_end(unsigned long long* at, float s, unsigned tag) {
  asm volatile("st.relaxed.gpu.global.b64 [%0], %1;" ::"l"(at), "l"(tagged(s, tag)) : "memory");
}
__device__ __forceinline__ ulonglong2 get_sum(const ulonglong2* at) {
  ulonglong2 v;
  asm volatile("ld.relaxed.gpu.global.v2.b64 {%0, %1}, [%2];" : "=l"(v.x), "=l"(v.y) : "l"(at) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long get_end(const unsigned long long* at) {
  unsigned long long v;
  asm volatile("ld.relaxed.gpu.global.b64 %0, [%1];" : "=l"(v) : "l"(at) : "memory");
  return v;
}
__device__ __forceinline__ float value_of(unsigned long long w) { return __uint_as_float((uint32_t)w); }
__device__ __forceinline__ bool has_tag(unsigned long long w, unsigned tag) { return (unsigned)(w >> 32) == tag; }

// State in front of a chunk for CPW channels of a warp; lane = depth group * CPW + channel.  `want`: this lane's channel
// asks; `n` chunks precede it, `sum` / `end` point at the nearest one's entries, `stride` entries further lies the one
// before that.  kLook chunks are read at once, spread over the depth groups.
template <int CPW, int kLook>
__device__ __forceinline__ float look_back(bool want, const ulonglong2* sum, const unsigned long long* end, long long stride,
                                           int n, unsigned tag, int* status) {
  constexpr int DG = 32 / CPW, NI = kLook / DG;
  const int depth = (threadIdx.x & 31) / CPW, ch = (threadIdx.x & 31) % CPW;
  float result = 0.f;
  bool open = want;
  for (uint32_t poll = 0; poll < kChainPolls; ++poll) {
    unsigned long long e[NI];
    ulonglong2 q[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int k = depth + DG * i;
      e[i] = 0, q[i] = make_ulonglong2(0, 0);
      if (open && k < n) {
        e[i] = get_end(end + k * stride);
        q[i] = get_sum(sum + k * stride);
      }
    }
    int found = kLook, gap = kLook;       // the nearest chunk with an end state, and without a summary
    float s = 0.f;
#pragma unroll
    for (int i = NI - 1; i >= 0; --i) {
      if (open && has_tag(e[i], tag)) found = depth + DG * i, s = value_of(e[i]);
      if (!(has_tag(q[i].x, tag) && has_tag(q[i].y, tag))) gap = depth + DG * i;
    }
    const int mine = found;
#pragma unroll
    for (int o = CPW; o < 32; o *= 2) {
      found = min(found, __shfl_xor_sync(0xffffffffu, found, o));
      gap = min(gap, __shfl_xor_sync(0xffffffffu, gap, o));
    }
    const unsigned has = __ballot_sync(0xffffffffu, mine == found);
    // the lane of this channel that holds the end state
    unsigned of_ch = 0;
#pragma unroll
    for (int d = 0; d < DG; ++d) of_ch |= has & (1u << (d * CPW + ch));
    s = __shfl_sync(0xffffffffu, s, of_ch != 0 ? __ffs(of_ch) - 1 : 0);
#pragma unroll
    for (int k = kLook - 1; k >= 0; --k) {
      const float A = __shfl_sync(0xffffffffu, value_of(q[k / DG].x), (k % DG) * CPW + ch);
      const float H = __shfl_sync(0xffffffffu, value_of(q[k / DG].y), (k % DG) * CPW + ch);
      if (k < found) s = fmaf(A, s, H);
    }
    if (open && found < kLook && gap >= found) {
      result = s;
      open = false;
    }
    if (!__any_sync(0xffffffffu, open)) return result;
    __nanosleep(20);
  }
  if (open) atomicExch(status, 1);
  return result;
}

// The same by a whole warp for one sequence: lane k looks at the k-th chunk back.
__device__ __forceinline__ float look_back_warp(const ulonglong2* sum, const unsigned long long* end, long long stride, int n,
                                                unsigned tag, int* status) {
  const int lane = threadIdx.x & 31;
  for (uint32_t poll = 0; poll < kChainPolls; ++poll) {
    unsigned long long e = 0;
    ulonglong2 q = make_ulonglong2(0, 0);
    if (lane < n) {
      e = get_end(end + lane * stride);
      q = get_sum(sum + lane * stride);
    }
    const unsigned ends = __ballot_sync(0xffffffffu, lane < n && has_tag(e, tag));
    const unsigned sums = __ballot_sync(0xffffffffu, lane < n && has_tag(q.x, tag) && has_tag(q.y, tag));
    const int found = __ffs(ends) - 1;
    if (found >= 0 && (sums & ((1u << found) - 1u)) == (1u << found) - 1u) {
      float s = __shfl_sync(0xffffffffu, value_of(e), found);
      for (int k = found - 1; k >= 0; --k)
        s = fmaf(__shfl_sync(0xffffffffu, value_of(q.x), k), s, __shfl_sync(0xffffffffu, value_of(q.y), k));
      return s;
    }
    __nanosleep(32);
  }
  if (lane == 0) atomicExch(status, 1);
  return 0.f;
}

// takes a ticket; all threads of the CTA get (tile, tag)
__device__ __forceinline__ unsigned take_ticket(ChainCtrl* ctrl, unsigned* shared2, unsigned& tag) {
  if (threadIdx.x == 0) {
    shared2[1] = *(volatile unsigned*)&ctrl->epoch + 1u;
    shared2[0] = atomicAdd(&ctrl->ticket, 1u);
  }
  __syncthreads();
  tag = shared2[1];
  return shared2[0];
}
// after a CTA's last use of the chain; the last one prepares the next call (tag 0 is what a fresh workspace holds)
__device__ __forceinline__ void leave_chain(ChainCtrl* ctrl, unsigned tag) {
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicAdd(&ctrl->done, 1u) == gridDim.x - 1) {
      ctrl->ticket = 0;
      ctrl->done = 0;
      ctrl->epoch = tag == 0xffffffffu ? 0u : tag;
    }
  }
}

template <typename T>
struct ScanArgs {
  const T *v, *g, *gh;
  const float *h0, *g_last;
  const int* lengths;
  T *h, *gv, *gg;
  float *h_last, *gh0, *ckpt;
  long long outer, L, inner, groups, total;     // groups of VEC channels per outer entry, outer * groups
  long long in_o, in_t, gr_o, gr_t;
  long long chains;            // CTAs side by side; each has `chunks` tiles one behind the other
  int chunks, sigmoid;
  // chained tiles (null: a CTA walks through its chunks by itself)
  ChainCtrl* ctrl;
  ulonglong2* sums;            // [chunks][outer * inner]: (A, tag), (H, tag) of a chunk
  unsigned long long* ends;    // [chunks][outer * inner]: (state behind a chunk, tag)
  int* status;
};

// a = 1 / (1 + e^-g) and b = 1 - a, each formed without cancellation.  The approximate exponential and reciprocal are good
// to about 2^-22; what they flush to zero (|g| > 87) is below the smallest normal number anyway.
__device__ __forceinline__ void gate_of(float g, float& a, float& b) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(g) * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  const float er = e * r;
  a = g >= 0.f ? r : er;
  b = g >= 0.f ? er : r;
}
// h_t = a h_{t-1} + b v_t
__device__ __forceinline__ void terms(int sigmoid, float g, float& a, float& b) {
  if (sigmoid) gate_of(g, a, b);
  else a = g, b = 1.f;
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
// [outer][L][inner], inner contiguous.  A tile is TX groups of VEC channels (groups run on across outer entries) times
// SLOTS runs of R steps, a run per thread.
template <int VEC_, int R_, int SLOTS_, int THREADS_>
struct ColShape {
  static constexpr int VEC = VEC_, R = R_, SLOTS = SLOTS_, THREADS = THREADS_;
  static constexpr int TX = THREADS / SLOTS, W = TX * VEC, LC = SLOTS * R;
  // while runs are joined a warp has CPW channels, DG lanes each, and a lane has JOIN neighbouring runs of its channel
  static constexpr int CPW = W / (THREADS / 32) < 32 ? W / (THREADS / 32) : 32, DG = 32 / CPW;
  static constexpr int JOIN = SLOTS >= DG ? SLOTS / DG : 1;
};
constexpr int kSave = 64;         // steps between saved states
constexpr int kColTile = 128;     // steps of a forward tile where a sequence has several

// joins (A, H) over the DG lanes of a channel, in lane order (UP) or against it; returns the summary of all of them and
// leaves in (A, H) that of the lanes before this one
template <int CPW, bool UP>
__device__ __forceinline__ float2 join_lanes(float& A, float& H) {
  const int d = (threadIdx.x & 31) / CPW;
  constexpr int DG = 32 / CPW;
#pragma unroll
  for (int o = 1; o < DG; o *= 2) {
    const float A1 = UP ? __shfl_up_sync(0xffffffffu, A, o * CPW) : __shfl_down_sync(0xffffffffu, A, o * CPW);
    const float H1 = UP ? __shfl_up_sync(0xffffffffu, H, o * CPW) : __shfl_down_sync(0xffffffffu, H, o * CPW);
    if (UP ? d >= o : d + o < DG) H = fmaf(A, H1, H), A *= A1;
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

// where a thread stands in its tile while it walks steps, and while it joins runs
template <typename T, class S>
struct ColPlace {
  int x, slot;              // group of the tile and run
  bool live;
  long long o, i0, end;     // outer entry, first channel, steps of the sequence
  int jx, jq;               // joining: channel of the tile, first run
  bool keeper, first;       // the channel exists; its first lane
  long long ch, ch_end;     // index of the channel's state, steps of its sequence
  __device__ __forceinline__ ColPlace(const ScanArgs<T>& p, long long g0) {
    x = threadIdx.x % S::TX, slot = threadIdx.x / S::TX;
    const long long gid = g0 + x;
    live = gid < p.total;
    o = live ? gid / p.groups : 0, i0 = live ? (gid - o * p.groups) * S::VEC : 0;
    end = live ? clamp_len(p.lengths, o, p.L) : 0;
    const int lane = threadIdx.x & 31;
    jx = (threadIdx.x / 32) * S::CPW + lane % S::CPW, jq = lane / S::CPW * S::JOIN;
    first = lane < S::CPW;
    const long long jg = g0 + jx / S::VEC;
    keeper = jg < p.total;
    const long long jo = keeper ? jg / p.groups : 0;
    ch = keeper ? jo * p.inner + (jg - jo * p.groups) * S::VEC + jx % S::VEC : 0;
    ch_end = keeper ? clamp_len(p.lengths, jo, p.L) : 0;
  }
};

template <typename T, class S, bool CHAIN>
__global__ void __launch_bounds__(S::THREADS, 1024 / S::THREADS) scan_cols_kernel(const ScanArgs<T> p) {
  constexpr int VEC = S::VEC, R = S::R, SLOTS = S::SLOTS, W = S::W, LC = S::LC;
  __shared__ float2 runs[SLOTS > 1 ? SLOTS : 1][SLOTS > 1 ? W : 1];     // (A, H) of every run; then its first state in x
  __shared__ unsigned ticket[2];
  pdl_trigger();
  pdl_wait();
  unsigned tag = 0, tile = blockIdx.x;
  if (CHAIN) tile = take_ticket(p.ctrl, ticket, tag);
  const int c_first = CHAIN ? (int)(tile / (unsigned)p.chains) : 0, c_end = CHAIN ? c_first + 1 : p.chunks;
  const long long g0 = (long long)(CHAIN ? tile % (unsigned)p.chains : tile) * S::TX;
  const ColPlace<T, S> at(p, g0);
  const T* v = p.v + at.o * p.in_o + at.i0;
  const T* g = p.g + at.o * p.in_o + at.i0;
  T* h = p.h + at.o * p.L * p.inner + at.i0;
  const long long states = p.outer * p.inner;
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(p.sigmoid);
  float state = SLOTS > 1 && at.keeper && c_first == 0 && p.h0 != nullptr ? p.h0[at.ch] : 0.f;

#pragma unroll 1
  for (int c = c_first; c < c_end; ++c) {
    const int t0 = c * LC + at.slot * R;
    Pack<T, VEC> pv[R], pg[R];
    const T *lv = v + t0 * p.in_t, *lg = g + t0 * p.in_t;
#pragma unroll
    for (int r = 0; r < R; ++r, lv += p.in_t, lg += p.in_t) {
      if (t0 + r < at.end) pv[r].load(lv), pg[r].load(lg);
      else pv[r].fill(none_v), pg[r].fill(none_g);
    }
    float a[R][VEC], u[R][VEC], s[VEC];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        terms(p.sigmoid, pg[r].get(j), a[r][j], u[r][j]);
        u[r][j] *= pv[r].get(j);
      }
    if constexpr (SLOTS == 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = at.live && p.h0 != nullptr ? p.h0[at.o * p.inner + at.i0 + j] : 0.f;
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float A = 1.f, H = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          A *= a[r][j];
          H = fmaf(a[r][j], H, u[r][j]);
        }
        runs[at.slot][at.x * VEC + j] = make_float2(A, H);
      }
      __syncthreads();
      float A = 1.f, H = 0.f;
      float2 m[S::JOIN];
#pragma unroll
      for (int q = 0; q < S::JOIN; ++q) {
        m[q] = runs[at.jq + q][at.jx];
        A *= m[q].x;
        H = fmaf(m[q].x, H, m[q].y);
      }
      const float2 all = join_lanes<S::CPW, true>(A, H);
      // a chunk in which a sequence has no step leaves its state alone, and nobody waits for it
      const bool active = at.keeper && c * LC < at.ch_end;
      const bool more = active && (c + 1) * (long long)LC < at.ch_end;
      const long long entry = c * states + at.ch;
      if (CHAIN && c > 0) {
        if (more && at.first) put_sum(p.sums + entry, all.x, all.y, tag);
        state = look_back<S::CPW, 32>(active, p.sums + entry - states, p.ends + entry - states, -states, c, tag, p.status);
      }
      float run = fmaf(A, state, H);
#pragma unroll
      for (int q = 0; q < S::JOIN; ++q) {
        runs[at.jq + q][at.jx].x = run;
        const int step = c * LC + (at.jq + q) * R;
        if (p.ckpt != nullptr && at.keeper && step % kSave == 0 && (step < at.ch_end || step == 0))
          p.ckpt[step / kSave * states + at.ch] = run;
        run = fmaf(m[q].x, run, m[q].y);
      }
      state = fmaf(all.x, state, all.y);
      if (at.first) {
        if (CHAIN && more) put_end(p.ends + entry, state, tag);
        if (at.keeper && (active || c == 0) && !more && p.h_last != nullptr) p.h_last[at.ch] = state;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = runs[at.slot][at.x * VEC + j].x;
    }
    T* sh = h + t0 * p.inner;
#pragma unroll
    for (int r = 0; r < R; ++r, sh += p.inner) {
      Pack<T, VEC> out;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        s[j] = fmaf(a[r][j], s[j], u[r][j]);
        out.put(j, t0 + r < at.end ? s[j] : 0.f);
      }
      if (at.live && t0 + r < p.L) out.store(sh);
    }
    if constexpr (SLOTS == 1) {
      if (at.live && p.h_last != nullptr) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.h_last[at.o * p.inner + at.i0 + j] = s[j];
      }
    } else if (!CHAIN) {
      __syncthreads();       // the runs' states are read before the next chunk's summaries replace them
    }
  }
  if (CHAIN) leave_chain(p.ctrl, tag);
}

template <typename T, class S, bool CHAIN>
__global__ void __launch_bounds__(S::THREADS, 512 / S::THREADS) scan_cols_backward_kernel(const ScanArgs<T> p) {
  constexpr int VEC = S::VEC, R = S::R, SLOTS = S::SLOTS, W = S::W, LC = S::LC;
  // (A, H) and D of every run; then the state in front of it (x) and the gradient that comes to it from behind
  __shared__ float2 runs[SLOTS > 1 ? SLOTS : 1][SLOTS > 1 ? W : 1];
  __shared__ float backs[SLOTS > 1 ? SLOTS : 1][SLOTS > 1 ? W : 1];
  __shared__ unsigned ticket[2];
  pdl_trigger();
  pdl_wait();
  unsigned tag = 0, tile = blockIdx.x;
  if (CHAIN) tile = take_ticket(p.ctrl, ticket, tag);
  // chunks from the last to the first
  const int n_first = CHAIN ? (int)(tile / (unsigned)p.chains) : 0, n_end = CHAIN ? n_first + 1 : p.chunks;
  const long long g0 = (long long)(CHAIN ? tile % (unsigned)p.chains : tile) * S::TX;
  const ColPlace<T, S> at(p, g0);
  const T* v = p.v + at.o * p.in_o + at.i0;
  const T* g = p.g + at.o * p.in_o + at.i0;
  const T* gh = p.gh + at.o * p.L * p.inner + at.i0;
  T* gv = p.gv + at.o * p.gr_o + at.i0;
  T* gg = p.gg + at.o * p.gr_o + at.i0;
  const long long states = p.outer * p.inner;
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(p.sigmoid);
  const int ch_last = at.ch_end > 0 ? (int)((at.ch_end - 1) / LC) : 0;     // the chunk of the sequence's last step
  float grad = SLOTS > 1 && at.keeper && p.g_last != nullptr ? p.g_last[at.ch] : 0.f;

#pragma unroll 1
  for (int n = n_first; n < n_end; ++n) {
    const int c = p.chunks - 1 - n;
    const int t0 = c * LC + at.slot * R;
    Pack<T, VEC> pv[R], pg[R], pd[R];
    const T *lv = v + t0 * p.in_t, *lg = g + t0 * p.in_t, *ld = gh + t0 * p.inner;
#pragma unroll
    for (int r = 0; r < R; ++r, lv += p.in_t, lg += p.in_t, ld += p.inner) {
      if (t0 + r < at.end) pv[r].load(lv), pg[r].load(lg), pd[r].load(ld);
      else pv[r].fill(none_v), pg[r].fill(none_g), pd[r].fill(none_v);
    }
    const bool active = at.keeper && c * LC < at.ch_end, mine = at.keeper && (active || c == 0);
    float before = 0.f;      // the state in front of the chunk: saved, or the sequence's own beginning
    if (SLOTS > 1 && mine) before = p.ckpt != nullptr ? p.ckpt[c * states + at.ch] : p.h0 != nullptr ? p.h0[at.ch] : 0.f;
    float a[R][VEC], w[R][VEC], s[VEC], d[VEC];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        terms(p.sigmoid, pg[r].get(j), a[r][j], w[r][j]);
        w[r][j] *= pv[r].get(j);
      }
    if constexpr (SLOTS == 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        s[j] = at.live && p.h0 != nullptr ? p.h0[at.o * p.inner + at.i0 + j] : 0.f;
        d[j] = at.live && p.g_last != nullptr ? p.g_last[at.o * p.inner + at.i0 + j] : 0.f;
      }
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float A = 1.f, H = 0.f, D = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          A *= a[r][j];
          H = fmaf(a[r][j], H, w[r][j]);
        }
#pragma unroll
        for (int r = R - 1; r >= 0; --r) D = a[r][j] * (D + pd[r].get(j));
        runs[at.slot][at.x * VEC + j] = make_float2(A, H);
        backs[at.slot][at.x * VEC + j] = D;
      }
      __syncthreads();
      float A = 1.f, H = 0.f, B = 1.f, D = 0.f;
      float2 m[S::JOIN];
      float md[S::JOIN];
#pragma unroll
      for (int q = 0; q < S::JOIN; ++q) {
        m[q] = runs[at.jq + q][at.jx];
        md[q] = backs[at.jq + q][at.jx];
        A *= m[q].x;
        H = fmaf(m[q].x, H, m[q].y);
      }
#pragma unroll
      for (int q = S::JOIN - 1; q >= 0; --q) D = fmaf(m[q].x, D, md[q]);
      B = A;
      join_lanes<S::CPW, true>(A, H);
      const float2 all = join_lanes<S::CPW, false>(B, D);
      if (CHAIN) {
        const long long entry = c * states + at.ch;
        const bool asks = active && c < ch_last;
        if (asks && c > 0 && at.first) put_sum(p.sums + entry, all.x, all.y, tag);
        const float in = look_back<S::CPW, 16>(asks, p.sums + entry + states, p.ends + entry + states, states, ch_last - c, tag, p.status);
        if (asks) grad = in;
      }
      float run = fmaf(A, before, H);
#pragma unroll
      for (int q = 0; q < S::JOIN; ++q) {
        runs[at.jq + q][at.jx].x = run;
        run = fmaf(m[q].x, run, m[q].y);
      }
      run = fmaf(B, grad, D);
#pragma unroll
      for (int q = S::JOIN - 1; q >= 0; --q) {
        backs[at.jq + q][at.jx] = run;
        run = fmaf(m[q].x, run, md[q]);
      }
      if (mine) grad = fmaf(all.x, grad, all.y);
      if (mine && at.first) {
        if (CHAIN && c > 0) put_end(p.ends + c * states + at.ch, grad, tag);
        if (c == 0 && p.gh0 != nullptr) p.gh0[at.ch] = grad;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = runs[at.slot][at.x * VEC + j].x, d[j] = backs[at.slot][at.x * VEC + j];
    }
    // forward once more: u is replaced by what delta is multiplied with for the gate's gradient
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float u = w[r][j];
        float aa, b;
        terms(p.sigmoid, pg[r].get(j), aa, b);
        w[r][j] = p.sigmoid ? (s[j] - pv[r].get(j)) * (a[r][j] * b) : s[j];
        s[j] = fmaf(a[r][j], s[j], u);
      }
    T *sv = gv + (t0 + R - 1) * p.gr_t, *sg = gg + (t0 + R - 1) * p.gr_t;
#pragma unroll
    for (int r = R - 1; r >= 0; --r, sv -= p.gr_t, sg -= p.gr_t) {
      Pack<T, VEC> ov, og;
      ov.zero();
      og.zero();
      if (t0 + r < at.end) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float delta = d[j] + pd[r].get(j);
          float aa, b;
          terms(p.sigmoid, pg[r].get(j), aa, b);
          ov.put(j, delta * b);
          og.put(j, delta * w[r][j]);
          d[j] = a[r][j] * delta;
        }
      }
      if (at.live && t0 + r < p.L) {
        ov.store(sv);
        og.store(sg);
      }
    }
    if constexpr (SLOTS == 1) {
      if (at.live && p.gh0 != nullptr) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.gh0[at.o * p.inner + at.i0 + j] = d[j];
      }
    } else if (!CHAIN) {
      __syncthreads();
    }
  }
  if (CHAIN) leave_chain(p.ctrl, tag);
}

// ------------------------------------------------------------------------------------------------ rows
// [outer][L], the steps contiguous, L >= 8.  A warp takes a unit of at most 512 neighbouring elements - whole rows, or a
// chunk of a long one - in 16-byte vectors straight from global memory: K vectors a lane, the k-th at (32 k + lane) V.  Each
// vector is composed in its lane, the lanes are joined by a warp scan that does not reach across a row's first step
// (forward) or last step (backward), and the K scans are joined one after the other.  No shared memory, no barriers.
// Where rows begin off a vector the unit starts at the vector before; the elements in front are left alone.
constexpr int kUnit = 512, kRowWarps = 8;

// steps of a chunk (a chunk of odd rows leaves room for a shifted beginning)
__host__ __device__ constexpr int row_chunk(long long L) { return L % 8 == 0 ? kUnit : kUnit - 8; }

enum RowMode { kWholeRows = 0, kWalk = 1, kChained = 2 };

// Vector k of a unit: its first element's index (below 0 in front of the unit) and step, and the element that is a row's
// first step (V: none; at most one, since L >= V).
template <int V>
struct RowVec {
  int rel, t, spos;
};

template <typename T, bool WIDE, int MODE, bool RAGGED>
struct RowUnit {
  static constexpr int V = 16 / (int)sizeof(T), K = kUnit / 32 / V;
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
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        r.v[i] = none;
        if (on(v, i)) r.v[i] = base[WIDE ? v.rel + i : offset(v, row, i, stride)];
      }
    }
  }
  __device__ __forceinline__ void store(const Pack<T, V>& r, const Vec& v, int row, T* base, long long stride) const {
    if (WIDE && full(v)) {
      r.store(base + v.rel);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (on(v, i)) base[WIDE ? v.rel + i : offset(v, row, i, stride)] = r.v[i];
    }
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
template <bool UP>
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
    if (o <= room) H = fmaf(A, H1, H), A *= A1;
  }
  return fresh;
}

// the unit of this warp; false if there is none.  `c` = its chunk, counted from the front.
template <class U, typename T, int MODE, bool BACK>
__device__ __forceinline__ bool first_unit(const ScanArgs<T>& p, U& u, int& c, unsigned& tag) {
  const long long id = (long long)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
  u.L = (int)p.L;
  u.magic = 0xffffffffu / (uint32_t)p.L + 1u;
  u.span = MODE == kWholeRows ? (u.L + U::V - 2) / U::V + 1 : 32;
  c = 0, tag = 0;
  if (MODE == kWholeRows) {
    u.row0 = id * p.groups;                       // groups: rows of a unit
    if (u.row0 >= p.outer) return false;
    u.n = (int)((p.outer - u.row0 < p.groups ? p.outer - u.row0 : p.groups) * p.L);
    u.t0 = 0;
  } else if (MODE == kWalk) {
    if (id >= p.outer) return false;
    u.row0 = id;
    c = BACK ? p.chunks - 1 : 0;
  } else {
    if (id >= p.outer * p.chunks) return false;   // as many tickets as units
    unsigned t = 0;
    if ((threadIdx.x & 31) == 0) {
      tag = *(volatile unsigned*)&p.ctrl->epoch + 1u;
      t = atomicAdd(&p.ctrl->ticket, 1u);
    }
    tag = __shfl_sync(0xffffffffu, tag, 0);
    t = __shfl_sync(0xffffffffu, t, 0);
    u.row0 = t % (unsigned)p.outer;
    c = (int)(t / (unsigned)p.outer);
    if (BACK) c = p.chunks - 1 - c;
  }
  return true;
}
template <class U, typename T, int MODE>
__device__ __forceinline__ void place_unit(const ScanArgs<T>& p, U& u, int c) {
  if (MODE != kWholeRows) {
    const int step = row_chunk(p.L);
    u.t0 = c * step;
    u.n = (int)(p.L - u.t0 < step ? p.L - u.t0 : step);
  }
  // rows that begin off a vector: only contiguous tensors are read wide then, all with the same shift
  u.shift = p.L % U::V == 0 ? 0 : (int)((u.row0 * p.L + u.t0) % U::V);
}
template <typename T>
__device__ __forceinline__ void leave_unit(const ScanArgs<T>& p, unsigned tag) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) {
    __threadfence();
    if (atomicAdd(&p.ctrl->done, 1u) == (unsigned)(p.outer * p.chunks) - 1u) {
      p.ctrl->ticket = 0;
      p.ctrl->done = 0;
      p.ctrl->epoch = tag == 0xffffffffu ? 0u : tag;
    }
  }
}

template <typename T, bool WIDE, int MODE, bool RAGGED>
__global__ void __launch_bounds__(32 * kRowWarps, 3) scan_rows_kernel(const ScanArgs<T> p) {
  using U = RowUnit<T, WIDE, MODE, RAGGED>;
  constexpr int V = U::V, K = U::K;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  U u;
  int c;
  unsigned tag;
  if (!first_unit<U, T, MODE, false>(p, u, c, tag)) return;
  const long long end = MODE == kWholeRows ? p.L : clamp_len(p.lengths, u.row0, p.L);
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(p.sigmoid);
  float carry = 0.f;
  if (MODE != kWholeRows && c == 0 && p.h0 != nullptr) carry = p.h0[u.row0];
#pragma unroll 1
  for (;; ++c) {
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
      for (int i = 0; i < V; ++i) {
        if (RAGGED && !(live[k] >> i & 1u)) pv[k].v[i] = none_v, pg[k].v[i] = none_g;
        terms(p.sigmoid, pg[k].get(i), a[k][i], b[k][i]);
        b[k][i] *= pv[k].get(i);
        if (MODE == kWholeRows && i == x[k].spos) H[k] = h0v[k];
        A[k] *= a[k][i];
        H[k] = fmaf(a[k][i], H[k], b[k][i]);
      }
      fresh[k] = segmented_scan<true>(A[k], H[k], MODE == kWholeRows ? __ballot_sync(0xffffffffu, x[k].spos < V) : 0u, u.span);
    }
    const bool active = MODE == kWholeRows || u.t0 < end, more = MODE != kWholeRows && u.t0 + u.n < end;
    const long long at = (long long)c * p.outer + u.row0;
    if (MODE == kChained && active && c > 0) {
      if (more) {           // the whole chunk's summary, the vectors joined in order
        float tA = 1.f, tH = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) tH = fmaf(A[k], tH, H[k]), tA *= A[k];
        if (lane == 31) put_sum(p.sums + at, tA, tH, tag);
      }
      carry = look_back_warp(p.sums + at - p.outer, p.ends + at - p.outer, -p.outer, c, tag, p.status);
    }
    if (MODE != kWholeRows && p.ckpt != nullptr && lane == 0 && (active || c == 0)) p.ckpt[at] = carry;
    float in[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const float s = fresh[k] ? H[k] : fmaf(A[k], carry, H[k]);
      in[k] = __shfl_up_sync(0xffffffffu, s, 1);
      if (lane == 0) in[k] = carry;
      carry = __shfl_sync(0xffffffffu, s, 31);
    }
    if (MODE == kChained && more && lane == 0) put_end(p.ends + at, carry, tag);
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
    if (MODE != kWalk || c + 1 == p.chunks) break;
  }
  if (MODE == kChained) leave_unit(p, tag);
}

template <typename T, bool WIDE, int MODE, bool RAGGED>
__global__ void __launch_bounds__(32 * kRowWarps, 2) scan_rows_backward_kernel(const ScanArgs<T> p) {
  using U = RowUnit<T, WIDE, MODE, RAGGED>;
  constexpr int V = U::V, K = U::K;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31;
  U u;
  int c;
  unsigned tag;
  if (!first_unit<U, T, MODE, true>(p, u, c, tag)) return;
  const long long end = MODE == kWholeRows ? p.L : clamp_len(p.lengths, u.row0, p.L);
  const int last = end > 0 ? (int)((end - 1) / row_chunk(p.L)) : 0;      // the chunk of the row's last step
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(p.sigmoid);
  float carry = 0.f;
  if (MODE != kWholeRows && p.g_last != nullptr) carry = p.g_last[u.row0];
#pragma unroll 1
  for (;; --c) {
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
    const bool active = MODE == kWholeRows || u.t0 < end;
    const long long at = (long long)c * p.outer + u.row0;
    float start = 0.f;            // the state in front of the chunk: saved, or the row's own beginning
    if (MODE != kWholeRows && (active || c == 0)) start = p.ckpt != nullptr ? p.ckpt[at] : p.h0 != nullptr ? p.h0[u.row0] : 0.f;
    float a[K][V], b[K][V], A[K], H[K], B[K], D[K];
    bool fresh_up[K], fresh_down[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      A[k] = 1.f, H[k] = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (RAGGED && !(live[k] >> i & 1u)) pv[k].v[i] = none_v, pg[k].v[i] = none_g, pd[k].v[i] = none_v;
        terms(p.sigmoid, pg[k].get(i), a[k][i], b[k][i]);
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
      fresh_up[k] = segmented_scan<true>(A[k], H[k], MODE == kWholeRows ? __ballot_sync(0xffffffffu, x[k].spos < V) : 0u, u.span);
      fresh_down[k] = segmented_scan<false>(B[k], D[k], MODE == kWholeRows ? __ballot_sync(0xffffffffu, u.ends(x[k])) : 0u, u.span);
    }
    if (MODE == kChained && active && c < last) {
      if (c > 0) {
        float tA = 1.f, tD = 0.f;
#pragma unroll
        for (int k = K - 1; k >= 0; --k) tD = fmaf(B[k], tD, D[k]), tA *= B[k];
        if (lane == 0) put_sum(p.sums + at, tA, tD, tag);
      }
      carry = look_back_warp(p.sums + at + p.outer, p.ends + at + p.outer, p.outer, last - c, tag, p.status);
    }
    float in[K], din[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const float s = fresh_up[k] ? H[k] : fmaf(A[k], start, H[k]);
      in[k] = __shfl_up_sync(0xffffffffu, s, 1);
      if (lane == 0) in[k] = start;
      start = __shfl_sync(0xffffffffu, s, 31);
    }
#pragma unroll
    for (int k = K - 1; k >= 0; --k) {
      const float d = fresh_down[k] ? D[k] : fmaf(B[k], carry, D[k]);
      din[k] = __shfl_down_sync(0xffffffffu, d, 1);
      if (lane == 31) din[k] = carry;
      carry = __shfl_sync(0xffffffffu, d, 0);
    }
    if (MODE == kChained && active && c > 0 && lane == 0) put_end(p.ends + at, carry, tag);
    if (MODE != kWholeRows && c == 0 && lane == 0 && p.gh0 != nullptr) p.gh0[u.row0] = carry;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float w[V], s = in[k], g0 = 0.f;
      float d = u.ends(x[k]) && u.L - x[k].t == V ? glv[k] : din[k];
#pragma unroll
      for (int i = 0; i < V; ++i) {       // what delta is multiplied with for the gate's gradient
        if (MODE == kWholeRows && i == x[k].spos) s = h0v[k];
        const float v = pv[k].get(i);
        w[i] = p.sigmoid ? (s - v) * (a[k][i] * b[k][i]) : s;
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
    if (MODE != kWalk || c == 0) break;
  }
  if (MODE == kChained) leave_unit(p, tag);
}

// length 0: the state passes through
__global__ void __launch_bounds__(256) scan_copy_kernel(const float* __restrict__ in, float* __restrict__ out, long long n) {
  pdl_trigger();
  pdl_wait();
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256)
    out[i] = in != nullptr ? in[i] : 0.f;
}

// bytes in front of the chain's entries: status word, then its control words
constexpr size_t kChainHead = kStatusBytes + 256;

// Whether the chunks of a sequence become chained tiles (true) or a CTA walks through them (false): see the rule below.
bool chained(long long ctas, long long chunks, long long tiles) {
  return chunks > 1 && tiles <= 0x7fffffff && ctas < 4 * (long long)num_sms();
}

template <typename T>
void chain(ScanArgs<T>& p, const ScanCall& c) {
  unsigned char* ws = static_cast<unsigned char*>(c.workspace);
  p.ctrl = reinterpret_cast<ChainCtrl*>(ws + kStatusBytes);
  p.sums = reinterpret_cast<ulonglong2*>(ws + kChainHead);
  p.ends = reinterpret_cast<unsigned long long*>(p.sums + (long long)p.chunks * c.outer * c.inner);
  p.status = reinterpret_cast<int*>(ws);
}

template <typename T, class S, bool BACK>
cudaError_t launch_cols(ScanArgs<T> p, const ScanCall& c, cudaStream_t st) {
  p.chains = (p.total + S::TX - 1) / S::TX;
  p.chunks = (int)((p.L + S::LC - 1) / S::LC);
  const dim3 block(S::THREADS);
  // only the longest tiles ever come in several
  if constexpr (S::LC >= kSave) {
    if (chained(p.chains, p.chunks, p.chains * p.chunks)) {
      chain(p, c);
      const dim3 grid((unsigned)(p.chains * p.chunks));
      if constexpr (BACK) return launch_pdl(scan_cols_backward_kernel<T, S, true>, grid, block, 0, st, p);
      else return launch_pdl(scan_cols_kernel<T, S, true>, grid, block, 0, st, p);
    }
  }
  const dim3 grid((unsigned)p.chains);
  if constexpr (BACK) return launch_pdl(scan_cols_backward_kernel<T, S, false>, grid, block, 0, st, p);
  else return launch_pdl(scan_cols_kernel<T, S, false>, grid, block, 0, st, p);
}

template <typename T, bool WIDE, int MODE, bool BACK>
cudaError_t launch_rows_kernel(const ScanArgs<T>& p, long long units, cudaStream_t st) {
  const dim3 grid((unsigned)((units + kRowWarps - 1) / kRowWarps)), block(32 * kRowWarps);
  if constexpr (BACK)
    return p.lengths != nullptr ? launch_pdl(scan_rows_backward_kernel<T, WIDE, MODE, true>, grid, block, 0, st, p)
                                : launch_pdl(scan_rows_backward_kernel<T, WIDE, MODE, false>, grid, block, 0, st, p);
  else
    return p.lengths != nullptr ? launch_pdl(scan_rows_kernel<T, WIDE, MODE, true>, grid, block, 0, st, p)
                                : launch_pdl(scan_rows_kernel<T, WIDE, MODE, false>, grid, block, 0, st, p);
}

template <typename T, bool BACK>
cudaError_t launch_rows(ScanArgs<T> p, const ScanCall& c, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  const int step = row_chunk(p.L);
  p.chunks = (int)((p.L + step - 1) / step);
  // one vector grid for all tensors: contiguous rows, or (a chunk is part of one row) rows that begin on vectors
  auto wide = [&](const void* base, long long stride) {
    return base == nullptr || (aligned_to(base, 16) && (stride == p.L || (p.chunks > 1 && p.L % V == 0 && stride % V == 0)));
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
    return w ? launch_rows_kernel<T, true, kWholeRows, BACK>(p, units, st) : launch_rows_kernel<T, false, kWholeRows, BACK>(p, units, st);
  }
  if (chained((p.outer + kRowWarps - 1) / kRowWarps, p.chunks, p.outer * p.chunks)) {
    chain(p, c);
    return w ? launch_rows_kernel<T, true, kChained, BACK>(p, p.outer * p.chunks, st)
             : launch_rows_kernel<T, false, kChained, BACK>(p, p.outer * p.chunks, st);
  }
  return w ? launch_rows_kernel<T, true, kWalk, BACK>(p, p.outer, st) : launch_rows_kernel<T, false, kWalk, BACK>(p, p.outer, st);
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
  p.total = c.outer * p.groups;
  // forward tiles of 128 steps, backward ones of the 64 between saved states; shorter ones for short sequences
  if (vec) {
    if (c.length <= 4) return launch_cols<T, ColShape<4, 4, 1, 256>, BACK>(p, c, st);
    if (c.length <= 32) return launch_cols<T, ColShape<4, 4, 8, 256>, BACK>(p, c, st);
    return launch_cols<T, ColShape<4, 4, BACK ? 16 : 32, BACK ? 256 : 512>, BACK>(p, c, st);
  }
  if (c.length <= 8) return launch_cols<T, ColShape<1, 8, 1, 256>, BACK>(p, c, st);
  if (c.length <= 32) return launch_cols<T, ColShape<1, 8, 4, 256>, BACK>(p, c, st);
  return launch_cols<T, ColShape<1, 8, BACK ? 8 : 16, BACK ? 256 : 512>, BACK>(p, c, st);
}

}  // namespace

// States are saved every 64 steps of [outer][L][inner] sequences, every 512 (or 504) of contiguous ones - or once, in
// front of a sequence that fits one tile.
long long scan_chunk(int, long long length, long long inner) {
  const long long lc = inner == 1 ? row_chunk(length) : kSave;
  return length <= lc ? (length < 1 ? 1 : length) : lc;
}

size_t scan_workspace_bytes(int dtype, long long outer, long long length, long long inner) {
  const long long lc = scan_chunk(dtype, length, inner), chunks = (length + lc - 1) / lc;
  if (chunks < 2) return kStatusBytes;
  return kChainHead + (size_t)chunks * (size_t)outer * (size_t)inner * (sizeof(ulonglong2) + sizeof(unsigned long long));
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
