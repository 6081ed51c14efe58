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

// a = 1 / (1 + e^-g) and b = 1 - a, each formed without cancellation
__device__ __forceinline__ void gate_of(float g, float& a, float& b) {
  const float e = __expf(-fabsf(g));
  const float r = __fdividef(1.0f, 1.0f + e);
  a = g >= 0.f ? r : e * r;
  b = g >= 0.f ? e * r : r;
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
  float state = SLOTS > 1 && at.keeper && c_first == 0 && p.h0 != nullptr ? p.h0[at.ch] : 0.f;

#pragma unroll 1
  for (int c = c_first; c < c_end; ++c) {
    const int t0 = c * LC + at.slot * R;
    Pack<T, VEC> pv[R], pg[R];
    const T *lv = v + t0 * p.in_t, *lg = g + t0 * p.in_t;
#pragma unroll
    for (int r = 0; r < R; ++r, lv += p.in_t, lg += p.in_t)
      if (t0 + r < at.end) pv[r].load(lv), pg[r].load(lg);
    float a[R][VEC], u[R][VEC], s[VEC];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        a[r][j] = 1.f, u[r][j] = 0.f;
        if (t0 + r < at.end) {
          if (p.sigmoid) {
            float b;
            gate_of(pg[r].get(j), a[r][j], b);
            u[r][j] = b * pv[r].get(j);
          } else {
            a[r][j] = pg[r].get(j), u[r][j] = pv[r].get(j);
          }
        }
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
  const int ch_last = at.ch_end > 0 ? (int)((at.ch_end - 1) / LC) : 0;     // the chunk of the sequence's last step
  float grad = SLOTS > 1 && at.keeper && p.g_last != nullptr ? p.g_last[at.ch] : 0.f;

#pragma unroll 1
  for (int n = n_first; n < n_end; ++n) {
    const int c = p.chunks - 1 - n;
    const int t0 = c * LC + at.slot * R;
    Pack<T, VEC> pv[R], pg[R], pd[R];
    const T *lv = v + t0 * p.in_t, *lg = g + t0 * p.in_t, *ld = gh + t0 * p.inner;
#pragma unroll
    for (int r = 0; r < R; ++r, lv += p.in_t, lg += p.in_t, ld += p.inner)
      if (t0 + r < at.end) pv[r].load(lv), pg[r].load(lg), pd[r].load(ld);
    const bool active = at.keeper && c * LC < at.ch_end, mine = at.keeper && (active || c == 0);
    float before = 0.f;      // the state in front of the chunk: saved, or the sequence's own beginning
    if (SLOTS > 1 && mine) before = p.ckpt != nullptr ? p.ckpt[c * states + at.ch] : p.h0 != nullptr ? p.h0[at.ch] : 0.f;
    float a[R][VEC], w[R][VEC], s[VEC], d[VEC];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        a[r][j] = 1.f, w[r][j] = 0.f;
        if (t0 + r < at.end) {
          if (p.sigmoid) {
            float b;
            gate_of(pg[r].get(j), a[r][j], b);
            w[r][j] = b * pv[r].get(j);
          } else {
            a[r][j] = pg[r].get(j), w[r][j] = pv[r].get(j);
          }
        }
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
        for (int r = R - 1; r >= 0; --r) D = a[r][j] * (D + (t0 + r < at.end ? pd[r].get(j) : 0.f));
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
        if (t0 + r < at.end) {
          if (p.sigmoid) {
            float aa, b;
            gate_of(pg[r].get(j), aa, b);
            w[r][j] = (s[j] - pv[r].get(j)) * aa * b;
          } else {
            w[r][j] = s[j];
          }
        }
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
          float b = 1.f;
          if (p.sigmoid) {
            float aa;
            gate_of(pg[r].get(j), aa, b);
          }
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
// [outer][L], the steps contiguous.  P neighbouring lanes share a row, 16 steps each; tiles come and go through
// shared memory with one word of padding behind every 16 steps (a warp's lanes then walk their runs without bank
// conflicts), the lanes' runs are joined by shuffles.  Global accesses are 16 bytes wide: a tile of whole rows is one
// contiguous piece of memory, cut into vectors regardless of where rows begin.
constexpr int kRowSteps = 16;
constexpr int kRowPitch = kRowSteps + 1;
constexpr int kTileFloats = kScanThreads * kRowPitch;

// A tile of `rows` rows of n steps, rows `stride` elements apart in memory.  WIDE: 16-byte accesses - the tile is one
// contiguous piece, or its rows begin and end on vectors; element by element otherwise.
template <typename T, int P, bool WIDE>
struct RowTile {
  static constexpr int V = 16 / (int)sizeof(T), N = kRowSteps / V;    // vectors per thread
  uint32_t rows, n, magic;          // magic: division by n through the high word of a product (exact below 2^16)
  __device__ __forceinline__ RowTile(uint32_t rows_, uint32_t n_) : rows(rows_), n(n_), magic(0xffffffffu / n_ + 1u) {}
  __device__ __forceinline__ void split(uint32_t e, uint32_t& row, uint32_t& t) const {
    row = n == 1 ? e : __umulhi(e, magic);
    t = e - row * n;
  }
  static __device__ __forceinline__ uint32_t place(uint32_t row, uint32_t t) { return row * (P * kRowPitch) + t + t / kRowSteps; }
  // global -> registers (WIDE; all loads of a tile are under way before the first is used)
  __device__ __forceinline__ void fetch(Pack<T, V> (&r)[N], const T* base, long long stride) const {
    if constexpr (WIDE) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        uint32_t row, t;
        const uint32_t e = (threadIdx.x + k * kScanThreads) * V;
        split(e, row, t);
        const T* at = base + row * stride + t;
        if (e + V <= rows * n) r[k].load(at);
        else if (e < rows * n) r[k].load_part(at, (int)(rows * n - e));
      }
    }
  }
  // registers (or, element by element, global) -> shared memory
  __device__ __forceinline__ void scatter(float* tile, const Pack<T, V> (&r)[N], const T* base, long long stride) const {
    if constexpr (WIDE) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        uint32_t row, t;
        split((threadIdx.x + k * kScanThreads) * V, row, t);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          if (row < rows) tile[place(row, t)] = r[k].get(i);
          if (++t == n) t = 0, ++row;
        }
      }
    } else {
#pragma unroll 4
      for (uint32_t e = threadIdx.x; e < rows * n; e += kScanThreads) {
        uint32_t row, t;
        split(e, row, t);
        tile[place(row, t)] = Elem<T>::get(base[row * stride + t]);
      }
    }
  }
  __device__ __forceinline__ void store(T* base, const float* tile, long long stride) const {
    if constexpr (WIDE) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        Pack<T, V> r;
        uint32_t row, t;
        const uint32_t e = (threadIdx.x + k * kScanThreads) * V;
        split(e, row, t);
        T* at = base + row * stride + t;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          if (row < rows) r.put(i, tile[place(row, t)]);
          if (++t == n) t = 0, ++row;
        }
        if (e + V <= rows * n) r.store(at);
        else if (e < rows * n) r.store_part(at, (int)(rows * n - e));
      }
    } else {
#pragma unroll 4
      for (uint32_t e = threadIdx.x; e < rows * n; e += kScanThreads) {
        uint32_t row, t;
        split(e, row, t);
        base[row * stride + t] = Elem<T>::put(tile[place(row, t)]);
      }
    }
  }
};

template <typename T, int P, bool WIDE, bool CHAIN>
__global__ void __launch_bounds__(kScanThreads, 3) scan_rows_kernel(const ScanArgs<T> p) {
  constexpr int ROWS = kScanThreads / P, LC = P * kRowSteps;
  using Tile = RowTile<T, P, WIDE>;
  __shared__ float sv[kTileFloats], sg[kTileFloats];
  __shared__ unsigned ticket[2];
  pdl_trigger();
  pdl_wait();
  unsigned tag = 0, tile = blockIdx.x;
  if (CHAIN) tile = take_ticket(p.ctrl, ticket, tag);
  const int c_first = CHAIN ? (int)(tile / (unsigned)p.chains) : 0, c_end = CHAIN ? c_first + 1 : p.chunks;
  const long long r0 = (long long)(CHAIN ? tile % (unsigned)p.chains : tile) * ROWS;
  const int slot = threadIdx.x % P;
  const long long row = r0 + threadIdx.x / P;
  const uint32_t rows = (uint32_t)(p.outer - r0 < ROWS ? p.outer - r0 : ROWS);
  const bool live = row < p.outer;
  const long long end = live ? clamp_len(p.lengths, row, p.L) : 0;
  float carry = live && p.h0 != nullptr ? p.h0[row] : 0.f;
  float* mv = sv + threadIdx.x * kRowPitch;
  float* mg = sg + threadIdx.x * kRowPitch;
#pragma unroll 1
  for (int c = c_first; c < c_end; ++c) {
    const long long t0 = (long long)c * LC;
    const Tile m(rows, (uint32_t)(p.L - t0 < LC ? p.L - t0 : LC));
    {
      const T *bv = p.v + r0 * p.in_o + t0, *bg = p.g + r0 * p.in_o + t0;
      Pack<T, Tile::V> rv[Tile::N], rg[Tile::N];
      m.fetch(rv, bv, p.in_o);
      m.fetch(rg, bg, p.in_o);
      m.scatter(sv, rv, bv, p.in_o);
      m.scatter(sg, rg, bg, p.in_o);
    }
    __syncthreads();
    float a[kRowSteps], u[kRowSteps], A = 1.f, H = 0.f;
    const long long ts = t0 + slot * kRowSteps;
    const int have = end - ts >= kRowSteps ? kRowSteps : end > ts ? (int)(end - ts) : 0;
#pragma unroll
    for (int r = 0; r < kRowSteps; ++r) {
      a[r] = 1.f, u[r] = 0.f;
      if (r < have) {
        if (p.sigmoid) {
          float b;
          gate_of(mg[r], a[r], b);
          u[r] = b * mv[r];
        } else {
          a[r] = mg[r], u[r] = mv[r];
        }
      }
      A *= a[r];
      H = fmaf(a[r], H, u[r]);
    }
#pragma unroll
    for (int k = 1; k < P; k *= 2) {
      const float A1 = __shfl_up_sync(0xffffffffu, A, k, P), H1 = __shfl_up_sync(0xffffffffu, H, k, P);
      if (slot >= k) H = fmaf(A, H1, H), A *= A1;
    }
    const long long at = (long long)c * p.outer + row;
    // a warp holds one row where tiles are chained, so the row's lanes look back together
    const bool active = t0 < end, more = t0 + LC < end;
    if (CHAIN && active && c > 0) {
      if (more && slot == P - 1) put_sum(p.sums + at, A, H, tag);
      carry = look_back_warp(p.sums + at - p.outer, p.ends + at - p.outer, -p.outer, c, tag, p.status);
    }
    if (p.ckpt != nullptr && live && slot == 0 && (active || c == 0)) p.ckpt[at] = carry;
    const float full = fmaf(A, carry, H);                  // the state behind this lane's run
    float s = __shfl_up_sync(0xffffffffu, full, 1, P);
    if (slot == 0) s = carry;
    carry = __shfl_sync(0xffffffffu, full, P - 1, P);
    if (CHAIN && more && slot == 0) put_end(p.ends + at, carry, tag);
    if (live && slot == 0 && p.h_last != nullptr && ((active && !more) || (c == 0 && end == 0))) p.h_last[row] = carry;
#pragma unroll
    for (int r = 0; r < kRowSteps; ++r) {
      s = fmaf(a[r], s, u[r]);
      mv[r] = r < have ? s : 0.f;
    }
    __syncthreads();
    m.store(p.h + r0 * p.L + t0, sv, p.L);
    if (!CHAIN) __syncthreads();
  }
  if (CHAIN) leave_chain(p.ctrl, tag);
}

template <typename T, int P, bool WIDE, bool CHAIN>
__global__ void __launch_bounds__(kScanThreads, 2) scan_rows_backward_kernel(const ScanArgs<T> p) {
  constexpr int ROWS = kScanThreads / P, LC = P * kRowSteps;
  using Tile = RowTile<T, P, WIDE>;
  extern __shared__ float tiles[];
  __shared__ unsigned ticket[2];
  float* sv = tiles;
  float* sg = sv + kTileFloats;
  float* sd = sg + kTileFloats;
  pdl_trigger();
  pdl_wait();
  unsigned tag = 0, tile = blockIdx.x;
  if (CHAIN) tile = take_ticket(p.ctrl, ticket, tag);
  const int n_first = CHAIN ? (int)(tile / (unsigned)p.chains) : 0, n_end = CHAIN ? n_first + 1 : p.chunks;
  const long long r0 = (long long)(CHAIN ? tile % (unsigned)p.chains : tile) * ROWS;
  const int slot = threadIdx.x % P;
  const long long row = r0 + threadIdx.x / P;
  const uint32_t rows = (uint32_t)(p.outer - r0 < ROWS ? p.outer - r0 : ROWS);
  const bool live = row < p.outer;
  const long long end = live ? clamp_len(p.lengths, row, p.L) : 0;
  const int last = end > 0 ? (int)((end - 1) / LC) : 0;     // the chunk of the row's last step
  float carry = live && p.g_last != nullptr ? p.g_last[row] : 0.f;
  float* mv = sv + threadIdx.x * kRowPitch;
  float* mg = sg + threadIdx.x * kRowPitch;
  float* md = sd + threadIdx.x * kRowPitch;
#pragma unroll 1
  for (int k0 = n_first; k0 < n_end; ++k0) {
    const int c = p.chunks - 1 - k0;
    const long long t0 = (long long)c * LC;
    const Tile m(rows, (uint32_t)(p.L - t0 < LC ? p.L - t0 : LC));
    {
      const T *bv = p.v + r0 * p.in_o + t0, *bg = p.g + r0 * p.in_o + t0, *bd = p.gh + r0 * p.L + t0;
      Pack<T, Tile::V> rv[Tile::N], rg[Tile::N], rd[Tile::N];
      m.fetch(rv, bv, p.in_o);
      m.fetch(rg, bg, p.in_o);
      m.fetch(rd, bd, p.L);
      m.scatter(sv, rv, bv, p.in_o);
      m.scatter(sg, rg, bg, p.in_o);
      m.scatter(sd, rd, bd, p.L);
    }
    const float* before = p.ckpt != nullptr ? p.ckpt + (long long)c * p.outer : p.h0;
    const bool active = t0 < end;
    const float start = live && before != nullptr && (active || c == 0) ? before[row] : 0.f;
    __syncthreads();
    float a[kRowSteps], w[kRowSteps], A = 1.f, H = 0.f, D = 0.f;
    const long long ts = t0 + slot * kRowSteps;
    const int have = end - ts >= kRowSteps ? kRowSteps : end > ts ? (int)(end - ts) : 0;
#pragma unroll
    for (int r = 0; r < kRowSteps; ++r) {
      a[r] = 1.f, w[r] = 0.f;
      if (r < have) {
        if (p.sigmoid) {
          float b;
          gate_of(mg[r], a[r], b);
          w[r] = b * mv[r];
          mg[r] = b;
        } else {
          a[r] = mg[r], w[r] = mv[r];
          mg[r] = 1.f;
        }
      }
      A *= a[r];
      H = fmaf(a[r], H, w[r]);
    }
#pragma unroll
    for (int r = kRowSteps - 1; r >= 0; --r) D = a[r] * (D + (r < have ? md[r] : 0.f));
    float Af = A, Ab = A;
#pragma unroll
    for (int k = 1; k < P; k *= 2) {
      const float A1 = __shfl_up_sync(0xffffffffu, Af, k, P), H1 = __shfl_up_sync(0xffffffffu, H, k, P);
      const float A2 = __shfl_down_sync(0xffffffffu, Ab, k, P), D2 = __shfl_down_sync(0xffffffffu, D, k, P);
      if (slot >= k) H = fmaf(Af, H1, H), Af *= A1;
      if (slot + k < P) D = fmaf(Ab, D2, D), Ab *= A2;
    }
    const long long at = (long long)c * p.outer + row;
    if (CHAIN && active && c < last) {
      if (c > 0 && slot == 0) put_sum(p.sums + at, Ab, D, tag);
      carry = look_back_warp(p.sums + at + p.outer, p.ends + at + p.outer, p.outer, last - c, tag, p.status);
    }
    float s = __shfl_up_sync(0xffffffffu, fmaf(Af, start, H), 1, P);
    if (slot == 0) s = start;
    const float all = fmaf(Ab, carry, D);
    float d = __shfl_down_sync(0xffffffffu, all, 1, P);
    if (slot == P - 1) d = carry;
    carry = __shfl_sync(0xffffffffu, all, 0, P);
    if (CHAIN && active && c > 0 && slot == 0) put_end(p.ends + at, carry, tag);
    if (c == 0 && live && slot == 0 && p.gh0 != nullptr) p.gh0[row] = carry;
    // forward once more: u is replaced by what delta is multiplied with for the gate's gradient
#pragma unroll
    for (int r = 0; r < kRowSteps; ++r) {
      const float u = w[r];
      if (r < have) w[r] = p.sigmoid ? (s - mv[r]) * a[r] * mg[r] : s;
      s = fmaf(a[r], s, u);
    }
#pragma unroll
    for (int r = kRowSteps - 1; r >= 0; --r) {
      const bool on = r < have;
      const float delta = d + (on ? md[r] : 0.f);
      mv[r] = on ? delta * mg[r] : 0.f;
      mg[r] = on ? delta * w[r] : 0.f;
      d = a[r] * delta;
    }
    __syncthreads();
    m.store(p.gv + r0 * p.gr_o + t0, sv, p.gr_o);
    m.store(p.gg + r0 * p.gr_o + t0, sg, p.gr_o);
    if (!CHAIN) __syncthreads();
  }
  if (CHAIN) leave_chain(p.ctrl, tag);
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

int row_lanes(long long length) {
  int P = 1;
  while (P < 32 && P * kRowSteps < length) P *= 2;
  return P;
}

// Whether the chunks of a sequence become chained tiles (true) or a CTA walks through them (false): see the rule below.
bool chained(long long chains, long long chunks) { return chunks > 1 && chains * chunks <= 0x7fffffff && chains < 4 * (long long)num_sms(); }

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
    if (chained(p.chains, p.chunks)) {
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

template <typename T, int P, bool WIDE, bool CHAIN, bool BACK>
cudaError_t launch_rows_kernel(const ScanArgs<T>& p, long long tiles, cudaStream_t st) {
  const dim3 grid((unsigned)tiles), block(kScanThreads);
  if constexpr (!BACK) return launch_pdl(scan_rows_kernel<T, P, WIDE, CHAIN>, grid, block, 0, st, p);
  constexpr int smem = 3 * (int)sizeof(float) * kTileFloats;
  cudaError_t e = cudaFuncSetAttribute(scan_rows_backward_kernel<T, P, WIDE, CHAIN>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return e != cudaSuccess ? e : launch_pdl(scan_rows_backward_kernel<T, P, WIDE, CHAIN>, grid, block, smem, st, p);
}

template <typename T, int P, bool BACK>
cudaError_t launch_rows(ScanArgs<T> p, const ScanCall& c, cudaStream_t st) {
  constexpr int V = 16 / (int)sizeof(T);
  p.chains = (p.outer + kScanThreads / P - 1) / (kScanThreads / P);
  p.chunks = (int)((p.L + P * kRowSteps - 1) / (P * kRowSteps));
  auto wide = [&](const void* base, long long stride) {   // tiles begin at multiples of 8 rows, chunks at multiples of 512 steps
    return base == nullptr || (aligned_to(base, 16) && ((p.chunks == 1 && stride == p.L) || (p.L % V == 0 && stride % V == 0)));
  };
  const bool w = wide(c.v, c.in_outer) && wide(c.g, c.in_outer) && wide(c.h, p.L) && wide(c.grad_h, p.L) &&
                 wide(c.grad_v, c.grad_outer) && wide(c.grad_g, c.grad_outer);
  if constexpr (P == 32) {
    if (chained(p.chains, p.chunks)) {
      chain(p, c);
      return w ? launch_rows_kernel<T, P, true, true, BACK>(p, p.chains * p.chunks, st)
               : launch_rows_kernel<T, P, false, true, BACK>(p, p.chains * p.chunks, st);
    }
  }
  return w ? launch_rows_kernel<T, P, true, false, BACK>(p, p.chains, st) : launch_rows_kernel<T, P, false, false, BACK>(p, p.chains, st);
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
  if (c.inner == 1) {
    switch (row_lanes(c.length)) {
      case 1: return launch_rows<T, 1, BACK>(p, c, st);
      case 2: return launch_rows<T, 2, BACK>(p, c, st);
      case 4: return launch_rows<T, 4, BACK>(p, c, st);
      case 8: return launch_rows<T, 8, BACK>(p, c, st);
      case 16: return launch_rows<T, 16, BACK>(p, c, st);
      default: return launch_rows<T, 32, BACK>(p, c, st);
    }
  }
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

// States are saved every 64 steps of [outer][L][inner] sequences, every 512 of contiguous ones - or once, in front of a
// sequence that fits one tile.
long long scan_chunk(int, long long length, long long inner) {
  const long long lc = inner == 1 ? kRowSteps * row_lanes(length) : kSave;
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
