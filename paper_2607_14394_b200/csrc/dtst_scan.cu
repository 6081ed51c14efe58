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
constexpr uint32_t kChainPolls = 1u << 18;

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

// Which earlier chunk to start from, by one warp: lane k looks at the hint of the k-th tile back (`hint` = the nearest
// one's, `stride` entries between them, `n` of them).  A hint is written when (most of) a tile's entries have been:
// kind 1 = its summary, 2 = its end state; the reader of the entries still checks their tags.  -1: gave up.
__device__ __forceinline__ int poll_hints(const unsigned long long* hint, long long stride, int n, unsigned tag) {
  const int lane = threadIdx.x & 31;
  for (uint32_t poll = 0; poll < kChainPolls; ++poll) {
    const unsigned long long w = lane < n ? get_end(hint + lane * stride) : 0ull;
    const bool mine = has_tag(w, tag);
    const unsigned ends = __ballot_sync(0xffffffffu, mine && (unsigned)w == 2u), any = __ballot_sync(0xffffffffu, mine);
    const int found = __ffs(ends) - 1;
    if (found >= 0 && (any & ((1u << found) - 1u)) == (1u << found) - 1u) return found;
    __nanosleep(20);
  }
  return -1;
}
__device__ __forceinline__ void put_hint(unsigned long long* at, unsigned kind, unsigned tag) { put_end(at, __uint_as_float(kind), tag); }

// State in front of a chunk for CPW channels of a warp, from the end state `found` (< 32, the same for the whole warp) chunks
// further back than the nearest one and the summaries in between; lane = depth group * CPW + channel.  `want`: this lane's
// channel exists; `sum` / `end` point at the nearest chunk's entries, `stride` entries further lies the one before that.
template <int CPW>
__device__ __forceinline__ float look_back(bool want, const ulonglong2* sum, const unsigned long long* end, long long stride,
                                           int found, unsigned tag, int* status) {
  constexpr int DG = 32 / CPW;
  const int depth = (threadIdx.x & 31) / CPW, ch = (threadIdx.x & 31) % CPW;
  float s = 0.f;
  bool ok = !want;
  for (uint32_t poll = 0; poll < kChainPolls && !ok; ++poll) {
    const unsigned long long e = get_end(end + found * stride);
    ok = has_tag(e, tag);
    s = value_of(e);
  }
  if (!ok) atomicExch(status, 1);
  for (int k0 = found - 1; k0 >= 0; k0 -= DG) {       // the farthest first, DG at once
    const int k = k0 - depth;
    float A = 1.f, H = 0.f;
    ok = !want || k < 0;
    for (uint32_t poll = 0; poll < kChainPolls && !ok; ++poll) {
      const ulonglong2 q = get_sum(sum + k * stride);
      ok = has_tag(q.x, tag) && has_tag(q.y, tag);
      A = value_of(q.x), H = value_of(q.y);
    }
    if (!ok) atomicExch(status, 1);
    __syncwarp();
    const int n = k0 + 1 < DG ? k0 + 1 : DG;
    for (int d = 0; d < n; ++d)
      s = fmaf(__shfl_sync(0xffffffffu, A, d * CPW + ch), s, __shfl_sync(0xffffffffu, H, d * CPW + ch));
  }
  return s;
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
  long long chains;            // tiles side by side, `chunks` of them one behind the other
  unsigned per_outer;          // chains of an outer entry
  int chunks, sigmoid;
  // chained tiles (null: a CTA walks through its chunks by itself)
  ChainCtrl* ctrl;
  ulonglong2* sums;            // [chunks][outer * inner]: (A, tag), (H, tag) of a chunk
  unsigned long long* ends;    // [chunks][outer * inner]: (state behind a chunk, tag)
  unsigned long long* hints;   // [chunks][chains] (columns)
  int* status;
};

// a = 1 / (1 + e^-g) and b = 1 - a = e^-g / (1 + e^-g), both without cancellation.  The exponent is kept below 2^126 (a NaN
// stays one); the approximate exponential and reciprocal are good to about 2^-22, and what they flush to zero (g > 87) is
// below the smallest normal number.
__device__ __forceinline__ void gate_of(float g, float& a, float& b) {
  float e, r;
  asm("{\n\t.reg .f32 x;\n\tmul.f32 x, %1, 0fBFB8AA3B;\n\tmin.NaN.f32 x, x, 0f42FC0000;\n\tex2.approx.ftz.f32 %0, x;\n\t}" : "=f"(e) : "f"(g));   // 2^min(-g log2 e, 126)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  a = r;
  b = e * r;
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
// [outer][L][inner], inner contiguous.  A tile is TX groups of VEC channels times SLOTS runs of R steps, a run per thread.
// Long sequences: the tiles of one outer entry lie side by side over its channels (a chain of chunks each).  Short ones
// (one tile holds them): groups run on across outer entries, so that few channels fill a CTA too.
template <int VEC_, int R_, int SLOTS_>
struct ColShape {
  static constexpr int VEC = VEC_, R = R_, SLOTS = SLOTS_;
  static constexpr int TX = kScanThreads / SLOTS, W = TX * VEC, LC = SLOTS * R;
  // while runs are joined a warp has CPW channels, DG lanes each, and a lane has JOIN neighbouring runs of its channel
  static constexpr int WARPS = kScanThreads / 32, CPW = W / WARPS < 32 ? W / WARPS : 32, DG = 32 / CPW;
  static constexpr int JOIN = SLOTS >= DG ? SLOTS / DG : 1;
};
constexpr int kColTile = 256;     // steps of a long sequence's tile, and between saved states
enum ColMode { kOneTile = 0, kColWalk = 1, kColChained = 2 };

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

// A thread's part of a tile on its way through shared memory: only the thread itself touches its slots, so the copies of
// the next tile start as soon as this one's are in registers, and no barrier is needed.
template <typename T, class S, int TENSORS>
struct ColSlots {
  static constexpr int VEC = S::VEC, R = S::R, BYTES = VEC * (int)sizeof(T);
  static constexpr bool ASYNC = BYTES >= 4;      // (cp.async moves 4, 8 or 16 bytes)
  static constexpr size_t SMEM = (size_t)TENSORS * R * kScanThreads * BYTES;
  using P = Pack<T, VEC>;
  unsigned char* base;
  __device__ __forceinline__ P* slot(int tensor, int r) const {
    return reinterpret_cast<P*>(base + ((size_t)(tensor * R + r) * kScanThreads + threadIdx.x) * BYTES);
  }
  // the first `have` steps from src on; `none` for the others
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
  static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
};

// Where a tile lies.  Long sequences: the same for all threads of the CTA.
struct ColTile {
  int c;               // chunk
  unsigned o;          // outer entry
  long long g0;        // first group in it
  int end;             // steps of the sequence
};

template <typename T, class S, int MODE>
__device__ __forceinline__ ColTile col_tile(const ScanArgs<T>& p, unsigned chain, int c) {
  ColTile t;
  t.c = c;
  t.o = MODE == kOneTile ? 0u : chain / p.per_outer;
  t.g0 = (long long)(MODE == kOneTile ? chain : chain - t.o * p.per_outer) * S::TX;
  t.end = MODE == kOneTile ? 0 : (int)clamp_len(p.lengths, t.o, p.L);
  return t;
}

// A group of a tile: its outer entry, first channel and steps (0: no such group)
struct ColGroup {
  long long o;
  int i0, end;
  bool live;
};
template <typename T, class S, int MODE>
__device__ __forceinline__ ColGroup col_group(const ScanArgs<T>& p, const ColTile& t, int x) {
  ColGroup g;
  if (MODE == kOneTile) {
    const long long gid = t.g0 + x;
    g.live = gid < p.total;
    g.o = g.live ? (p.total <= 0xffffffffll ? (long long)((unsigned)gid / (unsigned)p.groups) : gid / p.groups) : 0;
    g.i0 = g.live ? (int)(gid - g.o * p.groups) * S::VEC : 0;
    g.end = g.live ? (int)clamp_len(p.lengths, g.o, p.L) : 0;
  } else {
    g.live = t.g0 + x < p.groups;
    g.o = t.o;
    g.i0 = g.live ? (int)(t.g0 + x) * S::VEC : 0;
    g.end = g.live ? t.end : 0;
  }
  return g;
}

// The chained tiles of a CTA: by ticket, the next tile's ticket drawn and its loads started while a tile is worked on (a
// held ticket waits for earlier ones only, so the earliest unfinished tile is always being worked on).
struct ColDraw {
  ColTile tile;
  unsigned chain, tag;
  int more;            // the ticket is a tile
};

template <typename T, class S, bool BACK>
__device__ __forceinline__ void draw_tile(const ScanArgs<T>& p, unsigned ticket, ColDraw* out) {
  const unsigned chains = (unsigned)p.chains;
  const unsigned n = ticket / chains;
  out->more = n < (unsigned)p.chunks;
  out->chain = ticket - n * chains;
  if (out->more) out->tile = col_tile<T, S, kColChained>(p, out->chain, BACK ? p.chunks - 1 - (int)n : (int)n);
}

template <typename T, class S, int MODE>
__global__ void __launch_bounds__(kScanThreads, S::SLOTS > 1 ? 2 : 3) scan_cols_kernel(const ScanArgs<T> p) {
  constexpr int VEC = S::VEC, R = S::R, SLOTS = S::SLOTS, W = S::W, LC = S::LC;
  constexpr bool CHAIN = MODE == kColChained;
  using Slots = ColSlots<T, S, 2>;
  __shared__ float2 runs[SLOTS > 1 ? SLOTS : 1][SLOTS > 1 ? W : 1];     // (A, H) of every run; then its first state in x
  __shared__ ColDraw drawn[2];
  __shared__ int depth_s;
  extern __shared__ __align__(16) unsigned char raw[];
  const Slots slots{raw};
  pdl_trigger();
  pdl_wait();
  ColTile tile;
  unsigned tag = 0, chain = blockIdx.x;
  bool go = true;
  if (CHAIN) {
    if (threadIdx.x == 0) {
      drawn[1].tag = *(volatile unsigned*)&p.ctrl->epoch + 1u;
      draw_tile<T, S, false>(p, atomicAdd(&p.ctrl->ticket, 1u), &drawn[1]);
    }
    __syncthreads();
    tag = drawn[1].tag, tile = drawn[1].tile, chain = drawn[1].chain, go = drawn[1].more != 0;
  } else {
    tile = col_tile<T, S, MODE>(p, chain, 0);
  }
  const int slot = threadIdx.x / S::TX, x = threadIdx.x % S::TX;
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(p.sigmoid);
  const long long states = p.outer * p.inner;
  const int lane = threadIdx.x & 31;
  const int jx = (threadIdx.x / 32) * S::CPW + lane % S::CPW, jq = lane / S::CPW * S::JOIN;   // while joining: channel, first run
  const bool first = lane < S::CPW;
  auto fetch = [&](const ColTile& t) {
    const ColGroup g = col_group<T, S, MODE>(p, t, x);
    const int t0 = t.c * LC + slot * R;
    const long long from = g.o * p.in_o + g.i0 + t0 * p.in_t;
    slots.fetch(0, p.v + from, p.in_t, g.end - t0, none_v);
    slots.fetch(1, p.g + from, p.in_t, g.end - t0, none_g);
  };
  if (go) fetch(tile);
  float state = 0.f;

#pragma unroll 1
  while (go) {
    const int c = tile.c;
    const ColGroup at = col_group<T, S, MODE>(p, tile, x);
    unsigned draw = 0;
    if (CHAIN && threadIdx.x == 0) draw = atomicAdd(&p.ctrl->ticket, 1u);
    float a[R][VEC], u[R][VEC], s[VEC];
    Slots::wait();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float gv[VEC], vv[VEC];
      slots.slot(1, r)->unpack(gv);
      slots.slot(0, r)->unpack(vv);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        terms(p.sigmoid, gv[j], a[r][j], u[r][j]);
        u[r][j] *= vv[j];
      }
    }
    ColTile next;
    unsigned next_chain = 0;
    bool more_tiles = false;
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
        runs[slot][x * VEC + j] = make_float2(A, H);
      }
      if (CHAIN && threadIdx.x == 0) draw_tile<T, S, false>(p, draw, &drawn[0]);
      __syncthreads();
      if (CHAIN) {        // the next tile's values are on their way from here on
        next = drawn[0].tile, next_chain = drawn[0].chain, more_tiles = drawn[0].more != 0;
      } else {
        next = tile;
        ++next.c;
        more_tiles = next.c < p.chunks;
      }
      if (more_tiles) fetch(next);
      const ColGroup jg = col_group<T, S, MODE>(p, tile, jx / VEC);
      const long long ch = jg.o * p.inner + jg.i0 + jx % VEC;
      if (c == 0) state = jg.live && p.h0 != nullptr ? p.h0[ch] : 0.f;
      float A = 1.f, H = 0.f;
      float2 m[S::JOIN];
#pragma unroll
      for (int q = 0; q < S::JOIN; ++q) {
        m[q] = runs[jq + q][jx];
        A *= m[q].x;
        H = fmaf(m[q].x, H, m[q].y);
      }
      const float2 all = join_lanes<S::CPW, true>(A, H);
      // a chunk in which a sequence has no step leaves its state alone, and nobody waits for it
      const bool active = c * LC < jg.end, more = (c + 1) * (long long)LC < jg.end;
      const long long entry = c * states + ch;
      if (CHAIN && c > 0 && c * LC < tile.end) {
        if (more && first) put_sum(p.sums + entry, all.x, all.y, tag);
        if (threadIdx.x < 32) {
          unsigned long long* hint = p.hints + (long long)c * p.chains + chain;
          if (threadIdx.x == 0) put_hint(hint, 1u, tag);
          const int d = poll_hints(hint - p.chains, -p.chains, c, tag);
          if (threadIdx.x == 0) {
            depth_s = d < 0 ? 0 : d;
            if (d < 0) atomicExch(p.status, 1);
          }
        }
        __syncthreads();
        state = look_back<S::CPW>(active, p.sums + entry - states, p.ends + entry - states, -states, depth_s, tag, p.status);
      }
      float run = fmaf(A, state, H);
      if (MODE != kOneTile && p.ckpt != nullptr && first && jg.live && (active || c == 0)) p.ckpt[entry] = run;
#pragma unroll
      for (int q = 0; q < S::JOIN; ++q) {
        runs[jq + q][jx].x = run;
        run = fmaf(m[q].x, run, m[q].y);
      }
      state = fmaf(all.x, state, all.y);
      if (first && jg.live) {
        if (CHAIN && more) put_end(p.ends + entry, state, tag);
        if ((active || c == 0) && !more && p.h_last != nullptr) p.h_last[ch] = state;
      }
      if (CHAIN && threadIdx.x == 0) put_hint(p.hints + (long long)c * p.chains + chain, 2u, tag);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = runs[slot][x * VEC + j].x;
    }
    const int t0 = c * LC + slot * R, left = at.live ? (int)p.L - t0 : 0;
    T* h = p.h + (at.o * p.L + t0) * p.inner + at.i0;
#pragma unroll
    for (int r = 0; r < R; ++r, h += p.inner) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = fmaf(a[r][j], s[j], u[r][j]);
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
    tile = next, chain = CHAIN ? next_chain : chain, go = more_tiles;
  }
  if (CHAIN) leave_chain(p.ctrl, tag);
}

template <typename T, class S, int MODE>
__global__ void __launch_bounds__(kScanThreads, 2) scan_cols_backward_kernel(const ScanArgs<T> p) {
  constexpr int VEC = S::VEC, R = S::R, SLOTS = S::SLOTS, W = S::W, LC = S::LC;
  constexpr bool CHAIN = MODE == kColChained;
  using Slots = ColSlots<T, S, 3>;
  // (A, H) and D of every run; then the state in front of it (x) and the gradient that comes to it from behind
  __shared__ float2 runs[SLOTS > 1 ? SLOTS : 1][SLOTS > 1 ? W : 1];
  __shared__ float backs[SLOTS > 1 ? SLOTS : 1][SLOTS > 1 ? W : 1];
  __shared__ ColDraw drawn[2];
  __shared__ int depth_s;
  extern __shared__ __align__(16) unsigned char raw[];
  const Slots slots{raw};
  pdl_trigger();
  pdl_wait();
  ColTile tile;
  unsigned tag = 0, chain = blockIdx.x;
  bool go = true;
  if (CHAIN) {
    if (threadIdx.x == 0) {
      drawn[1].tag = *(volatile unsigned*)&p.ctrl->epoch + 1u;
      draw_tile<T, S, true>(p, atomicAdd(&p.ctrl->ticket, 1u), &drawn[1]);
    }
    __syncthreads();
    tag = drawn[1].tag, tile = drawn[1].tile, chain = drawn[1].chain, go = drawn[1].more != 0;
  } else {
    tile = col_tile<T, S, MODE>(p, chain, p.chunks - 1);        // chunks from the last to the first
  }
  const int slot = threadIdx.x / S::TX, x = threadIdx.x % S::TX;
  const T none_v = Elem<T>::put(0.f), none_g = neutral_gate<T>(p.sigmoid);
  const long long states = p.outer * p.inner;
  const int lane = threadIdx.x & 31;
  const int jx = (threadIdx.x / 32) * S::CPW + lane % S::CPW, jq = lane / S::CPW * S::JOIN;   // while joining: channel, first run
  const bool first = lane < S::CPW;
  auto fetch = [&](const ColTile& t) {
    const ColGroup g = col_group<T, S, MODE>(p, t, x);
    const int t0 = t.c * LC + slot * R;
    const long long from = g.o * p.in_o + g.i0 + t0 * p.in_t;
    slots.fetch(0, p.v + from, p.in_t, g.end - t0, none_v);
    slots.fetch(1, p.g + from, p.in_t, g.end - t0, none_g);
    slots.fetch(2, p.gh + (g.o * p.L + t0) * p.inner + g.i0, p.inner, g.end - t0, none_v);
  };
  if (go) fetch(tile);
  float grad = 0.f;

#pragma unroll 1
  while (go) {
    const int c = tile.c;
    const ColGroup at = col_group<T, S, MODE>(p, tile, x);
    unsigned draw = 0;
    if (CHAIN && threadIdx.x == 0) draw = atomicAdd(&p.ctrl->ticket, 1u);
    const ColGroup jg = col_group<T, S, MODE>(p, tile, jx / VEC);
    const long long ch = jg.o * p.inner + jg.i0 + jx % VEC, entry = c * states + ch;
    const int last = jg.end > 0 ? (jg.end - 1) / LC : 0;     // the chunk of the sequence's last step
    const bool active = c * LC < jg.end, mine = SLOTS > 1 && jg.live && (active || c == 0);
    float before = 0.f;      // the state in front of the chunk: saved, or the sequence's own beginning
    if (mine) {
      if (MODE != kOneTile && p.ckpt != nullptr) before = p.ckpt[entry];
      else if (p.h0 != nullptr) before = p.h0[ch];
      if (c >= last) grad = p.g_last != nullptr ? p.g_last[ch] : 0.f;
    }
    Slots::wait();
    // q: 1 - a (sigmoid) or a (decay); a is formed again where it is used
    float q[R][VEC], v[R][VEC], s[VEC], d[VEC];
    Pack<T, VEC> pd[R];
    const float ka = p.sigmoid ? -1.f : 1.f, kb = p.sigmoid ? 1.f : 0.f;
    auto a_of = [&](float qq) { return fmaf(qq, ka, kb); };
    auto b_of = [&](float qq) { return p.sigmoid ? qq : 1.f; };
#pragma unroll
    for (int r = 0; r < R; ++r) {
      pd[r] = *slots.slot(2, r);
      slots.slot(1, r)->unpack(q[r]);
      slots.slot(0, r)->unpack(v[r]);
      if (p.sigmoid) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          float a;
          gate_of(q[r][j], a, q[r][j]);
        }
      }
    }
    ColTile next;
    unsigned next_chain = 0;
    bool more_tiles = false;
    if constexpr (SLOTS == 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        s[j] = at.live && p.h0 != nullptr ? p.h0[at.o * p.inner + at.i0 + j] : 0.f;
        d[j] = at.live && p.g_last != nullptr ? p.g_last[at.o * p.inner + at.i0 + j] : 0.f;
      }
    } else {
      float D[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float A = 1.f, H = 0.f;
        D[j] = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float a = a_of(q[r][j]);
          A *= a;
          H = fmaf(a, H, b_of(q[r][j]) * v[r][j]);
        }
        runs[slot][x * VEC + j] = make_float2(A, H);
      }
#pragma unroll
      for (int r = R - 1; r >= 0; --r) {
        float gh[VEC];
        pd[r].unpack(gh);
#pragma unroll
        for (int j = 0; j < VEC; ++j) D[j] = a_of(q[r][j]) * (D[j] + gh[j]);
      }
#pragma unroll
      for (int j = 0; j < VEC; ++j) backs[slot][x * VEC + j] = D[j];
      if (CHAIN && threadIdx.x == 0) draw_tile<T, S, true>(p, draw, &drawn[0]);
      __syncthreads();
      if (CHAIN) {        // the next tile's values are on their way from here on
        next = drawn[0].tile, next_chain = drawn[0].chain, more_tiles = drawn[0].more != 0;
      } else {
        next = tile;
        --next.c;
        more_tiles = next.c >= 0;
      }
      if (more_tiles) fetch(next);
      float A = 1.f, H = 0.f, B = 1.f, E = 0.f;
      float2 m[S::JOIN];
      float md[S::JOIN];
#pragma unroll
      for (int k = 0; k < S::JOIN; ++k) {
        m[k] = runs[jq + k][jx];
        md[k] = backs[jq + k][jx];
        A *= m[k].x;
        H = fmaf(m[k].x, H, m[k].y);
      }
#pragma unroll
      for (int k = S::JOIN - 1; k >= 0; --k) E = fmaf(m[k].x, E, md[k]);
      B = A;
      join_lanes<S::CPW, true>(A, H);
      const float2 all = join_lanes<S::CPW, false>(B, E);
      if (CHAIN && tile.end > 0 && c < (tile.end - 1) / LC) {
        if (jg.live && c > 0 && first) put_sum(p.sums + entry, all.x, all.y, tag);
        if (threadIdx.x < 32) {
          unsigned long long* hint = p.hints + (long long)c * p.chains + chain;
          if (threadIdx.x == 0) put_hint(hint, 1u, tag);
          const int n = (tile.end - 1) / LC - c;
          const int dd = poll_hints(hint + p.chains, p.chains, n, tag);
          if (threadIdx.x == 0) {
            depth_s = dd < 0 ? 0 : dd;
            if (dd < 0) atomicExch(p.status, 1);
          }
        }
        __syncthreads();
        grad = look_back<S::CPW>(jg.live, p.sums + entry + states, p.ends + entry + states, states, depth_s, tag, p.status);
      }
      float run = fmaf(A, before, H);
#pragma unroll
      for (int k = 0; k < S::JOIN; ++k) {
        runs[jq + k][jx].x = run;
        run = fmaf(m[k].x, run, m[k].y);
      }
      run = fmaf(B, grad, E);
#pragma unroll
      for (int k = S::JOIN - 1; k >= 0; --k) {
        backs[jq + k][jx] = run;
        run = fmaf(m[k].x, run, md[k]);
      }
      if (mine) grad = fmaf(all.x, grad, all.y);
      if (mine && first) {
        if (CHAIN && c > 0) put_end(p.ends + entry, grad, tag);
        if (c == 0 && p.gh0 != nullptr) p.gh0[ch] = grad;
      }
      if (CHAIN && threadIdx.x == 0) put_hint(p.hints + (long long)c * p.chains + chain, 2u, tag);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = runs[slot][x * VEC + j].x, d[j] = backs[slot][x * VEC + j];
    }
    // forward once more: v is replaced by what delta is multiplied with for the gate's gradient
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float a = a_of(q[r][j]), u = b_of(q[r][j]) * v[r][j];
        v[r][j] = p.sigmoid ? (s[j] - v[r][j]) * (a * q[r][j]) : s[j];
        s[j] = fmaf(a, s[j], u);
      }
    const int t0 = c * LC + slot * R, left = at.live ? (int)p.L - t0 : 0;
    const long long back = at.o * p.gr_o + at.i0 + (t0 + R - 1) * p.gr_t;
    T *gv = p.gv + back, *gg = p.gg + back;
#pragma unroll
    for (int r = R - 1; r >= 0; --r, gv -= p.gr_t, gg -= p.gr_t) {
      float x1[VEC], x2[VEC];
      pd[r].unpack(x1);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float delta = d[j] + x1[j];
        x1[j] = delta * b_of(q[r][j]);
        x2[j] = delta * v[r][j];
        d[j] = a_of(q[r][j]) * delta;
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
    tile = next, chain = CHAIN ? next_chain : chain, go = more_tiles;
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
  p.hints = p.ends + (long long)p.chunks * c.outer * c.inner;
  p.status = reinterpret_cast<int*>(ws);
}

template <typename T, class S, int MODE, bool BACK>
cudaError_t launch_cols_kernel(const ScanArgs<T>& p, cudaStream_t st) {
  void (*kern)(const ScanArgs<T>);
  constexpr size_t smem = ColSlots<T, S, BACK ? 3 : 2>::SMEM;
  if constexpr (BACK) kern = scan_cols_backward_kernel<T, S, MODE>;
  else kern = scan_cols_kernel<T, S, MODE>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kern), smem + 4096 + sizeof(float) * 3 * S::SLOTS * S::W, allowed);
  if (e != cudaSuccess) return e;
  long long ctas = p.chains;
  if (MODE == kColChained) {       // as many CTAs as run at once (only a running CTA draws tickets, so none has to)
    const long long most = 2 * (long long)num_sms();
    ctas = p.chains * p.chunks < most ? p.chains * p.chunks : most;
  }
  return launch_pdl(kern, dim3((unsigned)ctas), dim3(kScanThreads), smem, st, p);
}

// sequences that fit one tile
template <typename T, class S, bool BACK>
cudaError_t launch_short_cols(ScanArgs<T> p, cudaStream_t st) {
  p.total = p.outer * p.groups;
  p.chains = (p.total + S::TX - 1) / S::TX;
  p.chunks = 1;
  return launch_cols_kernel<T, S, kOneTile, BACK>(p, st);
}
template <typename T, class S, bool BACK>
cudaError_t launch_long_cols(ScanArgs<T> p, const ScanCall& c, cudaStream_t st) {
  static_assert(S::LC == kColTile, "tiles end where states are saved");
  const long long per_outer = (p.groups + S::TX - 1) / S::TX;
  p.per_outer = (unsigned)per_outer;
  p.chains = p.outer * per_outer;
  if (p.chains > 0x7fffffff) return cudaErrorNotSupported;
  p.chunks = (int)((p.L + S::LC - 1) / S::LC);
  if (chained(p.chains, p.chunks, p.chains * p.chunks)) {
    chain(p, c);
    return launch_cols_kernel<T, S, kColChained, BACK>(p, st);
  }
  return launch_cols_kernel<T, S, kColWalk, BACK>(p, st);
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
  if (vec) {
    if (c.length <= 8) return launch_short_cols<T, ColShape<4, 8, 1>, BACK>(p, st);
    if (c.length <= 64) return launch_short_cols<T, ColShape<4, 8, 8>, BACK>(p, st);
    return launch_long_cols<T, ColShape<4, 8, 32>, BACK>(p, c, st);
  }
  if (c.length <= 8) return launch_short_cols<T, ColShape<1, 8, 1>, BACK>(p, st);
  if (c.length <= 64) return launch_short_cols<T, ColShape<1, 8, 8>, BACK>(p, st);
  return launch_long_cols<T, ColShape<1, 32, 8>, BACK>(p, c, st);
}

}  // namespace

// States are saved every 256 steps of [outer][L][inner] sequences, every 512 (or 504) of contiguous ones - or once, in
// front of a sequence that fits one tile.
long long scan_chunk(int, long long length, long long inner) {
  const long long lc = inner == 1 ? row_chunk(length) : kColTile;
  return length <= lc ? (length < 1 ? 1 : length) : lc;
}

size_t scan_workspace_bytes(int dtype, long long outer, long long length, long long inner) {
  const long long lc = scan_chunk(dtype, length, inner), chunks = (length + lc - 1) / lc;
  if (chunks < 2) return kStatusBytes;
  return kChainHead + (size_t)chunks * (size_t)outer * (size_t)inner * (sizeof(ulonglong2) + 2 * sizeof(unsigned long long));   // (at most one hint per state)
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
