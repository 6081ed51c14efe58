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

template <typename T>
struct ScanArgs {
  const T *v, *g, *gh;
  const float *h0, *g_last;
  const int* lengths;
  T *h, *gv, *gg;
  float *h_last, *gh0, *ckpt;
  long long outer, L, inner, groups, total;     // groups of VEC channels per outer entry, outer * groups
  long long in_o, in_t, gr_o, gr_t;
  int chunks, sigmoid;
};

// a = 1 / (1 + e^-g) and b = 1 - a, each formed without cancellation
__device__ __forceinline__ void gate_of(float g, float& a, float& b) {
  const float e = __expf(-fabsf(g));
  const float r = __fdividef(1.0f, 1.0f + e);
  a = g >= 0.f ? r : e * r;
  b = g >= 0.f ? e * r : r;
}

// Steps per thread: as many bytes for every type and width, and the same steps per tile (64 fp32, 128 of 16 bits)
// for both widths, since the tile is what a saved state belongs to.
template <typename T>
constexpr int kSteps4 = sizeof(T) == 4 ? 4 : 8;

__device__ __forceinline__ long long clamp_len(const int* lengths, long long o, long long L) {
  if (lengths == nullptr) return L;
  const long long n = lengths[o];
  return n < 0 ? 0 : (n < L ? n : L);
}

// ------------------------------------------------------------------------------------------------ columns
// [outer][L][inner], inner contiguous.  A CTA holds 256 / SLOTS groups of VEC channels (groups run on across outer
// entries) and SLOTS * R steps; it walks along L with the state in shared memory.
template <typename T, int VEC, int R, int SLOTS>
__global__ void __launch_bounds__(kScanThreads) scan_cols_kernel(const ScanArgs<T> p) {
  constexpr int TX = kScanThreads / SLOTS, W = TX * VEC, LC = SLOTS * R;
  __shared__ float sA[2][SLOTS][W], sH[2][SLOTS][W], carry[2][W];
  pdl_trigger();
  pdl_wait();
  const int x = threadIdx.x % TX, slot = threadIdx.x / TX;
  const long long gid = (long long)blockIdx.x * TX + x;
  const bool live = gid < p.total;
  const long long o = live ? gid / p.groups : 0, i0 = live ? (gid % p.groups) * VEC : 0;
  const long long f0 = o * p.inner + i0;                   // first of this thread's channels among all states
  const long long end = live ? clamp_len(p.lengths, o, p.L) : 0;
  const T* v = p.v + o * p.in_o + i0;
  const T* g = p.g + o * p.in_o + i0;
  T* h = p.h + o * p.L * p.inner + i0;
  if (slot == 0) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) carry[0][x * VEC + j] = live && p.h0 != nullptr ? p.h0[f0 + j] : 0.f;
  }
  for (int c = 0; c < p.chunks; ++c) {
    const long long t0 = (long long)c * LC + slot * R;
    Pack<T, VEC> pv[R], pg[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (t0 + r < end) {
        pv[r].load(v + (t0 + r) * p.in_t);
        pg[r].load(g + (t0 + r) * p.in_t);
      }
    float a[R][VEC], u[R][VEC], A[VEC], H[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) A[j] = 1.f, H[j] = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        a[r][j] = 1.f, u[r][j] = 0.f;
        if (t0 + r < end) {
          if (p.sigmoid) {
            float b;
            gate_of(pg[r].get(j), a[r][j], b);
            u[r][j] = b * pv[r].get(j);
          } else {
            a[r][j] = pg[r].get(j), u[r][j] = pv[r].get(j);
          }
        }
        A[j] *= a[r][j];
        H[j] = fmaf(a[r][j], H[j], u[r][j]);
      }
    const int buf = c & 1;
#pragma unroll
    for (int j = 0; j < VEC; ++j) sA[buf][slot][x * VEC + j] = A[j], sH[buf][slot][x * VEC + j] = H[j];
    __syncthreads();
    float s[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) s[j] = carry[buf][x * VEC + j];
    if (slot == 0 && live && p.ckpt != nullptr) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) p.ckpt[(long long)c * p.outer * p.inner + f0 + j] = s[j];
    }
    for (int q = 0; q < slot; ++q)
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = fmaf(sA[buf][q][x * VEC + j], s[j], sH[buf][q][x * VEC + j]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      Pack<T, VEC> out;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        s[j] = fmaf(a[r][j], s[j], u[r][j]);
        out.put(j, t0 + r < end ? s[j] : 0.f);
      }
      if (live && t0 + r < p.L) out.store(h + (t0 + r) * p.inner);
    }
    if (slot == SLOTS - 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) carry[buf ^ 1][x * VEC + j] = s[j];
      if (c == p.chunks - 1 && live && p.h_last != nullptr) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.h_last[f0 + j] = s[j];
      }
    }
  }
}

template <typename T, int VEC, int R, int SLOTS>
__global__ void __launch_bounds__(kScanThreads) scan_cols_backward_kernel(const ScanArgs<T> p) {
  constexpr int TX = kScanThreads / SLOTS, W = TX * VEC, LC = SLOTS * R;
  __shared__ float sA[2][SLOTS][W], sH[2][SLOTS][W], sD[2][SLOTS][W], carry[2][W];
  pdl_trigger();
  pdl_wait();
  const int x = threadIdx.x % TX, slot = threadIdx.x / TX;
  const long long gid = (long long)blockIdx.x * TX + x;
  const bool live = gid < p.total;
  const long long o = live ? gid / p.groups : 0, i0 = live ? (gid % p.groups) * VEC : 0;
  const long long f0 = o * p.inner + i0;
  const long long end = live ? clamp_len(p.lengths, o, p.L) : 0;
  const T* v = p.v + o * p.in_o + i0;
  const T* g = p.g + o * p.in_o + i0;
  const T* gh = p.gh + o * p.L * p.inner + i0;
  T* gv = p.gv + o * p.gr_o + i0;
  T* gg = p.gg + o * p.gr_o + i0;
  if (slot == 0) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) carry[0][x * VEC + j] = live && p.g_last != nullptr ? p.g_last[f0 + j] : 0.f;
  }
  for (int n = 0; n < p.chunks; ++n) {
    const int c = p.chunks - 1 - n;
    const long long t0 = (long long)c * LC + slot * R;
    Pack<T, VEC> pv[R], pg[R], pd[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (t0 + r < end) {
        pv[r].load(v + (t0 + r) * p.in_t);
        pg[r].load(g + (t0 + r) * p.in_t);
        pd[r].load(gh + (t0 + r) * p.inner);
      }
    float a[R][VEC], w[R][VEC], A[VEC], H[VEC], D[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) A[j] = 1.f, H[j] = 0.f, D[j] = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        a[r][j] = 1.f, w[r][j] = 0.f;
        if (t0 + r < end) {
          if (p.sigmoid) {
            float b;
            gate_of(pg[r].get(j), a[r][j], b);
            w[r][j] = b * pv[r].get(j);
          } else {
            a[r][j] = pg[r].get(j), w[r][j] = pv[r].get(j);
          }
        }
        A[j] *= a[r][j];
        H[j] = fmaf(a[r][j], H[j], w[r][j]);
      }
#pragma unroll
    for (int r = R - 1; r >= 0; --r)
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        D[j] = a[r][j] * (D[j] + (t0 + r < end ? pd[r].get(j) : 0.f));
    const int buf = n & 1;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      sA[buf][slot][x * VEC + j] = A[j], sH[buf][slot][x * VEC + j] = H[j], sD[buf][slot][x * VEC + j] = D[j];
    }
    // the state in front of the chunk: saved, or the sequence's own beginning
    const float* before = p.ckpt != nullptr ? p.ckpt + (long long)c * p.outer * p.inner : p.h0;
    float s[VEC], d[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) s[j] = live && before != nullptr ? before[f0 + j] : 0.f;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < VEC; ++j) d[j] = carry[buf][x * VEC + j];
    for (int q = 0; q < slot; ++q)
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] = fmaf(sA[buf][q][x * VEC + j], s[j], sH[buf][q][x * VEC + j]);
    for (int q = SLOTS - 1; q > slot; --q)
#pragma unroll
      for (int j = 0; j < VEC; ++j) d[j] = fmaf(sA[buf][q][x * VEC + j], d[j], sD[buf][q][x * VEC + j]);
    // forward once more: u is replaced by what delta is multiplied with for the gate's gradient
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float u = w[r][j];
        if (t0 + r < end) {
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
#pragma unroll
    for (int r = R - 1; r >= 0; --r) {
      Pack<T, VEC> ov, og;
      ov.zero();
      og.zero();
      if (t0 + r < end) {
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
      if (live && t0 + r < p.L) {
        ov.store(gv + (t0 + r) * p.gr_t);
        og.store(gg + (t0 + r) * p.gr_t);
      }
    }
    if (slot == 0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) carry[buf ^ 1][x * VEC + j] = d[j];
      if (c == 0 && live && p.gh0 != nullptr) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.gh0[f0 + j] = d[j];
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ rows
// [outer][L], the steps contiguous.  P neighbouring lanes share a row, 16 steps each; tiles come and go through
// shared memory (pitch 17: conflict-free both ways), the lanes' runs are joined by shuffles.
constexpr int kRowSteps = 16, kRowPitch = kRowSteps + 1;

// element e of a tile of rows x n steps -> its place in shared memory (n <= 16 P, P lanes a row)
struct TileMap {
  uint32_t n, magic;   // division by n through the high word of a product (e < 2^16)
  int lanes;
  __device__ __forceinline__ TileMap(uint32_t n_, int lanes_) : n(n_), magic(0xffffffffu / n_ + 1u), lanes(lanes_) {}
  __device__ __forceinline__ void split(uint32_t e, uint32_t& row, uint32_t& t) const {
    row = n == 1 ? e : __umulhi(e, magic);
    t = e - row * n;
  }
  __device__ __forceinline__ uint32_t place(uint32_t row, uint32_t t) const {
    return (row * lanes + t / kRowSteps) * kRowPitch + t % kRowSteps;
  }
};

template <typename T>
__device__ __forceinline__ void tile_in(float* dst, const T* src, long long row_stride, uint32_t rows, const TileMap& m) {
  for (uint32_t e = threadIdx.x; e < rows * m.n; e += kScanThreads) {
    uint32_t row, t;
    m.split(e, row, t);
    dst[m.place(row, t)] = Elem<T>::get(src[row * row_stride + t]);
  }
}
template <typename T>
__device__ __forceinline__ void tile_out(T* dst, const float* src, long long row_stride, uint32_t rows, const TileMap& m) {
  for (uint32_t e = threadIdx.x; e < rows * m.n; e += kScanThreads) {
    uint32_t row, t;
    m.split(e, row, t);
    dst[row * row_stride + t] = Elem<T>::put(src[m.place(row, t)]);
  }
}

template <typename T, int P>
__global__ void __launch_bounds__(kScanThreads) scan_rows_kernel(const ScanArgs<T> p) {
  constexpr int ROWS = kScanThreads / P, LC = P * kRowSteps;
  __shared__ float sv[kScanThreads * kRowPitch], sg[kScanThreads * kRowPitch];
  pdl_trigger();
  pdl_wait();
  const int slot = threadIdx.x % P;
  const long long r0 = (long long)blockIdx.x * ROWS, row = r0 + threadIdx.x / P;
  const uint32_t rows = (uint32_t)(p.outer - r0 < ROWS ? p.outer - r0 : ROWS);
  const bool live = row < p.outer;
  const long long end = live ? clamp_len(p.lengths, row, p.L) : 0;
  float carry = live && p.h0 != nullptr ? p.h0[row] : 0.f;
  for (int c = 0; c < p.chunks; ++c) {
    const long long t0 = (long long)c * LC;
    const TileMap m((uint32_t)(p.L - t0 < LC ? p.L - t0 : LC), P);
    tile_in(sv, p.v + r0 * p.in_o + t0, p.in_o, rows, m);
    tile_in(sg, p.g + r0 * p.in_o + t0, p.in_o, rows, m);
    __syncthreads();
    float a[kRowSteps], u[kRowSteps], A = 1.f, H = 0.f;
    const long long ts = t0 + slot * kRowSteps;
#pragma unroll
    for (int r = 0; r < kRowSteps; ++r) {
      a[r] = 1.f, u[r] = 0.f;
      if (ts + r < end) {
        const float gx = sg[threadIdx.x * kRowPitch + r], vx = sv[threadIdx.x * kRowPitch + r];
        if (p.sigmoid) {
          float b;
          gate_of(gx, a[r], b);
          u[r] = b * vx;
        } else {
          a[r] = gx, u[r] = vx;
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
    if (p.ckpt != nullptr && live && slot == 0) p.ckpt[(long long)c * p.outer + row] = carry;
    const float full = fmaf(A, carry, H);                  // the state behind this lane's run
    float s = __shfl_up_sync(0xffffffffu, full, 1, P);
    if (slot == 0) s = carry;
    carry = __shfl_sync(0xffffffffu, full, P - 1, P);
#pragma unroll
    for (int r = 0; r < kRowSteps; ++r) {
      s = fmaf(a[r], s, u[r]);
      sv[threadIdx.x * kRowPitch + r] = ts + r < end ? s : 0.f;
    }
    __syncthreads();
    tile_out(p.h + r0 * p.L + t0, sv, p.L, rows, m);
    __syncthreads();
  }
  if (live && slot == 0 && p.h_last != nullptr) p.h_last[row] = carry;
}

template <typename T, int P>
__global__ void __launch_bounds__(kScanThreads) scan_rows_backward_kernel(const ScanArgs<T> p) {
  constexpr int ROWS = kScanThreads / P, LC = P * kRowSteps;
  extern __shared__ float tiles[];
  float* sv = tiles;
  float* sg = sv + kScanThreads * kRowPitch;
  float* sd = sg + kScanThreads * kRowPitch;
  pdl_trigger();
  pdl_wait();
  const int slot = threadIdx.x % P;
  const long long r0 = (long long)blockIdx.x * ROWS, row = r0 + threadIdx.x / P;
  const uint32_t rows = (uint32_t)(p.outer - r0 < ROWS ? p.outer - r0 : ROWS);
  const bool live = row < p.outer;
  const long long end = live ? clamp_len(p.lengths, row, p.L) : 0;
  float carry = live && p.g_last != nullptr ? p.g_last[row] : 0.f;
  float* mv = sv + threadIdx.x * kRowPitch;
  float* mg = sg + threadIdx.x * kRowPitch;
  float* md = sd + threadIdx.x * kRowPitch;
  for (int c = p.chunks - 1; c >= 0; --c) {
    const long long t0 = (long long)c * LC;
    const TileMap m((uint32_t)(p.L - t0 < LC ? p.L - t0 : LC), P);
    tile_in(sv, p.v + r0 * p.in_o + t0, p.in_o, rows, m);
    tile_in(sg, p.g + r0 * p.in_o + t0, p.in_o, rows, m);
    tile_in(sd, p.gh + r0 * p.L + t0, p.L, rows, m);
    const float* before = p.ckpt != nullptr ? p.ckpt + (long long)c * p.outer : p.h0;
    const float start = live && before != nullptr ? before[row] : 0.f;
    __syncthreads();
    float a[kRowSteps], w[kRowSteps], A = 1.f, H = 0.f, D = 0.f;
    const long long ts = t0 + slot * kRowSteps;
#pragma unroll
    for (int r = 0; r < kRowSteps; ++r) {
      a[r] = 1.f, w[r] = 0.f;
      if (ts + r < end) {
        if (p.sigmoid) {
          float b;
          gate_of(mg[r], a[r], b);
          w[r] = b * mv[r];
        } else {
          a[r] = mg[r], w[r] = mv[r];
        }
      }
      A *= a[r];
      H = fmaf(a[r], H, w[r]);
    }
#pragma unroll
    for (int r = kRowSteps - 1; r >= 0; --r) D = a[r] * (D + (ts + r < end ? md[r] : 0.f));
    float Af = A, Ab = A;
#pragma unroll
    for (int k = 1; k < P; k *= 2) {
      const float A1 = __shfl_up_sync(0xffffffffu, Af, k, P), H1 = __shfl_up_sync(0xffffffffu, H, k, P);
      const float A2 = __shfl_down_sync(0xffffffffu, Ab, k, P), D2 = __shfl_down_sync(0xffffffffu, D, k, P);
      if (slot >= k) H = fmaf(Af, H1, H), Af *= A1;
      if (slot + k < P) D = fmaf(Ab, D2, D), Ab *= A2;
    }
    float s = __shfl_up_sync(0xffffffffu, fmaf(Af, start, H), 1, P);
    if (slot == 0) s = start;
    const float all = fmaf(Ab, carry, D);
    float d = __shfl_down_sync(0xffffffffu, all, 1, P);
    if (slot == P - 1) d = carry;
    carry = __shfl_sync(0xffffffffu, all, 0, P);
#pragma unroll
    for (int r = 0; r < kRowSteps; ++r) {
      const float u = w[r];
      if (ts + r < end) {
        if (p.sigmoid) {
          float aa, b;
          gate_of(mg[r], aa, b);
          w[r] = (s - mv[r]) * aa * b;
          mg[r] = b;
        } else {
          w[r] = s;
          mg[r] = 1.f;
        }
      }
      s = fmaf(a[r], s, u);
    }
#pragma unroll
    for (int r = kRowSteps - 1; r >= 0; --r) {
      const bool on = ts + r < end;
      const float delta = d + (on ? md[r] : 0.f);
      mv[r] = on ? delta * mg[r] : 0.f;
      mg[r] = on ? delta * w[r] : 0.f;
      d = a[r] * delta;
    }
    __syncthreads();
    tile_out(p.gv + r0 * p.gr_o + t0, sv, p.gr_o, rows, m);
    tile_out(p.gg + r0 * p.gr_o + t0, sg, p.gr_o, rows, m);
    __syncthreads();
  }
  if (live && slot == 0 && p.gh0 != nullptr) p.gh0[row] = carry;
}

// length 0: the state passes through
__global__ void __launch_bounds__(256) scan_copy_kernel(const float* __restrict__ in, float* __restrict__ out, long long n) {
  pdl_trigger();
  pdl_wait();
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256)
    out[i] = in != nullptr ? in[i] : 0.f;
}

template <typename T>
ScanArgs<T> scan_args(const ScanCall& c) {
  ScanArgs<T> p{};
  p.v = static_cast<const T*>(c.v), p.g = static_cast<const T*>(c.g), p.gh = static_cast<const T*>(c.grad_h);
  p.h0 = c.h0, p.g_last = c.grad_last, p.lengths = c.lengths;
  p.h = static_cast<T*>(c.h), p.gv = static_cast<T*>(c.grad_v), p.gg = static_cast<T*>(c.grad_g);
  p.h_last = c.h_last, p.gh0 = c.grad_h0, p.ckpt = c.checkpoints;
  p.outer = c.outer, p.L = c.length, p.inner = c.inner;
  p.in_o = c.in_outer, p.in_t = c.in_step, p.gr_o = c.grad_outer, p.gr_t = c.grad_step;
  p.sigmoid = c.gate == DTST_GATE_SIGMOID;
  const long long lc = scan_chunk(c.dtype, c.length, c.inner);
  p.chunks = (int)((c.length + lc - 1) / lc);
  return p;
}

int row_lanes(long long length) {
  int P = 1;
  while (P < 32 && P * kRowSteps < length) P *= 2;
  return P;
}

template <typename T, bool BACK>
cudaError_t scan_t(const ScanCall& c, cudaStream_t st) {
  ScanArgs<T> p = scan_args<T>(c);
  if (c.inner == 1) {
    const int P = row_lanes(c.length);
    const long long rows = kScanThreads / P;
    const dim3 grid((unsigned)((c.outer + rows - 1) / rows)), block(kScanThreads);
    const size_t smem = BACK ? 3 * sizeof(float) * kScanThreads * kRowPitch : 0;
#define DTST_SCAN_ROWS(N)                                                                                         \
  if (P == N) {                                                                                                   \
    if (!BACK) return launch_pdl(scan_rows_kernel<T, N>, grid, block, 0, st, p);                                  \
    cudaError_t e = cudaFuncSetAttribute(scan_rows_backward_kernel<T, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); \
    return e != cudaSuccess ? e : launch_pdl(scan_rows_backward_kernel<T, N>, grid, block, smem, st, p);          \
  }
    DTST_SCAN_ROWS(1)
    DTST_SCAN_ROWS(2)
    DTST_SCAN_ROWS(4)
    DTST_SCAN_ROWS(8)
    DTST_SCAN_ROWS(16)
    DTST_SCAN_ROWS(32)
#undef DTST_SCAN_ROWS
    return cudaErrorNotSupported;
  }
  constexpr int R4 = kSteps4<T>;
  const size_t need = 4 * sizeof(T);
  bool vec = c.inner % 4 == 0 && c.in_outer % 4 == 0 && c.in_step % 4 == 0 && aligned_to(c.v, need) && aligned_to(c.g, need);
  if (BACK) vec = vec && c.grad_outer % 4 == 0 && c.grad_step % 4 == 0 && aligned_to(c.grad_h, need) && aligned_to(c.grad_v, need) && aligned_to(c.grad_g, need);
  else vec = vec && aligned_to(c.h, need);
  p.groups = vec ? c.inner / 4 : c.inner;
  p.total = c.outer * p.groups;
#define DTST_SCAN_COLS(VEC, R, SLOTS)                                                                             \
  {                                                                                                               \
    constexpr int TX = kScanThreads / SLOTS;                                                                      \
    const dim3 grid((unsigned)((p.total + TX - 1) / TX)), block(kScanThreads);                                    \
    return BACK ? launch_pdl(scan_cols_backward_kernel<T, VEC, R, SLOTS>, grid, block, 0, st, p)                  \
                : launch_pdl(scan_cols_kernel<T, VEC, R, SLOTS>, grid, block, 0, st, p);                          \
  }
  if (vec) {
    if (c.length <= R4) DTST_SCAN_COLS(4, R4, 1)
    if (c.length <= 4 * R4) DTST_SCAN_COLS(4, R4, 4)
    DTST_SCAN_COLS(4, R4, 16)
  }
  if (c.length <= R4) DTST_SCAN_COLS(1, 2 * R4, 1)
  if (c.length <= 4 * R4) DTST_SCAN_COLS(1, 2 * R4, 2)
  DTST_SCAN_COLS(1, 2 * R4, 8)
#undef DTST_SCAN_COLS
}

}  // namespace

long long scan_chunk(int dtype, long long length, long long inner) {
  const long long lc = inner == 1 ? 16 * row_lanes(length) : dtype == DTST_F32 ? 64 : 128;
  return length <= lc ? (length < 1 ? 1 : length) : lc;
}

size_t scan_workspace_bytes(int, long long, long long, long long) { return kStatusBytes; }

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
