// Layer norm over channels, with the residual's addition in front:
//     s = x + r,   m = mean_c s,   rstd = 1 / sqrt(mean_c (s - m)^2 + eps),   n = (s - m) rstd,   y = n w + b
// and its backward pass, with g = w gy:
//     grad_x = rstd (g - mean_c g - n mean_c(g n)) + grad_s,   grad_w = sum over positions of gy n,   grad_b = sum of gy
// (the gradient of the residual is the same tensor).  Everything is in 32 bits; y is formed from the unrounded sum.  The
// variance is that of the differences from the mean, formed once the mean is known: a mean that is large next to the spread
// costs it no bits, which the mean of squares less the square of the mean would.
//
// Bound by memory.  The layouts are those of the root-mean-square norm: rows held by 32..512 threads in registers, the next
// row's loads under way while a row is summed; channels-first fields with the positions along the lanes and the channels
// spread over warps.  Against that norm a row takes two sums one after the other forward (mean, then variance) and two at
// once backward.  Rows and fields beyond the registers are read again for every sum.
// The parameters' gradients are summed in registers over all positions that a CTA visits and in a fixed order over CTAs
// by a second launch: same bits on every run.
#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_norm.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

// two sums at once
template <int TPR, int GROUPS>
__device__ __forceinline__ float2 row_sum2(float2 v, float2* red, int& phase) {
  v.x = warp_sum(v.x), v.y = warp_sum(v.y);
  if constexpr (TPR > 32) {
    constexpr int N = TPR / 32;
    const int group = GROUPS > 1 ? threadIdx.x / TPR : 0;
    float2* r = red + (phase * GROUPS + group) * N;
    phase ^= 1;
    if ((threadIdx.x & 31) == 0) r[(threadIdx.x % TPR) >> 5] = v;
    if constexpr (GROUPS > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
    else __syncthreads();
    float2 t = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i) t.x += r[i].x, t.y += r[i].y;
    v = t;
  }
  return v;
}

struct RowArgs {
  const void *x, *residual;
  const float *weight, *bias;
  void *s, *low, *y;        // low: what rounding took from s (16-bit types; may be null)
  float *mean, *rstd;
  long long rows, C;
  float eps;
};

template <typename T, int TPR, int ITEMS, int LAY>
__global__ void __launch_bounds__(kRowThreads<TPR>) layer_norm_rows_kernel(const RowArgs a) {
  constexpr int VEC = kVec<T>;
  constexpr int RPC = kRowThreads<TPR> / TPR;
  __shared__ float red[64];
  pdl_trigger();
  pdl_wait();
  const int tr = threadIdx.x % TPR;
  const float inv_c = 1.0f / (float)a.C;
  const T* x = static_cast<const T*>(a.x);
  const T* res = static_cast<const T*>(a.residual);
  const long long group = (long long)blockIdx.x * RPC + threadIdx.x / TPR, step = (long long)gridDim.x * RPC;
  const int shift = LAY == kShifted ? (int)(group * a.C % VEC) : 0;
  const long long c0 = (long long)tr * VEC - shift;
  Pack<T, VEC> px[ITEMS], pr[ITEMS];
  auto fetch = [&](long long row) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) load_group<T, LAY>(px[k], x + row * a.C, c0 + k * TPR * VEC, a.C);
    if (res != nullptr) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) load_group<T, LAY>(pr[k], res + row * a.C, c0 + k * TPR * VEC, a.C);
    }
  };
  if (group < a.rows) fetch(group);
  float w[ITEMS][VEC], b[ITEMS][VEC];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    load_weights<VEC>(w[k], a.weight, c0 + k * TPR * VEC, a.C, LAY == kAligned);
    if (a.bias != nullptr) {
      load_weights<VEC>(b[k], a.bias, c0 + k * TPR * VEC, a.C, LAY == kAligned);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) b[k][i] = 0.f;
    }
  }
  int phase = 0;
  for (long long row = group; row < a.rows; row += step) {
    float v[ITEMS][VEC];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      px[k].unpack(v[k]);
      if (res != nullptr) {
        float r[VEC];
        pr[k].unpack(r);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[k][i] += r[i];
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) sum += v[k][i];
    }
    if (row + step < a.rows) fetch(row + step);
    if (a.s != nullptr) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        Pack<T, VEC> out;
        out.pack(v[k]);
        store_group<T, LAY>(out, static_cast<T*>(a.s) + row * a.C, c0 + k * TPR * VEC, a.C);
        if (sizeof(T) == 2 && a.low != nullptr) {
          Pack<T, VEC> lo;
#pragma unroll
          for (int i = 0; i < VEC; ++i) lo.v[i] = LowBits<T>::take(v[k][i], out.v[i]);
          store_group<T, LAY>(lo, static_cast<T*>(a.low) + row * a.C, c0 + k * TPR * VEC, a.C);
        }
      }
    }
    const float mean = row_sum<TPR, RPC>(sum, red, phase) * inv_c;
    float var = 0.f;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const long long c = c0 + k * TPR * VEC + i;
        v[k][i] -= mean;
        // (places outside the row hold zeros, which are no differences from the mean)
        if (LAY == kAligned ? c < a.C : c >= 0 && c < a.C) var = fmaf(v[k][i], v[k][i], var);
      }
    const float rstd = rsqrtf(fmaf(row_sum<TPR, RPC>(var, red, phase), inv_c, a.eps));
    if (a.rstd != nullptr && tr == 0) a.mean[row] = mean, a.rstd[row] = rstd;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[k][i] = fmaf(v[k][i] * rstd, w[k][i], b[k][i]);
      Pack<T, VEC> out;
      out.pack(v[k]);
      store_group<T, LAY>(out, static_cast<T*>(a.y) + row * a.C, c0 + k * TPR * VEC, a.C);
    }
  }
}

// Rows longer than the register kernels hold: one CTA per row, the row read three times, twice from L2.
template <typename T>
__global__ void __launch_bounds__(512) layer_norm_long_rows_kernel(const RowArgs a) {
  __shared__ float red[64];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  const T* res = static_cast<const T*>(a.residual);
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.C;
    auto at = [&](long long c) {
      float v = Elem<T>::get(x[c]);
      if (res != nullptr) v += Elem<T>::get(res[row * a.C + c]);
      return v;
    };
    float sum = 0.f, var = 0.f;
    for (long long c = threadIdx.x; c < a.C; c += 512) sum += at(c);
    const float mean = row_sum<512>(sum, red, phase) / (float)a.C;
    for (long long c = threadIdx.x; c < a.C; c += 512) {
      const float d = at(c) - mean;
      var = fmaf(d, d, var);
    }
    const float rstd = rsqrtf(fmaf(row_sum<512>(var, red, phase), 1.0f / (float)a.C, a.eps));
    if (a.rstd != nullptr && threadIdx.x == 0) a.mean[row] = mean, a.rstd[row] = rstd;
    for (long long c = threadIdx.x; c < a.C; c += 512) {
      const float v = at(c);
      if (a.s != nullptr) {
        const T out = Elem<T>::put(v);
        static_cast<T*>(a.s)[row * a.C + c] = out;
        if (sizeof(T) == 2 && a.low != nullptr) static_cast<T*>(a.low)[row * a.C + c] = LowBits<T>::take(v, out);
      }
      static_cast<T*>(a.y)[row * a.C + c] =
          Elem<T>::put(fmaf((v - mean) * rstd, __ldg(a.weight + c), a.bias != nullptr ? __ldg(a.bias + c) : 0.f));
    }
  }
}

template <typename T, int TPR, int ITEMS, int LAY>
cudaError_t launch_rows_kernel(const RowArgs& a, cudaStream_t st) {
  constexpr int RPC = kRowThreads<TPR> / TPR;
  // as many CTAs as run at once, or a row each; a multiple of VEC, so that a group's rows begin alike
  static Resident seen;
  auto kern = layer_norm_rows_kernel<T, TPR, ITEMS, LAY>;
  const long long most = resident_ctas((const void*)kern, kRowThreads<TPR>, 0, seen) / kVec<T> * kVec<T>;
  long long ctas = (a.rows + RPC - 1) / RPC;
  if (ctas > most) ctas = most;
  return launch_pdl(kern, dim3((unsigned)ctas), dim3(kRowThreads<TPR>), 0, st, a);
}

template <typename T>
cudaError_t launch_rows(const RowArgs& a, cudaStream_t st) {
  RowLayout lay = row_layout<T>(a.C, a.C, {a.x, a.residual, a.s, a.low, a.y});
  if (lay == kAligned && (!aligned_to(a.weight, 16) || !aligned_to(a.bias, 16))) lay = kScalar;
  const long long groups = row_groups<T>(a.C, lay);
#define DTST_ROWS(TPR, ITEMS)                                                                                     \
  {                                                                                                               \
    if (lay == kAligned) return launch_rows_kernel<T, TPR, ITEMS, kAligned>(a, st);                               \
    if (lay == kShifted) return launch_rows_kernel<T, TPR, ITEMS, kShifted>(a, st);                               \
    return launch_rows_kernel<T, TPR, ITEMS, kScalar>(a, st);                                                     \
  }
  if (groups <= 32) DTST_ROWS(32, 1)
  if (groups <= 64) DTST_ROWS(32, 2)
  if (groups <= 128) DTST_ROWS(128, 1)
  if (groups <= 256) DTST_ROWS(128, 2)
  if (groups <= 512) DTST_ROWS(256, 2)
  if (groups <= 1024) DTST_ROWS(512, 2)
#undef DTST_ROWS
  const long long most = (long long)num_sms() * 4;
  return launch_pdl(layer_norm_long_rows_kernel<T>, dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(512), 0, st, a);
}

// ---- backward, rows
struct RowBackArgs {
  const void *gy, *s, *low, *gs;
  const float *weight, *mean, *rstd;
  void* gx;
  float* partial;   // [gridDim.x][2][C]: grad_w, grad_b
  long long rows, C;
};

// (Three CTAs an SM where 256 threads hold a row: bf16 [16384][2048] 78 -> 71 us; the other sizes would spill.)
template <typename T, int TPR, int ITEMS, int LAY>
__global__ void __launch_bounds__(kRowThreads<TPR>, TPR == 256 && LAY == kAligned ? 3 : 1) layer_norm_rows_backward_kernel(const RowBackArgs a) {
  constexpr int VEC = kVec<T>;
  constexpr int RPC = kRowThreads<TPR> / TPR;
  __shared__ float2 red[64];
  extern __shared__ float gw_s[];   // RPC > 1: [RPC][C]
  pdl_trigger();
  pdl_wait();
  const int tr = threadIdx.x % TPR;
  const float inv_c = 1.0f / (float)a.C;
  const T* gy = static_cast<const T*>(a.gy);
  const T* s = static_cast<const T*>(a.s);
  const T* gs = static_cast<const T*>(a.gs);
  const T* low = sizeof(T) == 2 ? static_cast<const T*>(a.low) : nullptr;
  const long long group = (long long)blockIdx.x * RPC + threadIdx.x / TPR, step = (long long)gridDim.x * RPC;
  const int shift = LAY == kShifted ? (int)(group * a.C % VEC) : 0;
  const long long c0 = (long long)tr * VEC - shift;
  Pack<T, VEC> pg[ITEMS], ps[ITEMS], pr[ITEMS], pl[ITEMS];
  float mean_next = 0.f, rstd_next = 0.f;
  auto fetch = [&](long long row) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const long long c = c0 + k * TPR * VEC;
      load_group<T, LAY>(pg[k], gy + row * a.C, c, a.C);
      load_group<T, LAY>(ps[k], s + row * a.C, c, a.C);
      if (gs != nullptr) load_group<T, LAY>(pr[k], gs + row * a.C, c, a.C);
      if (low != nullptr) load_group<T, LAY>(pl[k], low + row * a.C, c, a.C);
    }
    mean_next = __ldg(a.mean + row), rstd_next = __ldg(a.rstd + row);
  };
  if (group < a.rows) fetch(group);
  float gw[ITEMS][VEC], gb[ITEMS][VEC], w[ITEMS][VEC];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    load_weights<VEC>(w[k], a.weight, c0 + k * TPR * VEC, a.C, false);
#pragma unroll
    for (int i = 0; i < VEC; ++i) gw[k][i] = gb[k][i] = 0.f;
  }
  int phase = 0;
  for (long long row = group; row < a.rows; row += step) {
    const float rstd = rstd_next, mean = mean_next;
    float g[ITEMS][VEC], n[ITEMS][VEC];
    Pack<T, VEC> pq[ITEMS];
    float2 dot = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      pg[k].unpack(g[k]);
      ps[k].unpack(n[k]);
      if (low != nullptr) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) n[k][i] = LowBits<T>::join(ps[k].v[i], pl[k].v[i]);
      }
      if (gs != nullptr) pq[k] = pr[k];
      // (gy is zero outside the row: whatever n is there counts for nothing)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        n[k][i] = (n[k][i] - mean) * rstd;
        gw[k][i] = fmaf(g[k][i], n[k][i], gw[k][i]);
        gb[k][i] += g[k][i];
        g[k][i] *= w[k][i];
        dot.x += g[k][i];
        dot.y = fmaf(g[k][i], n[k][i], dot.y);
      }
    }
    if (row + step < a.rows) fetch(row + step);
    dot = row_sum2<TPR, RPC>(dot, red, phase);
    dot.x *= inv_c, dot.y *= inv_c;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      float q[VEC];
      if (gs != nullptr) pq[k].unpack(q);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        g[k][i] = rstd * (fmaf(-n[k][i], dot.y, g[k][i]) - dot.x);
        if (gs != nullptr) g[k][i] += q[i];
      }
      Pack<T, VEC> out;
      out.pack(g[k]);
      store_group<T, LAY>(out, static_cast<T*>(a.gx) + row * a.C, c0 + k * TPR * VEC, a.C);
    }
  }
  if (a.partial == nullptr) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* out = a.partial + ((long long)blockIdx.x * 2 + which) * a.C;
    if constexpr (RPC > 1) {   // the CTA's groups meet in shared memory, in order
      const int rw = threadIdx.x / TPR;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const long long c = c0 + k * TPR * VEC + i;
          if (c >= 0 && c < a.C) gw_s[rw * a.C + c] = which ? gb[k][i] : gw[k][i];
        }
      __syncthreads();
      for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < RPC; ++r) t += gw_s[r * a.C + c];
        out[c] = t;
      }
    } else {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const long long c = c0 + k * TPR * VEC + i;
          if (c >= 0 && c < a.C) out[c] = which ? gb[k][i] : gw[k][i];
        }
    }
  }
}

// Longer rows: the parameters' gradients column by column, then grad_x by one CTA per row (the row read twice).
template <typename T>
__global__ void __launch_bounds__(512) layer_norm_long_rows_backward_kernel(const RowBackArgs a) {
  __shared__ float2 red[64];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* gy = static_cast<const T*>(a.gy) + row * a.C;
    const float rstd = a.rstd[row], mean = a.mean[row];
    auto n = [&](long long c) { return (sum_at<T>(a.s, a.low, row * a.C + c) - mean) * rstd; };
    float2 dot = make_float2(0.f, 0.f);
    for (long long c = threadIdx.x; c < a.C; c += 512) {
      const float g = __ldg(a.weight + c) * Elem<T>::get(gy[c]);
      dot.x += g, dot.y = fmaf(g, n(c), dot.y);
    }
    dot = row_sum2<512, 1>(dot, red, phase);
    dot.x /= (float)a.C, dot.y /= (float)a.C;
    for (long long c = threadIdx.x; c < a.C; c += 512) {
      float g = rstd * (fmaf(-n(c), dot.y, __ldg(a.weight + c) * Elem<T>::get(gy[c])) - dot.x);
      if (a.gs != nullptr) g += Elem<T>::get(static_cast<const T*>(a.gs)[row * a.C + c]);
      static_cast<T*>(a.gx)[row * a.C + c] = Elem<T>::put(g);
    }
  }
}
template <typename T>
__global__ void __launch_bounds__(256) layer_norm_long_rows_weight_kernel(const RowBackArgs a) {
  pdl_trigger();
  pdl_wait();
  const long long c = (long long)blockIdx.x * 256 + threadIdx.x;   // blockIdx.y: a share of the rows
  if (c >= a.C) return;
  float t = 0.f, u = 0.f;
  for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float g = Elem<T>::get(static_cast<const T*>(a.gy)[row * a.C + c]);
    t = fmaf(g, (sum_at<T>(a.s, a.low, row * a.C + c) - __ldg(a.mean + row)) * __ldg(a.rstd + row), t);
    u += g;
  }
  a.partial[((long long)blockIdx.y * 2) * a.C + c] = t;
  a.partial[((long long)blockIdx.y * 2 + 1) * a.C + c] = u;
}

// ------------------------------------------------------------------------------------------------ fields
struct FieldArgs {
  const void *x, *residual, *gy, *gs;
  const float *weight, *bias;
  const float *mean_in, *rstd_in;
  void *s, *low, *y;    // backward: y is grad_x, x is s
  float *mean, *rstd, *partial;
  long long outer, C, inner, tiles;   // tiles per outer entry
  float eps;
};

// sums over the W warps (threadIdx.y) of a position's VEC partial sums
template <int W, int VEC>
__device__ __forceinline__ void field_sum(float (&v)[VEC], float (&red)[2][W][32 * VEC], int& phase) {
  const int lane = threadIdx.x;
#pragma unroll
  for (int i = 0; i < VEC; ++i) red[phase][threadIdx.y][lane * VEC + i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    float q = 0.f;
#pragma unroll
    for (int y = 0; y < W; ++y) q += red[phase][y][lane * VEC + i];
    v[i] = q;
  }
  phase ^= 1;
}

template <typename T, int W, int VEC, int NCH>
__global__ void __launch_bounds__(32 * W) layer_norm_field_kernel(const FieldArgs a) {
  __shared__ float red[2][W][32 * VEC];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x, wy = threadIdx.y, ny = W;
  const float inv_c = 1.0f / (float)a.C;
  const T* res = static_cast<const T*>(a.residual);
  int phase = 0;
  Pack<T, VEC> px[NCH], pr[NCH];
  const auto fetch = [&](long long t) {
    const long long o = t / a.tiles, p = (t % a.tiles) * (32 * VEC) + lane * VEC, base = o * a.C * a.inner + p;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = wy + k * ny;
      const bool on = p < a.inner && c < a.C;
      if (on) px[k].load(static_cast<const T*>(a.x) + base + c * a.inner); else px[k].zero();
      if (res != nullptr) {
        if (on) pr[k].load(res + base + c * a.inner); else pr[k].zero();
      }
    }
  };
  const long long all = a.outer * a.tiles;
  if (blockIdx.x < all) fetch(blockIdx.x);
  for (long long t = blockIdx.x; t < all; t += gridDim.x) {
    const long long o = t / a.tiles, p = (t % a.tiles) * (32 * VEC) + lane * VEC;
    const long long base = o * a.C * a.inner + p;
    const bool live = p < a.inner;
    float v[NCH][VEC], mean[VEC], rstd[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) mean[i] = rstd[i] = 0.f;
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[k][i] = px[k].get(i);
        if (res != nullptr) v[k][i] += pr[k].get(i);
        mean[i] += v[k][i];
      }
    // (in place: another CTA's tiles are other places)
    if (t + gridDim.x < all) fetch(t + gridDim.x);
    if (a.s != nullptr && live) {
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
        const int c = wy + k * ny;
        Pack<T, VEC> out;
#pragma unroll
        for (int i = 0; i < VEC; ++i) out.put(i, v[k][i]);
        if (c >= a.C) continue;
        out.store(static_cast<T*>(a.s) + base + c * a.inner);
        if (sizeof(T) == 2 && a.low != nullptr) {
          Pack<T, VEC> lo;
#pragma unroll
          for (int i = 0; i < VEC; ++i) lo.v[i] = LowBits<T>::take(v[k][i], out.v[i]);
          lo.store(static_cast<T*>(a.low) + base + c * a.inner);
        }
      }
    }
    field_sum<W, VEC>(mean, red, phase);
#pragma unroll
    for (int i = 0; i < VEC; ++i) mean[i] *= inv_c;
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[k][i] -= mean[i];
        if (wy + k * ny < a.C) rstd[i] = fmaf(v[k][i], v[k][i], rstd[i]);
      }
    field_sum<W, VEC>(rstd, red, phase);
#pragma unroll
    for (int i = 0; i < VEC; ++i) rstd[i] = rsqrtf(fmaf(rstd[i], inv_c, a.eps));
    if (!live) continue;
    if (a.rstd != nullptr && wy == 0) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) a.mean[o * a.inner + p + i] = mean[i], a.rstd[o * a.inner + p + i] = rstd[i];
    }
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = wy + k * ny;
      if (c >= a.C) continue;
      const float w = __ldg(a.weight + c), b = a.bias != nullptr ? __ldg(a.bias + c) : 0.f;
      Pack<T, VEC> out;
#pragma unroll
      for (int i = 0; i < VEC; ++i) out.put(i, fmaf(v[k][i] * rstd[i], w, b));
      out.store(static_cast<T*>(a.y) + base + c * a.inner);
    }
  }
}

// Four CTAs an SM where four warps hold the channels (fp32, 20 channels, 7.9e7 elements: 183 -> 164 us); three for eight channels of four
// positions a thread, which four would spill (fp32 [1][32][2^21], with and without grad_s: 265 and 221 us with four, 180 and 163 without a bound, 171
// and 142 with three).
template <typename T, int W, int VEC, int NCH>
__global__ void __launch_bounds__(32 * W, W == 4 ? (NCH * VEC == 32 ? 3 : 4) : 1) layer_norm_field_backward_kernel(const FieldArgs a) {
  __shared__ float red[2][2][W][32 * VEC];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x, wy = threadIdx.y, ny = W;
  const float inv_c = 1.0f / (float)a.C;
  const T* gs = static_cast<const T*>(a.gs);
  const T* low = sizeof(T) == 2 ? static_cast<const T*>(a.low) : nullptr;
  // the sums over a CTA's positions are compensated (Kahan): a thread adds thousands of tiles one by one
  float gw[NCH], lost_w[NCH], gb[NCH], lost_b[NCH], w[NCH];
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const int c = wy + k * ny;
    gw[k] = lost_w[k] = gb[k] = lost_b[k] = 0.f;
    w[k] = c < a.C ? __ldg(a.weight + c) : 0.f;
  }
  int phase = 0, phase2 = 0;
  for (long long t = blockIdx.x; t < a.outer * a.tiles; t += gridDim.x) {
    const long long o = t / a.tiles, p = (t % a.tiles) * (32 * VEC) + lane * VEC;
    const long long base = o * a.C * a.inner + p;
    const bool live = p < a.inner;
    Pack<T, VEC> pg[NCH], ps[NCH], pr[NCH], pl[NCH];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = wy + k * ny;
      const bool on = live && c < a.C;
      if (on) pg[k].load(static_cast<const T*>(a.gy) + base + c * a.inner); else pg[k].zero();
      if (on) ps[k].load(static_cast<const T*>(a.x) + base + c * a.inner); else ps[k].zero();
      if (gs != nullptr) {
        if (on) pr[k].load(gs + base + c * a.inner); else pr[k].zero();
      }
      if (low != nullptr) {
        if (on) pl[k].load(low + base + c * a.inner); else pl[k].zero();
      }
    }
    float rstd[VEC], mean[VEC], g1[VEC], g2[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      rstd[i] = live ? __ldg(a.rstd_in + o * a.inner + p + i) : 0.f;
      mean[i] = live ? __ldg(a.mean_in + o * a.inner + p + i) : 0.f;
      g1[i] = g2[i] = 0.f;
    }
    auto n_of = [&](int k, int i) {
      return ((low != nullptr ? LowBits<T>::join(ps[k].v[i], pl[k].v[i]) : ps[k].get(i)) - mean[i]) * rstd[i];
    };
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      float tw = -lost_w[k], tb = -lost_b[k];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float g = pg[k].get(i), n = n_of(k, i);
        tw = fmaf(g, n, tw);
        tb += g;
        g1[i] = fmaf(w[k], g, g1[i]);
        g2[i] = fmaf(w[k] * g, n, g2[i]);
      }
      const float sw = gw[k] + tw, sb = gb[k] + tb;
      lost_w[k] = (sw - gw[k]) - tw, lost_b[k] = (sb - gb[k]) - tb;
      gw[k] = sw, gb[k] = sb;
    }
    // one barrier for both sums
#pragma unroll
    for (int i = 0; i < VEC; ++i) red[1][phase2][wy][lane * VEC + i] = g2[i];
    field_sum<W, VEC>(g1, red[0], phase);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      float q = 0.f;
#pragma unroll
      for (int y = 0; y < W; ++y) q += red[1][phase2][y][lane * VEC + i];
      g1[i] *= inv_c, g2[i] = q * inv_c;
    }
    phase2 ^= 1;
    if (!live) continue;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = wy + k * ny;
      if (c >= a.C) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        float g = rstd[i] * (fmaf(-n_of(k, i), g2[i], w[k] * pg[k].get(i)) - g1[i]);
        if (gs != nullptr) g += pr[k].get(i);
        pg[k].put(i, g);
      }
      pg[k].store(static_cast<T*>(a.y) + base + c * a.inner);
    }
  }
  if (a.partial == nullptr) return;
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const int c = wy + k * ny;
    const float tw = warp_sum(gw[k]), tb = warp_sum(gb[k]);
    if (lane == 0 && c < a.C) {
      a.partial[((long long)blockIdx.x * 2) * a.C + c] = tw;
      a.partial[((long long)blockIdx.x * 2 + 1) * a.C + c] = tb;
    }
  }
}

// More channels than the register kernels hold (128): a thread per position, the channels walked again for every sum.
template <typename T>
__global__ void __launch_bounds__(128) layer_norm_wide_field_kernel(const FieldArgs a) {
  pdl_trigger();
  pdl_wait();
  const T* res = static_cast<const T*>(a.residual);
  const float inv_c = 1.0f / (float)a.C;
  const long long n = a.outer * a.inner;
  for (long long t = (long long)blockIdx.x * 128 + threadIdx.x; t < n; t += (long long)gridDim.x * 128) {
    const long long base = (t / a.inner) * a.C * a.inner + t % a.inner;
    auto at = [&](long long c) {
      float v = Elem<T>::get(static_cast<const T*>(a.x)[base + c * a.inner]);
      if (res != nullptr) v += Elem<T>::get(res[base + c * a.inner]);
      return v;
    };
    float sum = 0.f, var = 0.f;
    for (long long c = 0; c < a.C; ++c) sum += at(c);
    const float mean = sum * inv_c;
    for (long long c = 0; c < a.C; ++c) {
      const float d = at(c) - mean;
      var = fmaf(d, d, var);
    }
    const float rstd = rsqrtf(fmaf(var, inv_c, a.eps));
    if (a.rstd != nullptr) a.mean[t] = mean, a.rstd[t] = rstd;
    for (long long c = 0; c < a.C; ++c) {
      const float v = at(c);
      if (a.s != nullptr) {
        const T out = Elem<T>::put(v);
        static_cast<T*>(a.s)[base + c * a.inner] = out;
        if (sizeof(T) == 2 && a.low != nullptr) static_cast<T*>(a.low)[base + c * a.inner] = LowBits<T>::take(v, out);
      }
      static_cast<T*>(a.y)[base + c * a.inner] =
          Elem<T>::put(fmaf((v - mean) * rstd, __ldg(a.weight + c), a.bias != nullptr ? __ldg(a.bias + c) : 0.f));
    }
  }
}
template <typename T>
__global__ void __launch_bounds__(128) layer_norm_wide_field_backward_kernel(const FieldArgs a) {
  pdl_trigger();
  pdl_wait();
  const T* gy = static_cast<const T*>(a.gy);
  const T* gs = static_cast<const T*>(a.gs);
  const float inv_c = 1.0f / (float)a.C;
  const long long n = a.outer * a.inner;
  for (long long t = (long long)blockIdx.x * 128 + threadIdx.x; t < n; t += (long long)gridDim.x * 128) {
    const long long base = (t / a.inner) * a.C * a.inner + t % a.inner;
    const float rstd = a.rstd_in[t], mean = a.mean_in[t];
    auto g_of = [&](long long c) { return __ldg(a.weight + c) * Elem<T>::get(gy[base + c * a.inner]); };
    auto n_of = [&](long long c) { return (sum_at<T>(a.x, a.low, base + c * a.inner) - mean) * rstd; };
    float g1 = 0.f, g2 = 0.f;
    for (long long c = 0; c < a.C; ++c) {
      const float g = g_of(c);
      g1 += g, g2 = fmaf(g, n_of(c), g2);
    }
    g1 *= inv_c, g2 *= inv_c;
    for (long long c = 0; c < a.C; ++c) {
      float g = rstd * (fmaf(-n_of(c), g2, g_of(c)) - g1);
      if (gs != nullptr) g += Elem<T>::get(gs[base + c * a.inner]);
      static_cast<T*>(a.y)[base + c * a.inner] = Elem<T>::put(g);
    }
  }
}
// the parameters' gradients of one channel (blockIdx.x) over a share (blockIdx.y) of the positions
template <typename T>
__global__ void __launch_bounds__(256) layer_norm_wide_field_weight_kernel(const FieldArgs a) {
  __shared__ float2 red[64];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  const long long c = blockIdx.x, n = a.outer * a.inner;
  float2 t = make_float2(0.f, 0.f);
  for (long long p = (long long)blockIdx.y * 256 + threadIdx.x; p < n; p += (long long)gridDim.y * 256) {
    const long long at = (p / a.inner) * a.C * a.inner + c * a.inner + p % a.inner;
    const float g = Elem<T>::get(static_cast<const T*>(a.gy)[at]);
    t.x = fmaf(g, (sum_at<T>(a.x, a.low, at) - a.mean_in[p]) * a.rstd_in[p], t.x);
    t.y += g;
  }
  t = row_sum2<256, 1>(t, red, phase);
  if (threadIdx.x == 0) {
    a.partial[((long long)blockIdx.y * 2) * a.C + c] = t.x;
    a.partial[((long long)blockIdx.y * 2 + 1) * a.C + c] = t.y;
  }
}

template <typename T, bool BACK>
cudaError_t launch_field(FieldArgs a, int* parts, cudaStream_t st) {
  constexpr int WIDE = 16 / (int)sizeof(T) < 4 ? 16 / (int)sizeof(T) : 4;   // 16 bytes of fp32, 8 bytes of a 16-bit type
  if (a.C > kNormFieldChannels) {
    const long long n = a.outer * a.inner, most = (long long)num_sms() * 16;
    const long long ctas = (n + 127) / 128;
    const dim3 grid((unsigned)(ctas < most ? ctas : most));
    if (!BACK) return launch_pdl(layer_norm_wide_field_kernel<T>, grid, dim3(128), 0, st, a);
    cudaError_t e = cudaSuccess;
    if (a.partial != nullptr) {      // first: grad_x may take grad_y's place
      *parts = 8;
      e = launch_pdl(layer_norm_wide_field_weight_kernel<T>, dim3((unsigned)a.C, 8), dim3(256), 0, st, a);
    }
    if (e != cudaSuccess) return e;
    return launch_pdl(layer_norm_wide_field_backward_kernel<T>, grid, dim3(128), 0, st, a);
  }
  // positions in vectors where the rows allow it; two of them a thread where 16 warps share the channels (8 warps with four each left one
  // CTA on an SM: bf16 [8][64][65536] backward 367 us), and backward in 16 bits for 21 to 32 channels, whose low parts and conversions take
  // registers too (bf16 [1][32][2^21] with and without a residual: 523 and 270 us with four and spills, 231 and 180 with two)
  constexpr int WIDE8 = BACK && sizeof(T) == 2 ? 2 : WIDE;
  const int most_wide = a.C <= 20 ? WIDE : a.C <= 32 ? WIDE8 : 2;
  const size_t need = most_wide * sizeof(T);
  bool vec = a.inner % most_wide == 0;
  for (const void* p : {a.x, a.residual, a.gy, a.gs, (const void*)a.s, (const void*)a.low, (const void*)a.y}) vec = vec && aligned_to(p, need);
  const int ny = a.C <= 32 ? 4 : 16, nch = (int)((a.C + ny - 1) / ny);
  const int per = 32 * (vec ? most_wide : 1);
  a.tiles = (a.inner + per - 1) / per;
  const long long all = a.outer * a.tiles;
  const dim3 block(32, ny);
  const auto go = [&](auto kern, Resident& seen) {      // (backward: the parameters' partial sums are two rows per CTA)
    long long most = resident_ctas((const void*)kern, 32 * ny, 0, seen);
    if (BACK && most > kNormParts) most = kNormParts;
    const dim3 grid((unsigned)(all < most ? all : most));
    *parts = (int)grid.x;
    return launch_pdl(kern, grid, block, 0, st, a);
  };
#define DTST_FIELD(W, N, WIDTH)                                                                                   \
  if (nch <= N && ny == W) {                                                                                      \
    static Resident seen[2];                                                                                      \
    if constexpr (BACK)                                                                                           \
      return vec ? go(layer_norm_field_backward_kernel<T, W, WIDTH, N>, seen[0])                                  \
                 : go(layer_norm_field_backward_kernel<T, W, 1, N>, seen[1]);                                     \
    else                                                                                                          \
      return vec ? go(layer_norm_field_kernel<T, W, WIDTH, N>, seen[0]) : go(layer_norm_field_kernel<T, W, 1, N>, seen[1]); \
  }
  DTST_FIELD(4, 2, WIDE)
  DTST_FIELD(4, 5, WIDE)
  DTST_FIELD(4, 8, WIDE8)
  DTST_FIELD(16, 4, 2)
  DTST_FIELD(16, 8, 2)
#undef DTST_FIELD
  return cudaErrorNotSupported;
}

template <typename T, int TPR, int ITEMS, int LAY>
cudaError_t launch_rows_backward_kernel(const RowBackArgs& a, int* parts, cudaStream_t st) {
  constexpr int RPC = kRowThreads<TPR> / TPR;
  static Resident seen;
  auto kern = layer_norm_rows_backward_kernel<T, TPR, ITEMS, LAY>;
  const size_t smem = RPC > 1 ? sizeof(float) * RPC * a.C : 0;
  // as many CTAs as run at once (each leaves a row of partial sums); rows of a group that begin alike need a multiple of VEC
  long long most = resident_ctas((const void*)kern, kRowThreads<TPR>, RPC > 1 ? sizeof(float) * RPC * ITEMS * TPR * kVec<T> : 0, seen);
  if (most > kNormParts) most = kNormParts;
  most = most / kVec<T> * kVec<T>;
  const long long ctas = (a.rows + RPC - 1) / RPC;
  *parts = (int)(ctas < most ? ctas : most);
  return launch_pdl(kern, dim3((unsigned)*parts), dim3(kRowThreads<TPR>), smem, st, a);
}

template <typename T>
cudaError_t launch_rows_backward(const RowBackArgs& a, int* parts, cudaStream_t st) {
  RowLayout lay = row_layout<T>(a.C, a.C, {a.gy, a.s, a.low, a.gs, a.gx});
  // (a shifted row takes a vector more: not where that needs the kernel of twice the size)
  constexpr long long MOST = 1024;
  const long long wide = row_groups<T>(a.C, kShifted), plain = row_groups<T>(a.C, kScalar);
  if (lay == kShifted && wide <= MOST && row_size(wide) > row_size(plain)) lay = kScalar;
  const long long groups = row_groups<T>(a.C, lay);
#define DTST_ROWS(TPR, ITEMS)                                                                                     \
  {                                                                                                               \
    if (lay == kAligned) return launch_rows_backward_kernel<T, TPR, ITEMS, kAligned>(a, parts, st);               \
    if (lay == kShifted) return launch_rows_backward_kernel<T, TPR, ITEMS, kShifted>(a, parts, st);               \
    return launch_rows_backward_kernel<T, TPR, ITEMS, kScalar>(a, parts, st);                                     \
  }
  if (groups <= 32) DTST_ROWS(32, 1)
  if (groups <= 64) DTST_ROWS(32, 2)
  if (groups <= 128) DTST_ROWS(128, 1)
  if (groups <= 256) DTST_ROWS(256, 1)
  if (groups <= 512) DTST_ROWS(512, 1)
  if (groups <= 1024) DTST_ROWS(512, 2)
#undef DTST_ROWS
  // the parameters' gradients first: grad_x may take grad_y's place
  const long long most = (long long)num_sms() * 4;
  cudaError_t e = cudaSuccess;
  if (a.partial != nullptr) {
    *parts = (int)(a.rows < 64 ? a.rows : 64);
    e = launch_pdl(layer_norm_long_rows_weight_kernel<T>, dim3((unsigned)((a.C + 255) / 256), (unsigned)*parts), dim3(256), 0, st, a);
  }
  if (e != cudaSuccess) return e;
  return launch_pdl(layer_norm_long_rows_backward_kernel<T>, dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(512), 0, st, a);
}

template <typename T>
cudaError_t forward_t(const LayerNormCall& n, cudaStream_t st) {
  float* rstd = n.stats != nullptr ? n.stats + n.outer * n.inner : nullptr;
  if (n.inner == 1) {
    RowArgs a{n.x, n.residual, n.weight, n.bias, n.s, n.low, n.y, n.stats, rstd, n.outer, n.channels, n.eps};
    return launch_rows<T>(a, st);
  }
  FieldArgs a{};
  a.x = n.x, a.residual = n.residual, a.weight = n.weight, a.bias = n.bias, a.s = n.s, a.low = n.low, a.y = n.y;
  a.mean = n.stats, a.rstd = rstd, a.outer = n.outer, a.C = n.channels, a.inner = n.inner, a.eps = n.eps;
  int parts = 0;
  return launch_field<T, false>(a, &parts, st);
}

template <typename T>
cudaError_t backward_t(const LayerNormBackCall& n, cudaStream_t st) {
  int parts = 0;
  cudaError_t e;
  const bool sums = n.grad_weight != nullptr || n.grad_bias != nullptr;
  float* partial = sums ? n.partial : nullptr;
  const float* rstd = n.stats + n.outer * n.inner;
  if (n.inner == 1) {
    RowBackArgs a{n.grad_y, n.s, n.low, n.grad_s, n.weight, n.stats, rstd, n.grad_x, partial, n.outer, n.channels};
    e = launch_rows_backward<T>(a, &parts, st);
  } else {
    FieldArgs a{};
    a.x = n.s, a.gy = n.grad_y, a.gs = n.grad_s, a.weight = n.weight, a.mean_in = n.stats, a.rstd_in = rstd;
    a.low = const_cast<void*>(n.low), a.y = n.grad_x, a.partial = partial, a.outer = n.outer, a.C = n.channels, a.inner = n.inner;
    e = launch_field<T, true>(a, &parts, st);
  }
  if (e != cudaSuccess || !sums) return e;
  return launch_sum_parts(partial, parts, 2 * n.channels, {{n.grad_weight, n.channels}, {n.grad_bias, n.channels}}, st);
}

}  // namespace

cudaError_t launch_layer_norm(const LayerNormCall& n, cudaStream_t st) {
  switch (n.dtype) {
    case DTST_F32: return forward_t<float>(n, st);
    case DTST_BF16: return forward_t<__nv_bfloat16>(n, st);
    default: return forward_t<__half>(n, st);
  }
}

cudaError_t launch_layer_norm_backward(const LayerNormBackCall& n, cudaStream_t st) {
  switch (n.dtype) {
    case DTST_F32: return backward_t<float>(n, st);
    case DTST_BF16: return backward_t<__nv_bfloat16>(n, st);
    default: return backward_t<__half>(n, st);
  }
}

}  // namespace dtst
