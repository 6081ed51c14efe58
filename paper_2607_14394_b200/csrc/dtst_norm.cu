// Root-mean-square norm over channels, with the residual's addition in front and, on request, an output in 8 bits:
//     s = x + r,   rstd = 1 / sqrt(mean_c s^2 + eps),   y = s rstd w
//     q = e4m3(y 448 / amax),  scale = amax / 448,  amax over 128 neighbouring channels of a row
// and its backward pass, with n = s rstd:
//     grad_x = rstd (w gy - n mean_c(w gy n)) + grad_s,   grad_w = sum over positions of gy n
// (the gradient of the residual is the same tensor).  Everything is in 32 bits; y is formed from the unrounded sum,
// so a 16-bit s costs y nothing.
//
// All of it is bound by memory: 2..5 tensors in or out per pass, a few operations per element.  Two layouts:
//   rows      [rows][C], C contiguous (token-major): a row is held by 32..512 threads in registers, each thread a
//             16-byte group of channels every TPR groups, so a group of 128 channels is 16 (32 for fp32)
//             neighbouring lanes and its amax a few shuffles; the next row's loads are under way while a row is summed.
//             bf16 [16384][2048] with residual: 43.4 us into 8 bits (5.4 TB/s), 55.9 forward, 77 backward (6.0 and 4.4 TB/s);
//             without norm and residual into 8 bits 18.8 us (5.4 TB/s), a frame [4][2048] 1.5;
//   fields    [outer][C][inner], inner contiguous (channels-first): lanes run along the positions, warps share the
//             channels, the sums over channels meet in shared memory.  fp32 [1][20][3932160] with residual: 206 us
//             forward, 198 backward (6.1 and 6.4 TB/s).
// Rows that begin off a vector (kShifted) are read in vectors that begin earlier: fp16 [33520][1001] 40 us forward and 98
// backward (3.4 and 2.1 TB/s), against 102 and 124 element by element (kScalar, for tensors that do not begin on a vector, and
// for the backward pass of some rows).  Positions of a field in vectors where its rows allow it: fp32 [8][64][65536] 85 us, with
// 65537 positions 110.  Beyond what registers hold, the fallbacks read their input again: forward bf16 [4096][16392] 284 us
// ([16384]: 109), fp32 fields [8][136][65536] 339 us (128 channels: 173); backward bf16 [4096][16384] 647, fields 667 (218).
// The backward kernels of the longest rows spill: 144 to 192 bytes of 16-bit rows off a vector (by elements 144) above 4096
// channels, 92 to 188 of fp32 rows.
// The weight gradient is summed in registers over all positions a CTA visits and in a fixed order over CTAs by a
// second launch: same bits on every run.
#include <initializer_list>

#include "dtst_common.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

// ------------------------------------------------------------------------------------------------ rows
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

// Sum over the TPR threads of a row.  `red` holds two alternating sets of partial sums for each group of the CTA, so that one
// barrier (the group's own where there are several) is enough.
template <int TPR, int GROUPS = 1>
__device__ __forceinline__ float row_sum(float v, float* red, int& phase) {
  v = warp_sum(v);
  if constexpr (TPR > 32) {
    constexpr int N = TPR / 32;
    const int group = GROUPS > 1 ? threadIdx.x / TPR : 0;
    float* r = red + (phase * GROUPS + group) * N;
    phase ^= 1;
    if ((threadIdx.x & 31) == 0) r[(threadIdx.x % TPR) >> 5] = v;
    if constexpr (GROUPS > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(TPR) : "memory");
    else __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) t += r[i];
    v = t;
  }
  return v;
}

// threads of a CTA: four rows at once where a warp holds one, two where four warps do (more CTAs would make more partial
// sums of the weight gradient)
template <int TPR>
constexpr int kRowThreads = TPR <= 32 ? 128 : TPR <= 128 ? 256 : TPR;

// How a row's vectors lie.  kShifted: rows of C elements that begin off a vector, in tensors that all begin on one: a group of
// threads takes rows whose numbers are the same modulo VEC, so all its rows begin `shift` elements behind a vector, and its
// vectors, weights and sums stand `shift` elements in front of the row's own.
enum RowLayout { kScalar = 0, kAligned = 1, kShifted = 2 };

template <typename T, int LAY>
__device__ __forceinline__ void load_group(Pack<T, kVec<T>>& p, const T* row, long long c, long long C) {
  constexpr int VEC = kVec<T>;
  if (LAY == kAligned) {
    if (c < C) p.load(row + c); else p.zero();
  } else if (LAY == kShifted && c >= 0 && c + VEC <= C) {
    p.load(row + c);
  } else {
    p.zero();
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (c + i >= 0 && c + i < C) p.v[i] = row[c + i];
  }
}
template <typename T, int LAY>
__device__ __forceinline__ void store_group(const Pack<T, kVec<T>>& p, T* row, long long c, long long C) {
  constexpr int VEC = kVec<T>;
  if (LAY == kAligned) {
    if (c < C) p.store(row + c);
  } else if (LAY == kShifted && c >= 0 && c + VEC <= C) {
    p.store(row + c);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (c + i >= 0 && c + i < C) row[c + i] = p.v[i];
  }
}
template <int VEC>
__device__ __forceinline__ void load_weights(float (&w)[VEC], const float* weight, long long c, long long C, bool aligned) {
  if (aligned && c < C) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const float4 t = __ldg(reinterpret_cast<const float4*>(weight + c + i));
      w[i] = t.x, w[i + 1] = t.y, w[i + 2] = t.z, w[i + 3] = t.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) w[i] = c + i >= 0 && c + i < C ? __ldg(weight + c + i) : 0.f;
  }
}

// quantises the group of VEC values this thread holds; the threads of a 128-channel group are neighbours in a warp
template <int VEC>
__device__ __forceinline__ void quantise_store(const float (&y)[VEC], uint8_t* q_row, float* scale, long long c,
                                               long long C, long long scale_ld, long long row, bool q_aligned) {
  float amax = kAmaxFloor;
#pragma unroll
  for (int i = 0; i < VEC; ++i) amax = fmaxf(amax, fabsf(y[i]));
#pragma unroll
  for (int o = kFp8Block / VEC / 2; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (c >= C) return;
  const float inv = __fdiv_rn(kE4m3Max, amax);
  if (c % kFp8Block == 0) scale[(c / kFp8Block) * scale_ld + row] = __fdiv_rn(amax, kE4m3Max);
  uint32_t w[VEC / 4];
#pragma unroll
  for (int i = 0; i < VEC / 4; ++i)
    w[i] = pack_e4m3(y[4 * i] * inv, y[4 * i + 1] * inv, y[4 * i + 2] * inv, y[4 * i + 3] * inv);
  if (q_aligned && c + VEC <= C) {
    if constexpr (VEC == 8) *reinterpret_cast<uint2*>(q_row + c) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q_row + c) = w[0];
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (c + i < C) q_row[c + i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

struct RowArgs {
  const void *x, *residual;
  const float* weight;
  void *s, *low, *y;        // low: what rounding took from s (16-bit types; may be null)
  uint8_t* q;
  float *scale, *rstd;
  long long rows, C, x_ld, q_ld;
  float eps;
  int q_aligned;
};

// NORM false: quantise x as it is (no residual, no weight).  A group of TPR threads walks over rows, the next row's loads
// under way while a row is summed and written; the weights stay in registers.
template <typename T, int TPR, int ITEMS, bool QUANT, bool NORM, int LAY>
__global__ void __launch_bounds__(kRowThreads<TPR>) norm_rows_kernel(const RowArgs a) {
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
  Pack<T, VEC> px[ITEMS], pr[ITEMS];
  auto fetch = [&](long long row) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) load_group<T, LAY>(px[k], x + row * a.x_ld, (long long)(tr + k * TPR) * VEC - shift, a.C);
    if (NORM && res != nullptr) {
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) load_group<T, LAY>(pr[k], res + row * a.C, (long long)(tr + k * TPR) * VEC - shift, a.C);
    }
  };
  if (group < a.rows) fetch(group);
  float w[ITEMS][VEC];
  if (NORM) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) load_weights<VEC>(w[k], a.weight, (long long)(tr + k * TPR) * VEC - shift, a.C, LAY == kAligned);
  }
  int phase = 0;
  for (long long row = group; row < a.rows; row += step) {
    float v[ITEMS][VEC];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      px[k].unpack(v[k]);
      if (NORM && res != nullptr) {
        float r[VEC];
        pr[k].unpack(r);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[k][i] += r[i];
      }
#pragma unroll
      for (int i = 0; i < VEC; ++i) sum = fmaf(v[k][i], v[k][i], sum);
    }
    if (row + step < a.rows) fetch(row + step);
    float rstd = 1.f;
    if (NORM) {
      if (a.s != nullptr) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
          Pack<T, VEC> out;
          out.pack(v[k]);
          store_group<T, LAY>(out, static_cast<T*>(a.s) + row * a.C, (long long)(tr + k * TPR) * VEC - shift, a.C);
          if (sizeof(T) == 2 && a.low != nullptr) {
            Pack<T, VEC> lo;
#pragma unroll
            for (int i = 0; i < VEC; ++i) lo.v[i] = LowBits<T>::take(v[k][i], out.v[i]);
            store_group<T, LAY>(lo, static_cast<T*>(a.low) + row * a.C, (long long)(tr + k * TPR) * VEC - shift, a.C);
          }
        }
      }
      rstd = rsqrtf(fmaf(row_sum<TPR, RPC>(sum, red, phase), inv_c, a.eps));
      if (a.rstd != nullptr && tr == 0) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const long long c = (long long)(tr + k * TPR) * VEC - shift;
      if (NORM) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[k][i] = v[k][i] * rstd * w[k][i];
      }
      if (QUANT) {
        quantise_store<VEC>(v[k], a.q + row * a.q_ld, a.scale, c, a.C, a.rows, row, a.q_aligned != 0);
      } else {
        Pack<T, VEC> out;
        out.pack(v[k]);
        store_group<T, LAY>(out, static_cast<T*>(a.y) + row * a.C, c, a.C);
      }
    }
  }
}

// Rows longer than the register kernels hold (16384 channels, 8192 in fp32): one CTA per row, the row read twice,
// the second time from L2.
template <typename T, bool QUANT, bool NORM>
__global__ void __launch_bounds__(512) norm_long_rows_kernel(const RowArgs a) {
  __shared__ float red[64];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  const T* res = static_cast<const T*>(a.residual);
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    float rstd = 1.f;
    if (NORM) {
      float sum = 0.f;
      for (long long c = threadIdx.x; c < a.C; c += 512) {
        float v = Elem<T>::get(x[c]);
        if (res != nullptr) v += Elem<T>::get(res[row * a.C + c]);
        sum = fmaf(v, v, sum);
      }
      rstd = rsqrtf(fmaf(row_sum<512>(sum, red, phase), 1.0f / (float)a.C, a.eps));
      if (a.rstd != nullptr && threadIdx.x == 0) a.rstd[row] = rstd;
    }
    for (long long c0 = 0; c0 < a.C; c0 += 2048) {   // 16 warps x 128 channels, four to a lane
      const long long c = c0 + 4 * (long long)threadIdx.x;
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i] = 0.f;
        if (c + i < a.C) {
          float v = Elem<T>::get(x[c + i]);
          if (NORM) {
            if (res != nullptr) v += Elem<T>::get(res[row * a.C + c + i]);
            if (a.s != nullptr) {
              const T out = Elem<T>::put(v);
              static_cast<T*>(a.s)[row * a.C + c + i] = out;
              if (sizeof(T) == 2 && a.low != nullptr) static_cast<T*>(a.low)[row * a.C + c + i] = LowBits<T>::take(v, out);
            }
            v = v * rstd * __ldg(a.weight + c + i);
          }
          y[i] = v;
        }
      }
      if (QUANT) {
        quantise_store<4>(y, a.q + row * a.q_ld, a.scale, c, a.C, a.rows, row, a.q_aligned != 0);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < a.C) static_cast<T*>(a.y)[row * a.C + c + i] = Elem<T>::put(y[i]);
      }
    }
  }
}

// the layout of contiguous rows [rows][C] of all these tensors
template <typename T>
RowLayout row_layout(long long C, long long x_ld, std::initializer_list<const void*> tensors) {
  for (const void* t : tensors)
    if (!aligned_to(t, 16)) return kScalar;
  if (C % kVec<T> == 0 && x_ld % kVec<T> == 0) return kAligned;
  return x_ld == C ? kShifted : kScalar;
}

// Vectors that hold a row, and how many times 32 has to be doubled to hold them: the row kernels come in these sizes.
template <typename T>
long long row_groups(long long C, RowLayout lay) {
  return (C + (lay == kShifted ? kVec<T> - 1 : 0) + kVec<T> - 1) / kVec<T>;
}
inline int row_size(long long groups) {
  int size = 0;
  for (long long n = 32; n < groups; n *= 2) ++size;
  return size;
}

template <typename T, int TPR, int ITEMS, bool QUANT, bool NORM, int LAY>
cudaError_t launch_rows_kernel(const RowArgs& a, cudaStream_t st) {
  constexpr int RPC = kRowThreads<TPR> / TPR;
  auto kern = norm_rows_kernel<T, TPR, ITEMS, QUANT, NORM, LAY>;
  // as many CTAs as run at once, or a row each; a multiple of VEC, so that a group's rows begin alike
  const long long most = (long long)num_sms() * (2048 / kRowThreads<TPR> < 8 ? 2048 / kRowThreads<TPR> : 8) / kVec<T> * kVec<T>;
  long long ctas = (a.rows + RPC - 1) / RPC;
  if (ctas > most) ctas = most;
  return launch_pdl(kern, dim3((unsigned)ctas), dim3(kRowThreads<TPR>), 0, st, a);
}

template <typename T, bool QUANT, bool NORM>
cudaError_t launch_rows(const RowArgs& a, cudaStream_t st) {
  RowLayout lay = row_layout<T>(a.C, a.x_ld, {a.x, a.residual, a.s, a.low, QUANT ? nullptr : a.y});
  if (lay == kAligned && !aligned_to(a.weight, 16)) lay = kScalar;
  if (QUANT && lay == kShifted) lay = kScalar;       // blocks of 128 channels are counted from the row's beginning
  const long long groups = row_groups<T>(a.C, lay);
#define DTST_ROWS(TPR, ITEMS)                                                                                     \
  {                                                                                                               \
    if (lay == kAligned) return launch_rows_kernel<T, TPR, ITEMS, QUANT, NORM, kAligned>(a, st);                  \
    if constexpr (!QUANT)                                                                                         \
      if (lay == kShifted) return launch_rows_kernel<T, TPR, ITEMS, QUANT, NORM, kShifted>(a, st);                \
    return launch_rows_kernel<T, TPR, ITEMS, QUANT, NORM, kScalar>(a, st);                                        \
  }
  if (groups <= 32) DTST_ROWS(32, 1)
  if (groups <= 64) DTST_ROWS(32, 2)
  if (groups <= 128) DTST_ROWS(128, 1)
  if (groups <= 256) DTST_ROWS(128, 2)
  if (groups <= 512) DTST_ROWS(256, 2)
  if (groups <= 1024) DTST_ROWS(512, 2)
  if (groups <= 2048) DTST_ROWS(512, 4)
#undef DTST_ROWS
  const long long most = (long long)num_sms() * 32;
  return launch_pdl(norm_long_rows_kernel<T, QUANT, NORM>, dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(512), 0, st, a);
}

// ---- backward, rows
struct RowBackArgs {
  const void *gy, *s, *low, *gs;
  const float *weight, *rstd;
  void* gx;
  float* partial;   // [gridDim.x][C]
  long long rows, C;
};

template <typename T, int TPR, int ITEMS, int LAY>
__global__ void __launch_bounds__(kRowThreads<TPR>) norm_rows_backward_kernel(const RowBackArgs a) {
  constexpr int VEC = kVec<T>;
  constexpr int RPC = kRowThreads<TPR> / TPR;
  __shared__ float red[64];
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
  Pack<T, VEC> pg[ITEMS], ps[ITEMS], pr[ITEMS], pl[ITEMS];
  float rstd_next = 0.f;
  auto fetch = [&](long long row) {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const long long c = (long long)(tr + k * TPR) * VEC - shift;
      load_group<T, LAY>(pg[k], gy + row * a.C, c, a.C);
      load_group<T, LAY>(ps[k], s + row * a.C, c, a.C);
      if (gs != nullptr) load_group<T, LAY>(pr[k], gs + row * a.C, c, a.C);
      if (low != nullptr) load_group<T, LAY>(pl[k], low + row * a.C, c, a.C);
    }
    rstd_next = __ldg(a.rstd + row);
  };
  if (group < a.rows) fetch(group);
  float gw[ITEMS][VEC], w[ITEMS][VEC];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    load_weights<VEC>(w[k], a.weight, (long long)(tr + k * TPR) * VEC - shift, a.C, false);
#pragma unroll
    for (int i = 0; i < VEC; ++i) gw[k][i] = 0.f;
  }
  int phase = 0;
  for (long long row = group; row < a.rows; row += step) {
    const float rstd = rstd_next;
    float g[ITEMS][VEC], n[ITEMS][VEC];
    Pack<T, VEC> pq[ITEMS];
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      pg[k].unpack(g[k]);
      ps[k].unpack(n[k]);
      if (low != nullptr) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) n[k][i] = LowBits<T>::join(ps[k].v[i], pl[k].v[i]);
      }
      if (gs != nullptr) pq[k] = pr[k];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        n[k][i] *= rstd;
        gw[k][i] = fmaf(g[k][i], n[k][i], gw[k][i]);
        g[k][i] *= w[k][i];
        dot = fmaf(g[k][i], n[k][i], dot);
      }
    }
    if (row + step < a.rows) fetch(row + step);
    dot = row_sum<TPR, RPC>(dot, red, phase) * inv_c;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      float q[VEC];
      if (gs != nullptr) pq[k].unpack(q);
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        g[k][i] = rstd * fmaf(-n[k][i], dot, g[k][i]);
        if (gs != nullptr) g[k][i] += q[i];
      }
      Pack<T, VEC> out;
      out.pack(g[k]);
      store_group<T, LAY>(out, static_cast<T*>(a.gx) + row * a.C, (long long)(tr + k * TPR) * VEC - shift, a.C);
    }
  }
  if (a.partial == nullptr) return;
  float* out = a.partial + (long long)blockIdx.x * a.C;
  if constexpr (RPC > 1) {   // the CTA's groups meet in shared memory, in order
    const int rw = threadIdx.x / TPR;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int c = (tr + k * TPR) * VEC - shift + i;
        if (c >= 0 && c < a.C) gw_s[rw * a.C + c] = gw[k][i];
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
        const long long c = (long long)(tr + k * TPR) * VEC - shift + i;
        if (c >= 0 && c < a.C) out[c] = gw[k][i];
      }
  }
}

// the sum at element `at`, to 24 bits where its low part was kept
template <typename T>
__device__ __forceinline__ float sum_at(const void* s, const void* low, long long at) {
  const T v = static_cast<const T*>(s)[at];
  return sizeof(T) == 2 && low != nullptr ? LowBits<T>::join(v, static_cast<const T*>(low)[at]) : Elem<T>::get(v);
}

// Longer rows: the weight gradient column by column, then grad_x by one CTA per row (the row read twice).
template <typename T>
__global__ void __launch_bounds__(512) norm_long_rows_backward_kernel(const RowBackArgs a) {
  __shared__ float red[64];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* gy = static_cast<const T*>(a.gy) + row * a.C;
    const float rstd = a.rstd[row];
    float dot = 0.f;
    for (long long c = threadIdx.x; c < a.C; c += 512)
      dot = fmaf(__ldg(a.weight + c) * Elem<T>::get(gy[c]), sum_at<T>(a.s, a.low, row * a.C + c) * rstd, dot);
    dot = row_sum<512>(dot, red, phase) / (float)a.C;
    for (long long c = threadIdx.x; c < a.C; c += 512) {
      float g = rstd * fmaf(-(sum_at<T>(a.s, a.low, row * a.C + c) * rstd), dot, __ldg(a.weight + c) * Elem<T>::get(gy[c]));
      if (a.gs != nullptr) g += Elem<T>::get(static_cast<const T*>(a.gs)[row * a.C + c]);
      static_cast<T*>(a.gx)[row * a.C + c] = Elem<T>::put(g);
    }
  }
}
template <typename T>
__global__ void __launch_bounds__(256) norm_long_rows_weight_kernel(const RowBackArgs a) {
  pdl_trigger();
  pdl_wait();
  const long long c = (long long)blockIdx.x * 256 + threadIdx.x;   // blockIdx.y: a share of the rows
  if (c >= a.C) return;
  float t = 0.f;
  for (long long row = blockIdx.y; row < a.rows; row += gridDim.y)
    t = fmaf(Elem<T>::get(static_cast<const T*>(a.gy)[row * a.C + c]),
             sum_at<T>(a.s, a.low, row * a.C + c) * __ldg(a.rstd + row), t);
  a.partial[(long long)blockIdx.y * a.C + c] = t;
}

// ------------------------------------------------------------------------------------------------ fields
struct FieldArgs {
  const void *x, *residual, *gy, *gs;
  const float* weight;
  const float* rstd_in;
  void *s, *low, *y;    // backward: y is grad_x, x is s
  float *rstd, *partial;
  long long outer, C, inner, tiles;   // tiles per outer entry
  float eps;
};

template <typename T, int VEC, int NCH>
__global__ void __launch_bounds__(256) norm_field_kernel(const FieldArgs a) {
  __shared__ float red[2][8][32 * VEC];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x, wy = threadIdx.y, ny = blockDim.y;
  const float inv_c = 1.0f / (float)a.C;
  const T* res = static_cast<const T*>(a.residual);
  int phase = 0;
  for (long long t = blockIdx.x; t < a.outer * a.tiles; t += gridDim.x) {
    const long long o = t / a.tiles, p = (t % a.tiles) * (32 * VEC) + lane * VEC;
    const long long base = o * a.C * a.inner + p;
    const bool live = p < a.inner;
    Pack<T, VEC> px[NCH], pr[NCH];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = wy + k * ny;
      const bool on = live && c < a.C;
      if (on) px[k].load(static_cast<const T*>(a.x) + base + c * a.inner); else px[k].zero();
      if (res != nullptr) {
        if (on) pr[k].load(res + base + c * a.inner); else pr[k].zero();
      }
    }
    float v[NCH][VEC], sum[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[i] = 0.f;
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[k][i] = px[k].get(i);
        if (res != nullptr) v[k][i] += pr[k].get(i);
        sum[i] = fmaf(v[k][i], v[k][i], sum[i]);
      }
    if (a.s != nullptr && live) {
#pragma unroll
      for (int k = 0; k < NCH; ++k) {
        const int c = wy + k * ny;
#pragma unroll
        for (int i = 0; i < VEC; ++i) px[k].put(i, v[k][i]);
        if (c >= a.C) continue;
        px[k].store(static_cast<T*>(a.s) + base + c * a.inner);
        if (sizeof(T) == 2 && a.low != nullptr) {
          Pack<T, VEC> lo;
#pragma unroll
          for (int i = 0; i < VEC; ++i) lo.v[i] = LowBits<T>::take(v[k][i], px[k].v[i]);
          lo.store(static_cast<T*>(a.low) + base + c * a.inner);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) red[phase][wy][lane * VEC + i] = sum[i];
    __syncthreads();
    float rstd[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      float q = 0.f;
      for (int y = 0; y < ny; ++y) q += red[phase][y][lane * VEC + i];
      rstd[i] = rsqrtf(fmaf(q, inv_c, a.eps));
    }
    phase ^= 1;
    if (!live) continue;
    if (a.rstd != nullptr && wy == 0) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) a.rstd[o * a.inner + p + i] = rstd[i];
    }
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = wy + k * ny;
      if (c >= a.C) continue;
      const float w = __ldg(a.weight + c);
#pragma unroll
      for (int i = 0; i < VEC; ++i) px[k].put(i, v[k][i] * rstd[i] * w);
      px[k].store(static_cast<T*>(a.y) + base + c * a.inner);
    }
  }
}

template <typename T, int VEC, int NCH>
__global__ void __launch_bounds__(256) norm_field_backward_kernel(const FieldArgs a) {
  __shared__ float red[2][8][32 * VEC];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x, wy = threadIdx.y, ny = blockDim.y;
  const float inv_c = 1.0f / (float)a.C;
  const T* gs = static_cast<const T*>(a.gs);
  const T* low = sizeof(T) == 2 ? static_cast<const T*>(a.low) : nullptr;
  // the sums over a CTA's positions are compensated (Kahan): a thread adds thousands of tiles one by one
  float gw[NCH], lost[NCH], w[NCH];
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const int c = wy + k * ny;
    gw[k] = lost[k] = 0.f;
    w[k] = c < a.C ? __ldg(a.weight + c) : 0.f;
  }
  int phase = 0;
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
    auto sum_of = [&](int k, int i) { return low != nullptr ? LowBits<T>::join(ps[k].v[i], pl[k].v[i]) : ps[k].get(i); };
    float rstd[VEC], dot[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      rstd[i] = live ? __ldg(a.rstd_in + o * a.inner + p + i) : 0.f;
      dot[i] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      float t = -lost[k];
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float g = pg[k].get(i), n = sum_of(k, i) * rstd[i];
        t = fmaf(g, n, t);
        dot[i] = fmaf(w[k] * g, n, dot[i]);
      }
      const float sum = gw[k] + t;
      lost[k] = (sum - gw[k]) - t;
      gw[k] = sum;
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) red[phase][wy][lane * VEC + i] = dot[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      float q = 0.f;
      for (int y = 0; y < ny; ++y) q += red[phase][y][lane * VEC + i];
      dot[i] = q * inv_c;
    }
    phase ^= 1;
    if (!live) continue;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = wy + k * ny;
      if (c >= a.C) continue;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        float g = rstd[i] * fmaf(-(sum_of(k, i) * rstd[i]), dot[i], w[k] * pg[k].get(i));
        if (gs != nullptr) g += pr[k].get(i);
        ps[k].put(i, g);
      }
      ps[k].store(static_cast<T*>(a.y) + base + c * a.inner);
    }
  }
  if (a.partial == nullptr) return;
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const int c = wy + k * ny;
    const float t = warp_sum(gw[k]);
    if (lane == 0 && c < a.C) a.partial[(long long)blockIdx.x * a.C + c] = t;
  }
}

// More channels than the register kernels hold (128): a thread per position, the channels walked twice.
template <typename T>
__global__ void __launch_bounds__(128) norm_wide_field_kernel(const FieldArgs a) {
  pdl_trigger();
  pdl_wait();
  const T* res = static_cast<const T*>(a.residual);
  const float inv_c = 1.0f / (float)a.C;
  const long long n = a.outer * a.inner;
  for (long long t = (long long)blockIdx.x * 128 + threadIdx.x; t < n; t += (long long)gridDim.x * 128) {
    const long long base = (t / a.inner) * a.C * a.inner + t % a.inner;
    float sum = 0.f;
    for (long long c = 0; c < a.C; ++c) {
      float v = Elem<T>::get(static_cast<const T*>(a.x)[base + c * a.inner]);
      if (res != nullptr) v += Elem<T>::get(res[base + c * a.inner]);
      sum = fmaf(v, v, sum);
    }
    const float rstd = rsqrtf(fmaf(sum, inv_c, a.eps));
    if (a.rstd != nullptr) a.rstd[t] = rstd;
    for (long long c = 0; c < a.C; ++c) {
      float v = Elem<T>::get(static_cast<const T*>(a.x)[base + c * a.inner]);
      if (res != nullptr) v += Elem<T>::get(res[base + c * a.inner]);
      if (a.s != nullptr) {
        const T out = Elem<T>::put(v);
        static_cast<T*>(a.s)[base + c * a.inner] = out;
        if (sizeof(T) == 2 && a.low != nullptr) static_cast<T*>(a.low)[base + c * a.inner] = LowBits<T>::take(v, out);
      }
      static_cast<T*>(a.y)[base + c * a.inner] = Elem<T>::put(v * rstd * __ldg(a.weight + c));
    }
  }
}
template <typename T>
__global__ void __launch_bounds__(128) norm_wide_field_backward_kernel(const FieldArgs a) {
  pdl_trigger();
  pdl_wait();
  const T* gy = static_cast<const T*>(a.gy);
  const T* gs = static_cast<const T*>(a.gs);
  const float inv_c = 1.0f / (float)a.C;
  const long long n = a.outer * a.inner;
  for (long long t = (long long)blockIdx.x * 128 + threadIdx.x; t < n; t += (long long)gridDim.x * 128) {
    const long long base = (t / a.inner) * a.C * a.inner + t % a.inner;
    const float rstd = a.rstd_in[t];
    float dot = 0.f;
    for (long long c = 0; c < a.C; ++c)
      dot = fmaf(__ldg(a.weight + c) * Elem<T>::get(gy[base + c * a.inner]), sum_at<T>(a.x, a.low, base + c * a.inner) * rstd, dot);
    dot *= inv_c;
    for (long long c = 0; c < a.C; ++c) {
      float g = rstd * fmaf(-(sum_at<T>(a.x, a.low, base + c * a.inner) * rstd), dot,
                            __ldg(a.weight + c) * Elem<T>::get(gy[base + c * a.inner]));
      if (gs != nullptr) g += Elem<T>::get(gs[base + c * a.inner]);
      static_cast<T*>(a.y)[base + c * a.inner] = Elem<T>::put(g);
    }
  }
}
// weight gradient of one channel (blockIdx.x) over a share (blockIdx.y) of the positions
template <typename T>
__global__ void __launch_bounds__(256) norm_wide_field_weight_kernel(const FieldArgs a) {
  __shared__ float red[64];
  pdl_trigger();
  pdl_wait();
  int phase = 0;
  const long long c = blockIdx.x, n = a.outer * a.inner;
  float t = 0.f;
  for (long long p = (long long)blockIdx.y * 256 + threadIdx.x; p < n; p += (long long)gridDim.y * 256) {
    const long long at = (p / a.inner) * a.C * a.inner + c * a.inner + p % a.inner;
    t = fmaf(Elem<T>::get(static_cast<const T*>(a.gy)[at]), sum_at<T>(a.x, a.low, at) * a.rstd_in[p], t);
  }
  t = row_sum<256>(t, red, phase);
  if (threadIdx.x == 0) a.partial[(long long)blockIdx.y * a.C + c] = t;
}

// grad_w[c] = sum over parts, in a fixed order: 32 warps take every 32nd part, their sums meet in warp order.
__global__ void __launch_bounds__(1024) norm_weight_sum_kernel(const float* __restrict__ partial, float* __restrict__ gw,
                                                              int parts, long long C) {
  __shared__ float red[32][33];
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 32 + lane;
  float t = 0.f;
  if (c < C) {
#pragma unroll 8
    for (int p = w; p < parts; p += 32) t += partial[(long long)p * C + c];
  }
  red[w][lane] = t;
  __syncthreads();
  t = red[lane][w];                    // (turned round: warp w sums column w over the 32 parts' lanes)
  t = warp_sum(t);
  if (lane == 0 && (long long)blockIdx.x * 32 + w < C) gw[(long long)blockIdx.x * 32 + w] = t;
}

template <typename T, bool BACK>
cudaError_t launch_field(FieldArgs a, int* parts, cudaStream_t st) {
  constexpr int WIDE = 16 / (int)sizeof(T) < 4 ? 16 / (int)sizeof(T) : 4;   // 16 bytes of fp32, 8 bytes of a 16-bit type
  if (a.C > kNormFieldChannels) {
    const long long n = a.outer * a.inner, most = (long long)num_sms() * 16;
    const long long ctas = (n + 127) / 128;
    const dim3 grid((unsigned)(ctas < most ? ctas : most));
    if (!BACK) return launch_pdl(norm_wide_field_kernel<T>, grid, dim3(128), 0, st, a);
    cudaError_t e = cudaSuccess;
    if (a.partial != nullptr) {      // first: grad_x may take grad_y's place
      *parts = 8;
      e = launch_pdl(norm_wide_field_weight_kernel<T>, dim3((unsigned)a.C, 8), dim3(256), 0, st, a);
    }
    if (e != cudaSuccess) return e;
    return launch_pdl(norm_wide_field_backward_kernel<T>, grid, dim3(128), 0, st, a);
  }
  const size_t need = WIDE * sizeof(T);
  const bool vec = a.inner % WIDE == 0 && aligned_to(a.x, need) && aligned_to(a.residual, need) && aligned_to(a.gy, need) &&
                   aligned_to(a.gs, need) && aligned_to(a.s, need) && aligned_to(a.low, need) && aligned_to(a.y, need);
  const int ny = a.C <= 32 ? 4 : 8, nch = (int)((a.C + ny - 1) / ny);
  const int per = 32 * (vec ? WIDE : 1);
  a.tiles = (a.inner + per - 1) / per;
  // the weight gradient's partial sums are one row per CTA
  const long long most = BACK ? (long long)kNormParts : (long long)num_sms() * 32, all = a.outer * a.tiles;
  const dim3 grid((unsigned)(all < most ? all : most)), block(32, ny);
  *parts = (int)grid.x;
#define DTST_FIELD(N)                                                                                             \
  if (nch <= N) {                                                                                                 \
    if (BACK)                                                                                                     \
      return vec ? launch_pdl(norm_field_backward_kernel<T, WIDE, N>, grid, block, 0, st, a)                      \
                 : launch_pdl(norm_field_backward_kernel<T, 1, N>, grid, block, 0, st, a);                        \
    return vec ? launch_pdl(norm_field_kernel<T, WIDE, N>, grid, block, 0, st, a)                                 \
               : launch_pdl(norm_field_kernel<T, 1, N>, grid, block, 0, st, a);                                   \
  }
  DTST_FIELD(2)
  DTST_FIELD(5)
  DTST_FIELD(8)
  DTST_FIELD(16)
#undef DTST_FIELD
  return cudaErrorNotSupported;
}

template <typename T>
cudaError_t launch_rows_backward(const RowBackArgs& a, int* parts, cudaStream_t st) {
  RowLayout lay = row_layout<T>(a.C, a.C, {a.gy, a.s, a.low, a.gs, a.gx});
  // Element by element where the vector more that a shifted row takes needs the kernel of twice the size (2^25 elements, us
  // shifted and by elements: fp16 250 channels 184, 103; 511 168, 128; 1023 248, 123; 4095 224, 200; fp32 1023 139, 76), but
  // not where that is the kernel beyond the registers (fp16 8191: 162, 225).  In between 98, 124 (fp16 1001) to 91, 82 (fp32
  // 2001); the forward pass is faster shifted on both sides (fp16 250: 80, 113; 1023: 91).
  constexpr long long MOST = sizeof(T) == 4 ? 2048 : 1024;
  const long long wide = row_groups<T>(a.C, kShifted), plain = row_groups<T>(a.C, kScalar);
  if (lay == kShifted && wide <= MOST && row_size(wide) > row_size(plain)) lay = kScalar;
  const long long groups = row_groups<T>(a.C, lay);
#define DTST_ROWS(TPR, ITEMS)                                                                                     \
  {                                                                                                               \
    constexpr int RPC = kRowThreads<TPR> / TPR;                                                                   \
    const long long ctas = (a.rows + RPC - 1) / RPC;                                                              \
    *parts = (int)(ctas < kNormParts ? ctas : kNormParts);                                                        \
    const dim3 grid((unsigned)*parts), block(kRowThreads<TPR>);                                                   \
    const size_t smem = RPC > 1 ? sizeof(float) * RPC * a.C : 0;                                                  \
    if (lay == kAligned) return launch_pdl(norm_rows_backward_kernel<T, TPR, ITEMS, kAligned>, grid, block, smem, st, a); \
    if (lay == kShifted) return launch_pdl(norm_rows_backward_kernel<T, TPR, ITEMS, kShifted>, grid, block, smem, st, a); \
    return launch_pdl(norm_rows_backward_kernel<T, TPR, ITEMS, kScalar>, grid, block, smem, st, a);               \
  }
  if (groups <= 32) DTST_ROWS(32, 1)
  if (groups <= 64) DTST_ROWS(32, 2)
  if (groups <= 128) DTST_ROWS(128, 1)
  if (groups <= 256) DTST_ROWS(256, 1)
  if (groups <= 512) DTST_ROWS(512, 1)
  if (groups <= 1024) DTST_ROWS(512, 2)
  if constexpr (sizeof(T) == 4)       // (16 elements of a 16-bit type a thread would spill)
    if (groups <= 2048) DTST_ROWS(1024, 2)
#undef DTST_ROWS
  // the weight gradient first: grad_x may take grad_y's place
  const long long most = (long long)num_sms() * 4;
  cudaError_t e = cudaSuccess;
  if (a.partial != nullptr) {
    *parts = (int)(a.rows < 64 ? a.rows : 64);
    e = launch_pdl(norm_long_rows_weight_kernel<T>, dim3((unsigned)((a.C + 255) / 256), (unsigned)*parts), dim3(256), 0, st, a);
  }
  if (e != cudaSuccess) return e;
  return launch_pdl(norm_long_rows_backward_kernel<T>, dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(512), 0, st, a);
}

template <typename T>
cudaError_t forward_t(const NormCall& n, cudaStream_t st) {
  if (n.inner == 1 || n.q != nullptr) {
    RowArgs a{n.x, n.residual, n.weight, n.s, n.low, n.y, n.q, n.scale, n.rstd, n.outer, n.channels, n.x_ld, n.q_ld, n.eps, 0};
    if (n.q == nullptr) return launch_rows<T, false, true>(a, st);
    a.q_aligned = n.q_ld % 8 == 0 && aligned_to(n.q, 8);
    return n.weight != nullptr ? launch_rows<T, true, true>(a, st) : launch_rows<T, true, false>(a, st);
  }
  FieldArgs a{n.x, n.residual, nullptr, nullptr, n.weight, nullptr, n.s, n.low, n.y, n.rstd, nullptr, n.outer, n.channels, n.inner, 0, n.eps};
  int parts = 0;
  return launch_field<T, false>(a, &parts, st);
}

template <typename T>
cudaError_t backward_t(const NormBackCall& n, cudaStream_t st) {
  int parts = 0;
  cudaError_t e;
  float* partial = n.grad_weight != nullptr ? n.partial : nullptr;
  if (n.inner == 1) {
    RowBackArgs a{n.grad_y, n.s, n.low, n.grad_s, n.weight, n.rstd, n.grad_x, partial, n.outer, n.channels};
    e = launch_rows_backward<T>(a, &parts, st);
  } else {
    FieldArgs a{n.s, nullptr, n.grad_y, n.grad_s, n.weight, n.rstd, nullptr, const_cast<void*>(n.low), n.grad_x, nullptr, partial, n.outer, n.channels, n.inner, 0, 0.f};
    e = launch_field<T, true>(a, &parts, st);
  }
  if (e != cudaSuccess || partial == nullptr) return e;
  return launch_pdl(norm_weight_sum_kernel, dim3((unsigned)((n.channels + 31) / 32)), dim3(1024), 0, st,
                    static_cast<const float*>(partial), n.grad_weight, parts, (long long)n.channels);
}

}  // namespace

cudaError_t launch_norm_forward(const NormCall& n, cudaStream_t st) {
  switch (n.dtype) {
    case DTST_F32: return forward_t<float>(n, st);
    case DTST_BF16: return forward_t<__nv_bfloat16>(n, st);
    default: return forward_t<__half>(n, st);
  }
}

cudaError_t launch_norm_backward(const NormBackCall& n, cudaStream_t st) {
  switch (n.dtype) {
    case DTST_F32: return backward_t<float>(n, st);
    case DTST_BF16: return backward_t<__nv_bfloat16>(n, st);
    default: return backward_t<__half>(n, st);
  }
}

}  // namespace dtst
