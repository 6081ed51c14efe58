// Rows of channels as the norms' kernels hold them: sums over a row's threads, the layouts a row can have in memory, and the
// loads and stores of a thread's vectors.
#pragma once

#include <initializer_list>

#include "dtst_common.cuh"
#include "dtst_types.cuh"

namespace dtst {

namespace {

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

// the sum at element `at`, to 24 bits where its low part was kept
template <typename T>
__device__ __forceinline__ float sum_at(const void* s, const void* low, long long at) {
  const T v = static_cast<const T*>(s)[at];
  return sizeof(T) == 2 && low != nullptr ? LowBits<T>::join(v, static_cast<const T*>(low)[at]) : Elem<T>::get(v);
}

}  // namespace

}  // namespace dtst
