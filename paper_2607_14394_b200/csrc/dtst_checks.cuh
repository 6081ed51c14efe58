// Argument checks shared by the C entry points of the memory operators.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/dtst.h"
#include "dtst_types.cuh"

namespace dtst {

namespace {

constexpr int64_t kMostElements = (int64_t)1 << 46;   // keeps every product of extents and strides inside 64 bits
constexpr int64_t kMostCtas = 0x7fffffff;

bool known(int dtype) { return dtype == DTST_F32 || dtype == DTST_BF16 || dtype == DTST_F16; }
size_t elem(int dtype) { return dtype == DTST_F32 ? 4 : 2; }
bool fits(const void* p, int dtype) { return aligned_to(p, elem(dtype)); }
bool f32(const void* p) { return aligned_to(p, 4); }

// whether a * b * c stays within the range above (all non-negative)
bool small_product(int64_t a, int64_t b, int64_t c) {
  if (a == 0 || b == 0 || c == 0) return true;
  return a <= kMostElements && b <= kMostElements / a && c <= kMostElements / (a * b);
}

dtst_status done(cudaError_t e) {
  if (e == cudaSuccess) return DTST_OK;
  (void)cudaGetLastError();
  return e == cudaErrorNotSupported ? DTST_ERR_UNSUPPORTED : DTST_ERR_CUDA;
}

bool workspace_ok(const void* ws) { return ws != nullptr && aligned_to(ws, 256); }

}  // namespace

}  // namespace dtst
