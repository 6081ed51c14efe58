// C entry points of the recurrent-memory operators: argument checks, then one launch (two where a weight gradient is
// summed).  Nothing is launched when a check fails.
#include "dtst_checks.cuh"
#include "dtst_fused.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

using namespace dtst;

namespace {

dtst_status check_scan(const dtst_scan_desc* d) {
  if (d == nullptr || !known(d->dtype) || (d->gate != DTST_GATE_SIGMOID && d->gate != DTST_GATE_DECAY)) return DTST_ERR_INVALID_ARG;
  if (d->outer < 0 || d->length < 0 || d->inner < 1 || !small_product(d->outer, d->length, d->inner) ||
      !small_product(d->outer, d->inner, 1))
    return DTST_ERR_INVALID_ARG;
  for (int k = 0; k < 2; ++k)
    if (d->in_stride[k] < 0 || d->grad_stride[k] < 0 ||
        !small_product(d->in_stride[k], k == 0 ? d->outer : d->length, 1) ||
        !small_product(d->grad_stride[k], k == 0 ? d->outer : d->length, 1))
      return DTST_ERR_INVALID_ARG;
  if (d->inner == 1 && d->length > 1 && (d->in_stride[1] != 1 || d->grad_stride[1] != 1)) return DTST_ERR_INVALID_ARG;
  if (d->length > ((int64_t)1 << 30) || d->inner > ((int64_t)1 << 30) || d->outer * d->inner > ((int64_t)1 << 33)) return DTST_ERR_UNSUPPORTED;
  return DTST_OK;
}

// elements of a strided [outer, length, inner] tensor never coincide
bool distinct(const dtst_scan_desc* d) {
  const int64_t so = d->grad_stride[0], st = d->grad_stride[1];
  if (d->outer < 2) return d->length < 2 || st >= d->inner;
  if (d->length < 2) return so >= d->inner;
  return (st >= d->inner && so >= (d->length - 1) * st + d->inner) || (so >= d->inner && st >= (d->outer - 1) * so + d->inner);
}

ScanCall scan_call(const dtst_scan_desc* d) {
  ScanCall c{};
  c.dtype = d->dtype, c.gate = d->gate, c.outer = d->outer, c.length = d->length, c.inner = d->inner;
  c.in_outer = d->in_stride[0], c.in_step = d->in_stride[1];
  c.grad_outer = d->grad_stride[0], c.grad_step = d->grad_stride[1];
  return c;
}

}  // namespace

extern "C" {

dtst_status dtst_rms_norm(int dtype, int64_t outer, int64_t channels, int64_t inner, float eps, const void* x,
                          const void* residual, const float* weight, void* s, void* s_low, void* y, float* rstd,
                          void* stream) {
  if (!known(dtype) || outer < 0 || inner < 0 || channels < 1 || !(eps >= 0.f) || !small_product(outer, channels, inner))
    return DTST_ERR_INVALID_ARG;
  if (outer == 0 || inner == 0) return DTST_OK;
  if (x == nullptr || weight == nullptr || y == nullptr || y == s || y == residual || !fits(x, dtype) || !fits(residual, dtype) ||
      !fits(s, dtype) || !fits(y, dtype) || !f32(weight) || !f32(rstd))
    return DTST_ERR_INVALID_ARG;
  if (s_low != nullptr && (dtype == DTST_F32 || s == nullptr || s_low == s || s_low == y || s_low == x || s_low == residual || !fits(s_low, dtype)))
    return DTST_ERR_INVALID_ARG;
  NormCall n{dtype, outer, channels, inner, eps, x, residual, weight, s, s_low, y, nullptr, nullptr, rstd, channels, 0};
  return done(launch_norm_forward(n, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_rms_norm_scratch_bytes(int64_t channels, size_t* bytes) {
  if (channels < 1 || channels > kMostElements || bytes == nullptr) return DTST_ERR_INVALID_ARG;
  *bytes = (size_t)kNormParts * (size_t)channels * sizeof(float);
  return DTST_OK;
}

dtst_status dtst_rms_norm_backward(int dtype, int64_t outer, int64_t channels, int64_t inner, const void* grad_y,
                                   const void* s, const void* s_low, const float* weight, const float* rstd,
                                   const void* grad_s, void* grad_x, float* grad_weight, void* scratch, size_t scratch_bytes, void* stream) {
  if (!known(dtype) || outer < 0 || inner < 0 || channels < 1 || !small_product(outer, channels, inner) || !f32(grad_weight))
    return DTST_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (outer == 0 || inner == 0) {
    if (grad_weight == nullptr) return DTST_OK;
    return done(cudaMemsetAsync(grad_weight, 0, (size_t)channels * sizeof(float), st));   // an empty sum
  }
  if (grad_y == nullptr || s == nullptr || weight == nullptr || rstd == nullptr || grad_x == nullptr || grad_x == s ||
      (s_low != nullptr && (dtype == DTST_F32 || grad_x == s_low || !fits(s_low, dtype))) ||
      !fits(grad_y, dtype) || !fits(s, dtype) || !fits(grad_s, dtype) || !fits(grad_x, dtype) || !f32(weight) || !f32(rstd))
    return DTST_ERR_INVALID_ARG;
  if (grad_weight != nullptr) {
    size_t need = 0;
    dtst_rms_norm_scratch_bytes(channels, &need);
    if (scratch == nullptr || scratch_bytes < need) return DTST_ERR_WORKSPACE;
    if (!aligned_to(scratch, 16)) return DTST_ERR_INVALID_ARG;
  }
  NormBackCall n{dtype, outer, channels, inner, grad_y, s, s_low, grad_s, weight, rstd, grad_x, grad_weight, static_cast<float*>(scratch)};
  return done(launch_norm_backward(n, st));
}

dtst_status dtst_rms_norm_fp8(int dtype, int64_t rows, int64_t channels, float eps, const void* x, const void* residual,
                              const float* weight, void* s, void* q, int64_t q_ld, float* scale, void* stream) {
  if (!known(dtype) || rows < 0 || channels < 1 || q_ld < channels || !(eps >= 0.f) || !small_product(rows, q_ld, 1))
    return DTST_ERR_INVALID_ARG;
  if (rows == 0) return DTST_OK;
  if (x == nullptr || weight == nullptr || q == nullptr || scale == nullptr || q == x || q == s || q == residual ||
      !fits(x, dtype) || !fits(residual, dtype) || !fits(s, dtype) || !f32(weight) || !f32(scale))
    return DTST_ERR_INVALID_ARG;
  NormCall n{dtype, rows, channels, 1, eps, x, residual, weight, s, nullptr, nullptr, static_cast<uint8_t*>(q), scale, nullptr, channels, q_ld};
  return done(launch_norm_forward(n, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_quantize_fp8(int dtype, int64_t rows, int64_t channels, const void* x, int64_t x_ld, void* q,
                              int64_t q_ld, float* scale, void* stream) {
  if (!known(dtype) || rows < 0 || channels < 1 || q_ld < channels || x_ld < 0 || (rows > 1 && x_ld < channels) ||
      !small_product(rows, q_ld, 1) || !small_product(rows, x_ld, 1))
    return DTST_ERR_INVALID_ARG;
  if (rows == 0) return DTST_OK;
  if (x == nullptr || q == nullptr || scale == nullptr || q == x || !fits(x, dtype) || !f32(scale)) return DTST_ERR_INVALID_ARG;
  NormCall n{dtype, rows, channels, 1, 0.f, x, nullptr, nullptr, nullptr, nullptr, nullptr, static_cast<uint8_t*>(q), scale, nullptr, x_ld, q_ld};
  return done(launch_norm_forward(n, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_quantize_fp8_weight(int dtype, int64_t rows, int64_t cols, const void* w, int64_t w_ld, void* q,
                                     int64_t q_ld, float* scale, void* stream) {
  if (!known(dtype) || rows < 0 || cols < 1 || w_ld < cols || q_ld < cols || !small_product(rows, w_ld, 1) ||
      !small_product(rows, q_ld, 1))
    return DTST_ERR_INVALID_ARG;
  if (rows == 0) return DTST_OK;
  if (w == nullptr || q == nullptr || scale == nullptr || q == w || !fits(w, dtype) || !f32(scale)) return DTST_ERR_INVALID_ARG;
  if ((rows + 127) / 128 > 65535 || cols > kMostCtas) return DTST_ERR_UNSUPPORTED;
  return done(launch_quantize_weight(dtype, w, w_ld, static_cast<uint8_t*>(q), q_ld, scale, rows, cols, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_matmul_fp8(int out_dtype, int64_t m, int64_t n, int64_t k, const void* x, int64_t x_ld,
                            const float* x_scale, const void* w, int64_t w_ld, const float* w_scale, void* out,
                            int64_t out_ld, void* workspace, size_t workspace_bytes, void* stream) {
  if (!known(out_dtype) || m < 0 || n < 0 || k < 1 || x_ld < k || w_ld < k || out_ld < n || x_ld % 16 != 0 || w_ld % 16 != 0 ||
      !small_product(m, x_ld, 1) || !small_product(n, w_ld, 1) || !small_product(m, out_ld, 1))
    return DTST_ERR_INVALID_ARG;
  if (m == 0 || n == 0) return DTST_OK;
  if (x == nullptr || x_scale == nullptr || w == nullptr || w_scale == nullptr || out == nullptr || !aligned_to(x, 16) ||
      !aligned_to(w, 16) || !f32(x_scale) || !f32(w_scale) || !fits(out, out_dtype))
    return DTST_ERR_INVALID_ARG;
  if (workspace == nullptr || workspace_bytes < kStatusBytes) return DTST_ERR_WORKSPACE;
  if (!workspace_ok(workspace)) return DTST_ERR_INVALID_ARG;
  // tile counts, coordinates and rows are 32-bit inside the kernel
  const int64_t most = ((int64_t)1 << 31) - 256;
  if (m > most || n > most || k > most || x_ld > most || w_ld > most || ((m + 31) / 32) * ((n + 31) / 32) > most ||
      !matmul_fp8_available())
    return DTST_ERR_UNSUPPORTED;
  MatmulCall c{out_dtype, m, n, k, x_ld, w_ld, out_ld, static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(w),
               x_scale, w_scale, out, static_cast<int*>(workspace)};
  return done(launch_matmul_fp8(c, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_gated_scan_checkpoints(const dtst_scan_desc* d, int64_t* checkpoint_floats) {
  const dtst_status s = check_scan(d);
  if (s != DTST_OK) return s;
  if (checkpoint_floats == nullptr) return DTST_ERR_INVALID_ARG;
  const int64_t lc = scan_chunk(d->dtype, d->length, d->inner);
  *checkpoint_floats = (d->length + lc - 1) / lc * d->outer * d->inner;
  return DTST_OK;
}

dtst_status dtst_gated_scan(const dtst_scan_desc* d, const void* v, const void* g, const float* h0, const int32_t* lengths,
                            void* h, float* h_last, float* checkpoints, void* stream) {
  const dtst_status s = check_scan(d);
  if (s != DTST_OK) return s;
  if (!f32(h0) || !f32(h_last) || !f32(lengths) || !f32(checkpoints)) return DTST_ERR_INVALID_ARG;
  if (d->outer == 0) return DTST_OK;
  if (d->length > 0 && (v == nullptr || g == nullptr || h == nullptr || h == v || h == g || !fits(v, d->dtype) ||
                        !fits(g, d->dtype) || !fits(h, d->dtype) || (checkpoints != nullptr && checkpoints == h0)))
    return DTST_ERR_INVALID_ARG;
  ScanCall c = scan_call(d);
  c.v = v, c.g = g, c.h0 = h0, c.lengths = lengths, c.h = h, c.h_last = h_last, c.checkpoints = checkpoints;
  return done(launch_scan_forward(c, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_gated_scan_backward(const dtst_scan_desc* d, const void* grad_h, const float* grad_last, const void* v,
                                     const void* g, const float* h0, const int32_t* lengths, const float* checkpoints,
                                     void* grad_v, void* grad_g, float* grad_h0, void* stream) {
  const dtst_status s = check_scan(d);
  if (s != DTST_OK) return s;
  if (!f32(h0) || !f32(grad_last) || !f32(lengths) || !f32(checkpoints) || !f32(grad_h0)) return DTST_ERR_INVALID_ARG;
  if (d->outer == 0) return DTST_OK;
  if (d->length > 0) {
    if (!distinct(d) || grad_h == nullptr || v == nullptr || g == nullptr || grad_v == nullptr || grad_g == nullptr || grad_v == grad_g ||
        grad_v == v || grad_v == g || grad_g == v || grad_g == g || grad_v == grad_h || grad_g == grad_h ||
        !fits(grad_h, d->dtype) || !fits(v, d->dtype) || !fits(g, d->dtype) || !fits(grad_v, d->dtype) || !fits(grad_g, d->dtype))
      return DTST_ERR_INVALID_ARG;
    // a pass longer than one chunk restarts from saved states
    if (checkpoints == nullptr && d->length > scan_chunk(d->dtype, d->length, d->inner)) return DTST_ERR_INVALID_ARG;
  }
  ScanCall c = scan_call(d);
  c.grad_h = grad_h, c.grad_last = grad_last, c.v = v, c.g = g, c.h0 = h0, c.lengths = lengths;
  c.checkpoints = const_cast<float*>(checkpoints);
  c.grad_v = grad_v, c.grad_g = grad_g, c.grad_h0 = grad_h0;
  return done(launch_scan_backward(c, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_gated_scan_status(void* stream) {
  int word = 0;
  const dtst_status s = done(scan_status(&word, static_cast<cudaStream_t>(stream)));
  return s != DTST_OK ? s : word == 0 ? DTST_OK : DTST_ERR_DEVICE_TIMEOUT;
}

dtst_status dtst_workspace_status(void* workspace, void* stream) {
  if (!workspace_ok(workspace)) return DTST_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int word = 0;
  if (cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, st) != cudaSuccess ||
      cudaStreamSynchronize(st) != cudaSuccess || (word != 0 && cudaMemsetAsync(workspace, 0, sizeof(word), st) != cudaSuccess)) {
    (void)cudaGetLastError();
    return DTST_ERR_CUDA;
  }
  return word == 0 ? DTST_OK : DTST_ERR_DEVICE_TIMEOUT;
}

}  // extern "C"
