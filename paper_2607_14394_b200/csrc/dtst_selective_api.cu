// C entry points of the selective memory's operators (layer norm, causal convolution, selective scan) and of the gradients'
// norm: argument checks, then the launches.  Nothing is launched when a check fails.
#include <algorithm>
#include <new>
#include <vector>

#include "dtst_checks.cuh"
#include "dtst_memory.cuh"
#include "dtst_types.cuh"

using namespace dtst;

namespace {

// strides of a token-major tensor: entries and steps, neither of which may go backwards
bool strides_ok(const int64_t (&s)[2], int64_t batch, int64_t length) {
  return s[0] >= 0 && s[1] >= 0 && small_product(s[0], batch, 1) && small_product(s[1], length, 1);
}
// elements of a [batch][length][width] tensor of these strides never coincide
bool distinct(const int64_t (&s)[2], int64_t batch, int64_t length, int64_t width) {
  if (batch < 1 || length < 1) return true;
  if (batch < 2) return length < 2 || s[1] >= width;
  if (length < 2) return s[0] >= width;
  return (s[1] >= width && s[0] >= (length - 1) * s[1] + width) || (s[0] >= width && s[1] >= (batch - 1) * s[0] + width);
}

dtst_status check_conv(const dtst_conv_desc* d) {
  if (d == nullptr || !known(d->dtype) || (d->activation != DTST_ACT_NONE && d->activation != DTST_ACT_SILU)) return DTST_ERR_INVALID_ARG;
  if (d->batch < 0 || d->length < 0 || d->channels < 1 || d->width < 1 || !small_product(d->batch, d->length, d->channels) ||
      !small_product(d->batch, d->channels, 8) || !strides_ok(d->x_stride, d->batch, d->length) || !strides_ok(d->grad_stride, d->batch, d->length))
    return DTST_ERR_INVALID_ARG;
  if (d->width > kConvWidth || d->length > ((int64_t)1 << 30) || d->channels > ((int64_t)1 << 30) || d->batch > ((int64_t)1 << 30))
    return DTST_ERR_UNSUPPORTED;
  return DTST_OK;
}
ConvCall conv_call(const dtst_conv_desc* d) {
  ConvCall c{};
  c.dtype = d->dtype, c.width = d->width, c.silu = d->activation == DTST_ACT_SILU;
  c.batch = d->batch, c.length = d->length, c.channels = d->channels;
  for (int k = 0; k < 2; ++k) c.x_stride[k] = d->x_stride[k], c.grad_stride[k] = d->grad_stride[k];
  return c;
}

dtst_status check_selective(const dtst_selective_desc* d) {
  if (d == nullptr || !known(d->dtype) || d->batch < 0 || d->length < 0 || d->channels < 1 || d->states < 1 || d->groups < 1 ||
      d->channels % d->groups != 0 || !small_product(d->batch, d->length, d->channels) || !small_product(d->channels, d->states, 1) ||
      !small_product(d->batch, d->channels * d->states, 1) || !small_product(d->batch, d->length, d->groups * d->states))
    return DTST_ERR_INVALID_ARG;
  for (const auto* s : {&d->x_stride, &d->dt_stride, &d->z_stride, &d->b_stride, &d->c_stride, &d->grad_x_stride, &d->grad_dt_stride,
                        &d->grad_z_stride, &d->grad_b_stride, &d->grad_c_stride})
    if (!strides_ok(*s, d->batch, d->length)) return DTST_ERR_INVALID_ARG;
  if (d->states > kSelectiveStates || d->batch > 65535 || d->length > ((int64_t)1 << 30) || d->channels > ((int64_t)1 << 24))
    return DTST_ERR_UNSUPPORTED;
  return DTST_OK;
}
Rows rows(const void* p, const int64_t (&s)[2]) { return Rows{const_cast<void*>(p), s[0], s[1]}; }
SelectiveCall selective_call(const dtst_selective_desc* d) {
  SelectiveCall c{};
  c.dtype = d->dtype, c.softplus = d->softplus != 0;
  c.batch = d->batch, c.length = d->length, c.channels = d->channels, c.states = d->states, c.groups = d->groups;
  return c;
}
// what both passes read
bool inputs_ok(const dtst_selective_desc* d, const dtst_selective_inputs* in) {
  if (in == nullptr || in->A == nullptr || !f32(in->A) || !f32(in->D) || !f32(in->dt_bias) || !f32(in->h0) || !f32(in->lengths)) return false;
  if (d->length == 0) return true;
  for (const void* p : {in->x, in->dt, in->B, in->C})
    if (p == nullptr || !fits(p, d->dtype)) return false;
  return fits(in->z, d->dtype);
}
void set_inputs(SelectiveCall& c, const dtst_selective_desc* d, const dtst_selective_inputs* in) {
  c.x = rows(in->x, d->x_stride), c.dt = rows(in->dt, d->dt_stride), c.z = rows(in->z, d->z_stride);
  c.B = rows(in->B, d->b_stride), c.C = rows(in->C, d->c_stride);
  c.A = in->A, c.D = in->D, c.bias = in->dt_bias, c.h0 = in->h0, c.lengths = in->lengths;
}

}  // namespace

extern "C" {

dtst_status dtst_layer_norm(int dtype, int64_t outer, int64_t channels, int64_t inner, float eps, const void* x, const void* residual,
                            const float* weight, const float* bias, void* s, void* s_low, void* y, float* stats, void* stream) {
  if (!known(dtype) || outer < 0 || inner < 0 || channels < 1 || !(eps >= 0.f) || !small_product(outer, channels, inner))
    return DTST_ERR_INVALID_ARG;
  if (outer == 0 || inner == 0) return DTST_OK;
  if (x == nullptr || weight == nullptr || y == nullptr || y == s || y == residual || !fits(x, dtype) || !fits(residual, dtype) ||
      !fits(s, dtype) || !fits(y, dtype) || !f32(weight) || !f32(bias) || !f32(stats))
    return DTST_ERR_INVALID_ARG;
  if (s_low != nullptr && (dtype == DTST_F32 || s == nullptr || s_low == s || s_low == y || s_low == x || s_low == residual || !fits(s_low, dtype)))
    return DTST_ERR_INVALID_ARG;
  const LayerNormCall n{dtype, outer, channels, inner, eps, x, residual, weight, bias, s, s_low, y, stats};
  return done(launch_layer_norm(n, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_layer_norm_scratch_bytes(int64_t channels, size_t* bytes) {
  if (channels < 1 || channels > kMostElements || bytes == nullptr) return DTST_ERR_INVALID_ARG;
  *bytes = (size_t)2 * kNormParts * (size_t)channels * sizeof(float);
  return DTST_OK;
}

dtst_status dtst_layer_norm_backward(int dtype, int64_t outer, int64_t channels, int64_t inner, const void* grad_y, const void* s,
                                     const void* s_low, const float* weight, const float* stats, const void* grad_s, void* grad_x,
                                     float* grad_weight, float* grad_bias, void* scratch, size_t scratch_bytes, void* stream) {
  if (!known(dtype) || outer < 0 || inner < 0 || channels < 1 || !small_product(outer, channels, inner) || !f32(grad_weight) ||
      !f32(grad_bias) || (grad_weight != nullptr && grad_weight == grad_bias))
    return DTST_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (outer == 0 || inner == 0) {              // empty sums
    for (float* g : {grad_weight, grad_bias}) {
      const dtst_status e = g == nullptr ? DTST_OK : done(cudaMemsetAsync(g, 0, (size_t)channels * sizeof(float), st));
      if (e != DTST_OK) return e;
    }
    return DTST_OK;
  }
  if (grad_y == nullptr || s == nullptr || weight == nullptr || stats == nullptr || grad_x == nullptr || grad_x == s ||
      (s_low != nullptr && (dtype == DTST_F32 || grad_x == s_low || !fits(s_low, dtype))) || !fits(grad_y, dtype) || !fits(s, dtype) ||
      !fits(grad_s, dtype) || !fits(grad_x, dtype) || !f32(weight) || !f32(stats))
    return DTST_ERR_INVALID_ARG;
  if (grad_weight != nullptr || grad_bias != nullptr) {
    size_t need = 0;
    dtst_layer_norm_scratch_bytes(channels, &need);
    if (scratch == nullptr || scratch_bytes < need) return DTST_ERR_WORKSPACE;
    if (!aligned_to(scratch, 16)) return DTST_ERR_INVALID_ARG;
  }
  const LayerNormBackCall n{dtype, outer, channels, inner, grad_y, s, s_low, grad_s, weight, stats, grad_x, grad_weight, grad_bias, static_cast<float*>(scratch)};
  return done(launch_layer_norm_backward(n, st));
}

dtst_status dtst_causal_conv(const dtst_conv_desc* d, const void* x, const float* weight, const float* bias, const void* state,
                             const int32_t* lengths, void* y, void* state_out, void* stream) {
  const dtst_status s = check_conv(d);
  if (s != DTST_OK) return s;
  if (!f32(weight) || !f32(bias) || !f32(lengths) || !fits(state, d->dtype) || !fits(state_out, d->dtype)) return DTST_ERR_INVALID_ARG;
  if (d->batch == 0) return DTST_OK;
  if (weight == nullptr || (d->length > 0 && (x == nullptr || y == nullptr || y == x || y == state || y == state_out || x == state_out ||
                                              !fits(x, d->dtype) || !fits(y, d->dtype))))
    return DTST_ERR_INVALID_ARG;
  if (d->length == 0 && (d->width == 1 || state_out == nullptr)) return DTST_OK;
  ConvCall c = conv_call(d);
  c.x = x, c.weight = weight, c.bias = bias, c.state = state, c.lengths = lengths, c.y = y, c.state_out = state_out;
  return done(launch_conv_forward(c, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_causal_conv_scratch_bytes(const dtst_conv_desc* d, size_t* bytes) {
  const dtst_status s = check_conv(d);
  if (s != DTST_OK) return s;
  if (bytes == nullptr) return DTST_ERR_INVALID_ARG;
  *bytes = (size_t)conv_parts(d->channels) * (size_t)d->channels * (size_t)(d->width + 1) * sizeof(float);
  return DTST_OK;
}

dtst_status dtst_causal_conv_backward(const dtst_conv_desc* d, const void* grad_y, const void* grad_state_out, const void* x,
                                      const float* weight, const float* bias, const void* state, const int32_t* lengths, void* grad_x,
                                      float* grad_weight, float* grad_bias, void* grad_state, void* scratch, size_t scratch_bytes, void* stream) {
  const dtst_status s = check_conv(d);
  if (s != DTST_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!f32(weight) || !f32(bias) || !f32(lengths) || !f32(grad_weight) || !f32(grad_bias) || (grad_weight != nullptr && grad_weight == grad_bias) ||
      !fits(state, d->dtype) || !fits(grad_state, d->dtype) || !fits(grad_state_out, d->dtype) ||
      (grad_state != nullptr && (grad_state == grad_state_out || grad_state == state)))
    return DTST_ERR_INVALID_ARG;
  if (d->batch == 0) {                         // empty sums
    dtst_status e = DTST_OK;
    if (grad_weight != nullptr) e = done(cudaMemsetAsync(grad_weight, 0, (size_t)(d->channels * d->width) * sizeof(float), st));
    if (grad_bias != nullptr && e == DTST_OK) e = done(cudaMemsetAsync(grad_bias, 0, (size_t)d->channels * sizeof(float), st));
    return e;
  }
  if (weight == nullptr || !distinct(d->grad_stride, d->batch, d->length, d->channels) ||
      (d->length > 0 && (x == nullptr || grad_y == nullptr || grad_x == nullptr || grad_x == x || grad_x == grad_y || grad_x == state ||
                         grad_x == grad_state || grad_x == grad_state_out || !fits(x, d->dtype) || !fits(grad_y, d->dtype) || !fits(grad_x, d->dtype))))
    return DTST_ERR_INVALID_ARG;
  if (grad_weight != nullptr || grad_bias != nullptr) {
    size_t need = 0;
    dtst_causal_conv_scratch_bytes(d, &need);
    if (scratch == nullptr || scratch_bytes < need) return DTST_ERR_WORKSPACE;
    if (!aligned_to(scratch, 16)) return DTST_ERR_INVALID_ARG;
  }
  ConvCall c = conv_call(d);
  c.x = x, c.weight = weight, c.bias = bias, c.state = state, c.lengths = lengths, c.grad_y = grad_y, c.grad_state_out = grad_state_out;
  c.grad_x = grad_x, c.grad_state = grad_state, c.grad_weight = grad_weight, c.grad_bias = grad_bias, c.partial = static_cast<float*>(scratch);
  return done(launch_conv_backward(c, st));
}

dtst_status dtst_selective_scan_checkpoints(const dtst_selective_desc* d, int64_t* checkpoint_floats) {
  const dtst_status s = check_selective(d);
  if (s != DTST_OK) return s;
  if (checkpoint_floats == nullptr) return DTST_ERR_INVALID_ARG;
  *checkpoint_floats = d->batch * ((d->length + kSelectiveSave - 1) / kSelectiveSave) * d->channels * ((d->states + 3) / 4 * 4);
  return DTST_OK;
}

dtst_status dtst_selective_scan(const dtst_selective_desc* d, const dtst_selective_inputs* in, void* y, float* h_last, float* checkpoints,
                                void* scratch, size_t scratch_bytes, void* stream) {
  const dtst_status s = check_selective(d);
  if (s != DTST_OK) return s;
  if (d->batch == 0) return DTST_OK;
  if (!inputs_ok(d, in) || !f32(h_last) || !aligned_to(checkpoints, 16)) return DTST_ERR_INVALID_ARG;
  if (d->length > 0) {
    if (y == nullptr || !fits(y, d->dtype)) return DTST_ERR_INVALID_ARG;
    for (const void* p : {in->x, in->dt, in->z, in->B, in->C})
      if (p == y) return DTST_ERR_INVALID_ARG;
  }
  size_t need = 0;
  dtst_selective_scan_scratch_bytes(d, 0, &need);
  if (need > 0 && (scratch == nullptr || scratch_bytes < need)) return DTST_ERR_WORKSPACE;
  if (!aligned_to(scratch, 16)) return DTST_ERR_INVALID_ARG;
  SelectiveCall c = selective_call(d);
  set_inputs(c, d, in);
  c.scratch = static_cast<float*>(scratch);
  c.y = y, c.h_last = h_last, c.checkpoints = checkpoints;
  return done(launch_selective_forward(c, static_cast<cudaStream_t>(stream)));
}

dtst_status dtst_selective_scan_scratch_bytes(const dtst_selective_desc* d, int backward, size_t* bytes) {
  const dtst_status s = check_selective(d);
  if (s != DTST_OK) return s;
  if (bytes == nullptr) return DTST_ERR_INVALID_ARG;
  *bytes = (size_t)selective_scratch_floats(selective_call(d), backward != 0) * sizeof(float);
  return DTST_OK;
}

dtst_status dtst_selective_scan_backward(const dtst_selective_desc* d, const dtst_selective_inputs* in, const void* grad_y, const float* grad_last,
                                         const float* checkpoints, const dtst_selective_grads* g, void* scratch, size_t scratch_bytes, void* stream) {
  const dtst_status s = check_selective(d);
  if (s != DTST_OK) return s;
  if (g == nullptr || !f32(g->A) || !f32(g->D) || !f32(g->dt_bias) || !f32(g->h0)) return DTST_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (d->batch == 0) {                         // empty sums
    const struct { float* p; int64_t n; } sums[3] = {{g->A, d->channels * d->states}, {g->D, d->channels}, {g->dt_bias, d->channels}};
    for (const auto& q : sums) {
      const dtst_status e = q.p == nullptr ? DTST_OK : done(cudaMemsetAsync(q.p, 0, (size_t)q.n * sizeof(float), st));
      if (e != DTST_OK) return e;
    }
    return DTST_OK;
  }
  if (!inputs_ok(d, in) || !f32(grad_last)) return DTST_ERR_INVALID_ARG;
  if (d->length > 0) {
    if (grad_y == nullptr || !fits(grad_y, d->dtype) || checkpoints == nullptr || !aligned_to(checkpoints, 16)) return DTST_ERR_INVALID_ARG;
    const struct { const void* p; const int64_t (&s)[2]; int64_t width; } outs[5] = {
        {g->x, d->grad_x_stride, d->channels}, {g->dt, d->grad_dt_stride, d->channels}, {g->z, d->grad_z_stride, d->channels},
        {g->B, d->grad_b_stride, d->groups * d->states}, {g->C, d->grad_c_stride, d->groups * d->states}};
    for (int i = 0; i < 5; ++i) {
      if (i == 2 && in->z == nullptr) continue;
      if (outs[i].p == nullptr || !fits(outs[i].p, d->dtype) || !distinct(outs[i].s, d->batch, d->length, outs[i].width)) return DTST_ERR_INVALID_ARG;
      for (const void* p : {in->x, in->dt, in->z, in->B, in->C, grad_y})
        if (p == outs[i].p) return DTST_ERR_INVALID_ARG;
      for (int j = 0; j < i; ++j)
        if (outs[j].p == outs[i].p) return DTST_ERR_INVALID_ARG;
    }
  }
  size_t need = 0;
  dtst_selective_scan_scratch_bytes(d, 1, &need);
  if (scratch == nullptr || scratch_bytes < need) return DTST_ERR_WORKSPACE;
  if (!aligned_to(scratch, 16)) return DTST_ERR_INVALID_ARG;
  SelectiveCall c = selective_call(d);
  set_inputs(c, d, in);
  c.grad_y = grad_y, c.grad_last = grad_last, c.checkpoints = const_cast<float*>(checkpoints);
  c.grad_x = rows(g->x, d->grad_x_stride), c.grad_dt = rows(g->dt, d->grad_dt_stride), c.grad_z = rows(g->z, d->grad_z_stride);
  c.grad_B = rows(g->B, d->grad_b_stride), c.grad_C = rows(g->C, d->grad_c_stride);
  c.grad_A = g->A, c.grad_D = g->D, c.grad_bias = g->dt_bias, c.grad_h0 = g->h0, c.scratch = static_cast<float*>(scratch);
  return done(launch_selective_backward(c, st));
}

dtst_status dtst_grad_norm_scratch_bytes(int64_t count, size_t* bytes) {
  if (count < 0 || count > ((int64_t)1 << 20) || bytes == nullptr) return DTST_ERR_INVALID_ARG;
  *bytes = ((size_t)grad_launches(count) * kGradParts + 1) * sizeof(double);
  return DTST_OK;
}

dtst_status dtst_clip_grad_norm(const dtst_grad_tensor* list, int64_t count, float max_norm, float eps, float* norm, void* scratch,
                                size_t scratch_bytes, void* stream) {
  size_t need = 0;
  if (dtst_grad_norm_scratch_bytes(count, &need) != DTST_OK || (list == nullptr && count > 0) || norm == nullptr || !f32(norm) ||
      !(max_norm >= 0.f) || !(eps > 0.f))
    return DTST_ERR_INVALID_ARG;
  bool scale = false;
  // no exception leaves a C entry
  try {
    std::vector<GradEntry> entries;
    struct Span { uintptr_t from, to; int64_t of; };
    std::vector<Span> written, read;
    entries.reserve((size_t)count);
    const uintptr_t at = reinterpret_cast<uintptr_t>(norm);
    const auto holds_norm = [&](uintptr_t from, uintptr_t to) { return from < at + sizeof(float) && at < to; };
    for (int64_t k = 0; k < count; ++k) {
      const dtst_grad_tensor& t = list[k];
      if (!known(t.dtype) || t.n < 0 || t.n > kMostElements) return DTST_ERR_INVALID_ARG;
      if (t.n == 0) continue;
      if (t.grad == nullptr || !fits(t.grad, t.dtype) || !fits(t.out, t.dtype)) return DTST_ERR_INVALID_ARG;
      const uintptr_t bytes = (uintptr_t)t.n * elem(t.dtype), g = reinterpret_cast<uintptr_t>(t.grad), o = reinterpret_cast<uintptr_t>(t.out);
      if (holds_norm(g, g + bytes) || (t.out != nullptr && holds_norm(o, o + bytes))) return DTST_ERR_INVALID_ARG;
      read.push_back({g, g + bytes, k});
      if (t.out != nullptr) written.push_back({o, o + bytes, k});
      entries.push_back({t.grad, t.out, t.n, t.dtype});
    }
    scale = !written.empty();
    if (scale) {
      // what is written must be apart from everything else, but for a gradient's own place
      const auto by = [](const Span& a, const Span& b) { return a.from < b.from || (a.from == b.from && a.to < b.to); };
      std::sort(written.begin(), written.end(), by);
      for (size_t i = 1; i < written.size(); ++i)
        if (written[i].from < written[i - 1].to) return DTST_ERR_INVALID_ARG;
      for (const Span& r : read) {
        auto w = std::upper_bound(written.begin(), written.end(), r.from, [](uintptr_t v, const Span& s) { return v < s.to; });
        for (; w != written.end() && w->from < r.to; ++w)
          if (w->of != r.of || w->from != r.from) return DTST_ERR_INVALID_ARG;
      }
    }
    if (scratch == nullptr || scratch_bytes < need) return DTST_ERR_WORKSPACE;
    if (!aligned_to(scratch, 16)) return DTST_ERR_INVALID_ARG;
    return done(launch_grad_norm(entries.data(), (long long)entries.size(), max_norm, eps, scale, norm, static_cast<double*>(scratch),
                                 static_cast<cudaStream_t>(stream)));
  } catch (const std::bad_alloc&) {
    return DTST_ERR_ALLOC;
  }
}

}  // extern "C"
