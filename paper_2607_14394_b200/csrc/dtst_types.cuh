// Element types of the recurrent-memory operators (norm, 8-bit product, recurrence) and their vector loads/stores.
// Arithmetic is in 32 bits for every type; a value is rounded once, when it is stored.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace dtst {

// Two 32-bit operations in one instruction, each rounded as the single one is: half the issue slots for the same arithmetic.
__device__ __forceinline__ float2 mul_pair(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}


// the special function unit's powers of two and reciprocals: 2 units in the last place and 1
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T>
struct Elem;

template <>
struct Elem<float> {
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct Elem<__half> {
  static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};

template <int BYTES>
struct RawOf;
template <>
struct RawOf<2> { using type = uint16_t; };
template <>
struct RawOf<4> { using type = uint32_t; };
template <>
struct RawOf<8> { using type = uint2; };
template <>
struct RawOf<16> { using type = uint4; };
struct Words8 { uint32_t w[8]; };
template <>
struct RawOf<32> { using type = Words8; };

// N elements as they lie in memory.  `load` and `store` move them in one access (the address is aligned to N
// elements; 32 bytes are global memory's widest); the `_part` forms touch only the first `n` of them, one by one.
template <typename T, int N>
struct Pack {
  using Raw = typename RawOf<N * (int)sizeof(T)>::type;
  union {
    Raw raw;
    T v[N];
  };
  __device__ __forceinline__ Pack() {}
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (sizeof(Raw) == 32)
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(raw.w[0]), "=r"(raw.w[1]), "=r"(raw.w[2]), "=r"(raw.w[3]), "=r"(raw.w[4]), "=r"(raw.w[5]), "=r"(raw.w[6]), "=r"(raw.w[7])
                   : "l"(p)
                   : "memory");
    else raw = *reinterpret_cast<const Raw*>(p);
  }
  __device__ __forceinline__ void load_part(const T* p, int n) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? p[i] : Elem<T>::put(0.f);
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (sizeof(Raw) == 32)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(raw.w[0]), "r"(raw.w[1]), "r"(raw.w[2]),
                   "r"(raw.w[3]), "r"(raw.w[4]), "r"(raw.w[5]), "r"(raw.w[6]), "r"(raw.w[7])
                   : "memory");
    else *reinterpret_cast<Raw*>(p) = raw;
  }
  __device__ __forceinline__ void store_part(T* p, int n) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = v[i];
  }
  __device__ __forceinline__ float get(int i) const { return Elem<T>::get(v[i]); }
  __device__ __forceinline__ void put(int i, float x) { v[i] = Elem<T>::put(x); }
  // all elements at once, two 16-bit ones to an instruction
  __device__ __forceinline__ void unpack(float (&x)[N]) const {
    if constexpr (sizeof(T) == 2 && N >= 2) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&raw);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) unpack2(w[i], x[2 * i], x[2 * i + 1], T());
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = get(i);
    }
  }
  __device__ __forceinline__ void pack(const float (&x)[N]) {
    if constexpr (sizeof(T) == 2 && N >= 2) {
      uint32_t* w = reinterpret_cast<uint32_t*>(&raw);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) w[i] = pack2(x[2 * i], x[2 * i + 1], T());
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) put(i, x[i]);
    }
  }
  static __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b, __nv_bfloat16) {
    a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b, __half) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x, b = f.y;
  }
  static __device__ __forceinline__ void unpack2(uint32_t, float&, float&, float) {}
  static __device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t pack2(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint32_t pack2(float, float, float) { return 0u; }
  __device__ __forceinline__ void fill(T x) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = x;
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = Elem<T>::put(0.f);
  }
};

constexpr float kE4m3Max = 448.f;
constexpr float kAmaxFloor = 0x1p-100f;   // a block of zeros keeps a finite scale, and its values stay zero
constexpr int kFp8Block = 128;            // values that share a scale along the contracted dimension

// four fp32 values -> four e4m3 values in a word, to nearest even, the largest finite value beyond the range
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What rounding a 32-bit sum to 16 bits took from it, in 16 more bits: in units of 2^-16 of the rounded value's last place, so
// that the two give the sum back to 24 bits.  (Values below 2^-80 keep nothing.)
template <typename T>
struct LowBits {
  static __device__ __forceinline__ int unit(float s) {        // exponent field of that unit's inverse
    constexpr int M = sizeof(T) == 4 ? 23 : std::is_same<T, __half>::value ? 10 : 7, LEAST = M == 10 ? 127 - 14 : 0;
    const int e = (__float_as_uint(s) >> 23) & 0xff;
    return 270 + M - (e > LEAST ? e : LEAST);
  }
  static __device__ __forceinline__ T take(float sum, T rounded) {
    const float s = Elem<T>::get(rounded);
    const int u = unit(s);
    const int lo = u > 230 ? 0 : max(-32768, min(32767, __float2int_rn((sum - s) * __uint_as_float((uint32_t)u << 23))));
    const short b = (short)lo;
    return *reinterpret_cast<const T*>(&b);
  }
  static __device__ __forceinline__ float join(T rounded, T low) {
    const float s = Elem<T>::get(rounded);
    const int u = unit(s);
    return u > 230 ? s : fmaf((float)*reinterpret_cast<const short*>(&low), __uint_as_float((uint32_t)(254 - u) << 23), s);
  }
};

// thread-block clusters
__device__ __forceinline__ int cluster_size() {
  int n;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}
__device__ __forceinline__ int cluster_rank() {
  int n;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(n));
  return n;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the value at `p` in the shared memory of CTA `rank` of the cluster
__device__ __forceinline__ float2 cluster_read(const float2* p, int rank) {
  uint32_t at;
  float2 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float4 cluster_read4(const float* p, int rank) {
  uint32_t at;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}

__device__ __forceinline__ bool aligned_to_device(const void* p, uint32_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace dtst
