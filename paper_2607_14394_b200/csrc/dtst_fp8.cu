// Matrix product of 8-bit floating-point operands (e4m3) with a scale for each block of 128 along the contracted
// dimension:
//     out[m, n] = sum_kb  x_scale[kb, m] w_scale[n / 128, kb]  sum_{k in block kb} x[m, k] w[n, k]
// on the fifth-generation tensor cores.  A k-block of 128 values is 128 bytes: one row of a 128-byte-swizzled TMA
// tile and four tcgen05.mma (kind::f8f6f4, K = 32).  The scales differ from block to block, so the tensor core sums
// one block into tensor memory, and the epilogue warps add it, scaled, to fp32 sums in registers while the next block
// is multiplied into the other half of the tensor memory.
//
// A CTA computes tiles of 128 lanes x BN columns.  Warp 0 issues the TMA loads, warp 1 the products, the others hold
// the sums (a thread one lane x up to 128 columns).  Lanes are rows of x and columns rows of w, or the other way round
// (SWAP) where there are few rows of x: the tile's 128 lanes are then filled by the weights.
// Every wait is bounded: on expiry the kernel raises the status word, drains its loads and products, frees its tensor
// memory and returns.
#include <cuda.h>

#include "dtst_common.cuh"
#include "dtst_fused.cuh"
#include "dtst_memory.cuh"
#include "dtst_sm100.cuh"
#include "dtst_types.cuh"

namespace dtst {

using namespace sm100;

namespace {

constexpr int kLanes = 128;
constexpr uint32_t kWaitLimit = 1u << 20;

struct MatmulArgs {
  const float *x_scale, *w_scale;
  void* out;
  long long out_ld;
  int M, N, KB;             // rows of x, rows of w, blocks along the contracted dimension
  int lane_tiles, col_tiles;
  int vec_out;              // rows of out start on 16-byte boundaries
  int* status;
};

// bounded wait without sleeping (the hardware suspends the thread inside try_wait)
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  for (uint32_t it = 0; it < kWaitLimit; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 255u) == 255u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}

// K-major operand with the 128-byte swizzle: rows of 128 bytes, 8-row groups 1024 bytes apart
__device__ __forceinline__ uint64_t desc_sw128(uint32_t addr) {
  return (uint64_t)((addr >> 4) & 0x3fffu) | (1ull << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// kind::f8f6f4: fp32 accumulator, both operands e4m3 and K-major
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N) {
  return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void umma_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 16 columns of this thread's lane; the values are valid after tmem_wait on the same registers
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

template <int BN>
struct MatmulCfg {
  static constexpr int CW = BN < 128 ? BN : 128;           // columns of an epilogue thread
  static constexpr int EPI = BN > 128 ? 8 : 4;             // epilogue warps
  static constexpr int THREADS = 64 + 32 * EPI;
  static constexpr int A_BYTES = kLanes * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
  static constexpr int STAGES = STAGE > 32768 ? 4 : 6;
  static constexpr int TCOLS = 2 * BN < 32 ? 32 : 2 * BN;
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + 2 * BN * 4 + 256;
};

template <typename T, int BN, bool SWAP>
__global__ void __launch_bounds__(MatmulCfg<BN>::THREADS, 1)
matmul_fp8_kernel(const __grid_constant__ CUtensorMap lane_map, const __grid_constant__ CUtensorMap col_map, const MatmulArgs p) {
  using Cfg = MatmulCfg<BN>;
  pdl_trigger();
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  float* col_scale = reinterpret_cast<float*>(smem + (size_t)Cfg::STAGES * Cfg::STAGE);   // [2][BN], SWAP only
  uint64_t* full = reinterpret_cast<uint64_t*>(col_scale + 2 * BN);
  uint64_t* empty = full + Cfg::STAGES;
  uint64_t* done = empty + Cfg::STAGES;      // [2] products of a block complete
  uint64_t* freed = done + 2;                // [2] tensor-memory half read
  uint32_t* tmem_s = reinterpret_cast<uint32_t*>(freed + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_s + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < Cfg::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int k = 0; k < 2; ++k) {
      mbar_init(&done[k], 1);
      mbar_init(&freed[k], Cfg::EPI);
    }
    *abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&lane_map);
    prefetch_tensormap(&col_map);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_s)),
                 "r"((uint32_t)Cfg::TCOLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_s;

  const int tiles = p.lane_tiles * p.col_tiles;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
        const int l0 = (t % p.lane_tiles) * kLanes, c0 = (t / p.lane_tiles) * BN;
        for (int kb = 0; kb < p.KB; ++kb, ++it) {
          const uint32_t s = it % Cfg::STAGES;
          if (!wait_bar(&empty[s], ((it / Cfg::STAGES) & 1) ^ 1, abort_flag)) goto out;
          mbar_arrive_expect_tx(&full[s], (uint32_t)Cfg::STAGE);
          tma_load_2d(smem + (size_t)s * Cfg::STAGE, &lane_map, kb * 128, l0, &full[s]);
          tma_load_2d(smem + (size_t)s * Cfg::STAGE + Cfg::A_BYTES, &col_map, kb * 128, c0, &full[s]);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_e4m3(kLanes, BN);
      uint32_t it = 0;
      for (int t = blockIdx.x; t < tiles; t += gridDim.x)
        for (int kb = 0; kb < p.KB; ++kb, ++it) {
          const uint32_t s = it % Cfg::STAGES, half = it & 1;
          if (!wait_bar(&freed[half], ((it >> 1) & 1) ^ 1, abort_flag)) goto out;
          if (!wait_bar(&full[s], (it / Cfg::STAGES) & 1, abort_flag)) goto out;
          tc_fence_after();
          const uint32_t a = smem_u32(smem + (size_t)s * Cfg::STAGE), b = a + Cfg::A_BYTES;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            umma_f8(tmem + half * BN, desc_sw128(a + 32 * ks), desc_sw128(b + 32 * ks), idesc, ks > 0 ? 1u : 0u);
          umma_commit(&empty[s]);
          umma_commit(&done[half]);
        }
    }
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    const int ln = quarter * 32 + lane;               // this thread's lane of the tile
    const int et = threadIdx.x - 64;                  // 0 .. 32 EPI - 1
    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(part * Cfg::CW);
    uint32_t it = 0;
    for (int t = blockIdx.x; t < tiles; t += gridDim.x) {
      const int l0 = (t % p.lane_tiles) * kLanes, c0 = (t / p.lane_tiles) * BN;
      float acc[Cfg::CW];
#pragma unroll
      for (int i = 0; i < Cfg::CW; ++i) acc[i] = 0.f;
      const int row = l0 + ln, lanes_n = SWAP ? p.N : p.M;
      // one scale of the weights per block; of x one per lane, or one per column through shared memory
      const float* ws = p.w_scale + (long long)((SWAP ? l0 : c0 + part * Cfg::CW) / 128) * p.KB;
      const bool ws_on = SWAP || c0 + part * Cfg::CW < p.N;
      const float* xs = p.x_scale + row;
      const bool xs_on = !SWAP && row < p.M;
      float xs_next = xs_on ? __ldg(xs) : 0.f, ws_next = ws_on ? __ldg(ws) : 0.f;
      for (int kb = 0; kb < p.KB; ++kb, ++it) {
        const uint32_t half = it & 1;
        if (SWAP) {
          for (int c = et; c < BN; c += 32 * Cfg::EPI)
            col_scale[half * BN + c] = c0 + c < p.M ? __ldg(p.x_scale + (long long)kb * p.M + c0 + c) : 0.f;
          asm volatile("bar.sync 1, %0;" ::"n"(32 * Cfg::EPI) : "memory");
        }
        const float scale = SWAP ? ws_next : xs_next * ws_next;
        if (kb + 1 < p.KB) {
          ws_next = ws_on ? __ldg(ws + kb + 1) : 0.f;
          if (!SWAP) xs_next = xs_on ? __ldg(xs + (long long)(kb + 1) * p.M) : 0.f;
        }
        bool ok = wait_bar(&done[half], (it >> 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok) != 0;
        if (!ok) {
          *abort_flag = 1;
          if (!SWAP) goto out;
          // the other epilogue warps meet this one at the named barrier: keep step with them, without results
        }
        tc_fence_after();
        uint32_t r[2][16];
        tmem_ld16(taddr + half * BN, r[0]);
#pragma unroll
        for (int c = 0; c < Cfg::CW; c += 16) {
          uint32_t(&cur)[16] = r[(c / 16) & 1];
          tmem_wait(cur);
          if (c + 16 < Cfg::CW) tmem_ld16(taddr + half * BN + c + 16, r[((c / 16) & 1) ^ 1]);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float f = SWAP ? scale * col_scale[half * BN + part * Cfg::CW + c + i] : scale;
            acc[c + i] = fmaf(__uint_as_float(cur[i]), f, acc[c + i]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&freed[half]);
      }
      T* out = static_cast<T*>(p.out);
      if (row < lanes_n) {
        if (SWAP) {
#pragma unroll
          for (int c = 0; c < Cfg::CW; ++c) {
            const int m = c0 + part * Cfg::CW + c;
            if (m < p.M) out[(long long)m * p.out_ld + row] = Elem<T>::put(acc[c]);
          }
        } else {
          constexpr int V = 16 / (int)sizeof(T);
          T* o = out + (long long)row * p.out_ld + c0 + part * Cfg::CW;
          const int left = p.N - (c0 + part * Cfg::CW);
#pragma unroll
          for (int c = 0; c < Cfg::CW; c += V) {
            Pack<T, V> v;
#pragma unroll
            for (int i = 0; i < V; ++i) v.put(i, acc[c + i]);
            if (p.vec_out && c + V <= left) v.store(o + c);
            else v.store_part(o + c, left - c);
          }
        }
      }
    }
  }
out:
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) {
    for (int s = 0; s < Cfg::STAGES; ++s) mbar_wait_plain(&full[s], 0, 1u << 12), mbar_wait_plain(&full[s], 1, 1u << 12);
    for (int k = 0; k < 2; ++k) mbar_wait_plain(&done[k], 0, 1u << 12), mbar_wait_plain(&done[k], 1, 1u << 12);
    atomicExch(p.status, 1);
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)Cfg::TCOLS) : "memory");
  }
}

// weights [rows][cols] -> e4m3 with one scale per 128 x 128 block, scale[rows / 128][cols / 128]; a CTA per block
template <typename T>
__global__ void __launch_bounds__(256) quantize_weight_kernel(const T* __restrict__ w, long long w_ld, uint8_t* __restrict__ q,
                                                             long long q_ld, float* __restrict__ scale, long long rows,
                                                             long long cols) {
  __shared__ float red[8];
  pdl_trigger();
  pdl_wait();
  const long long c0 = (long long)blockIdx.x * 128, r0 = (long long)blockIdx.y * 128;
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5;
  float amax = kAmaxFloor;
  for (int i = threadIdx.x; i < 128 * 128; i += 256) {
    const long long r = r0 + i / 128, c = c0 + i % 128;
    if (r < rows && c < cols) amax = fmaxf(amax, fabsf(Elem<T>::get(w[r * w_ld + c])));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (lane == 0) red[wp] = amax;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) amax = fmaxf(amax, red[k]);
  if (threadIdx.x == 0) scale[(long long)blockIdx.y * gridDim.x + blockIdx.x] = __fdiv_rn(amax, kE4m3Max);
  const float inv = __fdiv_rn(kE4m3Max, amax);
  for (int i = threadIdx.x; i < 128 * 128; i += 256) {
    const long long r = r0 + i / 128, c = c0 + i % 128;
    if (r < rows && c < cols) q[r * q_ld + c] = (uint8_t)pack_e4m3(Elem<T>::get(w[r * w_ld + c]) * inv, 0.f, 0.f, 0.f);
  }
}

template <typename T, int BN, bool SWAP>
cudaError_t launch_tile(const MatmulCall& c, MatmulArgs p, cudaStream_t st) {
  using Cfg = MatmulCfg<BN>;
  CUtensorMap lane_map, col_map;
  const uint8_t* lane_base = SWAP ? c.w : c.x;
  const uint8_t* col_base = SWAP ? c.x : c.w;
  const long long lanes = SWAP ? c.n : c.m, cols = SWAP ? c.m : c.n;
  if (!make_bytes_map(&lane_map, lane_base, lanes, c.k, SWAP ? c.w_ld : c.x_ld, kLanes) ||
      !make_bytes_map(&col_map, col_base, cols, c.k, SWAP ? c.x_ld : c.w_ld, BN))
    return cudaErrorNotSupported;
  p.lane_tiles = (int)((lanes + kLanes - 1) / kLanes);
  p.col_tiles = (int)((cols + BN - 1) / BN);
  auto kern = matmul_fp8_kernel<T, BN, SWAP>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kern), Cfg::SMEM, allowed);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)p.lane_tiles * p.col_tiles;
  const int most = num_sms();
  return launch_pdl(kern, dim3((unsigned)(tiles < most ? tiles : most)), dim3(Cfg::THREADS), Cfg::SMEM, st, lane_map, col_map, p);
}

template <typename T>
cudaError_t matmul_t(const MatmulCall& c, cudaStream_t st) {
  MatmulArgs p{};
  p.x_scale = c.x_scale, p.w_scale = c.w_scale, p.out = c.out, p.out_ld = c.out_ld;
  p.M = (int)c.m, p.N = (int)c.n, p.KB = (int)((c.k + 127) / 128);
  p.vec_out = c.out_ld * sizeof(T) % 16 == 0 && aligned_to(c.out, 16);
  p.status = c.status;
  if (c.m <= 32) return launch_tile<T, 32, true>(c, p, st);
  return launch_tile<T, 128, false>(c, p, st);
}

}  // namespace

bool matmul_fp8_available() { return tma_encode_available(); }

cudaError_t launch_matmul_fp8(const MatmulCall& c, cudaStream_t st) {
  switch (c.out_dtype) {
    case DTST_F32: return matmul_t<float>(c, st);
    case DTST_BF16: return matmul_t<__nv_bfloat16>(c, st);
    default: return matmul_t<__half>(c, st);
  }
}

cudaError_t launch_quantize_weight(int dtype, const void* w, long long w_ld, uint8_t* q, long long q_ld, float* scale,
                                   long long rows, long long cols, cudaStream_t st) {
  const dim3 grid((unsigned)((cols + 127) / 128), (unsigned)((rows + 127) / 128));
  switch (dtype) {
    case DTST_F32:
      return launch_pdl(quantize_weight_kernel<float>, grid, dim3(256), 0, st, static_cast<const float*>(w), w_ld, q, q_ld, scale, rows, cols);
    case DTST_BF16:
      return launch_pdl(quantize_weight_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, static_cast<const __nv_bfloat16*>(w), w_ld, q, q_ld, scale, rows, cols);
    default:
      return launch_pdl(quantize_weight_kernel<__half>, grid, dim3(256), 0, st, static_cast<const __half*>(w), w_ld, q, q_ld, scale, rows, cols);
  }
}

}  // namespace dtst
