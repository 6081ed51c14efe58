// Matrix product of 8-bit floating-point operands (e4m3) with a scale for each block of 128 along the contracted
// dimension:
//     out[m, n] = sum_kb  x_scale[kb, m] w_scale[n / 128, kb]  sum_{k in block kb} x[m, k] w[n, k]
// on the fifth-generation tensor cores.  A k-block of 128 values is 128 bytes: one row of a 128-byte-swizzled TMA
// tile and four tcgen05.mma (kind::f8f6f4, K = 32).  The scales differ from block to block, so the tensor core sums
// one block into tensor memory, and the epilogue warps add it, scaled, to fp32 sums in registers while the next block
// is multiplied into the other half of the tensor memory.
//
// Two kernels.  Many rows: a pair of CTAs (cta_group::2) computes tiles of 256 x 256, each SM holding half of both
// operands, which halves the bytes an SM has to fetch per product.  Otherwise: one CTA computes tiles of 128 lanes x BN
// columns, lanes being rows of x and columns rows of w, or the other way round (SWAP) where there are few rows of x, so that
// the tile's lanes are filled by the weights; where there are few tiles the CTAs of a cluster share the k-blocks of one and
// add their sums through distributed shared memory, in rank order.
// Measured: 16384 x 4096 x 2048 in 147 us after a pause and 152 to 167 in long runs under the power limit (1.65 to 1.87 PFLOP/s;
// without the epilogue, its loads and products take 115), 2048^3 in 13.3, 1000 x 1111 x 1360 in 10.2; few rows of x read the
// weights once: 4 x 4096 x 2048 in 5.5 us, 64 rows in 6.9, 65 (not swapped) in 8.4.  Bound: many rows by the handing over of a
// block's sums every 128 values of k (8192 rows: tensor pipe 42 % busy, L2 27 %), few rows by latency.
// Warp 0 issues the TMA loads, warp 1 the products, the others hold the sums (a thread one lane x up to 128 columns).
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
  int split;                // CTAs that share a tile's k-blocks
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

// sums of one k-block, scaled, onto the fp32 sums: CW columns of this thread's lane from `taddr` on.  (Two sums an instruction:
// 152 -> 139 us for 16384 x 4096 x 2048 at the time, after a pause.  32 columns a load made it spill, 199 us.)
template <int CW, typename F>
__device__ __forceinline__ void add_block(float (&acc)[CW], uint32_t taddr, F factor) {
  uint32_t r[2][16];
  tmem_ld16(taddr, r[0]);
#pragma unroll
  for (int c = 0; c < CW; c += 16) {
    uint32_t(&cur)[16] = r[(c / 16) & 1];
    tmem_wait(cur);
    if (c + 16 < CW) tmem_ld16(taddr + c + 16, r[((c / 16) & 1) ^ 1]);
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float2 sum = fma_pair(make_float2(__uint_as_float(cur[i]), __uint_as_float(cur[i + 1])),
                                  make_float2(factor(c + i), factor(c + i + 1)), make_float2(acc[c + i], acc[c + i + 1]));
      acc[c + i] = sum.x, acc[c + i + 1] = sum.y;
    }
  }
}

// One lane's CW columns to out (row-major, this lane's row at `o`, `left` columns exist).  Rows on 16-byte boundaries: vector
// stores.  Otherwise the warp turns 16 columns at a time round in its 32 x 17 floats of shared memory and writes rows
// piece by piece, neighbouring lanes to neighbouring columns.
template <typename T, int CW>
__device__ __forceinline__ void store_lane(const float (&acc)[CW], T* out, long long ld, int row0, int rows, int col0, int left,
                                           bool vec, float* turn) {
  const int lane = threadIdx.x & 31;
  constexpr int V = 16 / (int)sizeof(T);
  if (vec) {
    if (lane < rows) {
      T* o = out + (long long)(row0 + lane) * ld + col0;
#pragma unroll
      for (int c = 0; c < CW; c += V) {
        float x[V];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = acc[c + i];
        Pack<T, V> v;
        v.pack(x);
        if (c + V <= left) v.store(o + c);
        else v.store_part(o + c, left - c);
      }
    }
    return;
  }
#pragma unroll
  for (int c = 0; c < CW; c += 16) {
    if (c >= left) break;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) turn[lane * 17 + i] = acc[c + i];
    __syncwarp();
    const int col = c + (lane & 15);
#pragma unroll 4
    for (int r = lane >> 4; r < 32; r += 2)
      if (r < rows && col < left) out[(long long)(row0 + r) * ld + col0 + col] = Elem<T>::put(turn[r * 17 + (lane & 15)]);
  }
}

template <int BN>
struct MatmulCfg {
  static constexpr int EPI = 4;                            // epilogue warps
  static constexpr int THREADS = 64 + 32 * EPI;
  static constexpr int A_BYTES = kLanes * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES;
  static constexpr int STAGES = BN <= 32 ? 8 : 6;
  static constexpr int NBUF = 4, TCOLS = NBUF * BN;         // buffers of tensor memory in turn
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + 2 * BN * 4 + EPI * 32 * 17 * 4 + 256;
};

template <typename T, int BN, bool SWAP>
__global__ void __launch_bounds__(MatmulCfg<BN>::THREADS, 1)
matmul_fp8_kernel(const __grid_constant__ CUtensorMap lane_map, const __grid_constant__ CUtensorMap col_map, const MatmulArgs p) {
  using Cfg = MatmulCfg<BN>;
  pdl_trigger();
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  float* col_scale = reinterpret_cast<float*>(smem + (size_t)Cfg::STAGES * Cfg::STAGE);   // [2][BN], SWAP only
  float* turn = col_scale + 2 * BN;                                                       // [EPI][32][17]
  uint64_t* full = reinterpret_cast<uint64_t*>(turn + Cfg::EPI * 32 * 17);
  uint64_t* empty = full + Cfg::STAGES;
  uint64_t* done = empty + Cfg::STAGES;      // [NBUF] products of a block complete
  uint64_t* freed = done + Cfg::NBUF;        // [NBUF] buffer of tensor memory read
  uint32_t* tmem_s = reinterpret_cast<uint32_t*>(freed + Cfg::NBUF);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_s + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < Cfg::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int k = 0; k < Cfg::NBUF; ++k) {
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

  // a cluster shares the k-blocks of one tile; a CTA by itself walks over tiles
  const int split = p.split, rank = split > 1 ? cluster_rank() : 0;
  const int kb0 = (int)((long long)p.KB * rank / split), kb1 = (int)((long long)p.KB * (rank + 1) / split);
  const int tiles = p.lane_tiles * p.col_tiles, first = blockIdx.x / split, step = split > 1 ? tiles : gridDim.x;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int t = first; t < tiles; t += step) {
        const int l0 = (t % p.lane_tiles) * kLanes, c0 = (t / p.lane_tiles) * BN;
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
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
      for (int t = first; t < tiles; t += step)
        for (int kb = kb0; kb < kb1; ++kb, ++it) {
          const uint32_t s = it % Cfg::STAGES, buf = it % Cfg::NBUF;
          if (!wait_bar(&freed[buf], ((it / Cfg::NBUF) & 1) ^ 1, abort_flag)) goto out;
          if (!wait_bar(&full[s], (it / Cfg::STAGES) & 1, abort_flag)) goto out;
          tc_fence_after();
          const uint32_t a = smem_u32(smem + (size_t)s * Cfg::STAGE), b = a + Cfg::A_BYTES;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            umma_f8(tmem + buf * BN, desc_sw128(a + 32 * ks), desc_sw128(b + 32 * ks), idesc, ks > 0 ? 1u : 0u);
          umma_commit(&empty[s]);
          umma_commit(&done[buf]);
        }
    }
  } else {
    const int quarter = warp & 3;
    const int ln = quarter * 32 + lane;               // this thread's lane of the tile
    const int et = threadIdx.x - 64;                  // 0 .. 32 EPI - 1
    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16);
    uint32_t it = 0;
    for (int t = first; t < tiles; t += step) {
      const int l0 = (t % p.lane_tiles) * kLanes, c0 = (t / p.lane_tiles) * BN;
      float acc[BN];
#pragma unroll
      for (int i = 0; i < BN; ++i) acc[i] = 0.f;
      const int row = l0 + ln;
      // one scale of the weights per block; of x one per lane, or one per column through shared memory
      const float* ws = p.w_scale + (long long)((SWAP ? l0 : c0) / 128) * p.KB;
      const float* xs = p.x_scale + row;
      const bool xs_on = !SWAP && row < p.M;
      const int xc = c0 + et;                         // SWAP: the row of x whose scale this thread hands out
      const bool xc_on = SWAP && et < BN && xc < p.M;
      float xs_next = 0.f, ws_next = 0.f;
      if (kb0 < kb1) {
        ws_next = __ldg(ws + kb0);
        xs_next = xs_on ? __ldg(xs + (long long)kb0 * p.M) : xc_on ? __ldg(p.x_scale + (long long)kb0 * p.M + xc) : 0.f;
      }
      for (int kb = kb0; kb < kb1; ++kb, ++it) {
        const uint32_t half = it & 1, buf = it % Cfg::NBUF;
        if (SWAP) {
          if (et < BN) col_scale[half * BN + et] = xs_next;
          asm volatile("bar.sync 1, %0;" ::"n"(32 * Cfg::EPI) : "memory");
        }
        const float scale = SWAP ? ws_next : xs_next * ws_next;
        if (kb + 1 < kb1) {
          ws_next = __ldg(ws + kb + 1);
          xs_next = xs_on ? __ldg(xs + (long long)(kb + 1) * p.M) : xc_on ? __ldg(p.x_scale + (long long)(kb + 1) * p.M + xc) : 0.f;
        }
        bool ok = wait_bar(&done[buf], (it / Cfg::NBUF) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok) != 0;
        if (!ok) {
          *abort_flag = 1;
          if (!SWAP) goto out;
          // the other epilogue warps meet this one at the named barrier: keep step with them, without results
        }
        tc_fence_after();
        const float* cs = col_scale + half * BN;
        add_block<BN>(acc, taddr + buf * BN, [&](int c) { return SWAP ? scale * cs[c] : scale; });
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&freed[buf]);
      }
      T* out = static_cast<T*>(p.out);
      if (split > 1) {       // this CTA's part of the sums; every load has landed and every product is done
        float* part = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int c = 0; c < BN; ++c) part[SWAP ? c * kLanes + ln : ln * (BN + 4) + c] = acc[c];
      } else if (SWAP) {
        if (row < p.N) {
#pragma unroll
          for (int c = 0; c < BN; ++c)
            if (c0 + c < p.M) out[(long long)(c0 + c) * p.out_ld + row] = Elem<T>::put(acc[c]);
        }
      } else {
        store_lane<T, BN>(acc, out, p.out_ld, l0 + quarter * 32, p.M - (l0 + quarter * 32), c0, p.N - c0, p.vec_out != 0,
                          turn + (warp - 2) * 32 * 17);
      }
    }
  }
out:
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) {
    for (int s = 0; s < Cfg::STAGES; ++s) mbar_wait_plain(&full[s], 0, 1u << 12), mbar_wait_plain(&full[s], 1, 1u << 12);
    for (int k = 0; k < Cfg::NBUF; ++k) mbar_wait_plain(&done[k], 0, 1u << 12), mbar_wait_plain(&done[k], 1, 1u << 12);
    atomicExch(p.status, 1);
  }
  __syncthreads();
  if (split > 1) {       // the parts in rank order, each CTA a share of the tile
    cluster_sync();
    const int l0 = (first % p.lane_tiles) * kLanes, c0 = (first / p.lane_tiles) * BN;
    const float* part = reinterpret_cast<const float*>(smem);
    T* out = static_cast<T*>(p.out);
    // four neighbouring outputs of a row at a time (SWAP: along the lanes)
    constexpr int QUADS = kLanes * BN / 4, ROW4 = (SWAP ? kLanes : BN) / 4;
    for (int e = QUADS * rank / split + threadIdx.x; e < QUADS * (rank + 1) / split; e += Cfg::THREADS) {
      const int r = e / ROW4, q = e % ROW4 * 4;
      const int m = SWAP ? c0 + r : l0 + r, n = SWAP ? l0 + q : c0 + q;
      if (m >= p.M || n >= p.N) continue;
      const float* at = part + (SWAP ? r * kLanes + q : r * (BN + 4) + q);
      float4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < split) v[k] = cluster_read4(at, k);
      float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < split) x[0] += v[k].x, x[1] += v[k].y, x[2] += v[k].z, x[3] += v[k].w;
      Pack<T, 4> o;
      o.pack(x);
      T* to = out + (long long)m * p.out_ld + n;
      if (p.vec_out && n + 4 <= p.N) o.store(to);
      else o.store_part(to, p.N - n);
    }
    cluster_sync();        // nobody leaves while its part may be read
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)Cfg::TCOLS) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ pairs of CTAs
// Tiles of 256 x 256: CTA r of the pair holds rows 128 r .. of both operands' tiles and lanes 128 r .. of the products.  The
// even CTA issues the products for both; its barriers collect both CTAs' loads and both CTAs' reads of tensor memory, and
// its commits arrive at both CTAs' barriers.
struct PairCfg {
  static constexpr int EPI = 8, THREADS = 64 + 32 * EPI, CW = 128;         // two epilogue warps to a lane quarter
  static constexpr int HALF = 128 * 128, STAGE = 2 * HALF, STAGES = 5;     // bytes of a CTA's share of one operand's tile
  static constexpr int BOX = 32 * 128;                                     // an epilogue warp's piece of the output, two of them
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + (size_t)EPI * 2 * BOX + 256;
};

// An epilogue warp's 32 rows x CW columns by TMA: in pieces of 128 bytes a row, through the warp's two swizzled boxes of
// shared memory in turn; the copy out runs on while the next tile's blocks are summed.  What lies beyond the tensor is not
// written.
template <typename T, int CW>
__device__ __forceinline__ void store_box(const float (&acc)[CW], const CUtensorMap* map, unsigned char* boxes, int row0, int col0, int cols) {
  constexpr int E = 16 / (int)sizeof(T), PIECE = 128 / (int)sizeof(T);
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c = 0; c < CW; c += PIECE) {
    if (c >= cols) break;
    unsigned char* box = boxes + (c / PIECE & 1) * PairCfg::BOX;
    if (lane == 0) tma_store_wait_read<1>();       // the piece before the last one has left its box
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      float x[E];
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = acc[c + k * E + i];
      Pack<T, E> v;
      v.pack(x);
      *reinterpret_cast<uint4*>(box + swz128(lane, k)) = v.raw;
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      tma_store_2d(map, col0 + c, row0, box);
      tma_store_commit();
    }
  }
}

__device__ __forceinline__ uint32_t pair_addr(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
// (what it announces - tensor memory has been read - is ordered by tcgen05.fence; a release at cluster scope would wait for
// the warp's global stores at every block: measured 320 us against 195 for 16384 x 4096 x 2048, when it was tried)
__device__ __forceinline__ void pair_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// 2-D tile into this CTA's shared memory, its bytes counted by a barrier of either CTA of the pair
__device__ __forceinline__ void pair_load_2d(void* dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
          smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void pair_umma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc)
      : "memory");
}
// arrives at the barrier of this offset in both CTAs when the products issued so far are complete
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
               "h"((uint16_t)3)
               : "memory");
}

template <typename T>
__global__ void __launch_bounds__(PairCfg::THREADS, 1) __cluster_dims__(2, 1, 1)
matmul_fp8_pair_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map,
                       const __grid_constant__ CUtensorMap out_map, const MatmulArgs p) {
  using Cfg = PairCfg;
  pdl_trigger();
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  unsigned char* boxes = smem + (size_t)Cfg::STAGES * Cfg::STAGE;
  uint64_t* full = reinterpret_cast<uint64_t*>(boxes + Cfg::EPI * 2 * Cfg::BOX);    // the even CTA's: both CTAs' loads
  uint64_t* empty = full + Cfg::STAGES;
  uint64_t* done = empty + Cfg::STAGES;
  uint64_t* freed = done + 2;                                                   // the even CTA's: both CTAs' epilogue warps
  uint32_t* tmem_s = reinterpret_cast<uint32_t*>(freed + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_s + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = (uint32_t)cluster_rank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < Cfg::STAGES; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int k = 0; k < 2; ++k) {
      mbar_init(&done[k], 1);
      mbar_init(&freed[k], 2 * Cfg::EPI);
    }
    *abort_flag = 0;
    fence_barrier_init();
    prefetch_tensormap(&x_map);
    prefetch_tensormap(&w_map);
    if (p.vec_out) prefetch_tensormap(&out_map);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_s)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  tc_fence_before();
  cluster_sync();          // both CTAs' barriers and tensor memory are ready
  tc_fence_after();
  const uint32_t tmem = *tmem_s;
  const int tiles = p.lane_tiles * p.col_tiles, first = blockIdx.x / 2, step = gridDim.x / 2;

  if (warp == 0) {
    if (lane == 0) {
      uint32_t it = 0;
      for (int t = first; t < tiles; t += step) {
        const int l0 = (t % p.lane_tiles) * 256 + (int)rank * 128, c0 = (t / p.lane_tiles) * 256 + (int)rank * 128;
        for (int kb = 0; kb < p.KB; ++kb, ++it) {
          const uint32_t s = it % Cfg::STAGES;
          if (!wait_bar(&empty[s], ((it / Cfg::STAGES) & 1) ^ 1, abort_flag)) goto out;
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2u * Cfg::STAGE);
          const uint32_t bar = pair_addr(&full[s], 0);
          pair_load_2d(smem + (size_t)s * Cfg::STAGE, &x_map, kb * 128, l0, bar);
          pair_load_2d(smem + (size_t)s * Cfg::STAGE + Cfg::HALF, &w_map, kb * 128, c0, bar);
        }
      }
      // the even CTA's last commits have arrived here before this CTA may leave
      for (uint32_t k = it > Cfg::STAGES ? it - Cfg::STAGES : 0; k < it; ++k)
        if (!wait_bar(&empty[k % Cfg::STAGES], (k / Cfg::STAGES) & 1, abort_flag)) goto out;
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = idesc_e4m3(256, 256);
      uint32_t it = 0;
      for (int t = first; t < tiles; t += step)
        for (int kb = 0; kb < p.KB; ++kb, ++it) {
          const uint32_t s = it % Cfg::STAGES, half = it & 1;
          if (!wait_bar(&freed[half], ((it >> 1) & 1) ^ 1, abort_flag)) goto out;
          if (!wait_bar(&full[s], (it / Cfg::STAGES) & 1, abort_flag)) goto out;
          tc_fence_after();
          const uint32_t a = smem_u32(smem + (size_t)s * Cfg::STAGE), b = a + Cfg::HALF;
#pragma unroll
          for (int ks = 0; ks < 4; ++ks)
            pair_umma(tmem + half * 256, desc_sw128(a + 32 * ks), desc_sw128(b + 32 * ks), idesc, ks > 0 ? 1u : 0u);
          pair_commit(&empty[s]);
          pair_commit(&done[half]);
        }
    }
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(part * Cfg::CW);
    const uint32_t freed0 = pair_addr(&freed[0], 0), freed1 = pair_addr(&freed[1], 0);
    uint32_t it = 0;
    for (int t = first; t < tiles; t += step) {
      const int l0 = (t % p.lane_tiles) * 256 + (int)rank * 128 + quarter * 32, c0 = (t / p.lane_tiles) * 256 + part * Cfg::CW;
      float acc[Cfg::CW];
#pragma unroll
      for (int i = 0; i < Cfg::CW; ++i) acc[i] = 0.f;
      const int row = l0 + lane;
      const float* ws = p.w_scale + (long long)(c0 / 128) * p.KB;
      const float* xs = p.x_scale + row;
      const bool ws_on = c0 < p.N, xs_on = row < p.M;
      float xs_next = xs_on ? __ldg(xs) : 0.f, ws_next = ws_on ? __ldg(ws) : 0.f;
      for (int kb = 0; kb < p.KB; ++kb, ++it) {
        const uint32_t half = it & 1;
        const float scale = xs_next * ws_next;
        if (kb + 1 < p.KB) {
          ws_next = ws_on ? __ldg(ws + kb + 1) : 0.f;
          xs_next = xs_on ? __ldg(xs + (long long)(kb + 1) * p.M) : 0.f;
        }
        bool ok = wait_bar(&done[half], (it >> 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok) != 0;
        if (!ok) goto out;
        tc_fence_after();
        add_block<Cfg::CW>(acc, taddr + half * 256, [&](int) { return scale; });
        tc_fence_before();
        __syncwarp();
        if (lane == 0) pair_arrive(half ? freed1 : freed0);
      }
      unsigned char* box = boxes + (warp - 2) * 2 * Cfg::BOX;
      if (!p.vec_out) {
        store_lane<T, Cfg::CW>(acc, static_cast<T*>(p.out), p.out_ld, l0, p.M - l0, c0, p.N - c0, false, reinterpret_cast<float*>(box));
      } else if (l0 < p.M) {
        store_box<T, Cfg::CW>(acc, &out_map, box, l0, c0, p.N - c0);
      }
    }
  }
out:
  // also on the way out of a wait that gave up: the copies out read this CTA's shared memory
  if (warp >= 2 && lane == 0) tma_store_wait_all<0>();
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) {
    for (int s = 0; s < Cfg::STAGES; ++s) mbar_wait_plain(&full[s], 0, 1u << 12), mbar_wait_plain(&full[s], 1, 1u << 12);
    for (int k = 0; k < 2; ++k) mbar_wait_plain(&done[k], 0, 1u << 12), mbar_wait_plain(&done[k], 1, 1u << 12);
    atomicExch(p.status, 1);
  }
  cluster_sync();          // neither CTA leaves while the other's loads, commits or arrivals may still reach it
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// weights [rows][cols] -> e4m3 with one scale per 128 x 128 block, scale[rows / 128][cols / 128]; a CTA per block
// (bf16 [4096][2048] 15 us, fp32 [8192][8192] 113: the block is read twice, by elements; once a model)
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

// few tiles: as many CTAs to a tile as the GPU has room for, each with two k-blocks at least
int split_of(long long tiles, int KB) {
  int split = 1;
  while (split < 8 && tiles * split * 2 <= num_sms() && KB >= 4 * split) split *= 2;
  return split;
}

template <typename T, int BN, bool SWAP>
cudaError_t launch_tile(const MatmulCall& c, MatmulArgs p, cudaStream_t st) {
  using Cfg = MatmulCfg<BN>;
  CUtensorMap lane_map, col_map;
  const long long lanes = SWAP ? c.n : c.m, cols = SWAP ? c.m : c.n;
  if (!make_tile_map(&lane_map, SWAP ? c.w : c.x, 1, lanes, c.k, SWAP ? c.w_ld : c.x_ld, kLanes) ||
      !make_tile_map(&col_map, SWAP ? c.x : c.w, 1, cols, c.k, SWAP ? c.x_ld : c.w_ld, BN))
    return cudaErrorNotSupported;
  p.lane_tiles = (int)((lanes + kLanes - 1) / kLanes);
  p.col_tiles = (int)((cols + BN - 1) / BN);
  auto kern = matmul_fp8_kernel<T, BN, SWAP>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kern), Cfg::SMEM, allowed);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)p.lane_tiles * p.col_tiles;
  const int sms = num_sms();
  p.split = split_of(tiles, p.KB);
  const long long grid = p.split > 1 ? tiles * p.split : (tiles < sms ? tiles : sms);
  return launch_clusters(kern, (unsigned)grid, p.split, Cfg::THREADS, Cfg::SMEM, st, lane_map, col_map, p);
}

template <typename T>
cudaError_t launch_pairs(const MatmulCall& c, MatmulArgs p, cudaStream_t st) {
  using Cfg = PairCfg;
  CUtensorMap x_map, w_map, out_map;
  if (!make_tile_map(&x_map, c.x, 1, c.m, c.k, c.x_ld, 128) || !make_tile_map(&w_map, c.w, 1, c.n, c.k, c.w_ld, 128)) return cudaErrorNotSupported;
  // (an output that TMA cannot address is written by the warps; the map is then another one's copy, and not used)
  if (p.vec_out) p.vec_out = make_tile_map(&out_map, c.out, sizeof(T), c.m, c.n, c.out_ld * (long long)sizeof(T), 32) ? 1 : 0;
  if (!p.vec_out) out_map = x_map;
  p.lane_tiles = (int)((c.m + 255) / 256);
  p.col_tiles = (int)((c.n + 255) / 256);
  auto kern = matmul_fp8_pair_kernel<T>;
  static std::atomic<uint64_t> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kern), Cfg::SMEM, allowed);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)p.lane_tiles * p.col_tiles, pairs = num_sms() / 2;
  return launch_clusters(kern, (unsigned)(2 * (tiles < pairs ? tiles : pairs)), 0, Cfg::THREADS, Cfg::SMEM, st, x_map, w_map, out_map, p);
}

template <typename T>
cudaError_t matmul_t(const MatmulCall& c, cudaStream_t st) {
  MatmulArgs p{};
  p.x_scale = c.x_scale, p.w_scale = c.w_scale, p.out = c.out, p.out_ld = c.out_ld;
  p.M = (int)c.m, p.N = (int)c.n, p.KB = (int)((c.k + 127) / 128), p.split = 1;
  p.vec_out = c.out_ld * sizeof(T) % 16 == 0 && aligned_to(c.out, 16);
  p.status = c.status;
  if (c.m <= 16) return launch_tile<T, 16, true>(c, p, st);
  if (c.m <= 32) return launch_tile<T, 32, true>(c, p, st);
  if (c.m <= 64) return launch_tile<T, 64, true>(c, p, st);
  // The tile with the least of an estimate in ns: waves of tiles, each a time per k-block and one to write the tile out (both
  // measured at 2048^3, 4096 x 4096 x 512 and 9029 x 220 x 3051: tiles of 64 columns took 32.0 / 31.4 / 29.2 us, of 128
  // 21.0 / 26.1 / 21.8, pairs 14.5 / 17.2 / 23.5).
  const long long sms = num_sms(), KB = p.KB;
  auto tiles = [&](long long a, long long b) { return ((c.m + a - 1) / a) * ((c.n + b - 1) / b); };
  auto cost = [&](long long n, long long block, long long out) {
    const long long split = split_of(n, p.KB);
    return (n * split + sms - 1) / sms * ((KB + split - 1) / split * block + out) + (split > 1 ? 2 * out : 0);
  };
  const long long t64 = cost(tiles(128, 64), 430, 400), t128 = cost(tiles(128, 128), 540, 1200);
  const long long pair = (tiles(256, 256) + sms / 2 - 1) / (sms / 2) * (KB * 650 + 800);
  if (pair <= t64 && pair <= t128) return launch_pairs<T>(c, p, st);
  if (t128 <= t64) return launch_tile<T, 128, false>(c, p, st);
  return launch_tile<T, 64, false>(c, p, st);
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
