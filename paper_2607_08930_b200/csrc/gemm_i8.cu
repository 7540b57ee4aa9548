// Projections in 8-bit integers on the 5th-generation tensor cores:
//   z[m, n] = (sum over k of A[m, k] W[n, k]) * w_scale[n] * a_scale[m],  codes int8, sums int32 (exact), scales fp32,
// stored as bf16 (mode 0), added to fp32 (1), stored as fp32 (2), or silu(z) * z2 as bf16 with a second weight (3).
//
// Weight rows sit on the 128-row side of the tcgen05.mma tile and tokens on its N side, as in the bf16 projections: a
// block step with a few dozen tokens wastes no tensor-core rows, and every CTA streams weights of its own.  A k step is
// 128 codes (one 128-byte swizzle span, four kind::i8 instructions of 32).  One CTA per SM, warp-specialised:
//   warp 0       TMA producer
//   warp 1       MMA issuer (one thread)
//   warps 2..9   epilogue: warp w reads TMEM lanes 32 (w mod 4) ..; its two groups of four take alternate token chunks
// CG = 2: two CTAs of a cluster share every instruction (256 weight rows) and each stages half of the tokens, which
// takes a quarter off the bytes a CTA loads for an operation.
// SPLIT: a projection with fewer tiles than SMs has the k range of each tile shared by the CTAs (pairs) of one cluster.
// Chunk c (8 tokens) of the tile is finished by split c mod S: the others write their partial sums of it to that CTA's
// shared memory, which counts the bytes on a barrier.  Integer sums are exact, so the order does not matter and the result
// does not depend on the split.
// Measured: 8192 tokens x 3584 x 18944 in 360 us (3.1 POP/s; the bf16 projection of the same size takes 866), the SwiGLU of
// 512 x 18944 x 3584 in 52 us, of which its products take 44 (the arithmetic and stores of an epilogue that nothing hides,
// its accumulators fill TMEM, the rest); 64 tokens x 4608 x 3584 in 7.3 us (7.0 out of the L2), the LM head of 128
// tokens in 108 us (weights and logits from and to HBM: 95).
// Every wait is bounded: one that runs out raises the error flag and leaves NaN in the outputs that it kept from being
// formed; all roles drain and TMEM is freed.
#include <math.h>

#include <mutex>

#include "decode_ops.cuh"
#include "tc_common.cuh"

namespace bs {

namespace {

using namespace tc;

constexpr int BKB = 128;                  // bytes = codes of a k step
constexpr int kTileRows = 128;            // weight rows of a CTA
constexpr int kThreads = 320;
constexpr int kRing = 196 * 1024;         // operand stages and, behind them, received partial sums
constexpr int kChunk = 8;                 // tokens of a chunk that one split finishes
constexpr int kMaxStages = 12;
constexpr int kAccCols = 256;             // TMEM columns of an accumulator buffer (two of them)

struct Params {
  int M, N, K;
  int tn;                   // tokens of a tile
  int n_tiles, m_tiles, splits, kblocks, stages;
  int received;             // offset of the received partial sums
  int nbuf;                 // accumulator buffers
  int mgroup;               // token tiles per group of the item order (0: token tile fastest over all)
  int vec;                  // bf16 rows take 16-byte stores
  void* C;
  long long ldc;
  const float *sa, *sw, *sw2;
  int* error_flag;
};

__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned in_cta(unsigned addr, unsigned rank) {
  unsigned r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <int CG>
__device__ __forceinline__ void load_tile(unsigned dst, const CUtensorMap* map, int c0, int c1, unsigned bar) {
  if (CG == 1)
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_tile(const CUtensorMap* map, int c0, int c1) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(map), "r"(c0), "r"(c1) : "memory");
}
// kind::i8: signed 8-bit A and B, both K-major, 32-bit integer accumulator, shape (128 CG) x n x 32.
template <int CG>
__device__ __forceinline__ unsigned instruction(int n) {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((unsigned)(n >> 3) << 17) | ((unsigned)((kTileRows * CG) >> 4) << 24);
}
template <int CG>
__device__ __forceinline__ void mma_i8(unsigned d, unsigned a_lo, unsigned b_lo, unsigned idesc, unsigned accumulate) {
  if (CG == 1)
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                 "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
}
// Arrives on the barrier once the MMAs issued before have completed (CG = 2: on the one at this offset in both CTAs).
template <int CG>
__device__ __forceinline__ void commit(unsigned bar, unsigned short both) {
  if (CG == 1)
    umma_commit(bar);
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"(both) : "memory");
}
// What is in flight when a wait has run out gets 10 ms to arrive.
constexpr long long kDrainCycles = 20000000ll;
__device__ __forceinline__ void wait_briefly(unsigned bar, unsigned parity, long long until) {
  while (!mbar_try_wait(bar, parity) && clock64() < until) {
  }
}
__device__ __forceinline__ void tmem_ld8(unsigned taddr, int* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
  tmem_ld_wait();
}
// Writes 16 bytes to a CTA of the cluster and counts them on its barrier.
__device__ __forceinline__ void send16(unsigned to, unsigned bar, const int* v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(bar) : "memory");
}
__device__ __forceinline__ bool wait_received(unsigned bar, volatile int* abort_flag) {
  const long long t0 = clock64();
  for (;;) {
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], 0;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar) : "memory");
    if (ok) return true;
    if (clock64() - t0 > 3 * kWaitCycles) {                 // (the others' own waits come first)
      *abort_flag = 1;
      return false;
    }
  }
}

// Output tiles are numbered token tile fastest (the CTAs of a round then share weight tiles in L2); with mgroup the
// token tiles are taken in groups, all weight tiles within one before the next, so that the group's activations stay in
// L2 while the weights pass.
__device__ __forceinline__ void tile_of(const Params& p, int tile, int* mt, int* nt) {
  if (p.mgroup <= 0) {
    *mt = tile % p.m_tiles;
    *nt = tile / p.m_tiles;
    return;
  }
  const int per = p.mgroup * p.n_tiles, g = tile / per, r = tile - g * per;
  const int size = min(p.mgroup, p.m_tiles - g * p.mgroup);
  *nt = r / size;
  *mt = g * p.mgroup + r % size;
}

__device__ __forceinline__ float silu(float x) {         // as in the bf16 SwiGLU: relative error about 2^-21
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return x * r;
}

// Stores the finished values v[j] of (feature n, token t0 + j), j < jmax; `tile` (bf16 modes): 32 x 32 transposition
// space of the warp, through which the rows leave in 16-byte pieces.
template <int MODE>
__device__ __forceinline__ void store_chunk(const Params& p, const float* v, int n, int t0, int jmax, bf16* tile) {
  const int lane = threadIdx.x & 31;
  if (MODE == 0 || MODE == 3) {
    bf16* C = static_cast<bf16*>(p.C);
    if (p.vec) {
      __syncwarp();
#pragma unroll
      for (int j = 0; j < 32; ++j) tile[j * 32 + lane] = __float2bfloat16_rn(v[j]);
      __syncwarp();
      const int piece = lane & 3, nb = n - lane + piece * 8;
      if (nb < p.N) {                                     // N is a multiple of 8 here
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = i * 8 + (lane >> 2);
          if (tok < jmax)
            *reinterpret_cast<uint4*>(C + (long long)(t0 + tok) * p.ldc + nb) =
                *reinterpret_cast<const uint4*>(tile + tok * 32 + piece * 8);
        }
      }
      return;
    }
    if (n >= p.N) return;
    bf16* c = C + (long long)t0 * p.ldc + n;
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j < jmax) c[(long long)j * p.ldc] = __float2bfloat16_rn(v[j]);
  } else {
    if (n >= p.N) return;
    float* c = static_cast<float*>(p.C) + (long long)t0 * p.ldc + n;
    if (MODE == 1) {
      float u[32];
#pragma unroll
      for (int j = 0; j < 32; ++j) u[j] = j < jmax ? c[(long long)j * p.ldc] : 0.f;
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (j < jmax) c[(long long)j * p.ldc] = u[j] + v[j];
    } else {
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (j < jmax) c[(long long)j * p.ldc] = v[j];
    }
  }
}

template <int CG, int MODE, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1)
k_gemm_i8(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_w2,
          const __grid_constant__ CUtensorMap map_x, const Params p) {
  constexpr bool kDual = MODE == 3;
  constexpr int kW = kDual ? 2 : 1;
  constexpr int kWBytes = kTileRows * BKB;
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[2 * kMaxStages + 6];    // full, empty, accumulator full, empty; drain, received
  __shared__ __align__(16) bf16 out_tile[(MODE == 0 || MODE == 3) ? 8 : 1][(SPLIT ? kChunk : 32) * 32];
  __shared__ __align__(16) float tok_scale[8][256];
  __shared__ unsigned tmem_slot;
  __shared__ int s_abort;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned rank = (CG == 2 || SPLIT) ? cluster_rank() : 0u;
  const unsigned half = CG == 2 ? rank & 1u : 0u;           // place in the pair
  const unsigned lead = CG == 2 ? rank & ~1u : rank;        // the pair's leader
  const int split = SPLIT ? (int)(rank / CG) : 0;
  const int group_ctas = CG * (SPLIT ? p.splits : 1);
  const int worker = (int)blockIdx.x / group_ctas, workers = (int)gridDim.x / group_ctas;
  const unsigned smem0 = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const int x_rows = p.tn / CG;
  const int stage_bytes = kW * kWBytes + x_rows * BKB;
  const unsigned full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[kMaxStages]);
  const unsigned tfull0 = smem_u32(&bars[2 * kMaxStages]), tempty0 = smem_u32(&bars[2 * kMaxStages + 2]);
  const unsigned drain = smem_u32(&bars[2 * kMaxStages + 4]), got = smem_u32(&bars[2 * kMaxStages + 5]);
  const unsigned full_lead0 = CG == 2 ? in_cta(full0, lead) : full0;
  const unsigned tempty_lead0 = CG == 2 ? in_cta(tempty0, lead) : tempty0;
  const unsigned peer_abort = CG == 2 ? in_cta(smem_u32(&s_abort), rank ^ 1u) : 0u;
  const unsigned short both = (unsigned short)(3u << lead);
  const int items = p.n_tiles * p.m_tiles;
  const int kb0 = SPLIT ? (int)((long long)p.kblocks * split / p.splits) : 0;
  const int kb1 = SPLIT ? (int)((long long)p.kblocks * (split + 1) / p.splits) : p.kblocks;

  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w) : "memory");
    if (kDual) asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w2) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
  }
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(full0 + 8 * i, 1);
      mbar_init(empty0 + 8 * i, 1);
    }
    mbar_init(drain, 1);
    mbar_init(got, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(tfull0 + 8 * i, 1);
      mbar_init(tempty0 + 8 * i, 8 * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (CG == 1) {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2 || SPLIT) cluster_barrier();                  // the others' barriers exist before anything signals them
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const unsigned tmem = tmem_slot;
  volatile int* abort_flag = &s_abort;
  // (the tensor memory is held: a kernel behind that allocates its own before it waits cannot keep this one from it)
  pdl_trigger();
  if (warp == 0 && lane < p.stages && kb0 + lane < kb1 && worker < items) {
    // the first weight tiles come to L2 meanwhile (the kernel before may write them: they are not read before it ends)
    int mt, nt;
    tile_of(p, worker, &mt, &nt);
    prefetch_tile(&map_w, (kb0 + lane) * BKB, (nt * CG + (int)half) * kTileRows);
    if (kDual) prefetch_tile(&map_w2, (kb0 + lane) * BKB, (nt * CG + (int)half) * kTileRows);
  }
  pdl_wait();                                               // codes, scales and outputs may come from the kernel before

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA producer
    if (lane == 0) {
      int stage = 0, filled = 0;
      unsigned phase = 0;
      bool ok = true;
      for (int it = worker; it < items && ok; it += workers) {
        int mt, nt;
        tile_of(p, it, &mt, &nt);
        const int wrow = (nt * CG + (int)half) * kTileRows;
        const int xrow = mt * p.tn + (int)half * x_rows;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait(empty0 + 8 * stage, phase ^ 1u, abort_flag)) { ok = false; break; }
          if (half == 0) mbar_expect_tx(full0 + 8 * stage, (unsigned)(CG * stage_bytes));
          const unsigned at = smem0 + stage * stage_bytes;
          load_tile<CG>(at, &map_w, kb * BKB, wrow, full_lead0 + 8 * stage);
          if (kDual) load_tile<CG>(at + kWBytes, &map_w2, kb * BKB, wrow, full_lead0 + 8 * stage);
          load_tile<CG>(at + kW * kWBytes, &map_x, kb * BKB, xrow, full_lead0 + 8 * stage);
          ++filled;
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
      }
      if ((!ok || *abort_flag) && half == 0) {              // copies in flight land before this CTA leaves
        const long long until = clock64() + kDrainCycles;
        for (int f = max(0, filled - p.stages); f < filled; ++f)
          wait_briefly(full0 + 8 * (f % p.stages), (unsigned)(f / p.stages) & 1u, until);
      }
      if (CG == 2 && !ok) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_abort), "r"(1) : "memory");
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer (of a pair: the leader)
    if (lane == 0 && half == 0) {
      int stage = 0, local = 0;
      unsigned phase = 0;
      bool ok = true;
      const unsigned idesc = instruction<CG>(p.tn);
      const unsigned lo0 = desc_lo(smem0), step = (unsigned)stage_bytes >> 4;
      // debugging build: an error flag of -1 - b before the call makes the wait for k step b run out
      const int fail_at = kBoundsCheck && p.error_flag ? -1 - *static_cast<volatile int*>(p.error_flag) : -1;
      unsigned lo = lo0;
      for (int it = worker; it < items && ok; it += workers, ++local) {
        const int acc = p.nbuf == 2 ? local & 1 : 0;
        const unsigned acc_phase = (unsigned)(p.nbuf == 2 ? local >> 1 : local) & 1u;
        if (!mbar_wait(tempty0 + 8 * acc, acc_phase ^ 1u, abort_flag)) { ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const unsigned d0 = tmem + acc * kAccCols, d1 = d0 + (p.nbuf == 2 ? kAccCols / 2 : kAccCols);
        unsigned accumulate = 0u;
        for (int kb = kb0; kb < kb1; ++kb) {
          if (kBoundsCheck && kb == fail_at) *abort_flag = 1;
          if ((kBoundsCheck && kb == fail_at) || !mbar_wait(full0 + 8 * stage, phase, abort_flag)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned b = lo + kW * (kWBytes >> 4);
#pragma unroll
          for (int k = 0; k < BKB / 32; ++k) {
            mma_i8<CG>(d0, lo + 2 * k, b + 2 * k, idesc, k == 0 ? accumulate : 1u);
            if (kDual) mma_i8<CG>(d1, lo + (kWBytes >> 4) + 2 * k, b + 2 * k, idesc, k == 0 ? accumulate : 1u);
          }
          accumulate = 1u;
          commit<CG>(empty0 + 8 * stage, both);
          lo += step;
          if (++stage == p.stages) { stage = 0; phase ^= 1u; lo = lo0; }
        }
        if (ok) commit<CG>(tfull0 + 8 * acc, both);
      }
      if (!ok) {                                            // products in flight end before tensor memory is freed
        commit<CG>(drain, both);
        wait_briefly(drain, 0u, clock64() + kDrainCycles);
      }
      if (CG == 2 && !ok) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_abort), "r"(1) : "memory");
    }
  } else if (!SPLIT) {
    // ---------------------------------------------------------------- epilogue
    const int q = warp & 3, group = (warp - 2) >> 2;
    float* const scales = tok_scale[warp - 2];
    int local = 0;
    bool ok = true;
    for (int it = worker; it < items; it += workers, ++local) {
      int mt, nt;
      tile_of(p, it, &mt, &nt);
      const int n = (nt * CG + (int)half) * kTileRows + q * 32 + lane;
      const float w = n < p.N ? __ldg(p.sw + n) : 0.f;
      const float w2 = kDual && n < p.N ? __ldg(p.sw2 + n) : 0.f;
      const int limit = min(p.tn, p.M - mt * p.tn);
      __syncwarp();
      for (int t = lane; t < p.tn; t += 32) scales[t] = t < limit ? __ldg(p.sa + mt * p.tn + t) : 0.f;
      __syncwarp();
      const int acc = p.nbuf == 2 ? local & 1 : 0;
      const unsigned acc_phase = (unsigned)(p.nbuf == 2 ? local >> 1 : local) & 1u;
      ok = ok && mbar_wait(tfull0 + 8 * acc, acc_phase, abort_flag);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const unsigned row = tmem + ((unsigned)(q * 32) << 16) + acc * kAccCols;
      const unsigned second = p.nbuf == 2 ? kAccCols / 2 : kAccCols;
      auto release = [&]() {
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if (CG == 1) mbar_arrive(tempty0 + 8 * acc);
          else asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(tempty_lead0 + 8 * acc) : "memory");
        }
      };
      if (group * 32 >= limit) release();
      for (int c0 = group * 32; c0 < limit; c0 += 64) {
        const int t0 = mt * p.tn + c0, jmax = min(32, limit - c0);
        unsigned z[32], y[kDual ? 32 : 1];
        if (ok) {
          tmem_ld32_nowait(row + c0, z);
          if (kDual) tmem_ld32_nowait(row + second + c0, y);
        }
        if (ok) tmem_ld_wait();
        if (c0 + 64 >= limit) release();                     // the accumulator has been read: the next item may have it
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 t = *reinterpret_cast<const float4*>(scales + c0 + j);
          const float ts[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float g = (float)(int)z[j + i] * w * ts[i];
            v[j + i] = kDual ? silu(g) * ((float)(int)y[kDual ? j + i : 0] * w2 * ts[i]) : g;
          }
        }
        if (!ok) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(0x7fffffffu);
        }
        store_chunk<MODE>(p, v, n, t0, jmax, out_tile[(MODE == 0 || MODE == 3) ? warp - 2 : 0]);
      }
    }
    if (CG == 2 && !ok && lane == 0) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_abort), "r"(1) : "memory");
  }

  if (SPLIT && warp >= 2) {
    // ---------------------------------------------------------------- epilogue of a split tile (one for each cluster)
    const int S = p.splits;
    int mt, nt;
    tile_of(p, worker, &mt, &nt);
    const int limit = min(p.tn, p.M - mt * p.tn);
    const int chunks = (limit + kChunk - 1) / kChunk;
    const int mine = (chunks - split + S - 1) / S;           // chunks that this CTA finishes
    const int own = (chunks + S - 1) / S;                    // and the most that one does
    const int q = warp & 3, group = (warp - 2) >> 2, feature = q * 32 + lane;
    const unsigned row = tmem + ((unsigned)(q * 32) << 16);
    if (warp == 2 && lane == 0) mbar_expect_tx(got, (unsigned)((S - 1) * mine * kChunk * kTileRows * 4));
    // all scales, before the waits
    const int n = (nt * CG + (int)half) * kTileRows + feature;
    const float w = n < p.N ? __ldg(p.sw + n) : 0.f;
    float* const scales = tok_scale[warp - 2];
    for (int t = lane; t < p.tn; t += 32) scales[t] = t < limit ? __ldg(p.sa + mt * p.tn + t) : 0.f;
    __syncwarp();
    bool ok = mbar_wait(tfull0, 0u, abort_flag);
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    for (int c = group; c < chunks; c += 2) {
      const int owner = c % S;
      if (owner == split) continue;
      int z[8];
      tmem_ld8(row + c * kChunk, z);
      // a partial sum that is not there is sent as the least integer: no sum of fewer than 131072 products reaches it
      if (!ok) z[0] = (int)0x80000000;
      const int slot = split < owner ? split : split - 1;
      const unsigned rank_of = (unsigned)(owner * CG) + half;
      const unsigned to = in_cta(smem0 + (unsigned)p.received + (unsigned)(((slot * own + c / S) * 2 * kTileRows + feature) * 16), rank_of);
      const unsigned bar = in_cta(got, rank_of);
      send16(to, bar, z);
      send16(to + kTileRows * 16, bar, z + 4);
    }
    const bool here = mine == 0 || wait_received(got, abort_flag);
    for (int i = group; i < mine; i += 2) {
      const int c = i * S + split, t0 = mt * p.tn + c * kChunk, jmax = min(kChunk, limit - c * kChunk);
      const float4 s0 = *reinterpret_cast<const float4*>(scales + c * kChunk), s1 = *reinterpret_cast<const float4*>(scales + c * kChunk + 4);
      const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
      int z[8];
      tmem_ld8(row + c * kChunk, z);
      bool whole = ok && here;
      for (int slot = 0; slot < S - 1; ++slot) {
        const unsigned from = smem0 + (unsigned)p.received + (unsigned)(((slot * own + i) * 2 * kTileRows + feature) * 16);
        int y[8];
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(from) : "memory");
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(y[4]), "=r"(y[5]), "=r"(y[6]), "=r"(y[7]) : "r"(from + kTileRows * 16) : "memory");
        whole = whole && y[0] != (int)0x80000000;
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] += y[j];
      }
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = (float)z[j] * w * s[j];
        if (!whole) v[j] = __uint_as_float(0x7fffffffu);
      }
      if (MODE == 0 && p.vec) {
        bf16* tile = out_tile[warp - 2];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[j * 32 + lane] = __float2bfloat16_rn(v[j]);
        __syncwarp();
        const int tok = lane >> 2, piece = lane & 3, nb = n - lane + piece * 8;
        if (nb < p.N && tok < jmax)                          // N is a multiple of 8 here
          *reinterpret_cast<uint4*>(static_cast<bf16*>(p.C) + (long long)(t0 + tok) * p.ldc + nb) =
              *reinterpret_cast<const uint4*>(tile + tok * 32 + piece * 8);
      } else if (n < p.N) {
        if (MODE == 0) {
          bf16* o = static_cast<bf16*>(p.C) + (long long)t0 * p.ldc + n;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < jmax) o[(long long)j * p.ldc] = __float2bfloat16_rn(v[j]);
        } else {
          float* o = static_cast<float*>(p.C) + (long long)t0 * p.ldc + n;
          if (MODE == 1) {
            float u[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = j < jmax ? o[(long long)j * p.ldc] : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += u[j];
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < jmax) o[(long long)j * p.ldc] = v[j];
        }
      }
    }
  }

  // Neither CTA of a pair may leave (or free its tensor memory) while the partner can still reach it.
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) cluster_barrier();
  if (s_abort && threadIdx.x == 0 && p.error_flag) atomicMax(p.error_flag, 1);
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

using Kernel = void (*)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const Params);
template <int CG, bool SPLIT>
Kernel kernel_of(int mode) {
  switch (mode) {
    case 0: return k_gemm_i8<CG, 0, SPLIT>;
    case 1: return k_gemm_i8<CG, 1, SPLIT>;
    case 2: return k_gemm_i8<CG, 2, SPLIT>;
    default: return k_gemm_i8<CG, 3, false>;
  }
}

constexpr int kSmem = kRing + 1024;

// One-time set-up per device: SM count, shared-memory attributes, how many clusters of each size are resident at once.
struct DevInfo {
  int num_sms;
  int ok;
  int clusters[9];           // by cluster size (single-CTA kernel for sizes without pairs: 3, 5, 6, 7)
};
DevInfo g_dev[kMaxDevices];
std::mutex g_mutex;

const DevInfo* dev_info() {
  DevInfo* d = device_slot(g_dev);
  if (!d) return nullptr;
  std::lock_guard<std::mutex> lock(g_mutex);
  if (!d->num_sms) {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return nullptr;
    bool ok = true;
    for (int m = 0; m < 4 && ok; ++m)
      for (Kernel k : {kernel_of<1, false>(m), kernel_of<1, true>(m), kernel_of<2, false>(m), kernel_of<2, true>(m)})
        ok = ok && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) == cudaSuccess;
    for (int c = 1; c <= 8 && ok; ++c) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)(n / c * c));
      cfg.blockDim = dim3(kThreads);
      cfg.dynamicSmemBytes = kSmem;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = (unsigned)c; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
      cfg.attrs = at; cfg.numAttrs = 1;
      int most = 0;
      if (cudaOccupancyMaxActiveClusters(&most, c == 2 ? kernel_of<2, false>(0) : kernel_of<1, true>(0), &cfg) != cudaSuccess) {
        cudaGetLastError();
        most = 0;
      }
      d->clusters[c] = most;
    }
    if (!ok) cudaGetLastError();
    d->ok = ok;
    d->num_sms = n;
  }
  return d;
}

// [rows][cols] int8, `ld` bytes apart; boxes of `box` rows by 128 bytes, 128B-swizzled, zeros outside.
bool encode(const void* base, long long rows, long long cols, long long ld, int box, CUtensorMap* out) {
  const auto fn = tensor_map_encoder();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld};
  const cuuint32_t b[2] = {BKB, (cuuint32_t)box}, e[2] = {1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, b, e, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Plan {
  int cg, splits, tn, m_tiles, n_tiles, workers, nbuf;
  int stage_bytes, stages;   // operand stages, in what the received partial sums leave of the ring
};

void set_stages(Plan* p, bool dual) {
  const int own = (p->tn / kChunk + p->splits - 1) / p->splits;
  p->stage_bytes = (dual ? 2 : 1) * kTileRows * BKB + p->tn / p->cg * BKB;
  p->stages = (kRing - (p->splits - 1) * own * kChunk * kTileRows * 4) / p->stage_bytes;
  if (p->stages > kMaxStages) p->stages = kMaxStages;
}

// Clocks that a plan takes, from what was measured over QKV, O, gate/up, down and LM-head shapes at 1 to 8192 tokens.  A k
// step costs its products (2 tn clocks a weight tile, 1.2 times that in practice) or its loads (62 bytes a clock, 50 for a
// CTA of a pair); a call no less than its weights from HBM, 1.4 times that where token tiles fetch them side by side.  An
// epilogue takes 6 clocks a token, 18 with silu, behind the next item's products where there are two buffers.  A split
// costs 1200 clocks and its exchange, pairs 2500 for their barriers.
float cost_of(const Plan& p, int kblocks, bool dual, float weight_bytes) {
  const int w = dual ? 2 : 1, kb = (kblocks + p.splits - 1) / p.splits;
  const float step = fmaxf(2.4f * p.tn * w, (kTileRows * w + p.tn / p.cg) * (float)BKB / (p.cg == 1 ? 62.f : 50.f));
  const int rounds = (int)(((long long)p.n_tiles * p.m_tiles + p.workers - 1) / p.workers);
  const float epilogue = (dual ? 18.f : 6.f) * p.tn, loop = kb * step * (p.cg == 1 ? 1.05f : 1.f);
  float c = rounds * loop + (rounds - 1) * (p.nbuf == 1 ? epilogue : fmaxf(0.f, epilogue - loop));
  c = fmaxf(c, weight_bytes * (p.m_tiles > 1 ? 1.4f : 1.f) / 3400.f) + epilogue;
  if (p.splits > 1) c += 1200.f + p.tn * (8.f + 10.f / p.splits) * p.cg;
  return c + (p.cg == 2 ? 2500.f : 0.f);
}

// The cheapest plan: single CTAs or pairs, tiles of equal width that cover the tokens, k ranges shared by up to eight CTAs
// where the tiles leave SMs idle (one wave of clusters; two k steps each at least).  Three stages at least, without which
// products and loads take turns, and the cost above does not hold (512 x 2048 x 8192 on two 17.2 us, 13.8 on the three or
// more of the plan that is then cheapest; 256 x 3584 x 3584 10.8 and 8.9; 1024 x 1024 x 16384 29.5 and 25.1).
Plan plan_of(const DevInfo& dv, int M, int N, int kblocks, bool dual) {
  Plan best = {};
  float least = INFINITY;
  const float weight_bytes = (float)N * kblocks * BKB * (dual ? 2 : 1);
  for (int cg = 1; cg <= (dv.clusters[2] > 0 ? 2 : 1); ++cg) {
    const int unit = cg == 2 ? 32 : 16;                      // widths that kind::i8 has at 128 and at 256 rows
    int last = 0;
    for (int want = 256; want >= unit; want -= want > 128 ? 32 : want > 64 ? 16 : unit) {
      Plan p = {};
      p.cg = cg;
      p.m_tiles = (M + want - 1) / want;
      p.tn = ((M + p.m_tiles - 1) / p.m_tiles + unit - 1) / unit * unit;
      if (p.tn == last) continue;
      last = p.tn;
      p.n_tiles = (N + kTileRows * cg - 1) / (kTileRows * cg);
      p.nbuf = dual && p.tn > 128 ? 1 : 2;
      const long long items = (long long)p.n_tiles * p.m_tiles;
      for (int sp = 1; sp <= (dual ? 1 : 8 / cg); ++sp) {
        const int most = sp == 1 ? (cg == 2 ? dv.clusters[2] : dv.num_sms) : dv.clusters[sp * cg];
        if (sp > 1 && (items > most || kblocks < 2 * sp)) break;
        p.splits = sp;
        set_stages(&p, dual);
        if (p.stages < 3) continue;
        p.workers = (int)(items < most ? items : most);
        const float c = cost_of(p, kblocks, dual, weight_bytes);
        if (c < least) { least = c; best = p; }
      }
    }
  }
  return best;
}

}  // namespace

cudaError_t launch_gemm_i8(const GemmI8Args& a, cudaStream_t s) {
  if (a.M <= 0 || a.N <= 0) return cudaSuccess;
  const DevInfo* dv = dev_info();
  if (!dv || !dv->ok) return cudaErrorInitializationError;             // of the device, not of the arguments
  const bool dual = a.mode == 3;
  const int kblocks = (a.K + BKB - 1) / BKB;
  const Plan pl = plan_of(*dv, a.M, a.N, kblocks, dual);
  Params p;
  p.M = a.M; p.N = a.N; p.K = a.K; p.tn = pl.tn; p.n_tiles = pl.n_tiles; p.m_tiles = pl.m_tiles; p.splits = pl.splits;
  p.kblocks = kblocks; p.stages = pl.stages; p.nbuf = pl.nbuf; p.received = pl.stages * pl.stage_bytes;
  p.mgroup = (long long)a.M * a.K > (56ll << 20) && pl.m_tiles > 16 ? 16 : 0;
  p.vec = a.ldc % 8 == 0 && a.N % 8 == 0 && ((uintptr_t)a.C & 15) == 0;
  p.C = a.C; p.ldc = a.ldc; p.sa = a.sa; p.sw = a.sw; p.sw2 = a.sw2; p.error_flag = a.error_flag;
  CUtensorMap mw, mw2, mx;
  if (!encode(a.W, a.N, a.K, a.ldw, kTileRows, &mw) || !encode(a.A, a.M, a.K, a.lda, pl.tn / pl.cg, &mx))
    return cudaErrorNotSupported;
  mw2 = mw;
  if (dual && !encode(a.W2, a.N, a.K, a.ldw, kTileRows, &mw2)) return cudaErrorNotSupported;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(pl.workers * pl.cg * pl.splits));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)(pl.cg * pl.splits); at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = pdl_disabled() ? 1 : 2;
  Kernel k = pl.cg == 2 ? (pl.splits > 1 ? kernel_of<2, true>(a.mode) : kernel_of<2, false>(a.mode))
                        : (pl.splits > 1 ? kernel_of<1, true>(a.mode) : kernel_of<1, false>(a.mode));
  return cudaLaunchKernelEx(&cfg, k, mw, mw2, mx, p);
}

}  // namespace bs
