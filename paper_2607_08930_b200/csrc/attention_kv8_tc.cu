// Ragged attention over the 8-bit KV cache on the 5th-generation tensor cores, for work items with more
// query rows than the streaming kernel takes: block steps with grouped heads, whole rows.  Formulas and the handling of
// the scales as in attention_kv8.cu.
//
// Work item = (row, span of its query tokens, kv head): up to NT tiles of 128 flattened (token, head-in-group) query
// rows, one row per thread of a softmax group and per tensor-memory lane.  One CTA per SM, warp-specialised:
//   warp 0        producer: 128-key tiles of K and V codes by TMA, each through a ring of its own
//   warp 1        issues the products.  S = Q K^T takes K's codes as they arrive (kind::f8f6f4, e4m3 x e4m3): a query
//                 element, after a power of two per query row has brought the row's largest into [128, 256), is the sum
//                 of two e4m3 values - the nearest one and the rest (4 + 4 significant bits, bf16 has 8: exact above
//                 2^-10 of the row's largest element, within 2^-17 of that element below) - so S is two products at
//                 twice the rate of one in fp16, and K is neither converted nor stored a second time
//   4 NT warps    softmax, four per query tile.  The weights w = 2^(t - M) go back to tensor memory as fp16, over the first
//                 half of their scores, as the A operand of O += W V
//   4 more warps  V's codes to fp16 (exact) in the layout of a B operand; rows behind the row's end become zeros
// A key tile's scores and weights go in halves of 64 keys: a softmax thread holds 64 scores in registers (read once, for
// the maximum and the weights), and while it works on one half the tensor cores take the other half's weights and then
// overwrite them with the next tile's scores.
// Weights are formed against a running reference that lags the maximum (kTcBias, kTcGrow): the output is rescaled only
// when a row's maximum has outgrown it.
//
// What bounds it: 6 rows of 1200 to 2304 tokens (28 / 4 heads, head_dim 128) 367 us, 782 TFLOP/s counted as a 16-bit
// attention, 47 % of the measured matrix rate.  Of a 128-key step of two query tiles, about 3900 clk, the tensor pipe
// works for 2600 (1024 per tile at the full rate; the halves of the scores, 128 x 64 x 32 from shared memory, take 49 clk
// instead of 32) and each scheduler's exponentials take 2048; the two softmax warps of a scheduler overlap them with their
// other work only in part.  Scores of 128 keys at once (two passes over them, no spare half) took 480 us where halves with
// the same way of issuing took 529, and 398 with products issued by an elected lane.  16 block steps of 32 tokens over 320
// to 800 keys, one query tile per CTA, 18.2 us, are bound by a CTA's beginning - indices, barriers, queries to two terms:
// 4 us - and by its chain of three to seven tiles.
// Every wait is bounded; when one runs out the flag is raised, all roles drain, the copies and products in flight are
// waited for, and the CTA's outputs are NaN.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <mutex>
#include <type_traits>

#include "kv8_line.cuh"
#include "tc_common.cuh"

namespace bs {

namespace {

using namespace tc;

constexpr int KT = 128;                              // keys per tile: four cache blocks
constexpr int kKStages = 3, kV8Stages = 2, kV16Stages = 2;
constexpr float kTcBias = 2.f, kTcGrow = 15.f;       // weights reach 2^15 at most, 2^2 when the reference is set
constexpr unsigned kOCol = 256;                      // tensor memory: outputs behind the scores, 128 columns per query tile

template <int DH, int NT>
struct TcLayout {
  static constexpr int threads = 128 + 128 * NT + 128;
  static constexpr int k8 = KT * DH;                 // one tile of codes
  static constexpr int v16 = KT * DH * 2;            // one tile of V in fp16: DH / 64 parts of 64 dims
  static constexpr int q_part = 128 * DH;            // one query tile's nearest values; the rests follow
  static constexpr int q = 0, k = q + NT * 2 * q_part, v8 = k + kKStages * k8, v = v8 + kV8Stages * k8;
  static constexpr int bytes = v + kV16Stages * v16;
  static constexpr int smem = bytes + 1024;
};

__device__ __forceinline__ void tma_load_4d(unsigned dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, unsigned bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
// High word of a descriptor of a K-major operand whose rows are row_bytes long (128 or 64, swizzled by as much).
template <int ROW>
__host__ __device__ constexpr unsigned desc_hi() { return (unsigned)(8 * ROW >> 4) | (1u << 14) | ((ROW == 128 ? 2u : 4u) << 29); }
// One lane of a converged warp, in the form that tells the compiler so: the products it issues then cost 15 to 20 cycles
// each (39 with both operands' descriptors), where a branch on the lane number costs 52, and 63 beside busy warps.
__device__ __forceinline__ bool elect_one() {
  unsigned r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// S: e4m3 x e4m3 (both K-major), fp32 accumulator, 128 x 64 x 32.
constexpr unsigned kIdescS = (1u << 4) | ((unsigned)(KT / 2 >> 3) << 17) | ((128u >> 4) << 24);
template <int DH>
__device__ __forceinline__ void umma_qk(unsigned d_tmem, unsigned a_lo, unsigned b_lo, unsigned accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 da, {%1, %5};\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], da, db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(kIdescS), "r"(accumulate), "r"(desc_hi<DH>()) : "memory");
}
// O: fp16 (A, tensor memory) x fp16 (B, MN-major), fp32 accumulator, 128 x DH x 16
template <int DH>
__device__ __forceinline__ void umma_pv(unsigned d_tmem, unsigned a_tmem, unsigned b_lo, unsigned accumulate) {
  constexpr unsigned idesc = (1u << 4) | (1u << 16) | ((unsigned)(DH >> 3) << 17) | ((128u >> 4) << 24);
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi) : "memory");
}
// two fp32 at a time
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(f32x2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void tmem_st32(unsigned taddr, const unsigned* w) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "r"(w[8]),
        "r"(w[9]), "r"(w[10]), "r"(w[11]), "r"(w[12]), "r"(w[13]), "r"(w[14]), "r"(w[15]), "r"(w[16]), "r"(w[17]),
        "r"(w[18]), "r"(w[19]), "r"(w[20]), "r"(w[21]), "r"(w[22]), "r"(w[23]), "r"(w[24]), "r"(w[25]), "r"(w[26]),
        "r"(w[27]), "r"(w[28]), "r"(w[29]), "r"(w[30]), "r"(w[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// two fp16 values -> two e4m3 codes, to nearest even
__device__ __forceinline__ unsigned encode_half2(__half2 x) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(*reinterpret_cast<const unsigned*>(&x)));
  return r;
}
__device__ __forceinline__ uint4 lds128(unsigned at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ void sts128(unsigned at, unsigned a, unsigned b, unsigned c, unsigned d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void sts64(unsigned at, unsigned a, unsigned b) {
  asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at), "r"(a), "r"(b) : "memory");
}
// generic-proxy writes to shared memory before tensor-core reads of it
__device__ __forceinline__ void fence_smem_for_mma() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

struct TcParams {
  const bf16* q;
  int q_ld;
  const float* k_scale;
  const float* v_scale;
  long long n_blocks;
  bf16* out;
  const int* cu_q;
  const int* kv_base;
  const int* vis;
  int n_rows, M, hq, hkv, G;   // G = hq / hkv
  int tq;            // query tokens per query tile
  int per_row;       // spans of a row that have a CTA of their own
  int chunks;        // key chunks per row; > 1: partials instead of the output
  float* part_o;     // [chunks][M][hq][DH]
  float2* part_ml;   // [chunks][M][hq] (reference, sum); sum 0: a chunk without keys
  int* error_flag;
};

// Whether row r's indices fit (a row whose do not is skipped).
__device__ __forceinline__ bool row_fits(const TcParams& p, int cq0, int cq1, int vis, int base) {
  return cq0 >= 0 && cq1 >= cq0 && cq1 <= p.M && vis >= 0 && base >= 0 && base % kKv8Block == 0 &&
         (long long)base + vis <= p.n_blocks * kKv8Block;
}

template <int DH, int NT>
__global__ void __launch_bounds__(TcLayout<DH, NT>::threads, 1)
k_attention_kv8_tc(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const TcParams p) {
  using L = TcLayout<DH, NT>;
  enum { B_KFULL = 0, B_KEMPTY = B_KFULL + kKStages, B_V8FULL = B_KEMPTY + kKStages, B_V8EMPTY = B_V8FULL + kV8Stages,
         B_VFULL = B_V8EMPTY + kV8Stages, B_VEMPTY = B_VFULL + kV16Stages, B_QFULL = B_VEMPTY + kV16Stages,
         B_SFULL = B_QFULL + 1, B_PFULL = B_SFULL + 2 * NT, B_OFULL = B_PFULL + 2 * NT, B_LAST = B_OFULL + 2 * NT, B_COUNT };
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[B_COUNT];
  __shared__ unsigned tmem_base_slot;
  __shared__ int s_abort;
  __shared__ float s_sc[NT * 128];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned smem0 = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const unsigned sQ = smem0 + L::q, sK = smem0 + L::k, sV8 = smem0 + L::v8, sV16 = smem0 + L::v;
  const unsigned bar0 = smem_u32(&bars[0]);
  auto bar = [&](int i) { return bar0 + 8u * (unsigned)i; };
  pdl_wait();

  // ---- the work item ----
  const int G = p.G, per_cta = NT * p.tq;
  // A CTA is (span, key chunk, kv head), heads next to each other.  Spans [0, n_rows per_row): the first per_row of every
  // row.  Behind them: the rest, if a row has any, by slots that need no prefix (row i's begin at cu[i] / per_cta + i).
  const int unit = (int)(blockIdx.x / (unsigned)p.hkv), kh = (int)blockIdx.x - unit * p.hkv;
  const int at = p.chunks == 1 ? unit : unit / p.chunks, chunk = unit - at * p.chunks;
  const int slot = at - p.n_rows * p.per_row;
  const int row = slot < 0 ? at / p.per_row
                           : warp_search(p.n_rows, slot, [&](int i) { return __ldcg(p.cu_q + i) / per_cta + i; });
  const int cq0 = __ldcg(p.cu_q + row), cq1 = __ldcg(p.cu_q + row + 1), vis = __ldcg(p.vis + row), base = __ldcg(p.kv_base + row);
  if (!row_fits(p, cq0, cq1, vis, base)) {
    if (threadIdx.x == 0 && p.error_flag) atomicMax(p.error_flag, 100 + SITE_ATTN_KV8);
    return;
  }
  const int span = slot < 0 ? at - row * p.per_row : slot - (cq0 / per_cta + row);
  const int t0 = cq0 + span * per_cta;
  const int nt = min(per_cta, cq1 - t0);                    // query tokens of this CTA
  if (nt <= 0 || span < (slot < 0 ? 0 : p.per_row)) return; // no tokens, or somebody else's
  const int n_qt = NT == 1 || nt <= p.tq ? 1 : 2;
  const int tiles_all = (vis + KT - 1) / KT;
  const int per_chunk = (tiles_all + p.chunks - 1) / p.chunks;
  const int kt0 = chunk * per_chunk;
  const int n_tiles = max(0, min(tiles_all, kt0 + per_chunk) - kt0);

  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < kKStages; ++i) { mbar_init(bar(B_KFULL + i), 1); mbar_init(bar(B_KEMPTY + i), 1); }
    for (int i = 0; i < kV8Stages; ++i) { mbar_init(bar(B_V8FULL + i), 1); mbar_init(bar(B_V8EMPTY + i), 4); }
    for (int i = 0; i < kV16Stages; ++i) { mbar_init(bar(B_VFULL + i), 4); mbar_init(bar(B_VEMPTY + i), 1); }
    mbar_init(bar(B_QFULL), 4 * NT);
    for (int i = 0; i < 2 * NT; ++i) {                       // [query tile][half of the key tile]
      mbar_init(bar(B_SFULL + i), 1);
      mbar_init(bar(B_PFULL + i), 4);
      mbar_init(bar(B_OFULL + i), 1);
    }
    mbar_init(bar(B_LAST), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&tmem_base_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  pdl_trigger();      // not before the tensor memory is here: the kernel behind may take its own before it waits for this grid
  constexpr unsigned tmem_base = 0;                         // the only place an allocation of all 512 columns can have
  volatile int* abort_flag = &s_abort;
  if (threadIdx.x == 0 && tmem_base_slot != 0) s_abort = 1;
  auto wait = [&](unsigned b, unsigned parity) { return !(kBoundsCheck && *abort_flag) && mbar_wait(b, parity, abort_flag); };
  const int blk0 = base / kKv8Block + kt0 * (KT / kKv8Block);      // cache block of the chunk's first key

  // Two query tiles: 4 x 128 registers a thread at launch become 56 + 2 x 192 + 72.
  const int group = warp >> 2;
  if (group == 0) {
    if (NT == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0 && n_tiles > 0) {
      int issued = 0;
      const int give_up = kBoundsCheck && p.error_flag ? -1 - *(volatile int*)p.error_flag : -1;      // (for tests)
      for (int t = 0; t < n_tiles; ++t) {
        if (kBoundsCheck && t == give_up) *abort_flag = 1;
        const int ks = t % kKStages, vs = t % kV8Stages;
        if (!wait(bar(B_KEMPTY + ks), (unsigned)((t / kKStages) & 1) ^ 1u)) break;
        if (!wait(bar(B_V8EMPTY + vs), (unsigned)((t / kV8Stages) & 1) ^ 1u)) break;
        mbar_expect_tx(bar(B_KFULL + ks), (unsigned)L::k8);
        tma_load_4d(sK + ks * L::k8, &map_k, 0, 0, kh, blk0 + 4 * t, bar(B_KFULL + ks));
        mbar_expect_tx(bar(B_V8FULL + vs), (unsigned)L::k8);
        tma_load_4d(sV8 + vs * L::k8, &map_v, 0, 0, kh, blk0 + 4 * t, bar(B_V8FULL + vs));
        issued = t + 1;
      }
      if (*abort_flag) {            // copies in flight end before the CTA does
        for (int t = max(0, issued - kKStages); t < issued; ++t) {
          const long long begin = clock64();
          while (!(mbar_try_wait(bar(B_KFULL + t % kKStages), (unsigned)(t / kKStages) & 1u) &&
                   (t < issued - kV8Stages || mbar_try_wait(bar(B_V8FULL + t % kV8Stages), (unsigned)(t / kV8Stages) & 1u))) &&
                 clock64() - begin < kWaitCycles / 64) {
          }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (n_tiles > 0 && elect_one()) {
      bool ok = true;
      // Scores of half h of key tile t for query tile x.  The place is free: the weights in it were read by the last
      // product issued before, and the tensor pipe runs one thread's instructions in order.
      auto scores = [&](int t, int x, int h) {
        if (x == 0 && h == 0 && !wait(bar(B_KFULL + t % kKStages), (unsigned)(t / kKStages) & 1u)) return false;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const unsigned q_hi = desc_lo(sQ + x * 2 * L::q_part), q_lo = desc_lo(sQ + x * 2 * L::q_part + L::q_part);
        const unsigned k_lo = desc_lo(sK + (t % kKStages) * L::k8 + h * (L::k8 / 2)), d = tmem_base + x * 128 + h * 64;
#pragma unroll
        for (int k = 0; k < DH / 32; ++k) {
          umma_qk<DH>(d, q_hi + 2 * k, k_lo + 2 * k, k ? 1u : 0u);
          umma_qk<DH>(d, q_lo + 2 * k, k_lo + 2 * k, 1u);
        }
        umma_commit(bar(B_SFULL + 2 * x + h));
        if (h == 1 && x == n_qt - 1) umma_commit(bar(B_KEMPTY + t % kKStages));
        return true;
      };
      ok = wait(bar(B_QFULL), 0);
      for (int i = 0; i < 2 * n_qt && ok; ++i) ok = scores(0, NT == 1 ? 0 : i % n_qt, NT == 1 ? i : i / n_qt);
      for (int t = 0; t < n_tiles && ok; ++t) {
        ok = wait(bar(B_VFULL + t % kV16Stages), (unsigned)(t / kV16Stages) & 1u);
        const unsigned v_lo = desc_lo(sV16 + (t % kV16Stages) * L::v16, KT * 128);
#pragma unroll 1
        for (int i = 0; i < 2 * n_qt && ok; ++i) {           // first halves of all query tiles, then the second ones
          const int x = NT == 1 || n_qt == 1 ? 0 : i & 1, h = NT == 1 || n_qt == 1 ? i : i >> 1;
          ok = wait(bar(B_PFULL + 2 * x + h), (unsigned)t & 1u);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned d = tmem_base + kOCol + x * 128, a = tmem_base + x * 128 + h * 64, v = v_lo + h * (KT / 32) * (2048 >> 4);
#pragma unroll
          for (int j = 0; j < KT / 32; ++j) umma_pv<DH>(d, a + j * 8, v + j * (2048 >> 4), (t || h || j) ? 1u : 0u);
          umma_commit(bar(B_OFULL + 2 * x + h));
          if (h == 1 && x == n_qt - 1) umma_commit(bar(B_VEMPTY + t % kV16Stages));
          if (t + 1 < n_tiles) ok = scores(t + 1, x, h);
        }
      }
      if (!ok) {                    // products in flight end before their operands and the tensor memory are given up
        umma_commit(bar(B_LAST));
        const long long begin = clock64();
        while (!mbar_try_wait(bar(B_LAST), 0) && clock64() - begin < kWaitCycles / 64) {
        }
      }
    }
  }
  } else if (group == 1 + NT) {
    // ------------------------------------------------------------------ V: codes -> fp16 B operand
    if (NT == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    constexpr int LPK = DH / 16;                             // lanes per key, 16 dims each
    const int c = (int)threadIdx.x & 127;
    const int j = c % LPK;
    for (int t = 0; t < n_tiles; ++t) {
      const int a = t % kV8Stages, b = t % kV16Stages;
      if (!wait(bar(B_V8FULL + a), (unsigned)(t / kV8Stages) & 1u)) break;
      if (!wait(bar(B_VEMPTY + b), (unsigned)((t / kV16Stages) & 1) ^ 1u)) break;
      const int left = vis - (kt0 + t) * KT;
      const unsigned src = sV8 + a * L::k8 + c * 16, dst = sV16 + b * L::v16 + (j >> 2) * (KT * 128);
#pragma unroll 1
      for (int i0 = 0; i0 < DH / 16; i0 += 4) {
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = lds128(src + (i0 + i) * 2048);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = (i0 + i) * (128 / LPK) + c / LPK;
          if (key >= left) w[i] = make_uint4(0, 0, 0, 0);
          unsigned y[8];
          kv8_decode4(w[i].x, y[0], y[1]);
          kv8_decode4(w[i].y, y[2], y[3]);
          kv8_decode4(w[i].z, y[4], y[5]);
          kv8_decode4(w[i].w, y[6], y[7]);
          // chunks 2 (j % 4) and + 1 of the key's 128-byte line; with two lines per key, half of a store's eight lanes
          // take them the other way round, so that the eight fall on different banks
          const bool flip = DH == 128 && j >= 4;
          if (flip) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const unsigned first = y[k];
              y[k] = y[k + 4];
              y[k + 4] = first;
            }
          }
          const unsigned line = dst + key * 128, c0 = 2 * (j & 3) + (flip ? 1 : 0), sw = key & 7;
          sts128(line + ((c0 ^ sw) << 4), y[0], y[1], y[2], y[3]);
          sts128(line + (((c0 ^ 1) ^ sw) << 4), y[4], y[5], y[6], y[7]);
        }
      }
      fence_smem_for_mma();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(B_V8EMPTY + a));
        mbar_arrive(bar(B_VFULL + b));
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax: one query row per thread
    if (NT == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
    const int x = group - 1, quad = warp & 3, r = quad * 32 + lane;
    const int nrows = x < n_qt ? min(p.tq, nt - x * p.tq) * G : 0;
    const bool warp_has_rows = quad * 32 < nrows;
    const int my_tiles = x < n_qt ? n_tiles : 0;
    const unsigned t_lane = tmem_base + ((unsigned)(quad * 32) << 16) + x * 128;
    const unsigned t_out = t_lane + kOCol;
    // ---- the warp's 32 queries, 8 dims per lane, to two e4m3 terms in place: a step's rows stand, as bf16, in the very
    // bytes that their nearest values (lower half of the lanes) and their rests (upper half) will take ----
    if (my_tiles > 0) {
      constexpr int LPR = DH / 8, RPI = 32 / LPR;            // lanes per row, rows per step
      const int pl = lane % LPR, f0 = quad * 32 + lane / LPR;
      const unsigned place = sQ + x * 2 * L::q_part + quad * 32 * DH;
      const unsigned mine = place + (lane >> 4) * L::q_part + (lane & 15) * 16;
      const unsigned by_G = (65536u + G - 1) / G;            // f / G = f by_G >> 16 for f < 128
#pragma unroll 4
      for (int i = 0; i < LPR; ++i) {
        const int f = f0 + i * RPI;
        const bool valid = f < nrows;
        const int tok = valid ? (int)(f * by_G >> 16) : 0, head = valid ? f - tok * G : 0;
        const bf16* src = p.q + (size_t)(t0 + x * p.tq + tok) * p.q_ld + (kh * G + head) * DH + pl * 8;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(mine + i * 256), "l"(src), "r"(valid ? 16 : 0) : "memory");
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      constexpr int FLY = 4;                                 // steps whose chains of shuffles and conversions overlap
#pragma unroll 1
      for (int i0 = 0; i0 < LPR; i0 += FLY) {
        uint4 raw[FLY];
        __nv_bfloat162 top2[FLY];
#pragma unroll
        for (int u = 0; u < FLY; ++u) raw[u] = lds128(mine + (i0 + u) * 256);
        __syncwarp();
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
          const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&raw[u]);
          top2[u] = __hmax2(__hmax2(__habs2(h[0]), __habs2(h[1])), __hmax2(__habs2(h[2]), __habs2(h[3])));
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1)
#pragma unroll
          for (int u = 0; u < FLY; ++u) top2[u] = __hmax2(top2[u], __shfl_xor_sync(0xffffffffu, top2[u], o));
#pragma unroll
        for (int u = 0; u < FLY; ++u) {
          const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&raw[u]);
          const float top = fmaxf(__low2float(top2[u]), __high2float(top2[u]));
          // (2^-60 at least, under which no score passes 2^-4: a factor times a K scale of 2^-40 stays a normal number, and
          // masked scores of -inf stay that)
          const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -60), 127);
          const float up = pow2i(7 - e);
          const int f = f0 + (i0 + u) * RPI;
          // (an infinite element would saturate: its row becomes NaN here, as its softmax is)
          const float sc = fminf(pow2i(e - 7) * (1.4426950408889634f * rsqrtf((float)DH)), kMaxFactor);
          if (pl == 0) s_sc[x * 128 + f] = top < INFINITY ? sc : __int_as_float(0x7fffffff);
          unsigned hi[2] = {0u, 0u}, lo[2] = {0u, 0u};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            // (fp16 holds the scaled element but for what lies 2^-32 under the row's largest)
            const float2 v = __bfloat1622float2(h[j]);
            const __half2 y = __floats2half2_rn(v.x * up, v.y * up);
            const unsigned near = encode_half2(y), back = kv8_decode2((unsigned short)near);
            hi[j >> 1] |= near << (16 * (j & 1));
            lo[j >> 1] |= encode_half2(__hsub2(y, *reinterpret_cast<const __half2*>(&back))) << (16 * (j & 1));
          }
          const int turn = DH == 128 ? f & 7 : (f >> 1) & 3;   // the swizzle of 128- and of 64-byte rows
          const unsigned at = sQ + x * 2 * L::q_part + f * DH + (((pl >> 1) ^ turn) << 4) + (pl & 1) * 8;
          sts64(at, hi[0], hi[1]);
          sts64(at + L::q_part, lo[0], lo[1]);
        }
      }
      fence_smem_for_mma();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(B_QFULL));
    const float sc = my_tiles > 0 ? s_sc[x * 128 + r] : 0.f;
    float ref = -FLT_MAX, sum = 0.f;                         // (under any score but -inf, whose weight it makes 0)
    bool ok = true;
    // whole warps go on or give up: the tensor-memory instructions want all lanes
    auto warp_wait = [&](int i, int phase) {
      if (__all_sync(0xffffffffu, !(kBoundsCheck && *abort_flag) && mbar_try_wait(bar(i), (unsigned)phase & 1u))) return true;
      return __all_sync(0xffffffffu, wait(bar(i), (unsigned)phase & 1u)) != 0;
    };
    // The tile's four pairs of scales: lane l looks after block l % 4, one tile ahead.
    float ksn = 1.f, vsn = 1.f;
    auto load_scales = [&](int t) {
      const size_t at = (size_t)min((long long)blk0 + 4 * t + (lane & 3), p.n_blocks - 1) * p.hkv + kh;   // (a tile may reach over the end)
      ksn = __ldcg(p.k_scale + at);
      vsn = __ldcg(p.v_scale + at);
    };
    if (my_tiles > 0) load_scales(0);
    // A key tile; false: a wait ran out.  A weight's exponent s f + (lv - ref) is rounded once, so what the reference, itself a
    // rounded sum, was rounded by stays in it: more than a weight's whole range once scores pass 2^23.  FAR (such scores are
    // possible: a score is at most 256 x 448 x 128 f, none of 2^23 where f is below 1/2 for all rows of the warp): s f + lv is
    // rounded first, for every use alike.  Rolled, as next to no call comes here (the other way: 6 whole rows 366 us, 364
    // without a choice, 369 with a vote on every row's own f).
    const float sc_top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(sc)));
    auto tile = [&](auto far, int t, float f, float lv, int left) {
      constexpr bool FAR = decltype(far)::value;
#pragma unroll (FAR ? 1 : 2)
      for (int h = 0; h < 2; ++h) {                          // 64 keys at a time: their scores fit the registers, read once
        // (These scores were issued after the weights that stood in their place were used, so no warp of the group - one
        // without query rows has nothing to hold it up - publishes here before all four have published there.)
        if (!warp_wait(B_SFULL + 2 * x + h, t)) return false;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (warp_has_rows) {
          unsigned y[64];
          tmem_ld32_nowait(t_lane + h * 64, y);
          tmem_ld32_nowait(t_lane + h * 64 + 32, y + 32);
          tmem_ld_wait();
          if (left < h * 64 + 64) {
#pragma unroll
            for (int j = 0; j < 64; ++j) y[j] = h * 64 + j < left ? y[j] : 0xff800000u;       // -inf
          }
          float fi[2], li[2], add[2], top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            fi[i] = __shfl_sync(0xffffffffu, f, 2 * h + i) * sc;
            li[i] = add[i] = __shfl_sync(0xffffffffu, lv, 2 * h + i);
            if (FAR) {
#pragma unroll
              for (int j = 0; j < 32; ++j) y[i * 32 + j] = __float_as_uint(fmaf(__uint_as_float(y[i * 32 + j]), fi[i], li[i]));
              fi[i] = 1.f;
              add[i] = 0.f;
            }
            float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int j = 0; j < 32; j += 2)
              m4[(j >> 1) & 3] = max3(m4[(j >> 1) & 3], __uint_as_float(y[i * 32 + j]), __uint_as_float(y[i * 32 + j + 1]));
            top = fmaxf(top, fmaf(max3(fmaxf(m4[0], m4[1]), m4[2], m4[3]), fi[i], add[i]));
          }
          const bool grow = top - ref > kTcGrow;             // (ref + kTcGrow may be rounded up to top)
          if (__any_sync(0xffffffffu, grow)) {
            float turn = 1.f;
            if (grow) {
              turn = exp2_fast(ref - (top - kTcBias));       // 0 on the first tile
              ref = top - kTcBias;
              sum *= turn;
            }
            if (t > 0 || h > 0) {
              // the output stands still once the product issued last is in it
              if (!warp_wait(B_OFULL + 2 * x + (h ^ 1), t - 1 + h)) return false;
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
              for (int c = 0; c < DH / 32; ++c) {
                unsigned o[32];
                tmem_ld32_nowait(t_out + c * 32, o);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * turn);
                tmem_st32(t_out + c * 32, o);
              }
            }
          }
          unsigned w[32];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const f32x2 f2 = pack2(fi[i], fi[i]), shift2 = pack2(add[i] - ref, add[i] - ref);
            unsigned* z = y + i * 32;
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float2 a = unpack2(fma2(pack2(__uint_as_float(z[j]), __uint_as_float(z[j + 1])), f2, shift2));
              z[j] = __float_as_uint(a.x);
              z[j + 1] = __float_as_uint(a.y);
            }
          }
#pragma unroll
          for (int j = 0; j < 64; ++j) asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+r"(y[j]));
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const unsigned* z = y + i * 32;
            f32x2 a4[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float e0 = __uint_as_float(z[j]), e1 = __uint_as_float(z[j + 1]);
              a4[(j >> 1) & 3] = add2(a4[(j >> 1) & 3], pack2(e0, e1));
              const __half2 hw = __floats2half2_rn(e0, e1);
              w[i * 16 + (j >> 1)] = *reinterpret_cast<const unsigned*>(&hw);
            }
            const float2 got = unpack2(add2(add2(a4[0], a4[1]), add2(a4[2], a4[3])));
            sum = fmaf(got.x + got.y, exp2_fast(-li[i]), sum);   // 2^-lv: the inverse of the V scale
          }
          tmem_st32(t_lane + h * 64, w);                     // over scores that were read before
          tmem_st_wait();
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PFULL + 2 * x + h));
      }
      return true;
    };
    for (int t = 0; t < my_tiles && ok; ++t) {
      const float f = kv8_clamp_scale(ksn), lv = log2_fast(kv8_clamp_scale(vsn));
      if (t + 1 < my_tiles) load_scales(t + 1);
      const int left = vis - (kt0 + t) * KT;
      ok = __any_sync(0xffffffffu, !(f * sc_top < 0.5f)) ? tile(std::true_type(), t, f, lv, left) : tile(std::false_type(), t, f, lv, left);
    }
    const bool have = ok && my_tiles > 0 && warp_wait(B_OFULL + 2 * x + 1, my_tiles - 1);
    if (warp_has_rows) {
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const bool valid = r < nrows;
      const int rr = valid ? r : 0;
      const size_t tok = (size_t)(t0 + x * p.tq + rr / G);
      const size_t at = (tok * p.hq + kh * G + rr % G) * DH;
      const size_t ml_at = ((size_t)chunk * p.M + tok) * p.hq + kh * G + rr % G;
      // no keys: zeros; a wait that ran out: NaN, here and in what is merged of it
      const float none = my_tiles > 0 ? __int_as_float(0x7fffffff) : 0.f;
      if (p.chunks > 1 && valid) p.part_ml[ml_at] = make_float2(have ? ref : -INFINITY, have ? sum : none);
      const float inv = have ? 1.0f / sum : 1.f;
      float* pdst = p.part_o + (size_t)chunk * p.M * p.hq * DH + at;
#pragma unroll 1
      for (int c = 0; c < DH / 32; ++c) {
        unsigned o[32];
        if (have) {
          tmem_ld32_nowait(t_out + c * 32, o);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(none);
        }
        if (!valid) continue;
        if (p.chunks > 1) {
          if (have) {
#pragma unroll
            for (int g = 0; g < 8; ++g)
              *reinterpret_cast<uint4*>(pdst + c * 32 + g * 4) = make_uint4(o[g * 4], o[g * 4 + 1], o[g * 4 + 2], o[g * 4 + 3]);
          }
        } else {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            uint4 v;
            __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
            for (int j = 0; j < 4; ++j)
              h[j] = __floats2bfloat162_rn(__uint_as_float(o[g * 8 + 2 * j]) * inv, __uint_as_float(o[g * 8 + 2 * j + 1]) * inv);
            *reinterpret_cast<uint4*>(p.out + at + c * 32 + g * 8) = v;
          }
        }
      }
    }
  }

  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (s_abort && threadIdx.x == 0 && p.error_flag) atomicMax(p.error_flag, 1);
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base_slot), "r"(512u) : "memory");
  }
}

// Merges the key chunks of every (token, head): out = sum_c 2^(m_c - m) o_c / sum_c 2^(m_c - m) l_c.  A warp per head.
constexpr int kMaxChunks = 16;
template <int DH>
__global__ void __launch_bounds__(256) k_attention_kv8_chunks(const TcParams p) {
  constexpr int V = DH / 32;                                 // dims per lane
  pdl_wait();
  pdl_trigger();
  const float* part_o = p.part_o;
  const float2* part_ml = p.part_ml;
  const int chunks = p.chunks, M = p.M, hq = p.hq;
  bf16* out = p.out;
  const long long unit = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (unit >= (long long)M * hq) return;
  const int lane = threadIdx.x & 31, tok = (int)(unit / hq);
  const int row = warp_search(p.n_rows, tok, [&](int i) { return __ldcg(p.cu_q + i); });
  const int cq0 = __ldcg(p.cu_q + row), cq1 = __ldcg(p.cu_q + row + 1);
  if (tok < cq0 || tok >= cq1 || !row_fits(p, cq0, cq1, __ldcg(p.vis + row), __ldcg(p.kv_base + row))) return;
  float2 ml[kMaxChunks];
  float v[kMaxChunks][V];
#pragma unroll
  for (int c = 0; c < kMaxChunks; ++c) {
    ml[c] = make_float2(-INFINITY, 0.f);
    if (c < chunks) ml[c] = __ldcg(part_ml + (long long)c * M * hq + unit);
    const float* src = part_o + ((long long)c * M * hq + unit) * DH + lane * V;
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      float2 y = make_float2(0.f, 0.f);
      if (c < chunks && ml[c].y != 0.f) y = __ldcg(reinterpret_cast<const float2*>(src + j));
      v[c][j] = y.x;
      v[c][j + 1] = y.y;
    }
  }
  float m = -INFINITY, l = 0.f, a[V];
#pragma unroll
  for (int c = 0; c < kMaxChunks; ++c) m = fmaxf(m, ml[c].x);
#pragma unroll
  for (int j = 0; j < V; ++j) a[j] = 0.f;
#pragma unroll
  for (int c = 0; c < kMaxChunks; ++c) {
    if (ml[c].y == 0.f) continue;
    const float w = ml[c].x > -INFINITY ? exp2_fast(ml[c].x - m) : 1.f;
    l += w * ml[c].y;
#pragma unroll
    for (int j = 0; j < V; ++j) a[j] += w * v[c][j];
  }
  const float inv = l != 0.f ? 1.0f / l : 0.f;
#pragma unroll
  for (int j = 0; j < V; j += 2)
    *reinterpret_cast<__nv_bfloat162*>(out + unit * DH + lane * V + j) = __floats2bfloat162_rn(a[j] * inv, a[j + 1] * inv);
}

// e4m3 codes [n_blocks][hkv][32][dh] as bytes; box: four blocks of one head
bool make_map(const unsigned char* ptr, int hkv, int dh, long long n_blocks, bool swizzle, CUtensorMap* out) {
  PFN_cuTensorMapEncodeTiled_v12000 encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)dh, (cuuint64_t)kKv8Block, (cuuint64_t)hkv, (cuuint64_t)n_blocks};
  const cuuint64_t strides[3] = {(cuuint64_t)dh, (cuuint64_t)kKv8Block * dh, (cuuint64_t)hkv * kKv8Block * dh};
  const cuuint32_t box[4] = {(cuuint32_t)dh, (cuuint32_t)kKv8Block, 1, KT / kKv8Block};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return encode(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<unsigned char*>(ptr), dims, strides, box, estr,
                CU_TENSOR_MAP_INTERLEAVE_NONE,
                !swizzle ? CU_TENSOR_MAP_SWIZZLE_NONE : dh == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int g_sms[kMaxDevices];      // per device; non-zero once the kernels' attributes are set there
std::mutex g_mutex;

template <int DH>
cudaError_t set_up(int* sms) {
  int dev = 0;
  cudaError_t r = cudaGetDevice(&dev);
  if (r == cudaSuccess) r = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
  if (r == cudaSuccess)
    r = cudaFuncSetAttribute(k_attention_kv8_tc<DH, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcLayout<DH, 1>::smem);
  if (r == cudaSuccess)
    r = cudaFuncSetAttribute(k_attention_kv8_tc<DH, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcLayout<DH, 2>::smem);
  return r;
}

template <int DH>
cudaError_t run_tc(const AttnKv8Args& a, float* part, size_t part_floats, int sms, cudaStream_t s) {
  CUtensorMap mk, mv;
  if (!make_map(a.cache.k, a.hkv, DH, a.cache.n_blocks, true, &mk) || !make_map(a.cache.v, a.hkv, DH, a.cache.n_blocks, false, &mv))
    return cudaErrorInvalidValue;
  const int G = a.hq / a.hkv;
  TcParams p;
  p.q = a.q; p.q_ld = a.q_ld; p.k_scale = a.cache.k_scale; p.v_scale = a.cache.v_scale; p.n_blocks = a.cache.n_blocks;
  p.out = a.out; p.cu_q = a.cu_q; p.kv_base = a.kv_base; p.vis = a.vis;
  p.n_rows = a.n_rows; p.M = a.M; p.hq = a.hq; p.hkv = a.hkv; p.G = G; p.error_flag = a.error_flag;
  p.tq = 128 / G;
  // Two query tiles per CTA share every key tile it loads and converts (6 rows of 1200 to 2304 tokens, 7 heads a group: 388
  // us, 546 with one; 3 rows of 600 to 700 48 and 67); one per CTA fills the SMs when there are few.
  const int nq = a.max_nq > 0 ? std::min(a.max_nq, a.M) : a.M;
  const long long singles = (long long)((nq + p.tq - 1) / p.tq) * a.n_rows * a.hkv;       // most query tiles there can be
  const bool two = singles > 2ll * sms && nq > p.tq;
  const int key_tiles = a.max_vis > 0 ? (a.max_vis + KT - 1) / KT : 1;
  // Few CTAs: the keys are cut, too, as long as a chunk keeps four key tiles (32 tokens, 4 kv heads: a row of 30,000 to 40,000
  // keys 45 us, 376 uncut, 4 rows of 1000 to 2000 24 and 33; 9 rows of 500 to 800 29 us in two chunks, 18 uncut).
  int chunks = 1;
  if (!two)
    while (chunks < kMaxChunks && singles * (chunks + 1) <= sms && key_tiles / (chunks + 1) >= kAttnKv8CutTiles / 2 &&
           (size_t)(chunks + 1) * a.M * a.hq * (DH + 2) <= part_floats)
      ++chunks;
  p.chunks = chunks;
  p.part_o = part;
  p.part_ml = reinterpret_cast<float2*>(part + (size_t)chunks * a.M * a.hq * DH);
  const int per_cta = (two ? 2 : 1) * p.tq;
  // CTAs by slots are as many as there could be spans, up to half of them empty; where the caller's largest row says where
  // the spans are, the CTAs that have work come first and the slots, for rows longer than that, last.
  const long long slots = (long long)a.M / per_cta + a.n_rows;
  const long long spans = a.max_nq > 0 ? (nq + per_cta - 1) / per_cta : 0;
  p.per_row = (int)(spans * a.n_rows <= slots ? spans : 0);
  const long long ctas = (slots + (long long)a.n_rows * p.per_row) * a.hkv * chunks;
  if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  const dim3 grid((unsigned)ctas);
  cudaError_t r = two ? launch_pdl(k_attention_kv8_tc<DH, 2>, grid, dim3(TcLayout<DH, 2>::threads), (size_t)TcLayout<DH, 2>::smem, s, mk, mv, p)
                      : launch_pdl(k_attention_kv8_tc<DH, 1>, grid, dim3(TcLayout<DH, 1>::threads), (size_t)TcLayout<DH, 1>::smem, s, mk, mv, p);
  if (r != cudaSuccess || chunks == 1) return r;
  return launch_pdl(k_attention_kv8_chunks<DH>, dim3((unsigned)(((long long)a.M * a.hq + 7) / 8)), dim3(256), 0, s, p);
}

}  // namespace

cudaError_t launch_attention_kv8_tc(const AttnKv8Args& a, float* part, size_t part_floats, cudaStream_t s) {
  int* sms = device_slot(g_sms);
  if (!sms) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(g_mutex);
    if (!*sms) {
      int n = 0;
      cudaError_t r = set_up<64>(&n);
      if (r == cudaSuccess) r = set_up<128>(&n);
      if (r != cudaSuccess) return r;
      *sms = n;
    }
  }
  return a.dh == 128 ? run_tc<128>(a, part, part_floats, *sms, s) : run_tc<64>(a, part, part_floats, *sms, s);
}

}  // namespace bs
