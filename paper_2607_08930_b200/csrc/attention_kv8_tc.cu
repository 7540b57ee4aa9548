// Ragged attention over the 8-bit KV cache on the 5th-generation tensor cores, for work items with more query rows than
// the streaming kernel takes: block steps, whole rows.  Formulas and the handling of the scales as in attention_kv8.cu.
//
// Work item = (row, kv head, tile of 128 flattened (token, head-in-group) query rows); a query row is a tensor-memory
// lane.  All items' key tiles (128 keys) form one line - an item counts a little more than its tiles - that the CTAs of
// one resident wave, one per SM, share evenly; cut items leave parts for the merge kernel (attention_kv8.cu).  A CTA is
// persistent and warp-specialised; the rings run on from one item to the next:
//   warp 0        producer: tiles of K and V codes by TMA, each through a ring of its own; the next item's query rows
//   warp 1        issues the products.  S = Q K^T takes K's codes as they arrive (kind::f8f6f4, e4m3 x e4m3): a query
//                 element, after a power of two per query row has brought the row's largest into [128, 256), is the sum
//                 of two e4m3 values - the nearest one and the rest (4 + 4 significant bits, bf16 has 8: exact above
//                 2^-10 of the row's largest element, within 2^-17 of that element below) - so S is two products at
//                 twice the rate of one in fp16, and K is neither converted nor stored a second time.  Q is an operand
//                 from tensor memory: read from shared memory it would take half of that memory's bandwidth.
//   2 x 4 warps   softmax, a query row per thread: one group takes the even tiles, the other the odd ones, each with a
//                 scores buffer of its own, so that the exponentials of one run under the loads, maxima and stores of
//                 the other.  The weights w = 2^(t - M) go back to tensor memory as fp16, over the first half of their
//                 scores, as the A operand of O += W V.
//   4 more warps  V's codes to fp16 (exact) in the layout of a B operand, rows behind the row's end as zeros; and the
//                 next item's queries to tensor memory.
// Weights are formed against a reference per row that lags the maximum (kTcBias, kTcGrow); the groups pass it to each
// other from tile to tile.  The output is rescaled only when a row's maximum has outgrown it.
// Every wait is bounded; on a timeout the flag is raised, all roles run through their loops without waiting, and the
// copies in flight are waited for.
#include <math.h>

#include <algorithm>
#include <mutex>

#include "kv8_line.cuh"
#include "tc_common.cuh"

namespace bs {

namespace {

using namespace tc;

constexpr int KT = 128;                              // keys per tile: four cache blocks
constexpr int kTcThreads = 512;
constexpr int kKStages = 4, kV8Stages = 3, kV16Stages = 2;
constexpr int kScaleStages = 8;                      // tiles whose scales are held; no ring runs that far ahead
constexpr int kQPad = 16;                            // bytes between query rows in shared memory: every lane its own banks
constexpr float kTcBias = 2.f, kTcGrow = 15.f;       // weights reach 2^15 at most, 2^2 when the reference is set
constexpr int kTcItemCost = 1;                       // tiles that an item counts beyond its own
constexpr unsigned kOCol = 256, kQCol = 384;         // tensor memory: two scores buffers, output, two query buffers

template <int DH>
struct TcLayout {
  static constexpr int k8 = KT * DH;                 // one tile of codes
  static constexpr int v16 = KT * DH * 2;            // one tile of V in fp16: DH / 64 parts of 64 dims
  static constexpr int q_row = DH * 2 + kQPad;
  static constexpr int k = 0, v8 = k + kKStages * k8, v = v8 + kV8Stages * k8, q = v + kV16Stages * v16,
                       bytes = q + 128 * q_row;
  static constexpr int smem = bytes + 1024;
  static constexpr int q_cols = DH / 2;              // tensor-memory columns of one query buffer (nearest values, rests)
};

__device__ __forceinline__ void tma_load_4d(unsigned dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, unsigned bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_load(unsigned dst, const void* src, unsigned bytes, unsigned bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// High word of a descriptor of an operand whose rows are row_bytes long (128 or 64, swizzled by as much), K-major.
template <int ROW>
__host__ __device__ constexpr unsigned desc_hi() { return (unsigned)(8 * ROW >> 4) | (1u << 14) | ((ROW == 128 ? 2u : 4u) << 29); }
// S: e4m3 (A, tensor memory) x e4m3 (B, K-major), fp32 accumulator, 128 x 128 x 32
constexpr unsigned kIdescS = (1u << 4) | ((unsigned)(KT >> 3) << 17) | ((128u >> 4) << 24);
// The issuing warp runs as a whole and one lane's instructions take effect: descriptors and addresses then stay in
// uniform registers, where the instruction wants them.
template <int DH>
__device__ __forceinline__ void umma_qk(unsigned d_tmem, unsigned a_tmem, unsigned b_lo, unsigned accumulate, unsigned leader) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %6, 0;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(kIdescS), "r"(accumulate), "r"(desc_hi<DH>()), "r"(leader) : "memory");
}
// O: fp16 (A, tensor memory) x fp16 (B, MN-major), fp32 accumulator, 128 x DH x 16
template <int DH>
__device__ __forceinline__ void umma_pv(unsigned d_tmem, unsigned a_tmem, unsigned b_lo, unsigned accumulate, unsigned leader) {
  constexpr unsigned idesc = (1u << 4) | (1u << 16) | ((unsigned)(DH >> 3) << 17) | ((128u >> 4) << 24);
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %6, 0;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi), "r"(leader) : "memory");
}
__device__ __forceinline__ void umma_commit_if(unsigned bar, unsigned leader) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader) : "memory");
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
__device__ __forceinline__ void tmem_st8(unsigned taddr, const unsigned* w) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ void tmem_ld16_nowait(unsigned taddr, unsigned* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint4 lds128(unsigned at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ void sts128(unsigned at, unsigned a, unsigned b, unsigned c, unsigned d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// generic-proxy writes to shared memory before tensor-core reads of it
__device__ __forceinline__ void fence_smem_for_mma() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// hand-over between the two warps that own the same query rows: one waits, the other has gone ahead
__device__ __forceinline__ void turn_wait(int id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ void turn_pass(int id) { asm volatile("barrier.cta.arrive %0, 64;" ::"r"(id) : "memory"); }

template <int DH>
__global__ void __launch_bounds__(kTcThreads, 1)
k_attention_kv8_tc(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const LineParams p) {
  using L = TcLayout<DH>;
  enum { B_KFULL = 0, B_KEMPTY = B_KFULL + kKStages, B_V8FULL = B_KEMPTY + kKStages, B_V8EMPTY = B_V8FULL + kV8Stages,
         B_VFULL = B_V8EMPTY + kV8Stages, B_VEMPTY = B_VFULL + kV16Stages, B_SFULL = B_VEMPTY + kV16Stages,
         B_PFULL = B_SFULL + 2, B_OFULL = B_PFULL + 2, B_LFULL = B_OFULL + 2, B_CFULL = B_LFULL + 2, B_TFULL = B_CFULL + 4,
         B_QFULL = B_TFULL + kScaleStages, B_QEMPTY = B_QFULL + 2, B_OEMPTY = B_QEMPTY + 2, B_RFULL = B_OEMPTY + 1,
         B_REMPTY = B_RFULL + 1, B_COUNT = B_REMPTY + 1 };
  extern __shared__ unsigned char smem_dyn[];
  __shared__ __align__(8) unsigned long long bars[B_COUNT];
  __shared__ unsigned tmem_base_slot;
  __shared__ int s_abort;
  __shared__ float2 s_scale[kScaleStages][4];        // (K scale, log2 of the V scale) of a tile's blocks
  __shared__ float s_sc[4][128];                     // score scale of every query row, by item
  __shared__ float s_ref[128];                       // reference of every query row
  __shared__ float2 s_part[2][128];                  // (reference, sum) of the group that does not write the item, by item parity
  __shared__ LineShared<kTcThreads, 1> s_line;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned smem0 = (smem_u32(smem_dyn) + 1023u) & ~1023u;
  const unsigned sK = smem0 + L::k, sV8 = smem0 + L::v8, sV16 = smem0 + L::v;
  const unsigned bar0 = smem_u32(&bars[0]);
  auto bar = [&](int i) { return bar0 + 8u * (unsigned)i; };
  if (threadIdx.x == 0) {
    s_abort = 0;
    for (int i = 0; i < kKStages; ++i) { mbar_init(bar(B_KFULL + i), 1); mbar_init(bar(B_KEMPTY + i), 1); }
    for (int i = 0; i < kV8Stages; ++i) { mbar_init(bar(B_V8FULL + i), 1); mbar_init(bar(B_V8EMPTY + i), 4); }
    for (int i = 0; i < kV16Stages; ++i) { mbar_init(bar(B_VFULL + i), 4); mbar_init(bar(B_VEMPTY + i), 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(B_SFULL + i), 1);
      mbar_init(bar(B_PFULL + i), 4);
      mbar_init(bar(B_OFULL + i), 1);
      mbar_init(bar(B_LFULL + i), 4);
      mbar_init(bar(B_QFULL + i), 4);
      mbar_init(bar(B_QEMPTY + i), 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(bar(B_CFULL + i), 4);
    for (int i = 0; i < kScaleStages; ++i) mbar_init(bar(B_TFULL + i), 1);
    mbar_init(bar(B_OEMPTY), 4);
    mbar_init(bar(B_RFULL), 1);
    mbar_init(bar(B_REMPTY), 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&tmem_base_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  pdl_trigger();

  // ---- this CTA's share of the line ----
  line_share<kTcThreads, 1, KT, DH>(p, kTcItemCost, 1, s_line);
  const LineShare share = s_line.share[0];
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  constexpr unsigned tmem_base = 0;                  // the only place an allocation of all 512 columns can have
  volatile int* abort_flag = &s_abort;
  const int G = p.hq / p.hkv;
  const bool work = share.units > 0;
  if (threadIdx.x == 0 && tmem_base_slot != 0) s_abort = 1;

  // 4 x 128 registers a thread at launch become 104 + 2 x 152 + 104.
  const int group = warp >> 2;
  if (group == 0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    if (warp == 0) {
      // ------------------------------------------------------------------ producer
      if (work) {
        int n = 0, items = 0;
        LineItem it;
        LineWalk w;
        w.begin<KT>(p, share);
        for (; w.next<KT>(p, kTcItemCost, it); ++items) {
          // (one lane's word counts for the warp: it stays together)
          if (!__shfl_sync(0xffffffffu, lane > 0 || mbar_wait(bar(B_REMPTY), (unsigned)(items & 1) ^ 1u, abort_flag), 0)) break;
          if (lane == 0) mbar_expect_tx(bar(B_RFULL), (unsigned)(it.nrows * DH * 2));
          __syncwarp();
          for (int f = lane; f < it.nrows; f += 32)
            bulk_load(smem0 + L::q + f * L::q_row, p.q + (size_t)(it.t0 + f / G) * p.q_ld + (it.head * G + f % G) * DH, DH * 2,
                      bar(B_RFULL));
          __syncwarp();
          const int blk0 = it.block0 + it.b0 * (KT / kKv8Block);
          for (int t = 0; t < it.b1 - it.b0; ++t, ++n) {
            // lanes 0 .. 3: the scales of the tile's blocks (which may reach over the cache's end)
            const size_t at = (size_t)min((long long)blk0 + 4 * t + (lane & 3), p.c.n_blocks - 1) * p.hkv + it.head;
            const float ks8 = __ldcg(p.c.k_scale + at), vs8 = __ldcg(p.c.v_scale + at);
            bool ok = true;
            if (lane == 0) {
              const int ks = n % kKStages, vs = n % kV8Stages;
              ok = mbar_wait(bar(B_KEMPTY + ks), (unsigned)((n / kKStages) & 1) ^ 1u, abort_flag) &&
                   mbar_wait(bar(B_V8EMPTY + vs), (unsigned)((n / kV8Stages) & 1) ^ 1u, abort_flag);
              if (ok) {
                mbar_expect_tx(bar(B_KFULL + ks), (unsigned)L::k8);
                tma_load_4d(sK + ks * L::k8, &map_k, 0, 0, it.head, blk0 + 4 * t, bar(B_KFULL + ks));
                mbar_expect_tx(bar(B_V8FULL + vs), (unsigned)L::k8);
                tma_load_4d(sV8 + vs * L::k8, &map_v, 0, 0, it.head, blk0 + 4 * t, bar(B_V8FULL + vs));
              }
            }
            if (!__shfl_sync(0xffffffffu, ok, 0)) break;
            // (the entry's tile before, eight back, is long done with: K's ring lets this one pass only behind its scores)
            if (lane < 4) s_scale[n % kScaleStages][lane] = make_float2(kv8_clamp_scale(ks8), log2_fast(kv8_clamp_scale(vs8)));
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_TFULL + n % kScaleStages));
          }
          if (__shfl_sync(0xffffffffu, *abort_flag, 0)) break;
        }
        if (lane == 0 && *abort_flag) {   // copies in flight end before the CTA does
          const long long begin = clock64();
          auto ended = [&](int barrier, int phase) {
            while (!mbar_try_wait(bar(barrier), (unsigned)phase & 1u) && clock64() - begin < kWaitCycles / 16) {
            }
          };
          for (int t = max(0, n - kKStages); t < n; ++t) ended(B_KFULL + t % kKStages, t / kKStages);
          for (int t = max(0, n - kV8Stages); t < n; ++t) ended(B_V8FULL + t % kV8Stages, t / kV8Stages);
          ended(B_RFULL, items);          // (where this item's was not issued, the wait runs out)
        }
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------------ MMA issuer
      if (work) {
        const unsigned leader = lane == 0;
        // Two walks over the same tiles: the scores run two tiles ahead of the products with V.  The scores buffer of
        // tile n is that of tile n - 2, whose weights the product issued just before has read: the tensor pipe runs
        // this thread's instructions in order.
        LineWalk ws, wv;
        ws.begin<KT>(p, share);
        wv = ws;
        LineItem is, iv;
        int ns = 0, ts = 0, items_s = 0;         // next scores: tile number, tile within the item, item number
        bool more = ws.next<KT>(p, kTcItemCost, is);
        auto scores = [&]() {
          if (!more) return;
          const int qb = items_s & 1;
          bool ok = ts > 0 || mbar_wait(bar(B_QFULL + qb), (unsigned)(items_s >> 1) & 1u, abort_flag);
          if (ok) ok = mbar_wait(bar(B_KFULL + ns % kKStages), (unsigned)(ns / kKStages) & 1u, abort_flag);
          if (!ok) { more = false; return; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const unsigned k_lo = desc_lo(sK + (ns % kKStages) * L::k8), d = tmem_base + (ns & 1) * 128;
          const unsigned q = tmem_base + kQCol + qb * 64;
#pragma unroll
          for (int k = 0; k < DH / 32; ++k) {
            umma_qk<DH>(d, q + k * 8, k_lo + 2 * k, k ? 1u : 0u, leader);
            umma_qk<DH>(d, q + L::q_cols / 2 + k * 8, k_lo + 2 * k, 1u, leader);
          }
          umma_commit_if(bar(B_SFULL + (ns & 1)), leader);
          umma_commit_if(bar(B_KEMPTY + ns % kKStages), leader);
          ++ns;
          if (++ts == is.b1 - is.b0) {
            umma_commit_if(bar(B_QEMPTY + qb), leader);
            ts = 0;
            ++items_s;
            more = ws.next<KT>(p, kTcItemCost, is);
          }
        };
        scores();
        scores();
        int n = 0, items = 0;
        while (!*abort_flag && wv.next<KT>(p, kTcItemCost, iv)) {
          for (int t = 0; t < iv.b1 - iv.b0; ++t, ++n) {
            const int vs = n % kV16Stages;
            if (t == 0 && items > 0 && !mbar_wait(bar(B_OEMPTY), (unsigned)(items - 1) & 1u, abort_flag)) break;
            if (!mbar_wait(bar(B_VFULL + vs), (unsigned)(n / kV16Stages) & 1u, abort_flag)) break;
            if (!mbar_wait(bar(B_PFULL + (n & 1)), (unsigned)(n >> 1) & 1u, abort_flag)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const unsigned v_lo = desc_lo(sV16 + vs * L::v16, KT * 128), a = tmem_base + (n & 1) * 128;
#pragma unroll
            for (int j = 0; j < KT / 16; ++j) umma_pv<DH>(tmem_base + kOCol, a + j * 8, v_lo + j * (2048 >> 4), (t || j) ? 1u : 0u, leader);
            umma_commit_if(bar(B_OFULL + (n & 1)), leader);
            umma_commit_if(bar(B_VEMPTY + vs), leader);
            scores();
          }
          ++items;
        }
      }
    }
  } else if (group == 3) {
    // ------------------------------------------------------------------ V: codes -> fp16 B operand; Q -> tensor memory
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    constexpr int LPK = DH / 16;                             // lanes per key, 16 dims each
    const int c = (int)threadIdx.x & 127;
    const int j = c % LPK;
    int n = 0, items = 0;
    LineItem it;
    if (work) {
      LineWalk w;
      w.begin<KT>(p, share);
      for (; w.next<KT>(p, kTcItemCost, it); ++items) {
        {   // query row c: 2 e4m3 values per element, four elements of a kind per column
          mbar_wait(bar(B_RFULL), (unsigned)items & 1u, abort_flag);
          const int qb = items & 1;
          mbar_wait(bar(B_QEMPTY + qb), (unsigned)((items >> 1) & 1) ^ 1u, abort_flag);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const bool valid = c < it.nrows;
          const unsigned src = smem0 + L::q + c * L::q_row;
          float top = 0.f;
#pragma unroll
          for (int i = 0; i < DH / 8; ++i) {
            const uint4 raw = lds128(src + i * 16);
            const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&raw);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float2 y = __bfloat1622float2(h[k]);
              top = fmaxf(top, fmaxf(fabsf(y.x), fabsf(y.y)));
            }
          }
          if (!valid) top = 0.f;
          const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 100);
          const float up = valid ? pow2i(7 - e) : 0.f;
          s_sc[items & 3][c] = pow2i(e - 7) * (1.4426950408889634f * rsqrtf((float)DH));
          const unsigned dst = tmem_base + ((unsigned)(c & 96) << 16) + kQCol + qb * 64;
#pragma unroll 1
          for (int i = 0; i < DH / 32; ++i) {
            unsigned hi[8], lo[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              hi[k] = lo[k] = 0u;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint4 raw = lds128(src + (i * 4 + k) * 16);
              if (!valid) raw = make_uint4(0, 0, 0, 0);      // (what was there before may be anything)
              const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&raw);
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                const float2 y = __bfloat1622float2(h[m]);
                const float a = y.x * up, b = y.y * up;
                const unsigned near = kv8_encode2(a, b), back = kv8_decode2((unsigned short)near);
                const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&back));
                hi[2 * k + (m >> 1)] |= near << (16 * (m & 1));
                lo[2 * k + (m >> 1)] |= kv8_encode2(a - z.x, b - z.y) << (16 * (m & 1));
              }
            }
            tmem_st8(dst + i * 8, hi);
            tmem_st8(dst + L::q_cols / 2 + i * 8, lo);
          }
          tmem_st_wait();
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(B_REMPTY));
            mbar_arrive(bar(B_QFULL + qb));
            mbar_arrive(bar(B_CFULL + (items & 3)));
          }
        }
        for (int t = it.b0; t < it.b1; ++t, ++n) {
          const int a = n % kV8Stages, b = n % kV16Stages;
          mbar_wait(bar(B_V8FULL + a), (unsigned)(n / kV8Stages) & 1u, abort_flag);
          mbar_wait(bar(B_VEMPTY + b), (unsigned)((n / kV16Stages) & 1) ^ 1u, abort_flag);
          const int left = it.vis - t * KT;
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
              const unsigned line = dst + key * 128, c0 = 2 * (j & 3) + (flip ? 1 : 0), sw = key & 7;
              sts128(line + ((c0 ^ sw) << 4), y[flip ? 4 : 0], y[flip ? 5 : 1], y[flip ? 6 : 2], y[flip ? 7 : 3]);
              sts128(line + (((c0 ^ 1) ^ sw) << 4), y[flip ? 0 : 4], y[flip ? 1 : 5], y[flip ? 2 : 6], y[flip ? 3 : 7]);
            }
          }
          fence_smem_for_mma();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(B_V8EMPTY + a));
            mbar_arrive(bar(B_VFULL + b));
          }
        }
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax: one query row per thread
    // (On a timeout nobody leaves the loops: the two warps of the same rows meet at the same barriers to the end.)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 152;");
    const int me = group - 1, quad = warp & 3, r = quad * 32 + lane;
    const int my_turn = 1 + 2 * quad + me, your_turn = 1 + 2 * quad + (me ^ 1);
    const unsigned t_lane = tmem_base + ((unsigned)(quad * 32) << 16), t_s = t_lane + me * 128, t_out = t_lane + kOCol;
    int n = 0, items = 0;                  // n: number of the item's first tile; group `me` takes the tiles of its parity
    unsigned lphase = 0;                   // phases of B_LFULL, which only items of two tiles and more use
    LineItem it;
    if (work) {
      if (me == 1) turn_pass(your_turn);
      LineWalk w;
        w.begin<KT>(p, share);
        for (; w.next<KT>(p, kTcItemCost, it); ++items) {
        const bool warp_has_rows = quad * 32 < it.nrows;
        const int end = n + it.b1 - it.b0;
        const int start = n + ((n ^ me) & 1);
        float ref = -INFINITY, sum = 0.f, sc = 0.f;
        for (int t = start; t < end; t += 2) {
          const int left = it.vis - (it.b0 + t - n) * KT;     // keys of this tile that the row sees
          const float2* scale = s_scale[t % kScaleStages];
          if (t == start) {
            mbar_wait(bar(B_CFULL + (items & 3)), (unsigned)(items >> 2) & 1u, abort_flag);
            sc = s_sc[items & 3][r];
          }
          mbar_wait(bar(B_TFULL + t % kScaleStages), (unsigned)(t / kScaleStages) & 1u, abort_flag);
          mbar_wait(bar(B_SFULL + me), (unsigned)(t >> 1) & 1u, abort_flag);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          // (The loops over 16 scores are kept rolled: unrolled, four roles' straight-line code does not fit the
          // instruction caches - 128 scores unrolled measured 1.5 times the whole kernel's time.  The next 16 are loaded
          // while these are worked on.)
          auto mask = [&](unsigned* x, int first) {
            if (left < first + 16) {
#pragma unroll
              for (int j = 0; j < 16; ++j) x[j] = first + j < left ? x[j] : 0xff800000u;      // -inf
            }
          };
          float top = -INFINITY;
          if (warp_has_rows) {
            unsigned ra[16], rb[16];
            auto largest = [&](unsigned* x, int first) {
              mask(x, first);
              float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
              for (int j = 0; j < 16; ++j) m4[j & 3] = fmaxf(m4[j & 3], __uint_as_float(x[j]));
              return fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            };
            tmem_ld16_nowait(t_s, ra);
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
              tmem_ld_wait();
              tmem_ld16_nowait(t_s + i * 32 + 16, rb);
              const float fi = scale[i].x * sc, li = scale[i].y;
              float m = largest(ra, i * 32);
              tmem_ld_wait();
              if (i < 3) tmem_ld16_nowait(t_s + (i + 1) * 32, ra);
              m = fmaxf(m, largest(rb, i * 32 + 16));
              top = fmaxf(top, fmaf(m, fi, li));
            }
          }
          // ---- the reference, after the tile before has settled it ----
          turn_wait(my_turn);
          if (warp_has_rows) {
            const float old = t == n ? -INFINITY : s_ref[r];
            const bool grow = top > old + kTcGrow;
            const float now = grow ? top - kTcBias : old;
            if (__any_sync(0xffffffffu, grow)) {
              s_ref[r] = now;
              if (t > n) {
                // the product of the tile before has to be done with the output
                mbar_wait(bar(B_OFULL + ((t - 1) & 1)), (unsigned)((t - 1) >> 1) & 1u, abort_flag);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const float turn = grow ? exp2_fast(old - now) : 1.f;
#pragma unroll 1
                for (int c = 0; c < DH / 32; ++c) {
                  unsigned o[32];
                  tmem_ld32_nowait(t_out + c * 32, o);
                  tmem_ld_wait();
#pragma unroll
                  for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * turn);
                  tmem_st32(t_out + c * 32, o);
                }
                tmem_st_wait();
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
              }
            } else if (t == n) {
              s_ref[r] = now;
            }
            if (now != ref) {
              sum = ref > -INFINITY ? sum * exp2_fast(ref - now) : sum;      // (a row of NaN keeps its NaN)
              ref = now;
            }
          }
          __syncwarp();
          turn_pass(your_turn);
          // ---- weights ----
          if (warp_has_rows) {
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {                      // 64 scores
              unsigned out[32];
              unsigned ra[32], rb[32];
              tmem_ld32_nowait(t_s + h * 64, ra);
              tmem_ld_wait();
              tmem_ld32_nowait(t_s + h * 64 + 32, rb);
              auto weights = [&](unsigned* x, int i, unsigned* w) {
                const int first = h * 64 + i * 32;
                const float fi = scale[2 * h + i].x * sc, li = scale[2 * h + i].y, shift = li - ref;
                if (left < first + 32) {
#pragma unroll
                  for (int j = 0; j < 32; ++j) x[j] = first + j < left ? x[j] : 0xff800000u;      // -inf
                }
                float a4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                  const float e0 = exp2_fast(fmaf(__uint_as_float(x[j]), fi, shift));
                  const float e1 = exp2_fast(fmaf(__uint_as_float(x[j + 1]), fi, shift));
                  a4[(j >> 1) & 3] += e0 + e1;
                  const __half2 v = __floats2half2_rn(e0, e1);
                  w[j >> 1] = *reinterpret_cast<const unsigned*>(&v);
                }
                sum = fmaf((a4[0] + a4[1]) + (a4[2] + a4[3]), exp2_fast(-li), sum);      // 2^-lv: the inverse of the V scale
              };
              weights(ra, 0, out);
              tmem_ld_wait();
              weights(rb, 1, out + 16);
              tmem_st32(t_s + h * 32, out);                    // (over columns that were read before)
            }
            tmem_st_wait();
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          if (t == end - 2) s_part[items & 1][r] = make_float2(ref, sum);      // the other group writes the item
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar(B_PFULL + me));
            if (t == end - 2) mbar_arrive(bar(B_LFULL + (items & 1)));
          }
        }
        // ---- output, by the group that took the last tile ----
        if (((end - 1) & 1) == me) {
          // (Warps without query rows wait for the item's last product too: they would otherwise report the next item
          // before the others have this one.)
          const bool ok = mbar_wait(bar(B_OFULL + ((end - 1) & 1)), (unsigned)((end - 1) >> 1) & 1u, abort_flag);
          if (end - n > 1) {
            mbar_wait(bar(B_LFULL + (items & 1)), (unsigned)(lphase >> (items & 1)) & 1u, abort_flag);
            lphase ^= 1u << (items & 1);
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          if (warp_has_rows) {
            float total = sum;
            if (end - n > 1) {
              const float2 o = s_part[items & 1][r];
              total += o.x > -INFINITY ? o.y * exp2_fast(o.x - ref) : o.y;
            }
            const bool valid = r < it.nrows && ok;
            const int rr = r < it.nrows ? r : 0;
            const bool whole = it.b0 == 0 && it.b1 == it.nb;
            const size_t slot = 2 * (size_t)blockIdx.x + (it.opens ? 0 : 1);
            bf16* dst = p.out + ((size_t)(it.t0 + rr / G) * p.hq + it.head * G + rr % G) * DH;
            float* part = p.part_o + (slot * 128 + rr) * DH;
            const float inv = 1.0f / total;
            if (!whole && valid) p.part_ml[slot * 128 + rr] = make_float2(ref, total);
#pragma unroll 1
            for (int c = 0; c < DH / 32; ++c) {
              unsigned o[32];
              tmem_ld32_nowait(t_out + c * 32, o);
              tmem_ld_wait();
              if (!valid) continue;
              if (!whole) {
#pragma unroll
                for (int g = 0; g < 8; ++g)
                  *reinterpret_cast<uint4*>(part + c * 32 + g * 4) = make_uint4(o[g * 4], o[g * 4 + 1], o[g * 4 + 2], o[g * 4 + 3]);
              } else {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                  uint4 v;
                  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    h[j] = __floats2bfloat162_rn(__uint_as_float(o[g * 8 + 2 * j]) * inv, __uint_as_float(o[g * 8 + 2 * j + 1]) * inv);
                  *reinterpret_cast<uint4*>(dst + c * 32 + g * 8) = v;
                }
              }
            }
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_OEMPTY));
        } else if (end - n > 1) {
          lphase ^= 1u << (items & 1);
        }
        n = end;
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

}  // namespace

// p: everything but the query tile; *ctas: how many partial-slot pairs the launch may use (two slots of 128 rows each).
cudaError_t launch_attention_kv8_tc(LineParams p, int dh, int max_ctas, int* ctas, cudaStream_t s) {
  int* sms = device_slot(g_sms);
  if (!sms) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(g_mutex);
    if (!*sms) {
      int dev = 0, n = 0;
      cudaError_t r = cudaGetDevice(&dev);
      if (r == cudaSuccess) r = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
      if (r == cudaSuccess)
        r = cudaFuncSetAttribute(k_attention_kv8_tc<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcLayout<64>::smem);
      if (r == cudaSuccess)
        r = cudaFuncSetAttribute(k_attention_kv8_tc<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcLayout<128>::smem);
      if (r != cudaSuccess) return r;
      *sms = n;
    }
  }
  CUtensorMap mk, mv;
  if (!make_map(p.c.k, p.hkv, dh, p.c.n_blocks, true, &mk) || !make_map(p.c.v, p.hkv, dh, p.c.n_blocks, false, &mv))
    return cudaErrorInvalidValue;
  *ctas = std::min(*sms, max_ctas);
  return dh == 128 ? launch_pdl(k_attention_kv8_tc<128>, dim3(*ctas), dim3(kTcThreads), (size_t)TcLayout<128>::smem, s, mk, mv, p)
                   : launch_pdl(k_attention_kv8_tc<64>, dim3(*ctas), dim3(kTcThreads), (size_t)TcLayout<64>::smem, s, mk, mv, p);
}

}  // namespace bs
