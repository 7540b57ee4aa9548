// Ragged attention over the 8-bit KV cache (layout in kv8.cuh): every query token of row i attends to cache rows
// [kv_base_i, kv_base_i + vis_i); no causal or padding mask; rows with vis_i = 0 give zeros.
//
//   s_j = q . k_j / sqrt(dh),   out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m)
//
// with k_j = ks_b c_j and v_j = vs_b c'_j for the codes c, c' and the two scales of cache block b.  No scale is rounded
// into an operand: ks_b multiplies the finished fp32 scores, and the weight that meets the codes of V is
//
//   w_j = vs_b e^(s_j - m) = 2^(t_j - M),   t_j = log2(e) s_j + log2(vs_b),   M: running maximum of t
//
// so that weights are largest where the summands w_j c'_j are; the denominator takes w_j / vs_b.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <mutex>

#include "kv8_line.cuh"
#include "tc_common.cuh"

namespace bs {

namespace {

__device__ __forceinline__ void mma_f16(float* c, const unsigned* a, unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 8 x 8 fp16 matrix across the warp (lane (g, c): row g, columns 2c, 2c + 1), transposed
__device__ __forceinline__ unsigned transpose8x8(unsigned x) {
  unsigned r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ unsigned pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&h);
}
// Weights, up to 2^kGrow: beyond 2^23 the sum ref + kGrow that they are compared with is rounded itself, and one may reach
// 2^16, just over fp16's range (held to 65504, a relative 2^-11).
__device__ __forceinline__ unsigned pack_weights(float a, float b) {
  unsigned r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
// 16 bytes to shared memory, or zeros (`real` = false; the source is then not read)
__device__ __forceinline__ void copy_async16(unsigned dst, const void* src, bool real) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint4 lds128(unsigned at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds64(unsigned at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}

// ---- streaming kernel ---------------------------------------------------------------------------------------
//
// Few query rows per kv head (single tokens, block steps without grouped heads): bound by the bytes of the cache.
// A work item is (row, kv head, tile of 8 NQ flattened (token, head-in-group) query rows).  All items' cache blocks
// form one line - an item counts a few blocks more than it has, about what starting and ending it costs - which the
// workers of a single resident wave share evenly: worker c takes units [c T / N, (c + 1) T / N), whatever the rows'
// lengths are.  An item that a worker holds whole is written out directly; a cut one leaves partial (output, reference,
// sum) parts, at most two per worker, that a second small kernel merges in order.  Where no row is long (DIRECT) every
// item has a worker of its own instead, and there is neither a line to lay out nor a second kernel.
//
// A worker is a CTA of four warps (W = 4: long items, few of them; the warps take the item's blocks in turn and add
// their parts up in shared memory) or a single warp (W = 1: many items, whose beginnings and ends would leave four
// warps waiting for one another).  Every warp moves its blocks (32 keys) through a ring of shared-memory stages that
// no other warp touches (cp.async, no barrier): the next blocks are on their way while this one is computed.  Rows
// behind the row's end arrive as zeros, whatever the cache holds there.
//
// What it reaches: 64 single-token rows of 1024 to 4096 keys (28 / 4 heads, 175 MB) 38.7 us, of which the merge takes 5 to 6;
// two rows of 50,001 and 65,536 keys 29.0 us, 6 of them merge.  64 rows x 32 tokens over up to 1024 keys of 32 heads, 116 us,
// wait on one another's instructions instead: with 16 query rows per item every block is fetched and decoded twice (530 MB
// read where 306 would do), each time for only 64 products, and two warps per scheduler fill 39 % of the issue slots and
// 32 % of the tensor pipe.
//
// Keys are the rows (M) of both products and the queries their columns (N), so that 8 query rows - a group of heads of
// one token - fill an instruction.  Codes go to the tensor cores as fp16, which holds every e4m3 value (the warp-level
// e4m3 product is no way around that: measured on B200, it runs as conversions and two fp16 products, 25 clk against 8).
// Queries become fp16 after a power of two per query row has brought their largest element into [1, 2), or [2, 4) in the
// type's last binade: bf16's 8 bits fit fp16's 11, and what drops below 2^-24 of the row's largest element is below the
// fp32 sum's own rounding.  Weights
// are fp16, transposed in registers (movmatrix).  The order of the dims in the scores' k index and of the dims in the
// output's m index is free, and is chosen so that a lane's 16-byte shared-memory loads hold its operand registers; a
// 16-byte chunk's place in its 128-byte line is turned by the line's number, which keeps those loads free of bank
// conflicts.
constexpr int kStreamWarps = 4;
constexpr int kStreamThreads = kStreamWarps * 32;
constexpr int kMaxStreamCtas = 592;
// Units an item counts beyond its blocks, in block times of one worker.
__host__ __device__ constexpr int item_cost(int w) { return w == 1 ? 3 : 8; }
// Weights are formed against a reference kBias below the running maximum (log2 units), which is moved only when the
// maximum has grown kGrow above it: they stay below 2^kGrow in fp16 and keep full precision down to 2^-20 of the
// largest one.
constexpr float kBias = 6.f, kGrow = 14.f;

template <int DH>
constexpr int kTileBytes = kKv8Block * DH;           // one block of one head, K or V
template <int DH, int NQ, int STAGES, int W>
struct StreamSmem {
  static constexpr int R = 8 * NQ, LDO = DH + 4, groups = kStreamWarps / W;
  static constexpr int ring = kStreamWarps * STAGES * 2 * kTileBytes<DH>;
  static constexpr int merge = W == 1 ? 0 : W * R * LDO * 4;       // the warps' outputs, over the ring when it is idle
  static constexpr int front = ring > merge ? ring : merge;
  static constexpr int q = NQ * (DH / 32) * 32 * 16;               // query fragments, two k steps in 16 bytes
  static constexpr int total = 128 + front + groups * (q + W * R * 8 + R * 4);
};
template <int DH, int NQ, int STAGES, int W, int MINB, bool DIRECT>
__global__ void __launch_bounds__(kStreamThreads, MINB) k_attention_kv8_stream(const LineParams p) {
  using L = StreamSmem<DH, NQ, STAGES, W>;
  constexpr int KP = DH / 32;            // pairs of k steps of the scores
  constexpr int MD = DH / 16;            // m tiles of the output
  constexpr int R = L::R, LDO = L::LDO, TB = kTileBytes<DH>, kCost = item_cost(W);
  extern __shared__ unsigned char smem_raw[];
  __shared__ LineShared<kStreamThreads, L::groups> s_line;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, c4 = lane & 3;
  const int G = p.hq / p.hkv;
  // this thread's worker: its number in the CTA, and the warp's and the thread's number in the worker
  const int wk = W == 1 ? warp : 0, member = W == 1 ? 0 : warp, wtid = W == 1 ? lane : tid;
  auto sync_worker = [&]() { if (W == 1) __syncwarp(); else __syncthreads(); };
  unsigned char* smem = smem_raw + ((128u - (tc::smem_u32(smem_raw) & 127u)) & 127u);
  float* s_o = reinterpret_cast<float*>(smem);                               // [warps][R][LDO] (W = 4)
  uint4* s_q = reinterpret_cast<uint4*>(smem + L::front + wk * (L::q + W * R * 8 + R * 4));    // [NQ][KP][32]
  float2* s_ml = reinterpret_cast<float2*>(s_q + L::q / 16);                 // [W][R]
  float* s_sc = reinterpret_cast<float*>(s_ml + W * R);                      // [R]
  pdl_wait();
  pdl_trigger();

  const size_t me = (size_t)blockIdx.x * L::groups + wk;
  LineItem it = {};
  LineWalk walk;
  int tile = 0;
  if constexpr (DIRECT) {
    if (!direct_item<kKv8Block>(p, (long long)me, wtid, it, walk.ri, tile)) return;
  } else {
    line_share<kStreamThreads, L::groups, kKv8Block, DH>(p, kCost, W, s_line);
    if (s_line.share[wk].units == 0) return;   // (from here on only the worker's own threads wait for one another)
    walk.begin<kKv8Block>(p, s_line.share[wk]);
  }
  auto next = [&]() {
    if constexpr (!DIRECT) return walk.next<kKv8Block>(p, kCost, it);
    for (; tile < walk.ri.tiles; tile += p.direct) {
      it.t0 = walk.ri.t0 + tile * p.tq;
      it.nrows = min(p.tq, walk.ri.t0 + walk.ri.n - it.t0) * G;
      if (it.nb > 0) {
        tile += p.direct;
        return true;
      }
      for (int i = wtid; i < it.nrows * (DH / 8); i += W * 32)       // a row that sees nothing
        reinterpret_cast<uint4*>(p.out + (size_t)(it.t0 + i / (DH / 8) / G) * (p.hq * DH) +
                                 (it.head * G + i / (DH / 8) % G) * DH)[i % (DH / 8)] = make_uint4(0, 0, 0, 0);
    }
    return false;
  };

  // this warp's ring, and this lane's part of a block's copy: 16 bytes i * 512 + lane * 16 of K and of V
  const unsigned ring = tc::smem_u32(smem) + (unsigned)warp * STAGES * 2 * TB;
  const unsigned put0 = (unsigned)((lane >> 3) * 128 + (((lane & 7) ^ (lane >> 3)) << 4));
  const unsigned put1 = (unsigned)((lane >> 3) * 128 + (((lane & 7) ^ (4 + (lane >> 3))) << 4));
  auto tile_of = [&](int b) { return ((size_t)it.block0 + b) * p.hkv + it.head; };
  auto fetch = [&](int stage, int b) {
    const size_t at = tile_of(b) * TB + lane * 16;
    const unsigned dst = ring + (unsigned)stage * 2 * TB;
    const int rows = it.vis - b * kKv8Block;
#pragma unroll
    for (int i = 0; i < TB / 512; ++i) {
      const bool real = (i * 512 + lane * 16) / DH < rows;
      const unsigned to = dst + i * 512 + ((i & 1) ? put1 : put0);
      copy_async16(to, p.c.k + at + i * 512, real);
      copy_async16(to + TB, p.c.v + at + i * 512, real);
    }
  };

  while (next()) {
    const int b0 = it.b0, b1 = it.b1, head = it.head, t0 = it.t0, nrows = it.nrows;
    sync_worker();                       // the previous segment's fragments, sums and outputs are no longer read
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) {
      if (b0 + member + i * W < b1) fetch(i, b0 + member + i * W);
      asm volatile("cp.async.commit_group;\n" ::: "memory");
    }
    float ks_next = 1.f, vs_next = 1.f;
    if (b0 + member < b1) {
      const size_t sa = tile_of(b0 + member);
      ks_next = __ldcg(p.c.k_scale + sa);
      vs_next = __ldcg(p.c.v_scale + sa);
    }
    // ---- queries: fp16 fragments in shared memory ----
    for (int nq = member; nq < NQ; nq += W) {
      const int f = nq * 8 + g;          // query row of this lane (n index of the scores)
      const bool valid = f < nrows;
      const bf16* src = p.q + (size_t)(t0 + (valid ? f / G : 0)) * p.q_ld + (head * G + (valid ? f % G : 0)) * DH + c4 * (DH / 4);
      uint4 raw[KP];
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < KP; ++k) {     // k step i of lane c4 stands for dims c4 DH / 4 + 4 i .. + 3
        raw[k] = valid ? __ldcg(reinterpret_cast<const uint4*>(src + k * 8)) : make_uint4(0, 0, 0, 0);
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&raw[k]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = __bfloat1622float2(h[j]);
          top = fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y)));
        }
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 126);     // 2^-126 is fp32's least normal power
      const float up = pow2i(-e);
      if (c4 == 0) s_sc[f] = fminf(pow2i(e) * (1.4426950408889634f * rsqrtf((float)DH)), kMaxFactor);
#pragma unroll
      for (int k = 0; k < KP; ++k) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&raw[k]);
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = __bfloat1622float2(h[j]);
          w[j] = pack_f16(x.x * up, x.y * up);
        }
        s_q[(nq * KP + k) * 32 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    sync_worker();

    float o[NQ][MD][4];
    float ref[NQ][2], sum[NQ][2], sc[NQ][2];         // of query rows nq * 8 + 2 c4 + {0, 1}
    uint4 qf[NQ == 1 ? KP : 1];
    if (NQ == 1) {
#pragma unroll
      for (int k = 0; k < KP; ++k) qf[NQ == 1 ? k : 0] = s_q[k * 32 + lane];
    }
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
      for (int i = 0; i < MD; ++i) o[nq][i][0] = o[nq][i][1] = o[nq][i][2] = o[nq][i][3] = 0.f;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        ref[nq][y] = -FLT_MAX;           // (under any score but -inf, whose weight it makes 0)
        sum[nq][y] = 0.f;
        sc[nq][y] = s_sc[nq * 8 + 2 * c4 + y];
      }
    }

    int stage = 0;
    for (int b = b0 + member; b < b1; b += W) {
      const float ks = kv8_clamp_scale(ks_next), vs = kv8_clamp_scale(vs_next);
      {
        const int nb = b + (STAGES - 1) * W;
        if (nb < b1) fetch(stage == 0 ? STAGES - 1 : stage - 1, nb);
        asm volatile("cp.async.commit_group;\n" ::: "memory");
        if (b + W < b1) {
          const size_t sa = tile_of(b + W);
          ks_next = __ldcg(p.c.k_scale + sa);
          vs_next = __ldcg(p.c.v_scale + sa);
        }
      }
      const float lv = log2_fast(vs), inv_vs = 1.0f / vs;
      const int left = it.vis - b * kKv8Block;         // keys of this block that the row sees (> 0)
      asm volatile("cp.async.wait_group %0;\n" ::"n"(STAGES - 1) : "memory");
      __syncwarp();
      const unsigned kt = ring + (unsigned)stage * 2 * TB, vt = kt + TB;
#pragma unroll
      for (int m = 0; m < 2; ++m) {                    // 16 keys: rows 16 m + g and 16 m + g + 8 of this lane
        float s[NQ][4];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) s[nq][0] = s[nq][1] = s[nq][2] = s[nq][3] = 0.f;
        float s_odd[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < KP / 2; ++h) {             // 16 bytes of both keys: four k steps
          uint4 kr[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int key = m * 16 + g + 8 * x;
            // dh 128: line = key, chunk 2 c4 + h; dh 64: two keys per line, chunk 4 (key & 1) + c4
            const int line = DH == 128 ? key : key >> 1, chunk = DH == 128 ? 2 * c4 + h : 4 * (key & 1) + c4;
            kr[x] = lds128(kt + line * 128 + ((chunk ^ (line & 7)) << 4));
          }
          unsigned a[4][4];              // [k step][key g: 2 dims, key g + 8, key g: next 2 dims, key g + 8]
          kv8_decode4(kr[0].x, a[0][0], a[0][2]); kv8_decode4(kr[1].x, a[0][1], a[0][3]);
          kv8_decode4(kr[0].y, a[1][0], a[1][2]); kv8_decode4(kr[1].y, a[1][1], a[1][3]);
          kv8_decode4(kr[0].z, a[2][0], a[2][2]); kv8_decode4(kr[1].z, a[2][1], a[2][3]);
          kv8_decode4(kr[0].w, a[3][0], a[3][2]); kv8_decode4(kr[1].w, a[3][1], a[3][3]);
          // a product's latency is that of two to three others: the chains of the query tiles (one tile: of even and
          // odd k steps) take turns
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint4 qv[NQ];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) qv[nq] = NQ == 1 ? qf[NQ == 1 ? 2 * h + i : 0] : s_q[(nq * KP + 2 * h + i) * 32 + lane];
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) mma_f16(s[nq], a[2 * i], qv[nq].x, qv[nq].y);
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) mma_f16(NQ == 1 ? s_odd : s[nq], a[2 * i + 1], qv[nq].z, qv[nq].w);
          }
        }
        if (NQ == 1) {
#pragma unroll
          for (int j = 0; j < 4; ++j) s[0][j] += s_odd[j];
        }
        unsigned pr[NQ][2];
        bool grow = false;
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {                // j & 1: query row, j >> 1: key
            s[nq][j] = m * 16 + g + 8 * (j >> 1) < left ? fmaf(s[nq][j], sc[nq][j & 1] * ks, lv) : -INFINITY;
            grow = grow || s[nq][j] > ref[nq][j & 1] + kGrow;
          }
        }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float mx = fmaxf(s[nq][y], s[nq][2 + y]);
              mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
              mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
              mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
              if (mx > ref[nq][y] + kGrow) {
                const float f = exp2_fast(ref[nq][y] - (mx - kBias));
                ref[nq][y] = mx - kBias;
                sum[nq][y] *= f;
#pragma unroll
                for (int i = 0; i < MD; ++i) {
                  o[nq][i][y] *= f;
                  o[nq][i][2 + y] *= f;
                }
              }
            }
        }
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
          const float e0 = exp2_fast(s[nq][0] - ref[nq][0]), e1 = exp2_fast(s[nq][1] - ref[nq][1]);
          const float e2 = exp2_fast(s[nq][2] - ref[nq][0]), e3 = exp2_fast(s[nq][3] - ref[nq][1]);
          sum[nq][0] = fmaf(e0 + e2, inv_vs, sum[nq][0]);
          sum[nq][1] = fmaf(e1 + e3, inv_vs, sum[nq][1]);
          pr[nq][0] = transpose8x8(pack_weights(e0, e1));
          pr[nq][1] = transpose8x8(pack_weights(e2, e3));
        }
        // ---- output: dims g DH / 8 + 2 i (row g of m tile i) and + 1 (row g + 8) ----
        unsigned vr[4][DH / 32];         // keys 16 m + 2 c4, + 1, + 8, + 9
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = m * 16 + 2 * c4 + (j & 1) + (j >> 1) * 8;
          if (DH == 128) {
            const uint4 v = lds128(vt + key * 128 + ((g ^ (key & 7)) << 4));
            vr[j][0] = v.x; vr[j][1] = v.y;
            vr[j][DH / 32 - 2] = v.z; vr[j][DH / 32 - 1] = v.w;
          } else {
            const int line = key >> 1, chunk = 4 * (key & 1) + (g >> 1);
            const uint2 v = lds64(vt + line * 128 + ((chunk ^ (line & 7)) << 4) + (g & 1) * 8);
            vr[j][0] = v.x; vr[j][1] = v.y;
          }
        }
#pragma unroll
        for (int w = 0; w < DH / 32; ++w)
#pragma unroll
          for (int z = 0; z < 2; ++z) {                // dims 4 w + 2 z, + 1: bytes of two keys side by side
            unsigned a[4];
            kv8_decode4(__byte_perm(vr[0][w], vr[1][w], z ? 0x7362 : 0x5140), a[0], a[1]);
            kv8_decode4(__byte_perm(vr[2][w], vr[3][w], z ? 0x7362 : 0x5140), a[2], a[3]);
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq) mma_f16(o[nq][2 * w + z], a, pr[nq][0], pr[nq][1]);
          }
      }
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      __syncwarp();                      // the stage may be filled again
    }

    const bool whole = DIRECT || (b0 == 0 && b1 == it.nb);
    const size_t slot = 2 * me + (it.opens ? 0 : 1);
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        sum[nq][y] += __shfl_xor_sync(0xffffffffu, sum[nq][y], 4);
        sum[nq][y] += __shfl_xor_sync(0xffffffffu, sum[nq][y], 8);
        sum[nq][y] += __shfl_xor_sync(0xffffffffu, sum[nq][y], 16);
      }
    if constexpr (W == 1) {
      // straight from the registers: lane (g, c4) holds 16 (head_dim 64: 8) dims of query rows 2 c4 and 2 c4 + 1
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int f = nq * 8 + 2 * c4 + y;
          if (f >= nrows) continue;
          if (whole) {
            const float inv = 1.0f / sum[nq][y];
            bf16* dst = p.out + (size_t)(t0 + f / G) * (p.hq * DH) + (head * G + f % G) * DH + g * (DH / 8);
#pragma unroll
            for (int i = 0; i < MD; i += 4) {
              uint4 w;
              __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&w);
#pragma unroll
              for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(o[nq][i + j][y] * inv, o[nq][i + j][2 + y] * inv);
              *reinterpret_cast<uint4*>(dst + 2 * i) = w;
            }
          } else {
            float* dst = p.part_o + (slot * R + f) * DH + g * (DH / 8);
#pragma unroll
            for (int i = 0; i < MD; i += 2)
              *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(o[nq][i][y], o[nq][i][2 + y], o[nq][i + 1][y], o[nq][i + 1][2 + y]);
            if (g == 0) p.part_ml[slot * R + f] = make_float2(ref[nq][y], sum[nq][y]);
          }
        }
    } else {
    // ---- the warps' parts of this segment become one ----
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int y = 0; y < 2; ++y)
        if (g == 0) s_ml[member * R + nq * 8 + 2 * c4 + y] = make_float2(ref[nq][y], sum[nq][y]);
    sync_worker();                       // (the ring is idle from here on)
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int f = nq * 8 + 2 * c4 + y;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) m = fmaxf(m, s_ml[w * R + f].x);
        const float turn = exp2_fast(ref[nq][y] - m);        // (a warp without blocks: zeros; NaN stays NaN)
        float* dst = s_o + (member * R + f) * LDO + g * (DH / 8);
#pragma unroll
        for (int i = 0; i < MD; i += 2)
          *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(o[nq][i][y] * turn, o[nq][i][2 + y] * turn,
                                                                o[nq][i + 1][y] * turn, o[nq][i + 1][2 + y] * turn);
      }
    sync_worker();
    for (int v = wtid; v < nrows * (DH / 4); v += W * 32) {
      const int f = v / (DH / 4), d = v % (DH / 4) * 4;
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) m = fmaxf(m, s_ml[w * R + f].x);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float2 ml = s_ml[w * R + f];
        l += ml.x > -INFINITY ? ml.y * exp2_fast(ml.x - m) : ml.y;
        const float4 x = *reinterpret_cast<const float4*>(s_o + (w * R + f) * LDO + d);
        acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
      }
      if (whole) {
        const float inv = 1.0f / l;
        uint2 w;
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&w);
        h[0] = __floats2bfloat162_rn(acc.x * inv, acc.y * inv);
        h[1] = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2*>(p.out + (size_t)(t0 + f / G) * (p.hq * DH) + (head * G + f % G) * DH + d) = w;
      } else {
        *reinterpret_cast<float4*>(p.part_o + (slot * R + f) * DH + d) = acc;
        if (d == 0) p.part_ml[slot * R + f] = make_float2(m, l);
      }
    }
    }
  }
}

// Items that more than one worker held: out = sum_c 2^(m_c - m) o_c / sum_c 2^(m_c - m) l_c over the parts in order.
// One CTA per boundary between two shares; the boundaries inside an item divide its output, in units of four dims of a
// query row, between them.  The parts' weights are formed once per row; then a unit is one thread, or, where there are
// fewer units than threads, up to 32 neighbouring lanes, each with every so-manieth part.
constexpr int kMergeThreads = 256;
// Weights of one CTA: parts x the rows it touches.  With b boundaries inside an item of at most R rows it is at most
// (b + 1) (R / b + 2) <= 2 b + 2 R + 2, with b < 4 x 592 and R <= 16.
constexpr int kMergeWeights = 2 * kMaxStreamCtas * kStreamWarps + 34;
template <int DH>
__global__ void __launch_bounds__(kMergeThreads) k_attention_kv8_merge(const LineParams p, int R) {
  __shared__ float s_w[kMergeWeights];
  pdl_wait();
  pdl_trigger();
  Cut c;
  reinterpret_cast<int4*>(&c)[0] = __ldcg(reinterpret_cast<const int4*>(p.cuts + blockIdx.x));
  reinterpret_cast<int4*>(&c)[1] = __ldcg(reinterpret_cast<const int4*>(p.cuts + blockIdx.x) + 1);
  if (c.nrows == 0) return;
  const int parts = c.c1 - c.c0 + 1, cuts = parts - 1, nth = (int)blockIdx.x - c.c0 - 1;
  const int units = c.nrows * (DH / 4);
  const int v0 = (int)((long long)units * nth / cuts), v1 = (int)((long long)units * (nth + 1) / cuts);
  if (v0 >= v1) return;
  const int f0 = v0 / (DH / 4), f1 = (v1 - 1) / (DH / 4);
  const int G = p.hq / p.hkv, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // the first holder's part is in its odd slot unless it began with the item; everybody else began with it
  auto slot_of = [&](int k) { return (size_t)2 * (c.c0 + k) + (k == 0 && !c.even ? 1 : 0); };
  for (int f = f0 + warp; f <= f1; f += kMergeThreads / 32) {
    // the first 128 parts' references and sums in registers, all on their way at once
    constexpr int KEEP = 4;
    float2 ml[KEEP];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) {
      const int k = lane + 32 * i;
      ml[i] = k < parts ? __ldcg(p.part_ml + slot_of(k) * R + f) : make_float2(-INFINITY, 0.f);
    }
#pragma unroll
    for (int i = 0; i < KEEP; ++i) m = fmaxf(m, ml[i].x);
    for (int k = lane + 32 * KEEP; k < parts; k += 32) m = fmaxf(m, __ldcg(p.part_ml + slot_of(k) * R + f).x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    auto weight = [&](float ref) { return ref > -INFINITY ? exp2_fast(ref - m) : 1.f; };     // (no part: its sum is 0)
#pragma unroll
    for (int i = 0; i < KEEP; ++i) l += weight(ml[i].x) * ml[i].y;
    for (int k = lane + 32 * KEEP; k < parts; k += 32) {
      const float2 x = __ldcg(p.part_ml + slot_of(k) * R + f);
      l += weight(x.x) * x.y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    const float inv = 1.0f / l;
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
      if (lane + 32 * i < parts) s_w[(f - f0) * parts + lane + 32 * i] = weight(ml[i].x) * inv;
    for (int k = lane + 32 * KEEP; k < parts; k += 32)
      s_w[(f - f0) * parts + k] = weight(__ldcg(p.part_ml + slot_of(k) * R + f).x) * inv;
  }
  __syncthreads();
  auto store = [&](int v, const float4& x) {
    const int f = v / (DH / 4), d = v % (DH / 4) * 4;
    uint2 w;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&w);
    h[0] = __floats2bfloat162_rn(x.x, x.y);
    h[1] = __floats2bfloat162_rn(x.z, x.w);
    *reinterpret_cast<uint2*>(p.out + (size_t)(c.t0 + f / G) * (p.hq * DH) + (c.head * G + f % G) * DH + d) = w;
  };
  int lanes = 1;
  while (lanes < 32 && 2 * lanes <= parts && 2 * lanes * (v1 - v0) <= kMergeThreads) lanes *= 2;
  if (lanes == 1) {                        // four units of a thread at a time: their loads are independent
    for (int base = v0 + (int)threadIdx.x; base < v1; base += 4 * kMergeThreads) {
      float4 acc[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
      for (int k = 0; k < parts; ++k) {
        const float* from = p.part_o + slot_of(k) * R * DH;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int v = min(base + j * kMergeThreads, v1 - 1);
          const float4 x = __ldcg(reinterpret_cast<const float4*>(from + 4 * v));
          const float w = s_w[(v / (DH / 4) - f0) * parts + k];
          acc[j].x += w * x.x; acc[j].y += w * x.y; acc[j].z += w * x.z; acc[j].w += w * x.w;
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (base + j * kMergeThreads < v1) store(base + j * kMergeThreads, acc[j]);
    }
    return;
  }
  const int sub = threadIdx.x & (lanes - 1), v = v0 + (int)threadIdx.x / lanes, vc = min(v, v1 - 1);   // v1 - v0 <= 256 / lanes
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = sub; k < parts; k += lanes) {
    const float4 x = __ldcg(reinterpret_cast<const float4*>(p.part_o + slot_of(k) * R * DH + 4 * vc));
    const float w = s_w[(vc / (DH / 4) - f0) * parts + k];
    acc.x += w * x.x; acc.y += w * x.y; acc.z += w * x.z; acc.w += w * x.w;
  }
  for (int o = 1; o < lanes; o <<= 1) {
    acc.x += __shfl_xor_sync(0xffffffffu, acc.x, o);
    acc.y += __shfl_xor_sync(0xffffffffu, acc.y, o);
    acc.z += __shfl_xor_sync(0xffffffffu, acc.z, o);
    acc.w += __shfl_xor_sync(0xffffffffu, acc.w, o);
  }
  if (sub == 0 && v < v1) store(v, acc);
}

constexpr size_t kCutBytes = (size_t)kMaxStreamCtas * kStreamWarps * sizeof(Cut);
// Query rows of all partial slots, two slots per worker: 592 CTAs of four single-warp workers with 16 rows.  A launch takes
// no more CTAs than these hold.
constexpr size_t kPartRows = 2 * (size_t)kStreamWarps * kMaxStreamCtas * 16;

// Per device: how many CTAs of each instantiation one wave holds (0: not asked yet).
struct DeviceInfo { int wave[16]; };
DeviceInfo g_dev[kMaxDevices];
std::mutex g_mutex;

template <int DH, int NQ, int STAGES, int W, int MINB, bool DIRECT>
cudaError_t run_as(const LineParams& p, cudaStream_t s) {
  constexpr int index = (DH == 128 ? 4 : 0) + (NQ - 1) * 2 + (W == 1 ? 1 : 0) + (DIRECT ? 8 : 0);
  constexpr auto kernel = k_attention_kv8_stream<DH, NQ, STAGES, W, MINB, DIRECT>;
  constexpr int smem = StreamSmem<DH, NQ, STAGES, W>::total;
  DeviceInfo* d = device_slot(g_dev);
  if (!d) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(g_mutex);
    if (!d->wave[index]) {
      int dev = 0, sms = 0, per = 0;
      cudaError_t r = cudaGetDevice(&dev);
      if (r == cudaSuccess) r = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
      if (r == cudaSuccess) r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (r == cudaSuccess) r = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, kStreamThreads, smem);
      if (r != cudaSuccess) return r;
      if (sms < 1 || per < 1) return cudaErrorInvalidDevice;
      d->wave[index] = std::min(std::min(sms * per, kMaxStreamCtas), (int)(kPartRows / (2 * 8 * NQ * (kStreamWarps / W))));
    }
  }
  if constexpr (DIRECT) {
    const long long ctas = ((long long)p.n_rows * p.hkv * p.direct + kStreamWarps / W - 1) / (kStreamWarps / W);
    if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
    return launch_pdl(kernel, dim3((unsigned)ctas), dim3(kStreamThreads), (size_t)smem, s, p);
  }
  cudaError_t r = launch_pdl(kernel, dim3(d->wave[index]), dim3(kStreamThreads), (size_t)smem, s, p);
  if (r != cudaSuccess) return r;
  return launch_pdl(k_attention_kv8_merge<DH>, dim3(d->wave[index] * (kStreamWarps / W)), dim3(kMergeThreads), 0, s, p, 8 * NQ);
}

template <int DH, int NQ, int STAGES, int W, int MINB>
cudaError_t run_stream(const LineParams& p, cudaStream_t s) {
  return p.direct ? run_as<DH, NQ, STAGES, W, MINB, true>(p, s) : run_as<DH, NQ, STAGES, W, MINB, false>(p, s);
}

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }


}  // namespace

// Scratch: the streaming kernel's cuts, partial outputs and sums; the tensor-core kernel uses the same bytes for its chunks.
size_t attention_kv8_scratch_bytes(int hq, int hkv, int dh) {
  (void)hq; (void)hkv;
  return up256(kCutBytes) + up256(kPartRows * dh * sizeof(float)) + up256(kPartRows * sizeof(float2));
}

namespace {

// The way of a call, from the sizes that the host knows.
struct Route {
  bool tensor, many;     // the tensor-core kernel; single-warp workers
  int nq, tq, direct;    // query tiles of 8 rows and query tokens per item; as in LineParams
};
Route route_of(int n_rows, int M, int hint_nq, int max_vis, int hq, int hkv, int dh) {
  Route w = {};
  const int G = hq / hkv;
  const int max_nq = hint_nq > 0 ? std::min(hint_nq, M) : M;
  const long long widest = (long long)max_nq * G;
  // Beyond 48 (head_dim 64: 96) query rows per kv head the 128-row tensor-core tiles pay (16 rows of 320 to 800 keys, 7
  // heads a group: 35 query rows 16.5 us, 14.6 by the streaming kernel, 49 16.8 and 16.2, 112 17.6 and 23.3; 32 heads: 48 query
  // rows 56 and 52, 64 57 and 66; head_dim 64: 96 query rows 14.5 and 12.8, 128 14.6 and 16.8).  The streaming kernel's tiles
  // hold a token's group of up to 16 heads.
  // Rows of up to 96 keys do not fill a key tile and are streamed whatever the width (16 rows x 32 tokens, 7 heads a group: 43
  // keys 8.4 us, tcgen05 10.8, 100 keys 11.3 and 10.8; 200 rows: 64 keys 81 and 102, 96 keys 90 and 102, 128 keys 103 and 99).
  const bool brief = max_vis > 0 && max_vis <= 96;
  w.tensor = G > 16 || (!brief && widest > (dh == 128 ? 48 : 96));
  if (w.tensor) return w;
  // 8 or 16 query rows per item.  (32, which reads a block once for all of a 32-token step, leaves two warps per scheduler
  // with 255 registers: a fifth slower on 20 rows x 32 tokens of 32 heads, no faster on 64 rows when it was tried.)
  w.nq = widest <= 8 ? 1 : 2;
  w.tq = 8 * w.nq / G;
  // Workers per (row, kv head), when every item has one: the tiles of the largest row.  A worker goes on to the next tile of
  // its row, so fewer do as well, and those that the tokens cannot fill are launched for nothing: without a hint one more than
  // the rows' mean (512 rows x 1 to 16 tokens of 32 heads over up to 64 keys: 2344 us by the largest row there could be, 94
  // by the mean, 66 with the hint), with one at most eight times as many as there can be items (a hint of M: 236 us).
  const long long filled = (long long)M / w.tq + n_rows;           // tiles of one kv head, at most
  const long long cap = hint_nq > 0 ? 8 * filled / n_rows : ((long long)M / n_rows + w.tq - 1) / w.tq + 1;
  const int tiles = (int)std::min<long long>((max_nq + w.tq - 1) / w.tq, cap);
  // Single-warp workers where there are many items and two query tiles make each of them work for a warp.  64 rows x 32
  // tokens, 32 heads, 4096 items: 200 to 512 keys 86 us (102 with four-warp workers), 96 to 1024 118 us (125); 1280 items: 96
  // to 500 keys 31 us (33), but 500 to 3000 110 us (98); 768 items of 96 to 500 keys 28 us (23).
  const long long items = (long long)n_rows * hkv * tiles;
  w.many = w.nq > 1 && items >= (max_vis > 0 && max_vis <= 512 ? 6 : 16) * 148;
  // Short rows have a worker per item and nothing to merge; so do rows of some length where there are about as many items
  // as workers fit the machine.  Four-warp workers, 4 items a row: 2 rows of up to 500 keys 7.1 us, 11.7 by the line; 1100 8.9
  // and 11.5; 2000 15.8 and 11.8; 15,778 68 and 14; 30 rows of up to 2000 18.0 and 18.0; 4000 29 and 24; 110 rows of up to
  // 2000 33 and 34; 4000 58 and 54.  Single-warp workers: 4096 items of up to 512 keys 86 us, 92 by the line; of up to 1024
  // 124 and 118.
  const int reach = w.many ? 512 : items >= 400 ? 4096 : 2048;
  w.direct = max_vis > 0 && max_vis <= reach ? tiles : 0;
  return w;
}

}  // namespace

bool attention_kv8_uses_scratch(int n_rows, int M, int max_nq, int max_vis, int hq, int hkv, int dh) {
  const Route w = route_of(n_rows, M, max_nq, max_vis, hq, hkv, dh);
  return w.tensor ? max_vis > (kAttnKv8CutTiles - 1) * 128 : w.direct == 0;
}

cudaError_t launch_attention_kv8(const AttnKv8Args& a, cudaStream_t s) {
  if (a.M <= 0 || a.n_rows <= 0) return cudaSuccess;
  const Route w = route_of(a.n_rows, a.M, a.max_nq, a.max_vis, a.hq, a.hkv, a.dh);
  if (w.tensor) return launch_attention_kv8_tc(a, static_cast<float*>(a.scratch), a.scratch_bytes / sizeof(float), s);
  LineParams p;
  p.q = a.q; p.q_ld = a.q_ld; p.c = a.cache; p.out = a.out;
  p.cu_q = a.cu_q; p.kv_base = a.kv_base; p.vis = a.vis;
  p.n_rows = a.n_rows; p.M = a.M; p.hq = a.hq; p.hkv = a.hkv;
  p.tq = w.tq;
  p.direct = w.direct;
  p.error_flag = a.error_flag;
  char* at = static_cast<char*>(a.scratch);              // (a worker per item uses none)
  p.cuts = reinterpret_cast<Cut*>(at);
  p.part_o = nullptr;
  p.part_ml = nullptr;
  if (at) {
    at += up256(kCutBytes);
    p.part_o = reinterpret_cast<float*>(at);
    at += up256(kPartRows * a.dh * sizeof(float));
    p.part_ml = reinterpret_cast<float2*>(at);
  }
  const int nq = w.nq;
  const bool many = w.many;
  // Stages and CTAs per SM.  One query tile, head_dim 128: three stages on two CTAs, 64 rows of 1000 to 4000 keys 36.8 us
  // (two on three 38.0); head_dim 64: two on three, 60 rows of 1000 to 8000 keys, 8 heads, 49 us (three on three 59).  Two query
  // tiles, head_dim 128, four-warp: two on three, 200 rows x 2 tokens 36 us (three on two 43); single-warp: two on two, 64
  // rows x 32 tokens 119 us (two on three, which spills, 127).
  if (a.dh == 128) {
    if (nq == 1) return run_stream<128, 1, 3, 4, 2>(p, s);
    return many ? run_stream<128, 2, 2, 1, 2>(p, s) : run_stream<128, 2, 2, 4, 3>(p, s);
  }
  if (nq == 1) return run_stream<64, 1, 2, 4, 3>(p, s);
  return many ? run_stream<64, 2, 2, 1, 3>(p, s) : run_stream<64, 2, 2, 4, 3>(p, s);
}

}  // namespace bs
