// Ragged attention over the 8-bit KV cache (layout in kv8.cuh): every query token of row i attends to cache rows
// [kv_base_i, kv_base_i + vis_i); no causal or padding mask; rows with vis_i = 0 give zeros.
//
//   s_j = q . k_j / sqrt(dh),   out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m)
//
// with k_j = ks_b c_j and v_j = vs_b c'_j for the codes c, c' and the two scales of cache block b.  The codes go to the
// tensor cores as fp16 (exact: e4m3 needs 4 significant bits and 2^-9 .. 448); ks_b multiplies the finished fp32 scores
// and vs_b the output accumulator, so no scale is ever rounded into an operand.  Queries become fp16 after a power of
// two per query row has brought their largest element into [1, 2): bf16's 8 bits fit fp16's 11, what drops below 2^-24
// of the row's largest element is far below the fp32 sum's own rounding.
#include <math.h>

#include <algorithm>
#include <mutex>

#include "kv8.cuh"
#include "tc_common.cuh"

namespace bs {

namespace {

__device__ __forceinline__ void mma_f16(float* c, const uint4& a, unsigned b0, unsigned b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ unsigned pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const unsigned*>(&h);
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint4 load_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load_stream2(const void* p) {
  uint2 v;
  asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

// ---- streaming kernel ---------------------------------------------------------------------------------------
//
// Few query rows per kv head (single tokens, block steps without grouped heads): bound by the bytes of the cache.
// A work item is (row, kv head, tile of 16 MT flattened (token, head-in-group) query rows); its cost is the row's
// number of cache blocks.  All items' blocks form one line, which the CTAs of a single resident wave share evenly:
// CTA c takes blocks [c T / G, (c + 1) T / G), whatever the rows' lengths are.  An item that a CTA holds whole is
// written out directly; a cut one leaves partial (output, maximum, sum) parts, at most two per CTA, that a second small
// kernel merges in order.
//
// Inside a CTA every warp takes whole cache blocks (32 keys) on its own, straight from global memory into registers:
// the order of the dims in the scores' k index and of the dims in the output's n index is free, and is chosen so that
// a lane's 16-byte loads are its mma.sync operand registers - no shared memory, no barrier, no shuffle of K or V.
constexpr int kStreamWarps = 4;
constexpr int kStreamThreads = kStreamWarps * 32;
constexpr int kMaxStreamCtas = 512;
// Probabilities are formed against a reference kBias below the running maximum (log2 units), which is moved only when
// the maximum has grown kGrow above it: they stay below 2^kGrow in fp16 and keep full precision down to 2^-20 of the
// largest one.
constexpr float kBias = 6.f, kGrow = 14.f;

struct StreamParams {
  const bf16* q;
  int q_ld;
  Kv8Cache c;
  bf16* out;
  const int* cu_q;
  const int* kv_base;
  const int* vis;
  int n_rows, M, hq, hkv, tq;
  long long* prefix;     // scratch: [n_rows + 1] blocks before each row, then the number of CTAs that share them
  float* part_o;         // scratch: [2 CTAs][16 MT][DH]
  float2* part_ml;       // scratch: [2 CTAs][16 MT]
  int* error_flag;
};

struct RowInfo { int t0, n, vis, nb, tiles; long long base; };

__device__ __forceinline__ bool row_info(const int* cu_q, const int* kv_base, const int* vis, long long n_blocks, int M,
                                         int tq, int r, RowInfo& w) {
  w.t0 = __ldg(cu_q + r);
  const int t1 = __ldg(cu_q + r + 1);
  w.n = t1 - w.t0;
  w.vis = __ldg(vis + r);
  const int base = __ldg(kv_base + r);
  w.base = (long long)base / kKv8Block;
  const bool ok = w.t0 >= 0 && w.n >= 0 && t1 <= M && w.vis >= 0 && base >= 0 && base % kKv8Block == 0 &&
                  (long long)base + w.vis <= n_blocks * kKv8Block;
  if (!ok) w.n = w.vis = 0;
  w.nb = (w.vis + kKv8Block - 1) / kKv8Block;
  w.tiles = (w.n + tq - 1) / tq;
  return ok;
}

// First block of CTA c's share, and the CTA that holds block u.
__device__ __forceinline__ long long share_start(long long c, long long total, long long ctas) { return c * total / ctas; }
__device__ __forceinline__ int share_of(long long u, long long total, long long ctas) { return (int)(((u + 1) * ctas - 1) / total); }

template <int DH, int MT>
constexpr int stream_smem() {
  return MT * (DH / 16) * 32 * 16 +                                   // query fragments
         kStreamWarps / 2 * 16 * MT * (DH + 4) * 4 +                  // outputs of half the warps
         kStreamWarps * 16 * MT * 8 + 16 * MT * 4 +                   // (reference, sum) per warp and row; query scales
         (kAttnKv8MaxRows + 1) * 8;                                   // prefix
}

template <int DH, int MT>
__global__ void __launch_bounds__(kStreamThreads, 2) k_attention_kv8_stream(StreamParams p) {
  constexpr int KS = DH / 16;            // k steps of the scores = 32-bit words of K per lane and key
  constexpr int NT = DH / 8;             // n tiles of the output
  constexpr int R = 16 * MT;
  constexpr int LDO = DH + 4;
  extern __shared__ __align__(16) unsigned char smem[];
  uint4* s_q = reinterpret_cast<uint4*>(smem);                               // [MT][KS][32]
  float* s_o = reinterpret_cast<float*>(s_q + MT * KS * 32);                 // [warps / 2][R][LDO]
  float2* s_ml = reinterpret_cast<float2*>(s_o + kStreamWarps / 2 * R * LDO);   // [warps][R]
  float* s_sc = reinterpret_cast<float*>(s_ml + kStreamWarps * R);           // [R]
  long long* s_pre = reinterpret_cast<long long*>(s_sc + R);                 // [n_rows + 1]
  __shared__ long long s_warp[kStreamWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, c4 = lane & 3;
  const int G = p.hq / p.hkv;
  pdl_wait();
  pdl_trigger();

  // ---- blocks before every row (exclusive prefix) ----
  long long total = 0;
  for (int base = 0; base < p.n_rows; base += kStreamThreads) {
    const int r = base + tid;
    long long w = 0;
    if (r < p.n_rows) {
      RowInfo ri;
      if (!row_info(p.cu_q, p.kv_base, p.vis, p.c.n_blocks, p.M, p.tq, r, ri) && blockIdx.x == 0 && p.error_flag)
        atomicMax(p.error_flag, 100 + SITE_ATTN_KV8);
      w = (long long)ri.tiles * p.hkv * ri.nb;
    }
    long long inc = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    long long before = total;
    for (int k = 0; k < kStreamWarps; ++k) {
      if (k < warp) before += s_warp[k];
      total += s_warp[k];
    }
    if (r < p.n_rows) s_pre[r] = before + inc - w;
    __syncthreads();
  }
  if (tid == 0) s_pre[p.n_rows] = total;
  __syncthreads();
  // a share of fewer blocks than warps would leave warps idle
  const long long ctas = max(1ll, min((long long)gridDim.x, (total + kStreamWarps - 1) / kStreamWarps));
  if (blockIdx.x == 0) {
    for (int r = tid; r <= p.n_rows; r += kStreamThreads) p.prefix[r] = s_pre[r];
    if (tid == 0) p.prefix[p.n_rows + 1] = ctas;
  }
  if (total == 0 || (long long)blockIdx.x >= ctas) return;
  const long long u0 = share_start(blockIdx.x, total, ctas), u1 = share_start((long long)blockIdx.x + 1, total, ctas);

  int row = 0;
  {   // the row that holds block u0: the last one whose prefix is <= u0 (rows without blocks share a prefix with the next)
    int lo = 0, hi = p.n_rows;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_pre[mid] <= u0) lo = mid; else hi = mid;
    }
    row = lo;
  }

  for (long long u = u0; u < u1;) {
    while (s_pre[row + 1] <= u) ++row;
    RowInfo ri;
    row_info(p.cu_q, p.kv_base, p.vis, p.c.n_blocks, p.M, p.tq, row, ri);
    const long long local = u - s_pre[row];
    const int item = (int)(local / ri.nb), b0 = (int)(local % ri.nb);
    const int head = item / ri.tiles, tile = item % ri.tiles;
    const int b1 = (int)min((long long)ri.nb, b0 + (u1 - u));
    const int t0 = ri.t0 + tile * p.tq, nt = min(p.tq, ri.t0 + ri.n - t0), nrows = nt * G;

    // ---- queries: fp16 fragments in shared memory ----
    __syncthreads();                     // the previous segment's fragments and sums are no longer read
    for (int mt = warp; mt < MT; mt += kStreamWarps) {
      uint2 raw[2][KS];
      float top[2] = {0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int f = mt * 16 + g + 8 * x;
        const bool valid = f < nrows;
        const bf16* src = p.q + (size_t)(t0 + (valid ? f / G : 0)) * p.q_ld + (head * G + (valid ? f % G : 0)) * DH;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          // k step k of lane c4 stands for dims (k / 4) 64 + 16 c4 + 4 (k % 4) ..+ 3
          raw[x][k] = valid ? *reinterpret_cast<const uint2*>(src + (k >> 2) * 64 + c4 * 16 + (k & 3) * 4) : make_uint2(0, 0);
          const float2 a = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&raw[x][k].x));
          const float2 b = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&raw[x][k].y));
          top[x] = fmaxf(fmaxf(top[x], fmaxf(fabsf(a.x), fabsf(a.y))), fmaxf(fabsf(b.x), fabsf(b.y)));
        }
        top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 1));
        top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 2));
      }
      float inv[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int e = min(max((int)(__float_as_uint(top[x]) >> 23) - 127, -100), 100);
        inv[x] = pow2i(-e);
        if (c4 == 0) s_sc[mt * 16 + g + 8 * x] = pow2i(e) * (1.4426950408889634f * rsqrtf((float)DH));
      }
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        unsigned w[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float2 a = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&raw[x][k].x));
          const float2 b = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&raw[x][k].y));
          w[x][0] = pack_f16(a.x * inv[x], a.y * inv[x]);
          w[x][1] = pack_f16(b.x * inv[x], b.y * inv[x]);
        }
        s_q[(mt * KS + k) * 32 + lane] = make_uint4(w[0][0], w[1][0], w[0][1], w[1][1]);
      }
    }
    __syncthreads();

    float o[MT][NT][4];
    float ref[MT][2], sum[MT][2], sc[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int i = 0; i < NT; ++i) o[mt][i][0] = o[mt][i][1] = o[mt][i][2] = o[mt][i][3] = 0.f;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        ref[mt][x] = -INFINITY;
        sum[mt][x] = 0.f;
        sc[mt][x] = s_sc[mt * 16 + g + 8 * x];
      }
    }
    float vs_cur = 1.f;                  // the accumulator is in units of this V scale

    for (int b = b0 + warp; b < b1; b += kStreamWarps) {
      const size_t tile_at = (size_t)(ri.base + b) * p.hkv + head;
      const unsigned char* kt = p.c.k + tile_at * (kKv8Block * DH);
      const unsigned char* vt = p.c.v + tile_at * (kKv8Block * DH);
      const float ks = kv8_clamp_scale(__ldg(p.c.k_scale + tile_at));
      const float vs = kv8_clamp_scale(__ldg(p.c.v_scale + tile_at));
      unsigned kr[4][KS];                // [key group of 8][word]
#pragma unroll
      for (int n = 0; n < 4; ++n) {
#pragma unroll
        for (int h = 0; h < KS / 4; ++h) {
          const uint4 v = load_stream(kt + (n * 8 + g) * DH + h * 64 + c4 * 16);
          kr[n][h * 4] = v.x; kr[n][h * 4 + 1] = v.y; kr[n][h * 4 + 2] = v.z; kr[n][h * 4 + 3] = v.w;
        }
      }
      unsigned vr[2][4][NT / 4];         // [16 keys][key 2c, 2c+1, 2c+8, 2c+9][word]: dims g NT ..
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned char* src = vt + (n * 16 + 2 * c4 + (j & 1) + (j >> 1) * 8) * DH + g * NT;
          if (NT == 16) {
            const uint4 v = load_stream(src);
            vr[n][j][0] = v.x; vr[n][j][1] = v.y;
            vr[n][j][NT / 4 - 2] = v.z; vr[n][j][NT / 4 - 1] = v.w;
          } else {
            const uint2 v = load_stream2(src);
            vr[n][j][0] = v.x; vr[n][j][1] = v.y;
          }
        }
      float s[MT][4][4];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int n = 0; n < 4; ++n) s[mt][n][0] = s[mt][n][1] = s[mt][n][2] = s[mt][n][3] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint4 a[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) a[mt] = s_q[(mt * KS + k) * 32 + lane];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          unsigned x0, x1;
          kv8_decode4(kr[n][k], x0, x1);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) mma_f16(s[mt][n], a[mt], x0, x1);
        }
      }
      const int left = ri.vis - b * kKv8Block;         // keys of this block that the row sees (> 0)
      unsigned pr[MT][4][2];                           // probabilities as A fragments
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const float f = sc[mt][x] * ks;
#pragma unroll
          for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float& v = s[mt][n][2 * x + j];
              v = n * 8 + 2 * c4 + j < left ? v * f : -INFINITY;
              mx[x] = fmaxf(mx[x], v);
            }
          mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 1));
          mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 2));
        }
        const bool grow0 = mx[0] > ref[mt][0] + kGrow, grow1 = mx[1] > ref[mt][1] + kGrow;
        if (__any_sync(0xffffffffu, grow0 || grow1 || vs != vs_cur)) {
          const float turn = vs_cur / vs;              // exact: both are powers of two
          float f0 = 1.f, f1 = 1.f;
          if (grow0) { f0 = exp2_fast(ref[mt][0] - (mx[0] - kBias)); ref[mt][0] = mx[0] - kBias; }
          if (grow1) { f1 = exp2_fast(ref[mt][1] - (mx[1] - kBias)); ref[mt][1] = mx[1] - kBias; }
          sum[mt][0] *= f0;
          sum[mt][1] *= f1;
          f0 *= turn;
          f1 *= turn;
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            o[mt][i][0] *= f0; o[mt][i][1] *= f0;
            o[mt][i][2] *= f1; o[mt][i][3] *= f1;
          }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float e0 = exp2_fast(s[mt][n][2 * x] - ref[mt][x]), e1 = exp2_fast(s[mt][n][2 * x + 1] - ref[mt][x]);
            sum[mt][x] += e0 + e1;
            pr[mt][n][x] = pack_f16(e0, e1);
          }
        }
      }
      vs_cur = vs;
      if (left < kKv8Block) {                          // codes behind the row's end may be anything: none of them counts
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (n * 16 + 2 * c4 + (j & 1) + (j >> 1) * 8 >= left) {
#pragma unroll
              for (int w = 0; w < NT / 4; ++w) vr[n][j][w] = 0u;
            }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) {
#pragma unroll
        for (int w = 0; w < NT / 4; ++w) {
          // bytes of two keys side by side: (key 2c, key 2c + 1) for each of four dims
          unsigned b0w[4], b1w[4];
          kv8_decode4(__byte_perm(vr[n][0][w], vr[n][1][w], 0x5140), b0w[0], b0w[1]);
          kv8_decode4(__byte_perm(vr[n][0][w], vr[n][1][w], 0x7362), b0w[2], b0w[3]);
          kv8_decode4(__byte_perm(vr[n][2][w], vr[n][3][w], 0x5140), b1w[0], b1w[1]);
          kv8_decode4(__byte_perm(vr[n][2][w], vr[n][3][w], 0x7362), b1w[2], b1w[3]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
              mma_f16(o[mt][w * 4 + i],
                      make_uint4(pr[mt][2 * n][0], pr[mt][2 * n][1], pr[mt][2 * n + 1][0], pr[mt][2 * n + 1][1]),
                      b0w[i], b1w[i]);
        }
      }
    }

    // ---- the warps' parts of this segment become one: (reference, sum) of every warp, then the outputs in two steps ----
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float l = sum[mt][x];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        sum[mt][x] = l;
        if (c4 == 0) s_ml[warp * R + mt * 16 + g + 8 * x] = make_float2(ref[mt][x], l);
      }
    __syncthreads();
    float m_all[MT][2], l_all[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int f = mt * 16 + g + 8 * x;
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < kStreamWarps; ++w) m = fmaxf(m, s_ml[w * R + f].x);
#pragma unroll
        for (int w = 0; w < kStreamWarps; ++w) {
          const float2 v = s_ml[w * R + f];
          if (v.x > -INFINITY) l += v.y * exp2_fast(v.x - m);
        }
        m_all[mt][x] = m;
        l_all[mt][x] = l;
        const float f2 = ref[mt][x] > -INFINITY ? exp2_fast(ref[mt][x] - m) * vs_cur : 0.f;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          o[mt][i][2 * x] *= f2;
          o[mt][i][2 * x + 1] *= f2;
        }
      }
#pragma unroll
    for (int half = kStreamWarps / 2; half > 0; half >>= 1) {
      // lane (g, c4) holds dims [2 c4 NT, 2 c4 NT + NT) in component 0 and the NT after them in component 1
      if (warp >= half && warp < 2 * half) {
        float* dst = s_o + (warp - half) * R * LDO;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
              for (int i = 0; i < NT; i += 4)
                *reinterpret_cast<float4*>(dst + (mt * 16 + g + 8 * x) * LDO + (2 * c4 + y) * NT + i) =
                    make_float4(o[mt][i][2 * x + y], o[mt][i + 1][2 * x + y], o[mt][i + 2][2 * x + y], o[mt][i + 3][2 * x + y]);
      }
      __syncthreads();
      if (warp < half) {
        const float* src = s_o + warp * R * LDO;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
              for (int i = 0; i < NT; i += 4) {
                const float4 v = *reinterpret_cast<const float4*>(src + (mt * 16 + g + 8 * x) * LDO + (2 * c4 + y) * NT + i);
                o[mt][i][2 * x + y] += v.x; o[mt][i + 1][2 * x + y] += v.y;
                o[mt][i + 2][2 * x + y] += v.z; o[mt][i + 3][2 * x + y] += v.w;
              }
      }
      if (half > 1) __syncthreads();
    }
    if (warp == 0) {
      const bool whole = b0 == 0 && b1 == ri.nb;
      const size_t slot = 2 * (size_t)blockIdx.x + (u > u0 ? 1 : 0);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int f = mt * 16 + g + 8 * x;
          if (f >= nrows) continue;
          if (whole) {
            const float inv = 1.0f / l_all[mt][x];
            bf16* dst = p.out + (size_t)(t0 + f / G) * (p.hq * DH) + (head * G + f % G) * DH + 2 * c4 * NT;
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
              for (int i = 0; i < NT; i += 8) {
                uint4 w;
                __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&w);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                  h[j] = __floats2bfloat162_rn(o[mt][i + 2 * j][2 * x + y] * inv, o[mt][i + 2 * j + 1][2 * x + y] * inv);
                *reinterpret_cast<uint4*>(dst + y * NT + i) = w;
              }
          } else {
            float* dst = p.part_o + (slot * R + f) * DH + 2 * c4 * NT;
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
              for (int i = 0; i < NT; i += 4)
                *reinterpret_cast<float4*>(dst + y * NT + i) =
                    make_float4(o[mt][i][2 * x + y], o[mt][i + 1][2 * x + y], o[mt][i + 2][2 * x + y], o[mt][i + 3][2 * x + y]);
            if (c4 == 0) p.part_ml[slot * R + f] = make_float2(m_all[mt][x], l_all[mt][x]);
          }
        }
    }
    u += b1 - b0;
  }
}

// Items that more than one CTA held: out = sum_c 2^(m_c - m) o_c / sum_c 2^(m_c - m) l_c over the parts in order.
// Rows that see nothing (vis = 0): zeros.  One CTA per (query tile slot, kv head), one warp per query row in turn.
template <int DH>
__global__ void __launch_bounds__(256) k_attention_kv8_merge(StreamParams p, int R) {
  constexpr int V = DH / 32;
  pdl_wait();
  pdl_trigger();
  const int slot = (int)blockIdx.x, head = blockIdx.y;
  const int row = warp_search(p.n_rows, slot, [&](int i) { return __ldg(p.cu_q + i) / p.tq + i; });
  RowInfo ri;
  row_info(p.cu_q, p.kv_base, p.vis, p.c.n_blocks, p.M, p.tq, row, ri);
  const int tile = slot - (__ldg(p.cu_q + row) / p.tq + row);
  if (tile < 0 || tile >= ri.tiles) return;
  const int G = p.hq / p.hkv, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t0 = ri.t0 + tile * p.tq, nrows = min(p.tq, ri.t0 + ri.n - t0) * G;
  const long long total = p.prefix[p.n_rows], ctas = p.prefix[p.n_rows + 1];
  const long long first = p.prefix[row] + ((long long)head * ri.tiles + tile) * ri.nb;
  int c0 = 0, c1 = -1;
  if (ri.nb > 0) {
    c0 = share_of(first, total, ctas);
    c1 = share_of(first + ri.nb - 1, total, ctas);
    if (c0 == c1) return;                  // held whole by one CTA, which wrote it
  }
  for (int f = warp + 8 * blockIdx.z; f < nrows; f += 8 * gridDim.z) {
    float acc[V];
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0.f;
    float m = -INFINITY, l = 0.f;
    for (int c = c0; c <= c1; c += 4) {
      float2 ml[4];
      float v[4][V];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int cc = min(c + k, c1);
        const size_t at = ((size_t)2 * cc + (first > share_start(cc, total, ctas) ? 1 : 0)) * R + f;
        ml[k] = p.part_ml[at];
        if (c + k > c1) ml[k] = make_float2(-INFINITY, 0.f);
        const float* src = p.part_o + at * DH + lane * V;
        if (V == 4) {
          const float4 w = *reinterpret_cast<const float4*>(src);
          v[k][0] = w.x; v[k][1] = w.y; v[k][V - 2] = w.z; v[k][V - 1] = w.w;
        } else {
          const float2 w = *reinterpret_cast<const float2*>(src);
          v[k][0] = w.x; v[k][1] = w.y;
        }
      }
      float nm = m;
#pragma unroll
      for (int k = 0; k < 4; ++k) nm = fmaxf(nm, ml[k].x);
      const float f0 = m > -INFINITY ? exp2_fast(m - nm) : 0.f;
      l *= f0;
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] *= f0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (c + k > c1) continue;
        const float w = ml[k].x > -INFINITY ? exp2_fast(ml[k].x - nm) : 1.f;   // (NaN sums stay NaN)
        l += w * ml[k].y;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += w * v[k][j];
      }
      m = nm;
    }
    const float inv = ri.nb > 0 ? 1.0f / l : 0.f;
    bf16* dst = p.out + (size_t)(t0 + f / G) * (p.hq * DH) + (head * G + f % G) * DH + lane * V;
#pragma unroll
    for (int j = 0; j < V; j += 2)
      *reinterpret_cast<__nv_bfloat162*>(dst + j) = __floats2bfloat162_rn(acc[j] * inv, acc[j + 1] * inv);
  }
}

// Per device: how many CTAs of each instantiation one wave holds (0: not asked yet).
struct DeviceInfo { int wave[4]; };
DeviceInfo g_dev[kMaxDevices];
std::mutex g_mutex;

template <int DH, int MT>
cudaError_t prepare_stream(int* wave) {
  int dev = 0, sms = 0, per = 0;
  cudaError_t r = cudaGetDevice(&dev);
  if (r == cudaSuccess) r = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (r == cudaSuccess)
    r = cudaFuncSetAttribute(k_attention_kv8_stream<DH, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, stream_smem<DH, MT>());
  if (r == cudaSuccess)
    r = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, k_attention_kv8_stream<DH, MT>, kStreamThreads, stream_smem<DH, MT>());
  if (r != cudaSuccess) return r;
  if (sms < 1 || per < 1) return cudaErrorInvalidDevice;
  *wave = std::min(sms * per, kMaxStreamCtas);
  return cudaSuccess;
}

template <int DH, int MT>
cudaError_t run_stream(StreamParams p, int index, cudaStream_t s) {
  DeviceInfo* d = device_slot(g_dev);
  if (!d) return cudaErrorInvalidDevice;
  {
    std::lock_guard<std::mutex> lock(g_mutex);
    if (!d->wave[index])
      if (cudaError_t r = prepare_stream<DH, MT>(&d->wave[index])) return r;
  }
  cudaError_t r = launch_pdl(k_attention_kv8_stream<DH, MT>, dim3(d->wave[index]), dim3(kStreamThreads),
                             (size_t)stream_smem<DH, MT>(), s, p);
  if (r != cudaSuccess) return r;
  const long long slots = (long long)p.M / p.tq + p.n_rows;
  return launch_pdl(k_attention_kv8_merge<DH>, dim3((unsigned)slots, p.hkv), dim3(256), 0, s, p, 16 * MT);
}

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t attention_kv8_scratch_bytes(int hq, int hkv, int dh) {
  (void)hq; (void)hkv;
  const size_t rows = (size_t)2 * kMaxStreamCtas * 32;
  return up256((kAttnKv8MaxRows + 2) * sizeof(long long)) + up256(rows * dh * sizeof(float)) + up256(rows * sizeof(float2));
}

cudaError_t launch_attention_kv8(const AttnKv8Args& a, cudaStream_t s) {
  if (a.M <= 0 || a.n_rows <= 0) return cudaSuccess;
  const int G = a.hq / a.hkv;
  const long long widest = (long long)(a.max_nq > 0 ? a.max_nq : a.M) * G;
  const int mt = widest <= 16 ? 1 : 2;
  StreamParams p;
  p.q = a.q; p.q_ld = a.q_ld; p.c = a.cache; p.out = a.out;
  p.cu_q = a.cu_q; p.kv_base = a.kv_base; p.vis = a.vis;
  p.n_rows = a.n_rows; p.M = a.M; p.hq = a.hq; p.hkv = a.hkv; p.tq = 16 * mt / G;
  p.error_flag = a.error_flag;
  char* at = static_cast<char*>(a.scratch);
  p.prefix = reinterpret_cast<long long*>(at);
  at += up256((kAttnKv8MaxRows + 2) * sizeof(long long));
  p.part_o = reinterpret_cast<float*>(at);
  at += up256((size_t)2 * kMaxStreamCtas * 32 * a.dh * sizeof(float));
  p.part_ml = reinterpret_cast<float2*>(at);
  if (a.dh == 128) return mt == 1 ? run_stream<128, 1>(p, 0, s) : run_stream<128, 2>(p, 1, s);
  return mt == 1 ? run_stream<64, 1>(p, 2, s) : run_stream<64, 2>(p, 3, s);
}

}  // namespace bs
