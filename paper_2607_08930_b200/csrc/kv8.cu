// Norms of every query / key head with the rotation and the cache write in one pass (bf16 or 8-bit cache), and the way
// from the 8-bit cache back to bf16.
//
//   y = gain * x / sqrt(mean(x^2) + eps) over a head's dims; (y_j, y_{j + dh/2}) turned by the token's angle
//
// All three are bound by memory: every element of qkv is read once and its result written once.  dh / 16 lanes own one
// head of one token, 8 dims of its first half and the 8 they are turned with: the rotation stays inside a lane, the
// norm's sum moves by shuffles inside those lanes, everything between the load and the one rounding at the end is fp32.
//
// Measured against a copy's 6.5 TB/s: norms and rotation into the bf16 cache, 16 rows of 320 to 1024 tokens (28 / 4 heads,
// head_dim 128, 191 MB) 35.6 us, 5.4 TB/s (three heads in flight per lane and CTAs of four warps; four heads 38 us, eight
// warps 40 us); the same pass into the 8-bit cache, 32 heads, 308 MB, 64 us, 4.8 TB/s (a tile waits for its scale and for its
// loads, and the instructions of norm, rotation, maximum and encoding take 62 % of the issue slots); reading back, 617 MB, 102
// us, 6.0 TB/s (a whole tile in flight per warp).  A single-token batch is latency: 64 tokens 2.7 us, three trips to memory.
#include <math.h>

#include <algorithm>

#include "kv8.cuh"

namespace bs {

namespace {

__device__ __forceinline__ void unpack8(const uint4& v, float* x) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __bfloat1622float2(h[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float* x) {
  uint4 v;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
  return v;
}

// A lane's part of one head: x[0..8) = dims [8 p, 8 p + 8), x[8..16) = dims dh / 2 + [8 p, 8 p + 8), p = the lane's place
// among the head's dh / 16 lanes.
struct HeadLoad { uint4 lo, hi; };
template <int DH>
__device__ __forceinline__ HeadLoad load_head(const bf16* head, int p) {
  const uint4* src = reinterpret_cast<const uint4*>(head) + p;
  HeadLoad v;
  v.lo = __ldcg(src);
  v.hi = __ldcg(src + DH / 16);
  return v;
}
template <int DH>
__device__ __forceinline__ void store_head(bf16* head, int p, const HeadLoad& v) {
  uint4* dst = reinterpret_cast<uint4*>(head) + p;
  dst[0] = v.lo;
  dst[DH / 16] = v.hi;
}
__device__ __forceinline__ void unpack16(const HeadLoad& v, float* x) {
  unpack8(v.lo, x);
  unpack8(v.hi, x + 8);
}
__device__ __forceinline__ HeadLoad no_head() {
  HeadLoad v;
  v.lo = v.hi = make_uint4(0, 0, 0, 0);
  return v;
}
// 1 / root mean square of the head.  All lanes of the warp call.
template <int DH>
__device__ __forceinline__ float head_rms(const float* x, float eps) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) ss += x[i] * x[i];
#pragma unroll
  for (int o = DH / 32; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  return rsqrtf(ss * (1.0f / DH) + eps);
}
template <int DH>
__device__ __forceinline__ void head_gain(float* x, float r, const bf16* gain, int p) {
  HeadLoad v;
  v.lo = __ldg(reinterpret_cast<const uint4*>(gain) + p);
  v.hi = __ldg(reinterpret_cast<const uint4*>(gain) + p + DH / 16);
  float g[16];
  unpack16(v, g);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = x[i] * r * g[i];
}
// cs: (cos, sin) of the lane's 8 pairs
__device__ __forceinline__ void head_rotate(float* x, const float2* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float u = x[i], v = x[i + 8];
    x[i] = u * cs[i].x - v * cs[i].y;
    x[i + 8] = v * cs[i].x + u * cs[i].y;
  }
}
template <int DH>
__device__ __forceinline__ void load_turn(const float* table, int pos, int p, float2* cs) {
  const float4* src = reinterpret_cast<const float4*>(table + (size_t)pos * DH + p * 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = __ldg(src + i);
    cs[2 * i] = make_float2(v.x, v.y);
    cs[2 * i + 1] = make_float2(v.z, v.w);
  }
}

__device__ __forceinline__ void bad_index(int* flag, int site) {
  if (flag) atomicMax(flag, 100 + site);
}

constexpr int kWarps = 4;       // of a CTA of the bf16 pass
constexpr int kUnroll = 3;      // heads in flight per lane

// One warp: heads [h0, h1) of token t.  BF16KV: k and v heads go to cache row `kv_row` of kc / vc; else h1 <= hq.
// wanted(): whether the token is to be handled, asked while its heads and position are on their way.
template <int DH, bool BF16KV, typename Wanted>
__device__ __forceinline__ void token_heads(const QkNormArgs& a, int t, int h0, int h1, size_t kv_row,
                                            bf16* kc, bf16* vc, Wanted wanted) {
  constexpr int LPH = DH / 16, HPW = 32 / LPH;     // lanes per head, heads per warp pass
  const int lane = threadIdx.x & 31, p = lane % LPH, mine = lane / LPH;
  const int heads = a.hq + 2 * a.hkv;
  const bf16* src = a.qkv + (size_t)t * heads * DH;
  const int pos = __ldcg(a.tok_pos + t);
  HeadLoad raw[kUnroll];
  auto fetch = [&](int h) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) raw[u] = h + u * HPW < h1 ? load_head<DH>(src + (size_t)(h + u * HPW) * DH, p) : no_head();
  };
  fetch(h0 + mine);                                // on its way beside the position and the angles
  if (!wanted()) return;
  if (pos < 0 || pos >= a.max_pos) {               // warp-uniform
    if (lane == 0) bad_index(a.error_flag, SITE_QK_NORM);
    return;
  }
  const bool norm = a.q_gain != nullptr;
  float2 cs[8];
  load_turn<DH>(a.table, pos, p, cs);
  for (int hb = h0 + mine; hb - mine < h1; hb += kUnroll * HPW) {
    if (hb != h0 + mine) fetch(hb);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = hb + u * HPW;
      float x[16];
      unpack16(raw[u], x);
      if (norm) head_gain<DH>(x, head_rms<DH>(x, a.eps), h < a.hq ? a.q_gain : a.k_gain, p);
      head_rotate(x, cs);
      if (h >= h1) continue;
      HeadLoad y;
      y.lo = pack8(x);
      y.hi = pack8(x + 8);
      if (h < a.hq) {
        store_head<DH>(a.q_out + (size_t)t * a.q_ld + h * DH, p, y);
      } else if (BF16KV) {
        if (h < a.hq + a.hkv)
          store_head<DH>(kc + (kv_row * a.hkv + (h - a.hq)) * DH, p, y);
        else
          store_head<DH>(vc + (kv_row * a.hkv + (h - a.hq - a.hkv)) * DH, p, raw[u]);
      }
    }
  }
}

// bf16 cache: warps of (token, share of the heads); tok_kv[t] < 0 marks a token that belongs to no row.
template <int DH>
__global__ void __launch_bounds__(kWarps * 32, 5) k_qk_norm_rope_kv(QkNormArgs a, const int* __restrict__ tok_kv, bf16* kc,
                                                                 bf16* vc, long long kv_rows, int shares, int per_share) {
  pdl_wait();
  pdl_trigger();
  const long long unit = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int t = (int)(unit / shares), part = (int)(unit % shares);
  if (t >= a.M) return;
  const int row = __ldcg(tok_kv + t);
  if (row < 0) return;
  if (row >= kv_rows) {
    if ((threadIdx.x & 31) == 0) bad_index(a.error_flag, SITE_QK_NORM);
    return;
  }
  const int heads = a.hq + 2 * a.hkv;
  token_heads<DH, true>(a, t, part * per_share, min(heads, (part + 1) * per_share), (size_t)row, kc, vc,
                        [] { return true; });
}

// ---- 8-bit cache -------------------------------------------------------------------------------------------

// The rows of a span of cache rows, cut at cache blocks: which row and which of its blocks a work slot stands for.
struct Slot {
  int row, t0, n, at, base, len;     // len: kv_len of the row (0 where the caller has none)
  long long block;     // cache block
  int first;           // cache position (offset from the row's base) of the block's row 0
};
// Whether a row of n > 0 tokens from t0 on fits its slab and the call.
__device__ __forceinline__ bool span_fits(int t0, int n, int base, int at, int M, long long n_blocks) {
  return t0 >= 0 && n > 0 && (long long)t0 + n <= M && base >= 0 && base % kKv8Block == 0 && at >= 0 &&
         (long long)base + at + n <= n_blocks * kKv8Block;
}
// Whether token t belongs to a row that fits, asked once by every warp of a CTA, as whole warps.  One warp looks the rows up
// for its CTA, the 32 around the first token's, all at once (by every warp, the same few lines of the L2 hold all of them up:
// 16 block steps 7.3 us, 6.8 so); a token behind those is looked up by its own warp.
struct RowSpan {
  int t0, t1, base, at;
  __device__ __forceinline__ void load(int r, const int* __restrict__ cu, const int* __restrict__ kv_base,
                                       const int* __restrict__ kv_at) {
    t0 = __ldcg(cu + r);
    t1 = __ldcg(cu + r + 1);
    base = __ldcg(kv_base + r);
    at = __ldcg(kv_at + r);
  }
  __device__ __forceinline__ int2 tokens(int M, long long n_blocks) const {       // none of a row that does not fit
    return span_fits(t0, t1 - t0, base, at, M, n_blocks) ? make_int2(t0, t1) : make_int2(0, 0);
  }
};
// false: the slot holds nothing (or indices that do not fit: flagged).  Every lane of the warp gets the same answer.
__device__ __forceinline__ bool find_slot(int slot, const int* __restrict__ cu, const int* __restrict__ kv_base,
                                          const int* __restrict__ kv_at, const int* __restrict__ kv_len, int n_rows,
                                          int M, long long n_blocks, int* flag, Slot& s) {
  s.row = warp_search(n_rows, slot, [&](int i) { return __ldcg(cu + i) / kKv8Block + 2 * i; });
  const int r = s.row;
  s.t0 = __ldcg(cu + r);
  const int t1 = __ldcg(cu + r + 1);
  s.n = t1 - s.t0;
  s.base = __ldcg(kv_base + r);
  s.at = __ldcg(kv_at + r);
  s.len = kv_len ? __ldcg(kv_len + r) : 0;
  if (s.n == 0) return false;
  if (!span_fits(s.t0, s.n, s.base, s.at, M, n_blocks)) {
    if ((threadIdx.x & 31) == 0) bad_index(flag, SITE_KV8);
    return false;
  }
  const int k = slot - (s.t0 / kKv8Block + 2 * r);
  const int b = s.at / kKv8Block + k;
  if (k < 0 || b > (s.at + s.n - 1) / kKv8Block) return false;
  s.first = b * kKv8Block;
  s.block = (long long)s.base / kKv8Block + b;
  return true;
}

template <int DH>
constexpr int kTileThreads = kKv8Block * (DH / 16);      // a thread per (row of a tile, lane of its head)

// 16 fp32 values -> their codes at two places
template <int DH>
__device__ __forceinline__ void store_codes(unsigned char* row, int p, const float* x, float inv) {
  uint2 w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float* y = x + 8 * i;
    w[i].x = kv8_encode2(y[0] * inv, y[1] * inv) | (kv8_encode2(y[2] * inv, y[3] * inv) << 16);
    w[i].y = kv8_encode2(y[4] * inv, y[5] * inv) | (kv8_encode2(y[6] * inv, y[7] * inv) << 16);
    *reinterpret_cast<uint2*>(row + i * (DH / 2) + p * 8) = w[i];
  }
}
// The codes of a lane's 16 dims, in a HeadLoad's first half.
template <int DH>
__device__ __forceinline__ HeadLoad load_codes(const unsigned char* row, int p) {
  const uint2 a = __ldcg(reinterpret_cast<const uint2*>(row + p * 8));
  const uint2 b = __ldcg(reinterpret_cast<const uint2*>(row + DH / 2 + p * 8));
  HeadLoad v = no_head();
  v.lo = make_uint4(a.x, a.y, b.x, b.y);
  return v;
}
__device__ __forceinline__ void decode16(const HeadLoad& v, float scale, float* x) {
  const unsigned w[4] = {v.lo.x, v.lo.y, v.lo.z, v.lo.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned h[2];
    kv8_decode4(w[i], h[0], h[1]);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float2 f = __half22float2(*reinterpret_cast<__half2*>(&h[j]));
      x[4 * i + 2 * j] = f.x * scale;
      x[4 * i + 2 * j + 1] = f.y * scale;
    }
  }
}
// Largest finite magnitude over the warp, as its bits (they order like the magnitudes; infinities and NaN count nothing).
// The maximum passes NaN by; where it is infinite, which is rare, every element is looked at.
__device__ __forceinline__ unsigned largest_finite(const float* x, float top, bool counts) {
  if (counts && top == INFINITY) {
    top = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (fabsf(x[j]) < INFINITY) top = fmaxf(top, fabsf(x[j]));
  }
  return __reduce_max_sync(0xffffffffu, counts ? __float_as_uint(top) : 0u);
}
__device__ __forceinline__ float largest16(const float* x) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 16; j += 2) asm("max.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(fabsf(x[j])), "f"(fabsf(x[j + 1])));
  return top;
}
__device__ __forceinline__ float largest16(const HeadLoad& v) {
  const __nv_bfloat162* a = reinterpret_cast<const __nv_bfloat162*>(&v.lo);
  const __nv_bfloat162* b = reinterpret_cast<const __nv_bfloat162*>(&v.hi);
  __nv_bfloat162 top = __floats2bfloat162_rn(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < 4; ++j) top = __hmax2(top, __hmax2(__habs2(a[j]), __habs2(b[j])));
  return fmaxf(__low2float(top), __high2float(top));
}

// Three CTAs of 256 threads per SM (80 registers; with two 16 whole rows of 32 heads take 87 us where three take 76).
// One CTA: the K and V tiles of kv heads [g0, g1) of one cache block.  A thread owns one row of the block and keeps its
// angles in registers from head to head; the next head's rows are fetched while this one's are turned.  New rows are
// formed in registers, kept rows decoded beside them, the largest magnitude of both gives the scale, and all are encoded
// against it.
// MIXED: the block also has rows that are not written - a span's first or last one.
template <int DH, bool MIXED>
__device__ __forceinline__ void write_tiles(const QkNormArgs& a, const Slot& s, const Kv8Cache& c, int g0, int g1,
                            unsigned (*s_max)[2][kTileThreads<DH> / 32], float4* s_gain) {
  constexpr int LPH = DH / 16, W = kTileThreads<DH> / 32;
  const int p = threadIdx.x % LPH, r = threadIdx.x / LPH, at = s.first + r;
  const int heads = a.hq + 2 * a.hkv;
  const bool fresh = !MIXED || (at >= s.at && at < s.at + s.n);
  int state = MIXED && !fresh && at < s.len ? 1 : 0;                // 0: not a valid row, 1: kept, 2: new
  const int t = fresh ? s.t0 + at - s.at : 0;
  const bf16* src = a.qkv + ((size_t)t * heads + a.hq) * DH;
  const size_t tile0 = (size_t)s.block * a.hkv;
  HeadLoad k = no_head(), v = no_head();
  float next_k = 0.f, next_v = 0.f;                        // scales of kept rows
  auto fetch = [&](int head) {
    if (fresh) {
      k = load_head<DH>(src + head * DH, p);
      v = load_head<DH>(src + (a.hkv + head) * DH, p);
    } else if (MIXED && state == 1) {
      const size_t at_row = ((tile0 + head) * kKv8Block + r) * DH;
      k = load_codes<DH>(c.k + at_row, p);
      v = load_codes<DH>(c.v + at_row, p);
    }
    if (MIXED) {
      next_k = __ldcg(c.k_scale + tile0 + head);
      next_v = __ldcg(c.v_scale + tile0 + head);
    }
  };
  fetch(g0);
  if (a.k_gain && threadIdx.x < DH) {
    const int d = threadIdx.x, lane_of = d % (DH / 2) / 8, q = d / (DH / 2) * 2 + d % 8 / 4;
    reinterpret_cast<float*>(s_gain)[(q * LPH + lane_of) * 4 + d % 4] = __bfloat162float(a.k_gain[d]);
  }
  __syncthreads();
  float2 cs[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) cs[j] = make_float2(1.f, 0.f);
  if (fresh) {
    const int pos = __ldcg(a.tok_pos + t);
    if (pos >= 0 && pos < a.max_pos) {
      state = 2;
      load_turn<DH>(a.table, pos, p, cs);
    } else if (p == 0) {
      bad_index(a.error_flag, SITE_KV8);
    }
  }
  for (int head = g0; head < g1; ++head) {
    const size_t tile = tile0 + head;
    unsigned char* row_k = c.k + (tile * kKv8Block + r) * DH;
    unsigned char* row_v = c.v + (tile * kKv8Block + r) * DH;
    const HeadLoad vc = v;                                 // V waits for its scale as it came
    const float old_k = kv8_clamp_scale(next_k), old_v = kv8_clamp_scale(next_v);
    float x[16];
    auto v_row = [&] {
      if (MIXED && state == 1) decode16(vc, old_v, x); else unpack16(vc, x);
    };
    float top = MIXED || !(largest16(vc) < INFINITY) ? (v_row(), largest16(x)) : largest16(vc);
    unsigned top_v = largest_finite(x, top, state != 0);
    if (MIXED && state == 1) decode16(k, old_k, x); else unpack16(k, x);
    if (head + 1 < g1) fetch(head + 1);
    const float rms = a.k_gain ? head_rms<DH>(x, a.eps) : 0.f;
    if (state == 2) {
      if (a.k_gain) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 g = s_gain[i * LPH + p];
          x[4 * i] *= rms * g.x;
          x[4 * i + 1] *= rms * g.y;
          x[4 * i + 2] *= rms * g.z;
          x[4 * i + 3] *= rms * g.w;
        }
      }
      head_rotate(x, cs);
    }
    unsigned top_k = largest_finite(x, largest16(x), state != 0);
    unsigned (*place)[W] = s_max[(head - g0) & 1];         // the head before the last is done with it: one barrier a head
    if ((threadIdx.x & 31) == 0) {
      place[0][threadIdx.x >> 5] = top_k;
      place[1][threadIdx.x >> 5] = top_v;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) {
      top_k = max(top_k, place[0][w]);
      top_v = max(top_v, place[1][w]);
    }
    const int ek = kv8_scale_exp(__uint_as_float(top_k)), ev = kv8_scale_exp(__uint_as_float(top_v));
    if (state == 2 || (MIXED && state == 1 && pow2i(ek) != old_k)) store_codes<DH>(row_k, p, x, pow2i(-ek));
    if (state == 2 || (MIXED && state == 1 && pow2i(ev) != old_v)) {
      v_row();
      store_codes<DH>(row_v, p, x, pow2i(-ev));
    }
    if (threadIdx.x == 0) {
      c.k_scale[tile] = pow2i(ek);
      c.v_scale[tile] = pow2i(ev);
    }
  }
}

// CTAs [0, q_ctas): query heads, a warp for (token, share of the heads).  CTAs beyond: the tiles of the work slots, one
// CTA for (slot, `per_cta` kv heads).
template <int DH>
__global__ void __launch_bounds__(kTileThreads<DH>, 768 / kTileThreads<DH>) k_qk_norm_rope_kv8(QkNormArgs a, const int* __restrict__ cu_q,
                                                                       const int* __restrict__ kv_base,
                                                                       const int* __restrict__ kv_at,
                                                                       const int* __restrict__ kv_len, int n_rows,
                                                                       Kv8Cache c, int q_ctas, int shares, int per_share,
                                                                       int per_cta) {
  __shared__ unsigned s_max[2][2][kTileThreads<DH> / 32];
  __shared__ int2 s_rows[32];
  __shared__ int s_first;
  __shared__ float4 s_gain[DH / 4];      // k_gain as floats, by the lanes' order: [four dims of a lane][lane]
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x < q_ctas) {
    const long long unit = (long long)blockIdx.x * (kTileThreads<DH> / 32) + (threadIdx.x >> 5);
    const int t = (int)(unit / shares), part = (int)(unit % shares), lane = threadIdx.x & 31;
    RowSpan mine = {0, 0, 0, 0};
    int first = 0;
    auto look = [&](int token) {
      if (n_rows > 32) first = 32 * warp_search((n_rows + 31) >> 5, token, [&](int i) { return __ldcg(cu_q + 32 * i); });
      if (first + lane < n_rows) mine.load(first + lane, cu_q, kv_base, kv_at);
    };
    if (threadIdx.x < 32) look((int)((long long)blockIdx.x * (kTileThreads<DH> / 32) / shares));
    auto holds = [&](int2 v) { return __any_sync(0xffffffffu, t >= v.x && t < v.y) != 0; };
    auto wanted = [&] {
      if (threadIdx.x < 32) s_rows[lane] = mine.tokens(a.M, c.n_blocks);
      if (threadIdx.x == 0) s_first = first;
      __syncthreads();
      if (holds(s_rows[lane])) return true;
      if (s_first + 32 >= n_rows) return false;
      mine = {0, 0, 0, 0};
      look(t);
      return holds(mine.tokens(a.M, c.n_blocks));
    };
    // Tokens behind the last row are left alone, and so are those of rows that do not fit (the tiles' CTAs flag them).
    if (t >= a.M)
      wanted();                                            // (for the barrier)
    else
      token_heads<DH, false>(a, t, part * per_share, min(a.hq, (part + 1) * per_share), 0, nullptr, nullptr, wanted);
    return;
  }
  const int unit = (int)blockIdx.x - q_ctas;
  const int groups = (a.hkv + per_cta - 1) / per_cta, slot = unit / groups, g0 = (unit - slot * groups) * per_cta;
  Slot s;
  if (!find_slot(slot, cu_q, kv_base, kv_at, kv_len, n_rows, a.M, c.n_blocks, a.error_flag, s)) return;
  const int g1 = min(a.hkv, g0 + per_cta);
  if (s.first < s.at || s.first + kKv8Block > s.at + s.n)
    write_tiles<DH, true>(a, s, c, g0, g1, s_max, s_gain);
  else
    write_tiles<DH, false>(a, s, c, g0, g1, s_max, s_gain);
}

// One warp: one (head, K or V) tile of a work slot at a time, all of it in flight at once; a CTA takes `per_cta` tiles of
// its slot.
template <int DH>
__global__ void __launch_bounds__(256, 2) k_kv8_read(Kv8Cache c, const int* __restrict__ cu, const int* __restrict__ kv_base,
                                                  const int* __restrict__ kv_at, int n_rows, int total, int hkv,
                                                  bf16* __restrict__ k_out, bf16* __restrict__ v_out, int* error_flag,
                                                  int per_cta) {
  pdl_wait();
  pdl_trigger();
  const int tiles = 2 * hkv, groups = (tiles + per_cta - 1) / per_cta;
  const int slot = (int)blockIdx.x / groups, w0 = ((int)blockIdx.x - slot * groups) * per_cta;
  Slot s;
  if (!find_slot(slot, cu, kv_base, kv_at, nullptr, n_rows, total, c.n_blocks, error_flag, s)) return;
  constexpr int LPR = DH / 8, RPP = 32 / LPR, PASSES = kKv8Block / RPP;      // lanes per row, rows per pass
  const int lane = threadIdx.x & 31, p = lane % LPR, sub = lane / LPR;
  const int lo = max(s.first, s.at) - s.first, hi = min(s.first + kKv8Block, s.at + s.n) - s.first;
  const long long t0 = (long long)s.t0 + s.first - s.at;                     // token of the block's row 0
  for (int w = w0 + (threadIdx.x >> 5); w < min(tiles, w0 + per_cta); w += 8) {
    const int head = w >> 1;
    const size_t tile = (size_t)s.block * hkv + head;
    const unsigned char* codes = ((w & 1) ? c.v : c.k) + tile * kKv8Block * DH;
    bf16* out = (w & 1) ? v_out : k_out;
    const float scale = kv8_clamp_scale(__ldcg(((w & 1) ? c.v_scale : c.k_scale) + tile));
    uint2 raw[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = i * RPP + sub;
      raw[i] = make_uint2(0, 0);
      if (r >= lo && r < hi) raw[i] = __ldcg(reinterpret_cast<const uint2*>(codes + r * DH) + p);
    }
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int r = i * RPP + sub;
      if (r < lo || r >= hi) continue;
      unsigned h[4];
      kv8_decode4(raw[i].x, h[0], h[1]);
      kv8_decode4(raw[i].y, h[2], h[3]);
      float x[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<__half2*>(&h[j]));
        x[2 * j] = f.x * scale;
        x[2 * j + 1] = f.y * scale;
      }
      __stcs(reinterpret_cast<uint4*>(out + ((t0 + r) * hkv + head) * DH) + p, pack8(x));
    }
  }
}

// Heads per warp: all of a token's heads when the tokens give every SM `warps` warps (the rotation's cos / sin are then
// loaded once per token), otherwise a share of them.
void head_shares(int M, int heads, int dh, int warps, int* shares, int* per_share) {
  const int per_pass = 32 / (dh / 16) * kUnroll;
  const int passes = (heads + per_pass - 1) / per_pass;
  int n = 1;
  while (n < passes && (long long)M * n < 148 * warps) ++n;
  const int each = (passes + n - 1) / n;
  *per_share = each * per_pass;
  *shares = (passes + each - 1) / each;
}
// Of `n` items of each of `slots` work slots: how many one CTA takes, so that a slot's indices and angles are fetched for
// as many as leave eight CTAs per SM (with three 16 whole rows are written in 81 us where eight take 76, read in 106 and 103).
int items_per_cta(long long slots, int n, int least) {
  int per = n;
  while (per > least && slots * ((n + per - 1) / per) < 148 * 8) per = (per + 1) / 2;
  return std::max(per, least);
}

}  // namespace

cudaError_t launch_qk_norm_rope_kv(const QkNormArgs& a, const int* tok_kv, bf16* kc, bf16* vc, long long kv_rows,
                                   cudaStream_t s) {
  if (a.M <= 0) return cudaSuccess;
  int shares, per_share;
  head_shares(a.M, a.hq + 2 * a.hkv, a.dh, 20, &shares, &per_share);
  const dim3 grid((unsigned)(((long long)a.M * shares + kWarps - 1) / kWarps));
  return launch_pdl(a.dh == 128 ? k_qk_norm_rope_kv<128> : k_qk_norm_rope_kv<64>, grid, dim3(kWarps * 32), 0, s, a, tok_kv,
                    kc, vc, kv_rows, shares, per_share);
}

cudaError_t launch_qk_norm_rope_kv8(const QkNormArgs& a, const int* cu_q, const int* kv_base, const int* kv_at,
                                    const int* kv_len, int n_rows, const Kv8Cache& c, cudaStream_t s) {
  if (a.M <= 0 || n_rows <= 0) return cudaSuccess;
  int shares, per_share;
  head_shares(a.M, a.hq, a.dh, 6, &shares, &per_share);
  const int threads = a.dh == 128 ? kTileThreads<128> : kTileThreads<64>;
  const long long q_ctas = ((long long)a.M * shares + threads / 32 - 1) / (threads / 32);
  const long long slots = kv8_span_slots(a.M, n_rows);
  const int per_cta = items_per_cta(slots, a.hkv, 1);
  const long long ctas = q_ctas + slots * ((a.hkv + per_cta - 1) / per_cta);
  if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_pdl(a.dh == 128 ? k_qk_norm_rope_kv8<128> : k_qk_norm_rope_kv8<64>, dim3((unsigned)ctas),
                    dim3(threads), 0, s, a, cu_q, kv_base, kv_at, kv_len, n_rows, c, (int)q_ctas, shares, per_share, per_cta);
}

cudaError_t launch_kv8_read(const Kv8Cache& c, const int* cu, const int* kv_base, const int* kv_at, int n_rows, int total,
                            int hkv, int dh, bf16* k_out, bf16* v_out, int* error_flag, cudaStream_t s) {
  if (total <= 0 || n_rows <= 0) return cudaSuccess;
  const long long slots = kv8_span_slots(total, n_rows);
  const int per_cta = items_per_cta(slots, 2 * hkv, 8);
  const long long ctas = slots * ((2 * hkv + per_cta - 1) / per_cta);
  if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_pdl(dh == 128 ? k_kv8_read<128> : k_kv8_read<64>, dim3((unsigned)ctas), dim3(256), 0, s, c, cu, kv_base,
                    kv_at, n_rows, total, hkv, k_out, v_out, error_flag, per_cta);
}

}  // namespace bs
