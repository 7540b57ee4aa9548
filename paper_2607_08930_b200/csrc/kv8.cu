// Norms of every query / key head with the rotation and the cache write in one pass (bf16 or 8-bit cache), and the way
// from the 8-bit cache back to bf16.
//
//   y = gain * x / sqrt(mean(x^2) + eps) over a head's dims; (y_j, y_{j + dh/2}) turned by the token's angle
//
// All three are bound by memory: every element of qkv is read once and its result written once.  dh / 8 lanes own one
// head of one token (16 bytes each); the norm's sum and the rotation's partner half move by shuffles inside those
// lanes, everything between the load and the one rounding at the end stays fp32.
#include <math.h>

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

// x: dims [8 p, 8 p + 8) of one head, p = this lane's place among the head's dh / 8 lanes.  All lanes of the warp call.
template <int DH>
__device__ __forceinline__ void head_norm(float* x, const uint4& gain, float eps) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss += x[i] * x[i];
#pragma unroll
  for (int o = DH / 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  const float r = rsqrtf(ss * (1.0f / DH) + eps);
  float g[8];
  unpack8(gain, g);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * g[i];
}
// cs: (cos, sin) of the pairs this lane's dims belong to; sign = -1 in the first half of the dims, +1 in the second
template <int DH>
__device__ __forceinline__ void head_rotate(float* x, const float2* cs, float sign) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = __shfl_xor_sync(0xffffffffu, x[i], DH / 16);
    x[i] = x[i] * cs[i].x + sign * y * cs[i].y;
  }
}
template <int DH>
__device__ __forceinline__ void load_turn(const float* table, int pos, int p, float2* cs) {
  const float4* src = reinterpret_cast<const float4*>(table + (size_t)pos * DH + (p % (DH / 16)) * 16);
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

constexpr int kWarps = 8;
constexpr int kUnroll = 4;      // heads in flight per lane

// One warp: heads [h0, h1) of token t.  BF16KV: k and v heads go to cache row `kv_row` of kc / vc; else h1 <= hq.
template <int DH, bool BF16KV>
__device__ __forceinline__ void token_heads(const QkNormArgs& a, int t, int h0, int h1, size_t kv_row,
                                            bf16* kc, bf16* vc) {
  constexpr int LPH = DH / 8, HPW = 32 / LPH;      // lanes per head, heads per warp pass
  const int lane = threadIdx.x & 31, p = lane % LPH;
  const int pos = __ldcg(a.tok_pos + t);
  if (pos < 0 || pos >= a.max_pos) {               // warp-uniform
    if (lane == 0) bad_index(a.error_flag, SITE_QK_NORM);
    return;
  }
  const bool norm = a.q_gain != nullptr;
  uint4 gq = make_uint4(0, 0, 0, 0), gk = gq;
  if (norm) {
    gq = __ldg(reinterpret_cast<const uint4*>(a.q_gain) + p);
    gk = __ldg(reinterpret_cast<const uint4*>(a.k_gain) + p);
  }
  const int heads = a.hq + 2 * a.hkv;
  const uint4* src = reinterpret_cast<const uint4*>(a.qkv + (size_t)t * heads * DH) + p;
  float2 cs[8];
  load_turn<DH>(a.table, pos, p, cs);
  const float sign = p < LPH / 2 ? -1.f : 1.f;
  for (int hb = h0 + lane / LPH; hb - lane / LPH < h1; hb += kUnroll * HPW) {
    uint4 raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = hb + u * HPW;
      raw[u] = h < h1 ? src[(size_t)h * LPH] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = hb + u * HPW;
      float x[8];
      unpack8(raw[u], x);
      if (norm) head_norm<DH>(x, h < a.hq ? gq : gk, a.eps);
      head_rotate<DH>(x, cs, sign);
      if (h >= h1) continue;
      if (h < a.hq) {
        *reinterpret_cast<uint4*>(a.q_out + (size_t)t * a.q_ld + h * DH + p * 8) = pack8(x);
      } else if (BF16KV) {
        if (h < a.hq + a.hkv)
          *(reinterpret_cast<uint4*>(kc + (kv_row * a.hkv + (h - a.hq)) * DH) + p) = pack8(x);
        else
          *(reinterpret_cast<uint4*>(vc + (kv_row * a.hkv + (h - a.hq - a.hkv)) * DH) + p) = raw[u];
      }
    }
  }
}

// bf16 cache: warps of (token, share of the heads); tok_kv[t] < 0 marks a token that belongs to no row.
template <int DH>
__global__ void __launch_bounds__(kWarps * 32) k_qk_norm_rope_kv(QkNormArgs a, const int* __restrict__ tok_kv, bf16* kc,
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
  token_heads<DH, true>(a, t, part * per_share, min(heads, (part + 1) * per_share), (size_t)row, kc, vc);
}

// ---- 8-bit cache -------------------------------------------------------------------------------------------

// The rows of a span of cache rows, cut at cache blocks: which row and which of its blocks a work slot stands for.
struct Slot {
  int row, t0, n, at, base;
  long long block;     // cache block
  int first;           // cache position (offset from the row's base) of the block's row 0
};
// false: the slot holds nothing (or indices that do not fit: flagged).  Every lane of the warp gets the same answer.
__device__ __forceinline__ bool find_slot(int slot, const int* __restrict__ cu, const int* __restrict__ kv_base,
                                          const int* __restrict__ kv_at, int n_rows, int M, long long n_blocks,
                                          int* flag, Slot& s) {
  s.row = warp_search(n_rows, slot, [&](int i) { return __ldcg(cu + i) / kKv8Block + 2 * i; });
  const int r = s.row;
  s.t0 = __ldcg(cu + r);
  const int t1 = __ldcg(cu + r + 1);
  s.n = t1 - s.t0;
  s.base = __ldcg(kv_base + r);
  s.at = __ldcg(kv_at + r);
  if (s.n == 0) return false;
  const bool ok = s.t0 >= 0 && s.n > 0 && t1 <= M && s.base >= 0 && s.base % kKv8Block == 0 && s.at >= 0 &&
                  (long long)s.base + s.at + s.n <= n_blocks * kKv8Block;
  if (!ok) {
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

constexpr int kTileThreads = 128;

// One CTA: one (cache block, kv head) tile of K or of V.  The tile's new rows are formed in registers, its kept rows
// decoded beside them, the largest magnitude of both gives the scale, and all of them are encoded against it.
template <int DH>
__device__ void write_tile(const QkNormArgs& a, const Slot& s, int kv_len, const Kv8Cache& c, int head, bool is_k,
                           float* s_max) {
  constexpr int LPH = DH / 8, TPP = kTileThreads / LPH, PASSES = kKv8Block / TPP;   // lanes / token, tokens / pass
  const int tid = threadIdx.x, p = tid % LPH, sub = tid / LPH;
  const size_t tile = (size_t)s.block * a.hkv + head;
  unsigned char* codes = (is_k ? c.k : c.v) + tile * kKv8Block * DH + p * 8;
  float* scale_at = (is_k ? c.k_scale : c.v_scale) + tile;
  const float old = kv8_clamp_scale(*scale_at);
  const bool norm = is_k && a.k_gain != nullptr;
  const uint4 gain = norm ? __ldg(reinterpret_cast<const uint4*>(a.k_gain) + p) : make_uint4(0, 0, 0, 0);
  const float sign = p < LPH / 2 ? -1.f : 1.f;
  const int heads = a.hq + 2 * a.hkv;
  float x[PASSES][8];
  int state[PASSES];                       // 0: not a valid row, 1: kept, 2: new
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int r = i * TPP + sub, at = s.first + r;
    state[i] = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
    float2 cs[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) cs[j] = make_float2(1.f, 0.f);
    if (at >= s.at && at < s.at + s.n) {
      const int t = s.t0 + at - s.at;
      const int pos = __ldcg(a.tok_pos + t);
      if (pos >= 0 && pos < a.max_pos) {
        state[i] = 2;
        const int h = a.hq + (is_k ? 0 : a.hkv) + head;
        unpack8(*(reinterpret_cast<const uint4*>(a.qkv + ((size_t)t * heads + h) * DH) + p), x[i]);
        if (is_k) load_turn<DH>(a.table, pos, p, cs);
      } else if (p == 0) {
        bad_index(a.error_flag, SITE_KV8);
      }
    } else if (at < kv_len) {
      state[i] = 1;
      const uint2 w = *reinterpret_cast<const uint2*>(codes + r * DH);
      unsigned h[4];
      kv8_decode4(w.x, h[0], h[1]);
      kv8_decode4(w.y, h[2], h[3]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(*reinterpret_cast<__half2*>(&h[j]));
        x[i][2 * j] = f.x * old;
        x[i][2 * j + 1] = f.y * old;
      }
    }
    if (is_k) {                            // shuffles stay inside a token's lanes, whose state is the same
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = x[i][j];
      if (norm) head_norm<DH>(y, gain, a.eps);
      head_rotate<DH>(y, cs, sign);
      if (state[i] == 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = y[j];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float m = fabsf(x[i][j]);
      if (m <= 3.402823466e38f) top = fmaxf(top, m);      // finite values only
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if ((tid & 31) == 0) s_max[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kTileThreads / 32; ++w) top = fmaxf(top, s_max[w]);
  const int k = kv8_scale_exp(top);
  const float scale = pow2i(k), inv = pow2i(-k);
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    if (state[i] == 0 || (state[i] == 1 && scale == old)) continue;
    uint2 w;
    w.x = kv8_encode2(x[i][0] * inv, x[i][1] * inv) | (kv8_encode2(x[i][2] * inv, x[i][3] * inv) << 16);
    w.y = kv8_encode2(x[i][4] * inv, x[i][5] * inv) | (kv8_encode2(x[i][6] * inv, x[i][7] * inv) << 16);
    *reinterpret_cast<uint2*>(codes + (i * TPP + sub) * DH) = w;
  }
  if (tid == 0) *scale_at = scale;
}

// CTAs [0, q_ctas): query heads, a warp for (token, share of the heads).  CTAs beyond: the K and V tiles of the work
// slots, one (slot, kv head, K or V) each.
template <int DH>
__global__ void __launch_bounds__(kTileThreads) k_qk_norm_rope_kv8(QkNormArgs a, const int* __restrict__ cu_q,
                                                                   const int* __restrict__ kv_base,
                                                                   const int* __restrict__ kv_at,
                                                                   const int* __restrict__ kv_len, int n_rows,
                                                                   Kv8Cache c, int q_ctas, int shares, int per_share) {
  __shared__ float s_max[kTileThreads / 32];
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x < q_ctas) {
    const long long unit = (long long)blockIdx.x * (kTileThreads / 32) + (threadIdx.x >> 5);
    const int t = (int)(unit / shares), part = (int)(unit % shares);
    if (t >= min(a.M, __ldcg(cu_q + n_rows))) return;      // tokens behind the last row are left alone
    token_heads<DH, false>(a, t, part * per_share, min(a.hq, (part + 1) * per_share), 0, nullptr, nullptr);
    return;
  }
  const int unit = (int)blockIdx.x - q_ctas;
  const int which = unit % (2 * a.hkv), slot = unit / (2 * a.hkv);
  Slot s;
  if (!find_slot(slot, cu_q, kv_base, kv_at, n_rows, a.M, c.n_blocks, a.error_flag, s)) return;
  write_tile<DH>(a, s, __ldcg(kv_len + s.row), c, which >> 1, (which & 1) == 0, s_max);
}

// One CTA: one work slot (a cache block's share of a row), all kv heads, K and V.
template <int DH>
__global__ void __launch_bounds__(256) k_kv8_read(Kv8Cache c, const int* __restrict__ cu, const int* __restrict__ kv_base,
                                                  const int* __restrict__ kv_at, int n_rows, int total, int hkv,
                                                  bf16* __restrict__ k_out, bf16* __restrict__ v_out, int* error_flag) {
  pdl_wait();
  pdl_trigger();
  Slot s;
  if (!find_slot(blockIdx.x, cu, kv_base, kv_at, n_rows, total, c.n_blocks, error_flag, s)) return;
  constexpr int LPH = DH / 8;
  const int lo = max(s.first, s.at) - s.first, hi = min(s.first + kKv8Block, s.at + s.n) - s.first;
  const int units = 2 * hkv * kKv8Block * LPH;
  for (int u = threadIdx.x; u < units; u += 256) {
    const int p = u % LPH, r = u / LPH % kKv8Block, hw = u / LPH / kKv8Block;
    const int head = hw >> 1;
    if (r < lo || r >= hi) continue;
    const size_t tile = (size_t)s.block * hkv + head;
    const unsigned char* codes = (hw & 1) ? c.v : c.k;
    const float scale = kv8_clamp_scale(__ldcg(((hw & 1) ? c.v_scale : c.k_scale) + tile));
    const uint2 w = *reinterpret_cast<const uint2*>(codes + (tile * kKv8Block + r) * DH + p * 8);
    unsigned h[4];
    kv8_decode4(w.x, h[0], h[1]);
    kv8_decode4(w.y, h[2], h[3]);
    float x[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = __half22float2(*reinterpret_cast<__half2*>(&h[j]));
      x[2 * j] = f.x * scale;
      x[2 * j + 1] = f.y * scale;
    }
    const size_t t = (size_t)(s.t0 + s.first + r - s.at);
    *(reinterpret_cast<uint4*>(((hw & 1) ? v_out : k_out) + (t * hkv + head) * DH) + p) = pack8(x);
  }
}

// Heads per warp: all of a token's heads when the tokens fill the machine (the rotation's cos / sin are then loaded
// once per token), otherwise a share of them.
void head_shares(int M, int heads, int dh, int* shares, int* per_share) {
  const int per_pass = 32 / (dh / 8) * kUnroll;
  const int passes = (heads + per_pass - 1) / per_pass;
  int n = 1;
  while (n < passes && (long long)M * n < 148 * 32) ++n;
  const int each = (passes + n - 1) / n;
  *per_share = each * per_pass;
  *shares = (passes + each - 1) / each;
}

}  // namespace

cudaError_t launch_qk_norm_rope_kv(const QkNormArgs& a, const int* tok_kv, bf16* kc, bf16* vc, long long kv_rows,
                                   cudaStream_t s) {
  if (a.M <= 0) return cudaSuccess;
  int shares, per_share;
  head_shares(a.M, a.hq + 2 * a.hkv, a.dh, &shares, &per_share);
  const dim3 grid((unsigned)(((long long)a.M * shares + kWarps - 1) / kWarps));
  return launch_pdl(a.dh == 128 ? k_qk_norm_rope_kv<128> : k_qk_norm_rope_kv<64>, grid, dim3(kWarps * 32), 0, s, a, tok_kv,
                    kc, vc, kv_rows, shares, per_share);
}

cudaError_t launch_qk_norm_rope_kv8(const QkNormArgs& a, const int* cu_q, const int* kv_base, const int* kv_at,
                                    const int* kv_len, int n_rows, const Kv8Cache& c, cudaStream_t s) {
  if (a.M <= 0 || n_rows <= 0) return cudaSuccess;
  int shares, per_share;
  head_shares(a.M, a.hq, a.dh, &shares, &per_share);
  const long long q_ctas = ((long long)a.M * shares + kTileThreads / 32 - 1) / (kTileThreads / 32);
  const long long ctas = q_ctas + kv8_span_slots(a.M, n_rows) * 2 * a.hkv;
  if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_pdl(a.dh == 128 ? k_qk_norm_rope_kv8<128> : k_qk_norm_rope_kv8<64>, dim3((unsigned)ctas),
                    dim3(kTileThreads), 0, s, a, cu_q, kv_base, kv_at, kv_len, n_rows, c, (int)q_ctas, shares, per_share);
}

cudaError_t launch_kv8_read(const Kv8Cache& c, const int* cu, const int* kv_base, const int* kv_at, int n_rows, int total,
                            int hkv, int dh, bf16* k_out, bf16* v_out, int* error_flag, cudaStream_t s) {
  if (total <= 0 || n_rows <= 0) return cudaSuccess;
  const dim3 grid((unsigned)kv8_span_slots(total, n_rows));
  return launch_pdl(dh == 128 ? k_kv8_read<128> : k_kv8_read<64>, grid, dim3(256), 0, s, c, cu, kv_base, kv_at, n_rows,
                    total, hkv, k_out, v_out, error_flag);
}

}  // namespace bs
