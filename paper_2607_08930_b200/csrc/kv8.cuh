// Layout and arithmetic of the 8-bit KV cache.
//
// K and V are e4m3 codes [kv_rows / 32][n_kv_heads][32][head_dim]: the 32 rows of one (block, head) are one contiguous
// tile, and each tile has one scale, scales [kv_rows / 32][n_kv_heads] fp32.  A value is code * scale.  The scale is
// the smallest power of two 2^k, kKv8MinExp <= k <= kKv8MaxExp, under which the tile's largest magnitude fits e4m3's
// 448.  e4m3 is a floating format, so a power of two loses no relative precision against amax / 448 (normal values
// keep 4 significant bits either way); in exchange code * scale is exact in bf16 and fp32, and a tile whose scale
// moves when rows are rewritten is re-encoded without a second rounding (except where values go subnormal).
//
// The kernels here may be on the device before the kernel in front of them has ended (programmatic dependent launch):
// what that one may have written - queries, scales, indices - is read past the L1 cache (__ldcg, cp.async.cg, TMA) and
// never through the read-only path, which is for weights and tables.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace bs {

constexpr int kKv8Block = 32;                       // cache rows per scale
constexpr int kKv8MinExp = -40, kKv8MaxExp = 40;    // range of the scale's exponent: scales, their inverses and the
                                                    // quotient of two stay far inside fp32's range
constexpr float kKv8Max = 448.0f;                   // largest e4m3 value

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }

// Exponent of the scale for a tile whose largest finite magnitude is amax (448 = 1.75 * 2^8).
__device__ __forceinline__ int kv8_scale_exp(float amax) {
  const unsigned b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 127;               // amax >= 0; subnormals fall below the clamp
  const int k = (b & 0x7fffffu) <= 0x600000u ? e - 8 : e - 7;
  return min(max(k, kKv8MinExp), kKv8MaxExp);
}

// Scales read from memory are brought into the range the kernels' arithmetic is laid out for.
__device__ __forceinline__ float kv8_clamp_scale(float s) {
  return fminf(fmaxf(s, 0x1p-40f), 0x1p40f);
}

// two floats -> two e4m3 codes (lo in the low byte), to nearest even, beyond +-448 to +-448, NaN to NaN
__device__ __forceinline__ unsigned kv8_encode2(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// two e4m3 codes (low 16 bits of x) -> two fp16 values (exact)
__device__ __forceinline__ unsigned kv8_decode2(unsigned short x) {
  unsigned r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(x));
  return r;
}
__device__ __forceinline__ void kv8_decode4(unsigned w, unsigned& a, unsigned& b) {
  a = kv8_decode2((unsigned short)(w & 0xffffu));
  b = kv8_decode2((unsigned short)(w >> 16));
}

// Largest r in [0, n) with key(r) <= item for a non-decreasing key with key(0) <= item: every lane of the calling warp
// takes part and gets the result.  32 probes at a time: two round trips to memory up to 1024 rows.
template <typename Item, typename Key>
__device__ __forceinline__ int warp_search(int n, Item item, Key key) {
  const int lane = threadIdx.x & 31;
  int lo = 0;
  for (int len = n; len > 1;) {
    const int step = (len + 31) >> 5;
    const int off = lane * step;
    const bool le = off < len && key(lo + off) <= item;
    const int c = max(__popc(__ballot_sync(0xffffffffu, le)), 1);
    const int skip = (c - 1) * step;
    lo += skip;
    len = min(step, len - skip);
  }
  return lo;
}

// Work slots of spans that are cut at cache-block boundaries: row i with packed tokens [cu[i], cu[i+1]) starts at slot
// cu[i] / 32 + 2 i, which leaves it n / 32 + 2 slots - at least as many as the blocks that n consecutive cache rows
// touch - so a launch needs no prefix over the rows' block counts.
__host__ __device__ inline long long kv8_span_slots(int M, int n_rows) { return (long long)M / kKv8Block + 2ll * n_rows; }

struct Kv8Cache {
  unsigned char* k;
  unsigned char* v;
  float* k_scale;
  float* v_scale;
  long long n_blocks;    // kv_rows / 32
};

struct QkNormArgs {
  const bf16* qkv;       // [M][hq + 2 hkv][dh]
  bf16* q_out;           // row stride q_ld
  int q_ld;
  const bf16* q_gain;    // [dh], nullptr: no norm
  const bf16* k_gain;
  float eps;
  const int* tok_pos;
  const float* table;    // [max_pos][dh / 2][2]
  int max_pos;
  int M, hq, hkv, dh;
  int* error_flag;
};
cudaError_t launch_qk_norm_rope_kv(const QkNormArgs& a, const int* tok_kv, bf16* kc, bf16* vc, long long kv_rows,
                                   cudaStream_t s);
cudaError_t launch_qk_norm_rope_kv8(const QkNormArgs& a, const int* cu_q, const int* kv_base, const int* kv_at,
                                    const int* kv_len, int n_rows, const Kv8Cache& c, cudaStream_t s);
cudaError_t launch_kv8_read(const Kv8Cache& c, const int* cu, const int* kv_base, const int* kv_at, int n_rows, int total,
                            int hkv, int dh, bf16* k_out, bf16* v_out, int* error_flag, cudaStream_t s);

struct AttnKv8Args {
  const bf16* q;
  int q_ld;
  Kv8Cache cache;
  bf16* out;             // [M][hq * dh]
  const int* cu_q;
  const int* kv_base;
  const int* vis;
  int n_rows, M, max_nq, max_vis, hq, hkv, dh;
  void* scratch;
  size_t scratch_bytes;
  int* error_flag;
};
size_t attention_kv8_scratch_bytes(int hq, int hkv, int dh);
// Whether a call of these sizes puts anything there.
bool attention_kv8_uses_scratch(int n_rows, int M, int max_nq, int max_vis, int hq, int hkv, int dh);
constexpr int kAttnKv8CutTiles = 8;      // key tiles (of 128) from which the tensor-core kernel may cut a row's keys
cudaError_t launch_attention_kv8(const AttnKv8Args& a, cudaStream_t s);
// tensor-core kernel for many query rows per kv head; part: scratch for partial results of key chunks
cudaError_t launch_attention_kv8_tc(const AttnKv8Args& a, float* part, size_t part_floats, cudaStream_t s);

}  // namespace bs
