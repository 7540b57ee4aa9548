// Rows (activations of a token, weights of an output channel) as 8-bit integer codes with one scale each.
//
//   y = x, or gain * x / sqrt(mean(x^2) + eps) with a gain;  s = max(max |y| * fp32(1 / 127), 2^-126) in fp32;
//   code = y / s rounded to the nearest integer, halves to the even one - of the exact quotient, not of a rounded one.
//
// Bound by memory: x is read once, a byte an element is written.  The threads of a row keep it in registers as it is stored
// (32 elements each, all loads in flight before the first use) between the maximum and the rounding; rows too long for that
// are read twice, the second time from L2.  Short rows share a CTA of up to 256 threads.  Measured: 4096 rows of 18944 bf16 in
// 42 us (5.5 TB/s of 6.56 copied), in fp32 in 58 (6.6), with norms in 74 and 85, 16 rows of 3584 in 2.2 us.
// A row with an infinite or NaN element, or y, has no scale: NaN, with zero codes, so that every product of it is NaN.
#include "decode_ops.cuh"

namespace bs {

namespace {

constexpr int kUnit = 8;            // elements a thread loads and rounds at a time
constexpr int kUnits = 4;           // units a thread keeps

// Eight elements as they are stored; those at and behind K are zero.
template <bool F32>
struct Unit {
  uint4 u[F32 ? 2 : 1];
};
template <bool F32, bool VEC>
__device__ __forceinline__ Unit<F32> load_unit(const void* row, int at, int K) {
  Unit<F32> r;
  if (VEC && at + kUnit <= K) {
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(row) + (size_t)at * (F32 ? 4 : 2));
    r.u[0] = __ldg(p);
    if (F32) r.u[F32 ? 1 : 0] = __ldg(p + 1);
  } else {
    unsigned w[8];
#pragma unroll
    for (int i = 0; i < kUnit; ++i) {
      w[i] = 0u;
      if (at + i < K)
        w[i] = F32 ? __ldg(static_cast<const unsigned*>(row) + at + i) : __ldg(static_cast<const unsigned short*>(row) + at + i);
    }
    if (F32) {
      r.u[0] = make_uint4(w[0], w[1], w[2], w[3]);
      r.u[F32 ? 1 : 0] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
      r.u[0] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    }
  }
  return r;
}
template <bool F32>
__device__ __forceinline__ void widen(const Unit<F32>& r, float* v) {
  const unsigned w[8] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w, r.u[F32 ? 1 : 0].x, r.u[F32 ? 1 : 0].y, r.u[F32 ? 1 : 0].z,
                         r.u[F32 ? 1 : 0].w};
#pragma unroll
  for (int i = 0; i < kUnit; ++i)
    v[i] = F32 ? __uint_as_float(w[i]) : __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}

// This unit's elements times the gain, and its share of the sum of squares before that.
template <bool F32>
__device__ __forceinline__ float gained(const Unit<F32>& r, const bf16* gain, int at, int K, float* v) {
  widen<F32>(r, v);
  float ss = 0.f, g[kUnit];
#pragma unroll
  for (int i = 0; i < kUnit; ++i) ss = fmaf(v[i], v[i], ss);
  widen<false>(load_unit<false, true>(gain, at, K), g);
#pragma unroll
  for (int i = 0; i < kUnit; ++i) v[i] *= g[i];
  return ss;
}

// |v| as an integer orders as the value does, with infinities and NaN above all numbers.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ unsigned long long pair(float a, float b) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// Codes of eight elements, y = v * r.  Adding 1.5 * 2^23 leaves the nearest integer of y * inv in the low bits; where the
// remainder y - q s (exact: a multiple of half a step of s, no larger than s) reaches half of s the quotient's own rounding
// may have decided, and the remainder decides instead.  Two elements an instruction.
template <bool NORM>
__device__ __forceinline__ uint2 round_unit(const float* v, float r, float s, float inv) {
  constexpr float kMagic = 12582912.f;
  const unsigned long long inv2 = pair(inv, inv), s2 = pair(-s, -s), magic = pair(kMagic, kMagic), one = pair(1.f, 1.f),
                           back = pair(-kMagic, -kMagic), zero = pair(-0.f, -0.f), r2 = pair(r, r);
  unsigned b[kUnit];
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < kUnit; i += 2) {
    unsigned long long y = pair(v[i], v[i + 1]);
    if (NORM) y = fma2(y, r2, zero);
    const unsigned long long t = fma2(y, inv2, magic);
    const unsigned long long rest = fma2(fma2(t, one, back), s2, y);
    float lo, hi;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(rest));
    most = fmaxf(fmaxf(most, fabsf(lo)), fabsf(hi));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(b[i]), "=r"(b[i + 1]) : "l"(t));
  }
  if (most + most >= s) {
#pragma unroll
    for (int i = 0; i < kUnit; ++i) {
      const float y = NORM ? v[i] * r : v[i];
      const float q = __uint_as_float(b[i]) - kMagic;
      const float rest = fmaf(-q, s, y), twice = fabsf(rest) + fabsf(rest);
      if (twice > s || (twice == s && (b[i] & 1u))) b[i] += rest > 0.f ? 1u : 0xffffffffu;
    }
  }
  uint2 out;
  out.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  out.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
  return out;
}

__device__ __forceinline__ void store_unit(int8_t* row, int at, int K, uint2 c) {
  if (at + kUnit <= K) {
    *reinterpret_cast<uint2*>(row + at) = c;
  } else {
    for (int i = 0; at + i < K; ++i) row[at + i] = (int8_t)((i < 4 ? c.x >> (8 * i) : c.y >> (8 * (i - 4))) & 0xffu);
  }
}

// The largest magnitude of a unit (joined with `top`), and its share of the sum of squares.
template <bool F32, bool NORM>
__device__ __forceinline__ unsigned largest(const Unit<F32>& r, const bf16* gain, int at, int K, unsigned top, float* ss) {
  if (NORM) {
    float v[kUnit];
    *ss += gained<F32>(r, gain, at, K, v);
#pragma unroll
    for (int i = 0; i < kUnit; ++i) top = max(top, magnitude(v[i]));
  } else if (F32) {
    float v[kUnit];
    widen<F32>(r, v);
#pragma unroll
    for (int i = 0; i < kUnit; ++i) top = max(top, magnitude(v[i]));
  } else {                                                  // two to a word: the same order, in 16 bits
    const unsigned w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __vmaxu2(top, w[i] & 0x7fff7fffu);
  }
  return top;
}

// Whether fp32 holds a row's sum of squares and its products with the gains: the mean of the squares (with eps) and the
// largest product lie where neither has overflowed, nor lost bits to the least numbers.  A row of zeros is one, too.
__device__ __forceinline__ bool in_range(float mean, float ss, unsigned top) {
  return mean >= 0x1p-100f && mean < INFINITY && top < 0x7f800000u &&
         (top >= __float_as_uint(0x1p-100f) || (top == 0u && ss == 0.f));
}

// A row that is not: its elements are scaled by a power of two to below one first, and the squares are summed in 64 bits.
// Every warp reads the whole row for itself (no barriers, for rows that share the CTA), and rounds its own units.
template <bool F32, bool VEC>
__device__ __noinline__ void far_row(const void* row, const bf16* gain, float eps, int8_t* out, float* scale, int K) {
  const int lane = threadIdx.x & 31;
  float v[kUnit], g[kUnit];
  unsigned top = 0u;
  for (int at = lane * kUnit; at < K; at += 32 * kUnit) {
    widen<F32>(load_unit<F32, VEC>(row, at, K), v);
#pragma unroll
    for (int i = 0; i < kUnit; ++i) top = max(top, magnitude(v[i]));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  const int e = max((int)(top >> 23), 1) - 126;              // the largest |x| is below 2^e
  const float f = e > 126 ? __uint_as_float(1u << (149 - e)) : __uint_as_float((unsigned)(127 - e) << 23);      // 2^-e
  auto scaled = [&](int at) {                                // v = gain x 2^-e; its share of the sum of squares
    double ss = 0.0;
    widen<F32>(load_unit<F32, VEC>(row, at, K), v);
    widen<false>(load_unit<false, true>(gain, at, K), g);
#pragma unroll
    for (int i = 0; i < kUnit; ++i) {
      v[i] *= f;
      ss += (double)v[i] * v[i];
      v[i] *= g[i];
    }
    return ss;
  };
  unsigned most = 0u;
  double ss = 0.0;
  for (int at = lane * kUnit; at < K; at += 32 * kUnit) {
    ss += scaled(at);
#pragma unroll
    for (int i = 0; i < kUnit; ++i) most = max(most, magnitude(v[i]));
  }
  most = __reduce_max_sync(0xffffffffu, most);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  const float rms = (float)(1.0 / sqrt(ss / K + ldexp((double)eps, -2 * e)));
  const float big = __uint_as_float(most) * rms;
  const bool real = top < 0x7f800000u && most < 0x7f800000u && big < INFINITY;
  const float s = fmaxf(__fmul_rn(big, 1.f / 127.f), 0x1p-126f);
  if (threadIdx.x == 0) *scale = real ? s : __uint_as_float(0x7fffffffu);
  for (int at = threadIdx.x * kUnit; at < K; at += blockDim.x * kUnit) {
    scaled(at);
    store_unit(out, at, K, real ? round_unit<true>(v, rms, s, __frcp_rn(s)) : make_uint2(0u, 0u));
  }
}

// Two CTAs an SM at least: of up to 1024 threads with 32 registers each for plain bf16 rows (three of 592: 4096 x
// 18944 47 -> 42 us), where the others would spill; those have up to 640 threads (4096 x 18944 fp32 with 1024: one CTA, 81 us,
// so 58; norms of bf16 rows 106 and 73, unaligned ones 133 and 79).
template <bool F32, bool VEC, bool NORM, bool LONG>
constexpr int kMost = F32 || NORM || !VEC || LONG ? 640 : 1024;
template <bool F32, bool VEC, bool NORM, bool LONG>
__global__ void __launch_bounds__(kMost<F32, VEC, NORM, LONG>, 2) k_quant_i8(const QuantI8Args a) {
  __shared__ unsigned s_max[32];
  __shared__ float s_sum[32];
  pdl_wait();
  pdl_trigger();
  const int m = blockIdx.x * blockDim.y + threadIdx.y;       // (a row has whole warps)
  bool here = m < a.M;
  long long from = m;
  if (a.idx && here) {
    from = __ldg(a.idx + m);
    here = from >= 0 && from < a.x_rows;
    if (!here && threadIdx.x == 0 && a.error_flag) atomicMax(a.error_flag, 100 + SITE_QUANT_I8);
  }
  const int K = here ? a.K : 0;
  const void* row = static_cast<const char*>(a.x) + from * a.ldx * (F32 ? 4 : 2);
  const int step = blockDim.x * kUnit;
  Unit<F32> r[kUnits];
  unsigned top = 0;
  float ss = 0.f;
  if (!LONG) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = threadIdx.x * kUnit + u * step;
      if (at < K) r[u] = load_unit<F32, VEC>(row, at, K);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = threadIdx.x * kUnit + u * step;
      if (at < K) top = largest<F32, NORM>(r[u], a.gain, at, K, top, &ss);
    }
  } else {
    for (int at = threadIdx.x * kUnit; at < K; at += step)
      top = largest<F32, NORM>(load_unit<F32, VEC>(row, at, K), a.gain, at, K, top, &ss);
  }
  if (!F32 && !NORM) top = max(top & 0xffffu, top >> 16) << 16;
  top = __reduce_max_sync(0xffffffffu, top);
  if (NORM) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  }
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  if (warps > 1) {
    if (lane == 0) {
      s_max[threadIdx.y * warps + (threadIdx.x >> 5)] = top;
      if (NORM) s_sum[threadIdx.y * warps + (threadIdx.x >> 5)] = ss;
    }
    __syncthreads();
    top = __reduce_max_sync(0xffffffffu, lane < warps ? s_max[threadIdx.y * warps + lane] : 0u);
    if (NORM) {
      ss = lane < warps ? s_sum[threadIdx.y * warps + lane] : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    }
  }
  if (!here) return;
  const float mean = ss / (float)a.K + a.eps;
  // (by a vote, so that the units' registers need not outlive it: norms of 4096 x 18944 fp32 89 -> 85 us, without this case 81)
  if (NORM && __any_sync(0xffffffffu, !in_range(mean, ss, top))) {
    far_row<F32, VEC>(row, a.gain, a.eps, a.codes + (long long)m * a.ldc, a.scale + m, K);
    return;
  }
  // rounding is monotonic: the largest |gain x| times r is the largest |y|
  const float rms = NORM ? rsqrtf(mean) : 1.f;
  const float big = NORM ? __uint_as_float(top) * rms : __uint_as_float(top);
  const bool real = top < 0x7f800000u && big < INFINITY;
  const float s = fmaxf(__fmul_rn(big, 1.f / 127.f), 0x1p-126f);
  const float inv = __frcp_rn(s);
  if (threadIdx.x == 0) a.scale[m] = real ? s : __uint_as_float(0x7fffffffu);
  int8_t* out = a.codes + (long long)m * a.ldc;
  auto finish = [&](const Unit<F32>& u, int at) {
    float v[kUnit];
    if (NORM) gained<F32>(u, a.gain, at, K, v);
    else widen<F32>(u, v);
    store_unit(out, at, K, real ? round_unit<NORM>(v, rms, s, inv) : make_uint2(0u, 0u));
  };
  if (!LONG) {
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = threadIdx.x * kUnit + u * step;
      if (at < K) finish(r[u], at);
    }
  } else {
    for (int at = threadIdx.x * kUnit; at < K; at += step) finish(load_unit<F32, VEC>(row, at, K), at);
  }
}

template <bool F32, bool VEC>
cudaError_t launch_typed(const QuantI8Args& a, cudaStream_t s) {
  const int units = (a.K + kUnit - 1) / kUnit;
  int threads = ((units + kUnits - 1) / kUnits + 31) / 32 * 32;
  const bool lng = threads > (a.gain ? kMost<F32, VEC, true, false> : kMost<F32, VEC, false, false>);
  if (lng) threads = kMost<F32, VEC, false, true>;
  void (*k)(const QuantI8Args);
  if (a.gain) k = lng ? k_quant_i8<F32, VEC, true, true> : k_quant_i8<F32, VEC, true, false>;
  else k = lng ? k_quant_i8<F32, VEC, false, true> : k_quant_i8<F32, VEC, false, false>;
  // 256 threads to a CTA where there are rows enough (a CTA of one warp a row: 16384 x 384 18 us)
  int rows = threads < 256 ? 256 / threads : 1;
  while (rows > 1 && a.M < 512 * rows) --rows;
  return launch_pdl(k, dim3((unsigned)((a.M + rows - 1) / rows)), dim3((unsigned)threads, (unsigned)rows), 0, s, a);
}

}  // namespace

cudaError_t launch_quant_i8(const QuantI8Args& a, cudaStream_t s) {
  if (a.M <= 0 || a.K <= 0) return cudaSuccess;
  const bool vec = ((uintptr_t)a.x & 15) == 0 && (a.ldx * (a.f32 ? 4 : 2)) % 16 == 0;
  if (a.f32) return vec ? launch_typed<true, true>(a, s) : launch_typed<true, false>(a, s);
  return vec ? launch_typed<false, true>(a, s) : launch_typed<false, false>(a, s);
}

}  // namespace bs
