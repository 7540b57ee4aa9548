// The rules of constrained decoding on logits, and the confidence pass under them.  For a row of request i:
//   y = z;  token in the context:  y = y > 0 ? y / rho : y rho;  generated c > 0 times:  y = y - (phi c + alpha);
//   y = y + bias;  not allowed by the row's grammar mask, or the mask id:  y = -inf,
// every step rounded to fp32.  The first operator stores y; the second reduces it to tok = argmax y (the lowest of equal
// ones) and conf = exp(max - logsumexp) without storing it.
//
// Bound by memory: a row of logits is read once.  The rules touch few entries of a row (the context's tokens, the
// biases), so a pass over all entries only looks up one bit an entry, and the touched ones are taken one by one.  A
// vocabulary is cut into up to eight chunks; the CTA of a chunk keeps, for one request at a time, a count for every entry
// of the chunk in shared memory (context tokens are counted by shared-memory atomics: integers, so their order does not
// matter) and the bits of the entries that no rule but the grammar touches.  It walks the consecutive rows of its span
// and builds the table anew when the request changes.  For the confidence the CTAs of a span are a cluster; every warp
// leaves (max, sum, argmax) of its part of a row in shared memory, and these are joined in a fixed order over distributed
// shared memory, so that one launch without scratch does.
#include <math.h>

#include <mutex>

#include "decode_ops.cuh"
#include "tc_common.cuh"

namespace bs {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kRowsAtOnce = 32;            // rows whose parts are kept before they are joined
constexpr int kMaxChunks = 8;
constexpr unsigned kInPrompt = 0x80000000u;

constexpr int kListed = 4096;              // touched entries that a table lists (those beyond are found by their bits)

struct Part {
  float m, s;
  int at;
};

struct Plan {
  int chunks;            // CTAs that share a row (a cluster for the confidence)
  int chunk;             // entries of a chunk: a multiple of 32
  int spans;
};

__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float y) { *p = y; }
__device__ __forceinline__ void put(bf16* p, float y) { *p = __float2bfloat16_rn(y); }

// E elements of 16 bytes, as fp32.
template <typename T>
struct Vec {
  static constexpr int E = 16 / sizeof(T);
};
__device__ __forceinline__ void widen(const uint4& u, float* v, const float*) {
  v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void widen(const uint4& u, float* v, const bf16*) {
  const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// The table of one request's rules over the entries [c0, c0 + n) of a CTA.
struct Table {
  unsigned* plain;       // bit set: only the grammar decides about this entry; the word behind the last is zero
  unsigned* biased;      // bit set: the request has a bias for this entry
  unsigned* count;       // kInPrompt | times generated
  unsigned* list;        // the touched entries in ascending order: entry | (1 + place of its first bias, or 0) << 16
  int listed;            // how many of them
  int cut;               // the touched entries of words from this one on are not listed
  int c0, n, words;
  int bias_lo, bias_hi;  // the request's biases (all of them)
  float rho, alpha, phi;
};

__device__ __forceinline__ unsigned in_range(const Table& t, int w, int mask_id) {
  const int left = t.n - w * 32;
  unsigned bits = left >= 32 ? 0xffffffffu : (left <= 0 ? 0u : (1u << left) - 1u);
  const int m = mask_id - t.c0;
  if (m >= 0 && (m >> 5) == w) bits &= ~(1u << (m & 31));
  return bits;
}

__device__ void raise(const RulesArgs& a) {
  if (a.error_flag) atomicMax(a.error_flag, 100 + SITE_RULES);
}

// The place of the first bias of token id (ids ascend), bias_hi if there is none.
__device__ __forceinline__ int find_bias(const RulesArgs& a, const Table& t, int id) {
  int lo = t.bias_lo, hi = t.bias_hi;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(a.bias_tok + mid) < id) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

// All threads of the CTA; req < 0: no rules but the grammar.
__device__ void build_table(const RulesArgs& a, Table& t, int req) {
  __shared__ int s_first[kWarps + 1], s_cut;
  int begin = 0, gen = 0, end = 0, lo = 0, hi = 0;
  t.rho = 1.f; t.alpha = 0.f; t.phi = 0.f;
  if (req >= 0 && a.ctx) {
    begin = __ldg(a.ctx_begin + req); gen = __ldg(a.ctx_gen + req); end = __ldg(a.ctx_end + req);
    if (a.repetition) t.rho = __ldg(a.repetition + req);
    if (a.presence) t.alpha = __ldg(a.presence + req);
    if (a.frequency) t.phi = __ldg(a.frequency + req);
  }
  if (req >= 0 && a.bias_at) { lo = __ldg(a.bias_at + req); hi = __ldg(a.bias_at + req + 1); }
  __syncthreads();                                           // the rows before are done with the table
  for (int w = threadIdx.x; w < t.words; w += kThreads) {
    t.plain[w] = in_range(t, w, a.mask_id);
    t.biased[w] = 0u;
  }
  if (a.ctx)
    for (int i = threadIdx.x * 4; i < t.words * 32; i += kThreads * 4) *reinterpret_cast<uint4*>(t.count + i) = make_uint4(0, 0, 0, 0);
  if (threadIdx.x == 0) s_cut = t.words;
  if (begin < 0 || gen < begin || end < gen || end > a.ctx_total || lo < 0 || hi < lo || hi > a.bias_total) {
    if (threadIdx.x == 0 && t.c0 == 0) raise(a);
    if (begin < 0 || gen < begin || end < gen || end > a.ctx_total) begin = gen = end = 0;
    if (lo < 0 || hi < lo || hi > a.bias_total) lo = hi = 0;
  }
  t.bias_lo = lo; t.bias_hi = hi;
  __syncthreads();
  for (int i = begin + threadIdx.x; i < end; i += kThreads) {
    const int id = __ldg(a.ctx + i), e = id - t.c0;
    if ((unsigned)id >= (unsigned)a.vocab) {
      if (t.c0 == 0) raise(a);
    } else if (e >= 0 && e < t.n && id != a.mask_id) {
      if (i >= gen) atomicAdd(t.count + e, 1u);
      else atomicOr(t.count + e, kInPrompt);
      atomicAnd(t.plain + (e >> 5), ~(1u << (e & 31)));
    }
  }
  for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
    const int id = __ldg(a.bias_tok + i), e = id - t.c0;
    if ((unsigned)id >= (unsigned)a.vocab || (i > lo && __ldg(a.bias_tok + i - 1) > id)) {
      if (t.c0 == 0) raise(a);
    } else if (e >= 0 && e < t.n && id != a.mask_id) {
      atomicOr(t.biased + (e >> 5), 1u << (e & 31));
      atomicAnd(t.plain + (e >> 5), ~(1u << (e & 31)));
    }
  }
  __syncthreads();
  // list the touched entries in order: thread i takes `each` words
  const int each = (t.words + kThreads - 1) / kThreads, lane = threadIdx.x & 31;
  int mine = 0;
  for (int w = threadIdx.x * each; w < min(t.words, (int)(threadIdx.x + 1) * each); ++w)
    mine += __popc(in_range(t, w, a.mask_id) & ~t.plain[w]);
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) s_first[threadIdx.x >> 5] = upto;
  __syncthreads();
  int before = lane < kWarps ? s_first[lane] : 0;
  const int total = __reduce_add_sync(0xffffffffu, before);
  before = __reduce_add_sync(0xffffffffu, lane < (int)(threadIdx.x >> 5) ? before : 0);
  int at = before + upto - mine;
  if (mine)
    for (int w = threadIdx.x * each; w < min(t.words, (int)(threadIdx.x + 1) * each); ++w) {
      unsigned bits = in_range(t, w, a.mask_id) & ~t.plain[w];
      const unsigned with = t.biased[w];
      if (at + __popc(bits) > kListed) {
        if (bits) atomicMin(&s_cut, w);
        break;
      }
      for (; bits; bits &= bits - 1) {
        const int b = __ffs(bits) - 1, e = w * 32 + b;
        unsigned place = 0u;
        if ((with >> b) & 1u) place = (unsigned)min(find_bias(a, t, t.c0 + e) - t.bias_lo + 1, 0xffff);
        t.list[at++] = (unsigned)e | place << 16;
      }
    }
  __syncthreads();
  t.cut = s_cut;
  t.listed = total;
  if (t.cut < t.words) {                                     // entries of the words before: count them again
    int n = 0;
    for (int w = lane; w < t.cut; w += 32) n += __popc(in_range(t, w, a.mask_id) & ~t.plain[w]);
    t.listed = __reduce_add_sync(0xffffffffu, n);
  }
}

// y of entry e (of the chunk), which some rule touches, from its logit; place: where its first bias is, as listed.
__device__ __forceinline__ float touched(const RulesArgs& a, const Table& t, int e, unsigned place, float z) {
  float y = z;
  if (a.ctx) {
    const unsigned c = t.count[e];
    if (c) {
      y = y > 0.f ? __fdiv_rn(y, t.rho) : __fmul_rn(y, t.rho);
      const unsigned made = c & ~kInPrompt;
      if (made) y = __fsub_rn(y, __fadd_rn(__fmul_rn(t.phi, (float)made), t.alpha));
    }
  }
  if (place) {
    const int id = t.c0 + e;
    for (int i = place < 0xffffu ? t.bias_lo + (int)place - 1 : find_bias(a, t, id); i < t.bias_hi && __ldg(a.bias_tok + i) == id; ++i)
      y = __fadd_rn(y, __ldg(a.bias_val + i));
  }
  return y;
}

// Calls f(entry, place) for the touched entries that the mask (nullable) allows, each by one thread of the CTA.
template <typename F>
__device__ __forceinline__ void each_touched(const RulesArgs& a, const Table& t, const unsigned* mask, F f) {
  for (int i = threadIdx.x; i < t.listed; i += kThreads) {
    const unsigned r = t.list[i], e = r & 0xffffu;
    if (!mask || ((__ldg(mask + (e >> 5)) >> (e & 31)) & 1u)) f((int)e, r >> 16);
  }
  for (int w = t.cut + threadIdx.x; w < t.words; w += kThreads) {
    unsigned bits = in_range(t, w, a.mask_id) & ~t.plain[w];
    if (mask && bits) bits &= __ldg(mask + w);
    for (; bits; bits &= bits - 1) {
      const int b = __ffs(bits) - 1;
      f(w * 32 + b, (t.biased[w] >> b) & 1u ? 0xffffu : 0u);
    }
  }
}

// E bits from entry p of the chunk on, of a row of bits with a word behind the last.
template <bool ALIGNED, typename F>
__device__ __forceinline__ unsigned bits_at(int p, F word) {
  const int w = p >> 5;
  if (ALIGNED) return word(w) >> (p & 31);
  return __funnelshift_r(word(w), word(w + 1), p & 31);
}

// A row's chunk as vectors: entries [first, first + E nv) start at 16-byte boundaries; up to 2 E - 2 are left over.
struct Cut {
  int first, nv;
};
template <typename T, bool ALIGNED>
__device__ __forceinline__ Cut cut_of(const T* z, int n) {
  constexpr int E = Vec<T>::E;
  const int shift = ALIGNED ? 0 : (int)(((uintptr_t)z & 15) / sizeof(T));
  const int first = min(n, (E - shift) % E);
  return Cut{first, (n - first) / E};
}
// The i-th entry left over, or -1.
template <int E>
__device__ __forceinline__ int left_over(const Cut& c, int n, int i) {
  const int e = i < c.first ? i : c.first + c.nv * E + i - c.first;
  return e < n ? e : -1;
}

__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

// Request and grammar mask of a row, -1: none.
struct Row {
  int req, mask;
};
__device__ __forceinline__ Row row_of(const RulesArgs& a, int row) {
  return Row{a.row_req ? __ldg(a.row_req + row) : row, a.allowed ? (a.row_mask ? __ldg(a.row_mask + row) : row) : -1};
}
__device__ __forceinline__ bool valid(const RulesArgs& a, const Row& r) {
  return r.req >= -1 && r.req < a.n_reqs && r.mask >= -1 && r.mask < a.n_masks;
}

__device__ __forceinline__ unsigned ordered(float m) {       // unsigned order of floats (no NaN)
  const unsigned u = __float_as_uint(m);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(unsigned u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
// exp(m - top) of a part's maximum, 1 where they are equal (infinities too).
__device__ __forceinline__ float weight(float m, float top) { return m == top ? 1.f : __expf(m - top); }

// Joins (m, s, at) over the lanes of a warp; at = lowest index among the parts that hold the maximum.
__device__ __forceinline__ Part join_lanes(Part p) {
  const float top = unordered(__reduce_max_sync(0xffffffffu, ordered(p.m)));
  float s = p.s * weight(p.m, top);
  const unsigned at = __reduce_min_sync(0xffffffffu, p.m == top ? (unsigned)p.at : 0x7fffffffu);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return Part{top, s, (int)at};
}

__device__ Table make_table(const RulesArgs& a, const Plan& pl, int chunk, unsigned* smem) {
  Table t;
  t.c0 = chunk * pl.chunk;
  t.n = max(0, min(pl.chunk, a.vocab - t.c0));
  t.words = pl.chunk / 32;
  t.list = smem;
  t.count = smem + kListed;
  t.plain = t.count + (a.ctx ? pl.chunk : 0);
  t.biased = t.plain + t.words + 4;
  if (threadIdx.x < 4) t.plain[t.words + threadIdx.x] = 0u;
  return t;
}

// Joins one more value into a running (max, sum, argmax) whose entries come in ascending order.
__device__ __forceinline__ void join_one(Part& p, float y, int at) {
  if (y > p.m) {
    p.s = p.s * weight(p.m, y) + 1.f;
    p.m = y;
    p.at = at;
  } else if (y > -INFINITY || y != y) {
    p.s += weight(y, p.m);
  }
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, 2) k_rules_confidence(const RulesArgs a, const Plan pl, int* tok, float* conf) {
  constexpr int E = Vec<T>::E, kBatch = E == 4 ? 5 : 3;      // vectors a thread has in flight
  extern __shared__ __align__(16) unsigned smem[];
  __shared__ Part parts[kRowsAtOnce][kWarps];
  pdl_wait();
  pdl_trigger();
  const int chunk = pl.chunks > 1 ? (int)cluster_rank() : 0;
  const int span = blockIdx.x / pl.chunks;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r0 = (int)((long long)a.n_rows * span / pl.spans), r1 = (int)((long long)a.n_rows * (span + 1) / pl.spans);
  Table t = make_table(a, pl, chunk, smem);
  const T* logits = static_cast<const T*>(a.logits);
  int cur = -2;
  Row next = row_of(a, r0);
  for (int rb = r0; rb < r1; rb += kRowsAtOnce) {
    const int re = min(r1, rb + kRowsAtOnce);
    for (int row = rb; row < re; ++row) {
      const Row me = next;
      if (row + 1 < r1) next = row_of(a, row + 1);
      if (!valid(a, me)) {
        if (threadIdx.x == 0 && chunk == 0) raise(a);
        if (lane == 0) parts[row - rb][warp] = Part{-INFINITY, 0.f, 0x7fffffff};
        continue;
      }
      const T* z = logits + (long long)row * a.ld + t.c0;
      if (me.req != cur) {
        build_table(a, t, me.req);
        cur = me.req;
      }
      const unsigned* mask = me.mask < 0 ? nullptr : a.allowed + me.mask * a.allowed_ld + (t.c0 >> 5);
      const Cut c = cut_of<T, ALIGNED>(z, t.n);
      auto usable = [&](int w) -> unsigned {
        const unsigned p = t.plain[w];
        return mask && p ? p & __ldg(mask + w) : p;
      };
      float m = -INFINITY, s = 0.f;
      int best = 0;                                          // first entry of the vector that holds m
      for (int j0 = threadIdx.x; j0 < c.nv; j0 += kThreads * kBatch) {
        unsigned bits[kBatch];
        uint4 u[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int j = j0 + b * kThreads;
          bits[b] = 0u;
          u[b] = make_uint4(0u, 0u, 0u, 0u);
          if (j < c.nv) u[b] = __ldcs(reinterpret_cast<const uint4*>(z + c.first) + j);
          if (j < c.nv) bits[b] = bits_at<ALIGNED>(c.first + j * E, usable);
        }
        float v[kBatch][E];
        float top = m;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          widen(u[b], v[b], z);
#pragma unroll
          for (int e = 0; e < E; ++e) v[b][e] = (bits[b] >> e) & 1u ? v[b][e] : -INFINITY;
          float vm = v[b][0];
#pragma unroll
          for (int e = 1; e < E; ++e) vm = fmaxf(vm, v[b][e]);
          if (vm > top) {
            top = vm;
            best = c.first + (j0 + b * kThreads) * E;
          }
        }
        if (top > m) {
          s *= weight(m, top);
          m = top;
        }
        if (m == INFINITY) {
#pragma unroll
          for (int b = 0; b < kBatch; ++b)
#pragma unroll
            for (int e = 0; e < E; ++e) s += v[b][e] == INFINITY ? 1.f : (v[b][e] == v[b][e] ? 0.f : v[b][e]);
        } else {
          const float ref = m > -INFINITY ? m : 0.f;
#pragma unroll
          for (int b = 0; b < kBatch; ++b)
#pragma unroll
            for (int e = 0; e < E; ++e) s += __expf(v[b][e] - ref);
        }
      }
      Part one{-INFINITY, 0.f, 0x7fffffff};
      if (threadIdx.x < 2 * E) {
        const int e = left_over<E>(c, t.n, threadIdx.x);
        if (e >= 0 && ((usable(e >> 5) >> (e & 31)) & 1u)) join_one(one, value(z + e), t.c0 + e);
      }
      Part some{-INFINITY, 0.f, 0x7fffffff};
      each_touched(a, t, mask, [&](int e, unsigned place) { join_one(some, touched(a, t, e, place, value(z + e)), t.c0 + e); });
      // the warp's part: the lowest entry among the lanes that hold the maximum
      const float top = unordered(__reduce_max_sync(0xffffffffu, ordered(fmaxf(m, fmaxf(one.m, some.m)))));
      unsigned at = 0x7fffffffu;
      if (m == top && top > -INFINITY) {
#pragma unroll
        for (int e = E - 1; e >= 0; --e) {
          const int p = best + e;
          if (((usable(p >> 5) >> (p & 31)) & 1u) && value(z + p) == top) at = (unsigned)(t.c0 + p);
        }
      }
      if (one.m == top) at = min(at, (unsigned)one.at);
      if (some.m == top) at = min(at, (unsigned)some.at);
      at = __reduce_min_sync(0xffffffffu, at);
      s = s * weight(m, top) + one.s * weight(one.m, top) + some.s * weight(some.m, top);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0) parts[row - rb][warp] = Part{top, s, (int)at};
    }
    // join the parts of these rows: row i by CTA i mod chunks
    if (pl.chunks > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
    for (int i = chunk + warp * pl.chunks; i < re - rb; i += kWarps * pl.chunks) {
      Part p{-INFINITY, 0.f, 0x7fffffff};
      for (int k = lane; k < kWarps * pl.chunks; k += 32) {
        const int c = k / kWarps, w = k % kWarps;
        Part o;
        if (pl.chunks > 1) {
          const unsigned from = tc::smem_u32(&parts[i][w]);
          unsigned far;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(far) : "r"(from), "r"(c));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(o.m) : "r"(far) : "memory");
          asm volatile("ld.shared::cluster.f32 %0, [%1+4];" : "=f"(o.s) : "r"(far) : "memory");
          asm volatile("ld.shared::cluster.s32 %0, [%1+8];" : "=r"(o.at) : "r"(far) : "memory");
        } else {
          o = parts[i][w];
        }
        const float top = fmaxf(p.m, o.m);
        p.at = o.m > p.m ? o.at : (o.m == p.m ? min(p.at, o.at) : p.at);
        p.s = p.s * weight(p.m, top) + o.s * weight(o.m, top);
        p.m = top;
      }
      p = join_lanes(p);
      if (lane == 0) {
        tok[rb + i] = p.m > -INFINITY ? p.at : -1;
        conf[rb + i] = p.m > -INFINITY ? __fdiv_rn(1.f, p.s) : (p.s == p.s ? 0.f : p.s);
      }
    }
    if (pl.chunks > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
  }
}

__device__ __forceinline__ uint4 narrow(const float* v, const float*) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 narrow(const float* v, const bf16*) {
  unsigned w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
    w[k] = *reinterpret_cast<const unsigned*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Stores y.  In place only entries that change are written: the touched ones and those that are not allowed.
template <typename T, bool ALIGNED, bool INPLACE>
__global__ void __launch_bounds__(kThreads, 2) k_logit_rules(const RulesArgs a, const Plan pl, T* out, long long out_ld) {
  constexpr int E = Vec<T>::E, kBatch = INPLACE ? 1 : 4;
  constexpr unsigned kAll = (1u << E) - 1u;
  extern __shared__ __align__(16) unsigned smem[];
  pdl_wait();
  pdl_trigger();
  const int chunk = (int)blockIdx.x % pl.chunks, span = (int)blockIdx.x / pl.chunks;
  const int r0 = (int)((long long)a.n_rows * span / pl.spans), r1 = (int)((long long)a.n_rows * (span + 1) / pl.spans);
  Table t = make_table(a, pl, chunk, smem);
  int cur = -2;
  Row next = row_of(a, r0);
  for (int row = r0; row < r1; ++row) {
    const Row me = next;
    if (row + 1 < r1) next = row_of(a, row + 1);
    if (!valid(a, me)) {
      if (threadIdx.x == 0 && chunk == 0) raise(a);
      continue;
    }
    const T* z = static_cast<const T*>(a.logits) + (long long)row * a.ld + t.c0;
    T* y = out + (long long)row * out_ld + t.c0;
    if (me.req != cur) {
      build_table(a, t, me.req);
      cur = me.req;
    }
    const unsigned* mask = me.mask < 0 ? nullptr : a.allowed + me.mask * a.allowed_ld + (t.c0 >> 5);
    const Cut c = cut_of<T, ALIGNED>(z, t.n);
    // bits of the entries that may stay, and of those that no other rule touches
    auto allow = [&](int w) -> unsigned {
      const unsigned in = in_range(t, w, a.mask_id);
      return mask && in ? in & __ldg(mask + w) : in;
    };
    auto plain = [&](int w) -> unsigned { return t.plain[w]; };
    for (int j0 = threadIdx.x; j0 < c.nv; j0 += kThreads * kBatch) {
      uint4 u[kBatch];
      unsigned keep[kBatch], calm[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int j = j0 + b * kThreads;
        keep[b] = calm[b] = 0u;
        if (j < c.nv) {
          if (!INPLACE) u[b] = __ldcs(reinterpret_cast<const uint4*>(z + c.first) + j);
          keep[b] = bits_at<ALIGNED>(c.first + j * E, allow) & kAll;
          calm[b] = bits_at<ALIGNED>(c.first + j * E, plain) & keep[b];
        }
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int j = j0 + b * kThreads, p = c.first + j * E;
        if (j >= c.nv) break;
        const unsigned put_now = (INPLACE ? 0u : calm[b]) | (kAll & ~keep[b]);    // the others come below
        float v[E];
        if (!INPLACE) widen(u[b], v, z);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = !INPLACE && ((keep[b] >> e) & 1u) ? v[e] : -INFINITY;
        if (put_now == kAll && (ALIGNED || INPLACE)) {
          __stcs(reinterpret_cast<uint4*>(y + p), narrow(v, z));
        } else if (put_now) {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if ((put_now >> e) & 1u) put(y + p + e, v[e]);
        }
      }
    }
    if (threadIdx.x < 2 * E) {
      const int e = left_over<E>(c, t.n, threadIdx.x);
      if (e >= 0) {
        const bool stays = (allow(e >> 5) >> (e & 31)) & 1u, alone = (t.plain[e >> 5] >> (e & 31)) & 1u;
        if (!stays) put(y + e, -INFINITY);
        else if (alone && !INPLACE) put(y + e, value(z + e));
      }
    }
    each_touched(a, t, mask, [&](int e, unsigned place) { put(y + e, touched(a, t, e, place, value(z + e))); });
  }
}

// One-time set-up per device.
struct DevInfo {
  int num_sms;
  int ok;
};
DevInfo g_dev[kMaxDevices];
std::mutex g_mutex;

constexpr int kMaxSmem = 208 * 1024;         // the table of an eighth of the largest vocabulary

template <typename T>
using ConfKernel = void (*)(const RulesArgs, const Plan, int*, float*);
template <typename T>
using RuleKernel = void (*)(const RulesArgs, const Plan, T*, long long);

template <typename T>
bool allow_smem() {
  bool ok = true;
  for (ConfKernel<T> k : {k_rules_confidence<T, true>, k_rules_confidence<T, false>})
    ok = ok && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) == cudaSuccess;
  for (RuleKernel<T> k : {k_logit_rules<T, true, true>, k_logit_rules<T, true, false>, k_logit_rules<T, false, true>, k_logit_rules<T, false, false>})
    ok = ok && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) == cudaSuccess;
  return ok;
}

const DevInfo* dev_info() {
  DevInfo* d = device_slot(g_dev);
  if (!d) return nullptr;
  std::lock_guard<std::mutex> lock(g_mutex);
  if (!d->num_sms) {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return nullptr;
    d->ok = allow_smem<float>() && allow_smem<bf16>();
    if (!d->ok) cudaGetLastError();
    d->num_sms = n;
  }
  return d;
}

size_t smem_of(const RulesArgs& a, int chunk) { return (kListed + (a.ctx ? (size_t)chunk : 0) + 2 * (size_t)(chunk / 32) + 8) * 4; }

Plan plan_of(const RulesArgs& a, int num_sms) {
  Plan pl;
  pl.chunks = 1;
  while (pl.chunks < kMaxChunks && a.vocab > 16384 * pl.chunks) pl.chunks *= 2;
  pl.chunk = ((a.vocab + pl.chunks - 1) / pl.chunks + 31) / 32 * 32;
  int per_sm = (int)(225 * 1024 / (smem_of(a, pl.chunk) + 8 * 1024));
  if (per_sm > 2) per_sm = 2;
  int spans = num_sms * per_sm / pl.chunks;
  pl.spans = spans < a.n_rows ? spans : a.n_rows;
  return pl;
}

template <typename T>
cudaError_t launch_conf(const RulesArgs& a, const Plan& pl, int* tok, float* conf, cudaStream_t s) {
  const bool aligned = (a.ld * sizeof(T)) % 16 == 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(pl.spans * pl.chunks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem_of(a, pl.chunk);
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)pl.chunks; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, aligned ? k_rules_confidence<T, true> : k_rules_confidence<T, false>, a, pl, tok, conf);
}

template <typename T>
cudaError_t launch_rules(const RulesArgs& a, const Plan& pl, T* out, long long out_ld, cudaStream_t s) {
  const bool aligned = (a.ld * sizeof(T)) % 16 == 0 && (out_ld * sizeof(T)) % 16 == 0, inplace = out == a.logits;
  RuleKernel<T> k = inplace ? (aligned ? k_logit_rules<T, true, true> : k_logit_rules<T, false, true>)
                            : (aligned ? k_logit_rules<T, true, false> : k_logit_rules<T, false, false>);
  return launch_pdl(k, dim3((unsigned)(pl.spans * pl.chunks)), dim3(kThreads), smem_of(a, pl.chunk), s, a, pl, out, out_ld);
}

}  // namespace

cudaError_t launch_rules_confidence(const RulesArgs& a, int* tok, float* conf, cudaStream_t s) {
  if (a.n_rows <= 0) return cudaSuccess;
  const DevInfo* d = dev_info();
  if (!d || !d->ok) return cudaErrorNotSupported;
  const Plan pl = plan_of(a, d->num_sms);
  return a.bf16_logits ? launch_conf<bf16>(a, pl, tok, conf, s) : launch_conf<float>(a, pl, tok, conf, s);
}

cudaError_t launch_logit_rules(const RulesArgs& a, void* out, long long out_ld, cudaStream_t s) {
  if (a.n_rows <= 0) return cudaSuccess;
  const DevInfo* d = dev_info();
  if (!d || !d->ok) return cudaErrorNotSupported;
  const Plan pl = plan_of(a, d->num_sms);
  return a.bf16_logits ? launch_rules<bf16>(a, pl, (bf16*)out, out_ld, s) : launch_rules<float>(a, pl, (float*)out, out_ld, s);
}

}  // namespace bs
