// The line of work that the attention kernels over the 8-bit cache share: every item (row, kv head, tile of query rows)
// stands for its key tiles, in order, after a few units for what starting and ending it costs; worker c of N takes units
// [c T / N, (c + 1) T / N) of the line's T, whatever the rows' lengths are.
#pragma once
#include "kv8.cuh"

namespace bs {

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_fast(float x) {      // exact for powers of two
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A cut item: the workers that hold parts of it, its first query token, number of query rows (0: nothing is cut) and
// kv head; whether worker c0 began with it (its part is then in the even slot, as everybody else's is).
struct Cut { int c0, c1, t0, nrows, head, even, pad0, pad1; };

struct LineParams {
  const bf16* q;
  int q_ld;
  Kv8Cache c;
  bf16* out;
  const int* cu_q;
  const int* kv_base;
  const int* vis;
  int n_rows, M, hq, hkv;
  int tq;                // query tokens per tile
  Cut* cuts;             // scratch: [workers] the item that the boundary in front of a worker's share cuts
  float* part_o;         // scratch: [2 workers][rows of a tile][DH]
  float2* part_ml;       // scratch: [2 workers][rows of a tile] (reference, sum)
  int* error_flag;
};

struct RowInfo {
  int t0, n, vis, nb, tiles;     // first token, tokens, visible keys, key tiles, query tiles
  int block0;                    // first cache block
  __device__ __forceinline__ int item_units(int cost) const { return nb > 0 ? nb + cost : 0; }
  __device__ __forceinline__ long long units(int hkv, int cost) const { return (long long)tiles * hkv * item_units(cost); }
};
// false: indices that do not fit; the row then counts nothing
template <int KEYS>
__device__ __forceinline__ bool row_info(const LineParams& p, int r, RowInfo& w) {
  w.t0 = __ldcg(p.cu_q + r);
  const int t1 = __ldcg(p.cu_q + r + 1);
  w.n = t1 - w.t0;
  w.vis = __ldcg(p.vis + r);
  const int base = __ldcg(p.kv_base + r);
  w.block0 = base / kKv8Block;
  const bool ok = w.t0 >= 0 && w.n >= 0 && t1 <= p.M && w.vis >= 0 && base >= 0 && base % kKv8Block == 0 &&
                  (long long)base + w.vis <= p.c.n_blocks * kKv8Block;
  if (!ok) w.n = w.vis = 0;
  w.nb = (w.vis + KEYS - 1) / KEYS;
  w.tiles = (w.n + p.tq - 1) / p.tq;
  return ok;
}

// First unit of worker c's share, and the worker that holds unit u.
__device__ __forceinline__ long long share_start(long long c, long long total, long long n) { return c * total / n; }
__device__ __forceinline__ int share_of(long long u, long long total, long long n) { return (int)(((u + 1) * n - 1) / total); }

template <int THREADS, int GROUPS>
struct LineShared {
  long long warp[THREADS / 32];
  long long first[GROUPS];       // units before row[]
  int row[GROUPS];
};
struct LineShare {
  long long u0, u1;              // this worker's units; empty for idle workers
  long long first;               // units before `row`
  long long total, workers;
  int row;
};

// The share of worker blockIdx.x * GROUPS + wk, by all THREADS threads of the CTA (GROUPS workers per CTA, at least
// `least` units beyond the cost per share); also flags rows that do not fit and writes zeros for rows that see nothing.
template <int THREADS, int GROUPS, int KEYS, int DH>
__device__ __forceinline__ void line_share(const LineParams& p, int item_cost, int least, LineShared<THREADS, GROUPS>& s, int wk,
                                           LineShare& out) {
  constexpr int kPer = kAttnKv8MaxRows / THREADS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  long long before[kPer], cost[kPer];
  long long total = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (i * THREADS >= p.n_rows) break;
    const int r = i * THREADS + tid;
    long long w = 0;
    if (r < p.n_rows) {
      RowInfo ri;
      if (!row_info<KEYS>(p, r, ri) && blockIdx.x == 0 && p.error_flag) atomicMax(p.error_flag, 100 + SITE_ATTN_KV8);
      w = ri.units(p.hkv, item_cost);
    }
    long long inc = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    if (lane == 31) s.warp[warp] = inc;
    __syncthreads();
    long long b = total;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) {
      if (k < warp) b += s.warp[k];
      total += s.warp[k];
    }
    before[i] = b + inc - w;
    cost[i] = w;
    __syncthreads();
  }
  const long long workers = max(1ll, min((long long)gridDim.x * GROUPS, total / (item_cost + least)));
#pragma unroll
  for (int k = 0; k < GROUPS; ++k) {
    const long long u = share_start((long long)blockIdx.x * GROUPS + k, total, workers);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (i * THREADS >= p.n_rows) break;
      if (before[i] <= u && u < before[i] + cost[i]) {     // (rows behind the last one count nothing); one thread at most
        s.row[k] = i * THREADS + tid;
        s.first[k] = before[i];
      }
    }
  }
  for (int r = blockIdx.x; r < p.n_rows; r += gridDim.x) {
    RowInfo z;
    row_info<KEYS>(p, r, z);
    if (z.nb == 0) {
      uint4* dst = reinterpret_cast<uint4*>(p.out + (size_t)z.t0 * (p.hq * DH));
      for (long long i = tid; i < (long long)z.n * (p.hq * DH / 8); i += THREADS) dst[i] = make_uint4(0, 0, 0, 0);
    }
  }
  __syncthreads();
  const long long me = (long long)blockIdx.x * GROUPS + wk;
  out.total = total;
  out.workers = workers;
  out.u0 = out.u1 = 0;
  out.first = 0;
  out.row = 0;
  if (total > 0 && me < workers) {
    out.u0 = share_start(me, total, workers);
    out.u1 = share_start(me + 1, total, workers);
    out.row = s.row[wk];
    out.first = s.first[wk];
  }
}

// One stretch of an item that a worker holds: key tiles [b0, b1) of nb.
struct LineItem {
  int head, t0, nrows, vis, nb, b0, b1, block0;
  bool opens;                    // the worker's first stretch (its partial slot is the even one)
};
struct LineWalk {
  long long u, u0, u1, first;
  int row;
  RowInfo ri;
  bool fresh;
  __device__ __forceinline__ explicit LineWalk(const LineShare& s) : u(s.u0), u0(s.u0), u1(s.u1), first(s.first), row(s.row), fresh(true) {}
  template <int KEYS>
  __device__ __forceinline__ bool next(const LineParams& p, int cost, LineItem& it) {
    const int G = p.hq / p.hkv;
    while (u < u1) {
      if (fresh) row_info<KEYS>(p, row, ri);
      fresh = false;
      for (long long w; u - first >= (w = ri.units(p.hkv, cost));) {
        first += w;
        ++row;
        row_info<KEYS>(p, row, ri);
      }
      const long long local = u - first;
      const int per = ri.item_units(cost);
      const int item = local < 0x7fffffffll ? (int)local / per : (int)(local / per);
      const int at = (int)(local - (long long)item * per);
      it.b0 = max(0, at - cost);                                  // an item's first `cost` units hold no key tile
      it.b1 = (int)min((long long)ri.nb, max(0ll, at + (u1 - u) - cost));
      it.opens = u == u0;
      u += per - at;
      if (it.b1 <= it.b0) continue;
      it.head = item / ri.tiles;
      const int tile = item - it.head * ri.tiles;
      it.t0 = ri.t0 + tile * p.tq;
      it.nrows = min(p.tq, ri.t0 + ri.n - it.t0) * G;
      it.vis = ri.vis;
      it.nb = ri.nb;
      it.block0 = ri.block0;
      return true;
    }
    return false;
  }
};

// Writes down whether the share begins inside an item's key tiles (one thread of a worker that has one).
template <int KEYS>
__device__ __forceinline__ void line_cut(const LineParams& p, int cost, const LineShare& s, int worker) {
  RowInfo ri;
  row_info<KEYS>(p, s.row, ri);
  const int per = ri.item_units(cost), item = (int)((s.u0 - s.first) / per), at = (int)((s.u0 - s.first) % per);
  Cut c = {};
  if (at > cost) {
    const long long begin = s.u0 - at;                     // the item's first unit; its key tiles begin `cost` later
    c.c0 = share_of(begin + cost, s.total, s.workers);
    c.c1 = share_of(begin + per - 1, s.total, s.workers);
    c.even = begin <= share_start(c.c0, s.total, s.workers);
    c.head = item / ri.tiles;
    c.t0 = ri.t0 + item % ri.tiles * p.tq;
    c.nrows = min(p.tq, ri.t0 + ri.n - c.t0) * (p.hq / p.hkv);
  }
  p.cuts[worker] = c;
}

cudaError_t launch_attention_kv8_tc(LineParams p, int dh, int max_ctas, int* ctas, cudaStream_t s);

}  // namespace bs
