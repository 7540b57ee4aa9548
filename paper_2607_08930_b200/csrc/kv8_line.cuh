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

// Largest factor of a query row's scores: times a K scale of at most 2^40 it stays finite.  Rows held to it (their largest
// element is 2^90 at least) have all their scores scaled down alike; any two that differ are still so far apart, by 2^14
// at least, that the softmax is the larger one's alone.
constexpr float kMaxFactor = 0x1p87f;

// A cut item: the workers that hold parts of it, its first query token, number of query rows (0: nothing is cut) and
// kv head; whether worker c0 began with it (its part is then in the even slot, as everybody else's is).
struct alignas(16) Cut { int c0, c1, t0, nrows, head, even, pad0, pad1; };

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
  int direct;            // 0: the line of work.  > 0: workers of whole items, this many for the tiles of a (row, kv head)
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

// A worker's share: `units` of the line from unit `at` of the item (row, head, tile) on; 0 units: an idle worker.
struct LineShare {
  long long units;
  int row, head, tile, at;
};
template <int THREADS, int GROUPS>
struct LineShared {
  long long warp[THREADS / 32];
  LineShare share[GROUPS];
};

// Forms the shares of the CTA's GROUPS workers (by all THREADS threads; at least `least` units beyond the cost each) and
// writes their cuts down; also flags rows that do not fit and writes zeros for rows that see nothing.  The divisions are
// all here, in one place: the walk below has none.
template <int THREADS, int GROUPS, int KEYS, int DH>
__device__ __forceinline__ void line_share(const LineParams& p, int item_cost, int least, LineShared<THREADS, GROUPS>& s) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per_thread = (p.n_rows + THREADS - 1) / THREADS;       // consecutive rows
  const int r0 = min(tid * per_thread, p.n_rows), r1 = min(r0 + per_thread, p.n_rows);
  long long mine = 0;
#pragma unroll 1
  for (int r = r0; r < r1; ++r) {
    RowInfo ri;
    if (!row_info<KEYS>(p, r, ri) && blockIdx.x == 0 && p.error_flag) atomicMax(p.error_flag, 100 + SITE_ATTN_KV8);
    mine += ri.units(p.hkv, item_cost);
  }
  long long inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) s.warp[warp] = inc;
  if (tid < GROUPS) s.share[tid].units = 0;
  __syncthreads();
  long long total = 0, before = inc - mine;
#pragma unroll 4
  for (int k = 0; k < THREADS / 32; ++k) {
    if (k < warp) before += s.warp[k];
    total += s.warp[k];
  }
  const long long workers = max(1ll, min((long long)gridDim.x * GROUPS, total / (item_cost + least)));
#pragma unroll 1
  for (int k = 0; k < GROUPS; ++k) {
    const long long me = (long long)blockIdx.x * GROUPS + k;
    const bool idle = total == 0 || me >= workers;
    if (idle && tid == 0) p.cuts[me].nrows = 0;
    if (idle) continue;
    const long long u = share_start(me, total, workers);
    if (u < before || u >= before + mine) continue;                // one thread of the CTA goes on
    long long first = before;                                      // units before row r
    RowInfo ri;
    int r = r0;
    for (;; ++r) {
      row_info<KEYS>(p, r, ri);
      if (u - first < ri.units(p.hkv, item_cost)) break;
      first += ri.units(p.hkv, item_cost);
    }
    const int per = ri.item_units(item_cost), item = (int)((u - first) / per), at = (int)((u - first) - (long long)item * per);
    LineShare sh;
    sh.units = share_start(me + 1, total, workers) - u;
    sh.row = r;
    sh.head = item / ri.tiles;
    sh.tile = item - sh.head * ri.tiles;
    sh.at = at;
    s.share[k] = sh;
    Cut c = {};
    if (at > item_cost) {                                          // inside the item's key tiles
      const long long begin = u - at;                              // its first unit; its key tiles begin item_cost later
      c.c0 = share_of(begin + item_cost, total, workers);
      c.c1 = share_of(begin + per - 1, total, workers);
      c.even = begin <= share_start(c.c0, total, workers);
      c.head = sh.head;
      c.t0 = ri.t0 + sh.tile * p.tq;
      c.nrows = min(p.tq, ri.t0 + ri.n - c.t0) * (p.hq / p.hkv);
    }
    p.cuts[me] = c;
  }
#pragma unroll 1
  for (int r = blockIdx.x; r < p.n_rows; r += gridDim.x) {
    RowInfo z;
    row_info<KEYS>(p, r, z);
    if (z.nb == 0) {
      uint4* dst = reinterpret_cast<uint4*>(p.out + (size_t)z.t0 * (p.hq * DH));
#pragma unroll 1
      for (long long i = tid; i < (long long)z.n * (p.hq * DH / 8); i += THREADS) dst[i] = make_uint4(0, 0, 0, 0);
    }
  }
  __syncthreads();
}

// One stretch of an item that a worker holds: key tiles [b0, b1) of nb.
struct LineItem {
  int head, t0, nrows, vis, nb, b0, b1, block0;
  bool opens;                    // the worker's first stretch (its partial slot is the even one)
};
// The worker's item when every item has a worker of its own; false: none.  Flags rows that do not fit.
template <int KEYS>
__device__ __forceinline__ bool direct_item(const LineParams& p, long long worker, int lane, LineItem& it, RowInfo& ri, int& tile) {
  const long long unit = worker / p.direct;                // (row, kv head)
  const int r = (int)(unit / p.hkv);
  tile = (int)(worker - unit * p.direct);
  if (r >= p.n_rows) return false;
  it.head = (int)(unit - (long long)r * p.hkv);
  if (!row_info<KEYS>(p, r, ri) && lane == 0 && p.error_flag) atomicMax(p.error_flag, 100 + SITE_ATTN_KV8);
  it.vis = ri.vis;
  it.nb = it.b1 = ri.nb;
  it.b0 = 0;
  it.block0 = ri.block0;
  it.opens = true;
  return tile < ri.tiles;
}

struct LineWalk {
  long long left;                // units still to go
  int row, head, tile, at;       // the next item; units of it that belong to the worker before
  bool opens;
  RowInfo ri;
  template <int KEYS>
  __device__ __forceinline__ void begin(const LineParams& p, const LineShare& s) {
    left = s.units;
    row = s.row; head = s.head; tile = s.tile; at = s.at;
    opens = true;
    if (left > 0) row_info<KEYS>(p, row, ri);
  }
  template <int KEYS>
  __device__ __forceinline__ bool next(const LineParams& p, int cost, LineItem& it) {
    while (left > 0) {
      while (tile == ri.tiles || ri.nb == 0) {     // on to the next head, or the next row that has anything
        tile = 0;
        if (ri.tiles == 0 || ri.nb == 0 || ++head == p.hkv) {
          head = 0;
          row_info<KEYS>(p, ++row, ri);
        }
      }
      const int per = ri.nb + cost;
      it.b0 = max(0, at - cost);                   // an item's first `cost` units hold no key tile
      it.b1 = left < per - at ? max(0, at + (int)left - cost) : ri.nb;
      it.opens = opens;
      it.head = head;
      it.t0 = ri.t0 + tile * p.tq;
      it.nrows = min(p.tq, ri.t0 + ri.n - it.t0) * (p.hq / p.hkv);
      it.vis = ri.vis;
      it.nb = ri.nb;
      it.block0 = ri.block0;
      left -= per - at;
      at = 0;
      ++tile;
      opens = false;
      if (it.b1 > it.b0) return true;
    }
    return false;
  }
};

}  // namespace bs
