// The rules of constrained decoding on logits, and the confidence pass under them.  For a row of request i:
//   y = z;  token in the context:  y = y > 0 ? y / rho : y rho;  generated c > 0 times:  y = y - (phi c + alpha);
//   y = y + bias;  not allowed by the row's grammar mask, or the mask id:  y = -inf,
// every step rounded to fp32.  The first operator stores y; the second reduces it to tok = argmax y (the lowest of equal
// ones) and conf = exp(max - logsumexp) without storing it.
//
// Bound by memory: a row of logits is read once.  The rules touch few entries of a row (the context's tokens, the
// biases): the touched ones are taken one by one from a list, and the pass over all entries passes them over (one bit an
// entry) for the confidence; for the logits it writes them as if no rule touched them, and they are written again.  A vocabulary is dealt in blocks of 512 entries to up to eight CTAs (in turn, because the frequent tokens of a
// vocabulary have its low ids).  A CTA keeps a table of one request at a time in shared memory: the bits of the entries
// that some rule touches, and a list of those entries with how often each was generated.  Every warp queues the context
// tokens of the CTA's share among those it reads; they first set their bits, a prefix sum over the words makes the bits
// places in the list, and the tokens are counted there (shared-memory atomics: integers, so their order does not matter).
// The CTA walks the consecutive rows of its span and builds the table anew when the request changes.  For the confidence
// the CTAs of a span are a cluster; every warp sends (max, sum, argmax) of its part of a row to the CTA that joins the row
// (st.async: nobody waits in between), and the parts of up to 32 rows are joined at a time, in a fixed order: one launch
// without scratch.
//
// Measured on logits [rows][vocabulary]: the confidence of 317 rows of 152064 (16 requests, a grammar on nine rows of ten)
// takes 48 us, 40 without any rule (29 at the copy rate), of 64 single rows of 126464 with contexts of 512 to 4096 tokens 19
// us (17.5 out of the L2); the logits of 64 such rows of 152064 take 20 us (12), of 318 rows of 126464 in 16 bits 43 us (30;
// 35 without the grammar, 29 bare; in place 37 with half of the entries forbidden, 16 without a grammar).  Of the
// confidence's 48 us, 6 pass before and after the rows, 5 building tables, 7.5 for every row of a span (5.8 TB/s), and spans
// have 4 or 5 rows.  Fewer spans of equal lengths: 128 rows 27.3 -> 24.7 us, but 315 rows 49.2 -> 51.4.  Rows that are not
// aligned, 317 of 152063: confidence 50 us without rules, logits 81 (aligned 40 and 69).
#include <math.h>

#include <mutex>
#include <type_traits>

#include "decode_ops.cuh"
#include "tc_common.cuh"

namespace bs {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBlock = 512;                // entries dealt to a CTA at a time
constexpr int kBlockWords = kBlock / 32;
constexpr int kRowsAtOnce = 32;            // rows whose parts are kept before they are joined
constexpr int kPerSm = 4;                  // CTAs of an SM
constexpr int kMaxChunks = 8;
constexpr int kListed = 2944;              // touched entries that are listed at a time
constexpr int kTokens = 8;                 // context tokens a thread has in flight
constexpr int kQueue = 192;                // tokens of a CTA's share that a warp keeps (if it reads more, it reads them twice)
constexpr unsigned kInPrompt = 0x80000000u, kGenerated = 0x80000000u;
constexpr float kLog2e = 1.4426950408889634f;

struct Part {
  float m, s;
  int at;
};
struct __align__(16) Slot {
  Part part;
  int unused;
};

struct Plan {
  int chunks, lg;        // CTAs that share a row (a cluster for the confidence): 1 << lg
  int blocks;            // blocks of a CTA's share (the last may lie behind the vocabulary)
  int listed;            // room in the list
  int spans;
  int early;             // the launch may overlap the kernel before: clusters that fill the device do not all fit beside
                         // one that is leaving, and the last would wait for a first to end (16 x 32 rows: 61 us, else 48)
};

__device__ __forceinline__ float value(const float* p) { return *p; }
__device__ __forceinline__ float value(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float* p, float y) { *p = y; }
__device__ __forceinline__ void put(bf16* p, float y) { *p = __float2bfloat16_rn(y); }

__device__ __forceinline__ float exp2_fast(float x) {        // relative error 2^-22; results below 2^-126 are zero
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// A load that happens only if `on`, without a branch: a loop's loads then all leave before the first is waited for.
__device__ __forceinline__ unsigned load1_if(const void* p, bool on, unsigned otherwise) {
  unsigned u = otherwise;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.nc.u32 %0, [%1];\n\t}"
               : "+r"(u) : "l"(p), "r"((unsigned)on));
  return u;
}
// One logit as it is stored, and its value.  (An ordinary load: in place, other entries of its sector are being written.)
__device__ __forceinline__ unsigned load_bits(const float* p, bool on) {
  unsigned u = 0u;
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.u32 %0, [%1];\n\t}" : "+r"(u) : "l"(p), "r"((unsigned)on) : "memory");
  return u;
}
__device__ __forceinline__ unsigned load_bits(const bf16* p, bool on) {
  unsigned u = 0u;
  asm volatile("{\n\t.reg .pred p;\n\t.reg .u16 h;\n\tsetp.ne.u32 p, %2, 0;\n\tmov.u16 h, 0;\n\t@p ld.global.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}"
               : "=r"(u) : "l"(p), "r"((unsigned)on) : "memory");
  return u;
}
__device__ __forceinline__ float from_bits(unsigned u, const float*) { return __uint_as_float(u); }
__device__ __forceinline__ float from_bits(unsigned u, const bf16*) { return __uint_as_float(u << 16); }
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ unsigned in_cta(unsigned addr, unsigned rank) {
  unsigned r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// Writes a slot of CTA `rank` of the cluster, which counts its 16 bytes on its barrier.
__device__ __forceinline__ void send(const Slot* to, unsigned long long* bar, unsigned rank, float m, float s, unsigned at) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(in_cta(tc::smem_u32(to), rank)), "r"(__float_as_uint(m)), "r"(__float_as_uint(s)), "r"(at), "r"(0u),
                 "r"(in_cta(tc::smem_u32(bar), rank)) : "memory");
}
// Bounded: false if the parts do not arrive in time.  The CTAs of a cluster read the same lists but need not have the same
// work: a list's tokens may all be in one CTA's share, and equal biases are added one by one (a million of them in one row:
// 0.11 s).  So the limit grows with the longest list (context and biases), by a thousand clocks a token and row.
__device__ __forceinline__ bool wait_parts(unsigned long long* bar, unsigned parity, unsigned longest) {
  const long long t0 = clock64(), limit = tc::kWaitCycles + 1024ll * kRowsAtOnce * longest;
  for (;;) {
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(tc::smem_u32(bar)), "r"(parity) : "memory");
    if (ok) return true;
    if (clock64() - t0 > limit) return false;
  }
}

// ---- a request's table ---------------------------------------------------------------------------------------

// Entry e of a CTA's share is token id_of(e).
struct Table {
  unsigned* plain;       // bit set: only the grammar decides about this entry
  unsigned* touched;     // bit set: some other rule does
  unsigned short* place; // of a word's first touched entry among all of them
  unsigned* count;       // of a listed entry (touched, in ascending order): kInPrompt | times generated
  unsigned short* list;  // the entry
  unsigned short* bias;  // 1 + place of its first bias, or 0
  unsigned* queue;       // this warp's tokens of the share: entry | kGenerated
  int queued;            // how many (more than kQueue: they are not all there)
  int total;             // touched entries
  int begin, gen, end;   // the request's context
  int bias_lo, bias_hi;  // its biases
  int chunk, lg, words, vocab, mask_id;
  float rho, alpha, phi;

  __device__ __forceinline__ int id_of(int e) const {
    return ((((e >> 9) << lg) | chunk) << 9) | (e & (kBlock - 1));
  }
  __device__ __forceinline__ bool owns(int id) const { return ((id >> 9) & ((1 << lg) - 1)) == chunk; }
  __device__ __forceinline__ int entry_of(int id) const { return ((id >> 9) >> lg) << 9 | (id & (kBlock - 1)); }
  // the bits of word w that are entries of the vocabulary and not the mask id
  __device__ __forceinline__ unsigned in_range(int w) const {
    const int id = id_of(w * 32), left = vocab - id;
    unsigned bits = left >= 32 ? 0xffffffffu : (left <= 0 ? 0u : (1u << left) - 1u);
    if ((mask_id >> 5) == (id >> 5)) bits &= ~(1u << (mask_id & 31));
    return bits;
  }
  // whether a rule for token id is this CTA's to keep
  __device__ __forceinline__ bool takes(int id) const { return owns(id) && (unsigned)id < (unsigned)vocab && id != mask_id; }
};

__device__ void raise(const RulesArgs& a) {
  if (a.error_flag) atomicMax(a.error_flag, 100 + SITE_RULES);
}

__device__ Table make_table(const RulesArgs& a, const Plan& pl, int chunk, unsigned* smem) {
  Table t;
  t.chunk = chunk; t.lg = pl.lg; t.vocab = a.vocab; t.mask_id = a.mask_id;
  t.words = pl.blocks * kBlockWords;
  t.count = smem;
  t.plain = t.count + pl.listed;
  t.touched = t.plain + t.words;
  t.list = reinterpret_cast<unsigned short*>(t.touched + t.words);
  t.bias = t.list + pl.listed;
  t.place = t.bias + pl.listed;
  t.queue = reinterpret_cast<unsigned*>(t.place + t.words) + (threadIdx.x >> 5) * kQueue;
  t.total = t.queued = 0;
  return t;
}

// Lists the touched entries from the `from`-th on, as many as there is room for.  All threads of the CTA.
__device__ __forceinline__ void list_touched(const RulesArgs& a, const Table& t, const Plan& pl, int from) {
  const int n = min(t.total - from, pl.listed);
  for (int i = threadIdx.x; i < n; i += kThreads) {
    t.count[i] = 0u;
    t.bias[i] = 0;
  }
  __syncthreads();
  // the place of entry e (tokens that occur often write the same entry), or something out of [0, n)
  auto listed = [&](int e) {
    const int at = t.place[e >> 5] + __popc(t.touched[e >> 5] & ((1u << (e & 31)) - 1u)) - from;
    if (at >= 0 && at < n) t.list[at] = (unsigned short)e;
    return at;
  };
  auto counted = [&](int e, bool generated) {
    const int at = listed(e);
    if (at >= 0 && at < n) {
      if (generated) atomicAdd(t.count + at, 1u);
      else atomicOr(t.count + at, kInPrompt);
    }
  };
  if (t.queued <= kQueue) {
    for (int i = threadIdx.x & 31; i < t.queued; i += 32) counted((int)(t.queue[i] & 0xffffu), t.queue[i] & kGenerated);
  } else {
    for (int i = t.begin + threadIdx.x; i < t.end; i += kThreads) {
      const int id = __ldg(a.ctx + i);
      if (t.takes(id)) counted(t.entry_of(id), i >= t.gen);
    }
  }
  for (int i = t.bias_lo + threadIdx.x; i < t.bias_hi; i += kThreads) {
    const int id = __ldg(a.bias_tok + i);
    if (t.takes(id) && (i == t.bias_lo || __ldg(a.bias_tok + i - 1) < id)) {
      const int at = listed(t.entry_of(id));
      if (at >= 0 && at < n) t.bias[at] = (unsigned short)min(i - t.bias_lo + 1, 0xffff);
    }
  }
  __syncthreads();
}

// The table of a request (req < 0: no rules but the grammar).  All threads of the CTA.
__device__ __forceinline__ void build_table(const RulesArgs& a, Table& t, const Plan& pl, int req) {
  __shared__ int s_first[kWarps];
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
  for (int w = threadIdx.x; w < t.words; w += kThreads) t.touched[w] = 0u;
  const bool bad_ctx = begin < 0 || gen < begin || end < gen || end > a.ctx_total;
  const bool bad_bias = lo < 0 || hi < lo || hi > a.bias_total;
  if (bad_ctx) begin = gen = end = 0;
  if (bad_bias) lo = hi = 0;
  if ((bad_ctx || bad_bias) && threadIdx.x == 0 && t.chunk == 0) raise(a);
  t.begin = begin; t.gen = gen; t.end = end; t.bias_lo = lo; t.bias_hi = hi;
  __syncthreads();
  bool bad = false;
  const int lane = threadIdx.x & 31;
  auto touch = [&](int e) { atomicOr(t.touched + (e >> 5), 1u << (e & 31)); };
  // (a thread's first biases are fetched along with the first tokens)
  int b_id = (int)load1_if(a.bias_tok + lo + threadIdx.x, lo + (int)threadIdx.x < hi, 0xffffffffu);
  int b_before = (int)load1_if(a.bias_tok + lo + threadIdx.x - 1, threadIdx.x > 0 && lo + (int)threadIdx.x < hi, 0xffffffffu);
  t.queued = 0;
  for (int i0 = begin + threadIdx.x; i0 - lane < end; i0 += kThreads * kTokens) {
    int id[kTokens];
#pragma unroll
    for (int k = 0; k < kTokens; ++k) id[k] = i0 + k * kThreads < end ? __ldg(a.ctx + i0 + k * kThreads) : -1;
#pragma unroll
    for (int k = 0; k < kTokens; ++k) {
      if (i0 - lane + k * kThreads >= end) break;            // (the same for a warp)
      const bool mine = t.takes(id[k]);
      const unsigned all = __ballot_sync(0xffffffffu, mine);
      const int at = t.queued + __popc(all & ((1u << lane) - 1u));
      if (mine) {
        const int e = t.entry_of(id[k]);
        if (at < kQueue) t.queue[at] = (unsigned)e | (i0 + k * kThreads >= gen ? kGenerated : 0u);
        else touch(e);
      }
      t.queued += __popc(all);
      bad = bad || (i0 + k * kThreads < end && (unsigned)id[k] >= (unsigned)t.vocab);
    }
  }
  __syncwarp();
  for (int i = lane; i < min(t.queued, kQueue); i += 32) touch((int)(t.queue[i] & 0xffffu));
  for (int i = lo + threadIdx.x; i < hi; i += kThreads) {
    // (the first of equal ones, as list_touched has it: each place of the list has a writer whatever the order is)
    if (t.takes(b_id) && b_before < b_id) touch(t.entry_of(b_id));
    bad = bad || (unsigned)b_id >= (unsigned)t.vocab || b_before > b_id;
    b_id = (int)load1_if(a.bias_tok + i + kThreads, i + kThreads < hi, 0xffffffffu);
    b_before = (int)load1_if(a.bias_tok + i + kThreads - 1, i + kThreads < hi, 0xffffffffu);
  }
  if (bad && t.chunk == 0) raise(a);
  __syncthreads();
  const int each = (t.words + kThreads - 1) / kThreads;
  const int w0 = threadIdx.x * each, w1 = min(t.words, w0 + each);
  int mine = 0;
  for (int w = w0; w < w1; ++w) {
    const unsigned bits = t.touched[w];
    t.plain[w] = t.in_range(w) & ~bits;
    mine += __popc(bits);
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) s_first[threadIdx.x >> 5] = upto;
  __syncthreads();
  const int sum = lane < kWarps ? s_first[lane] : 0;
  t.total = __reduce_add_sync(0xffffffffu, sum);
  int at = __reduce_add_sync(0xffffffffu, lane < (int)(threadIdx.x >> 5) ? sum : 0) + upto - mine;
  for (int w = w0; w < w1; ++w) {
    t.place[w] = (unsigned short)at;
    at += __popc(t.touched[w]);
  }
  __syncthreads();
  if (t.total > 0 && t.total <= pl.listed) list_touched(a, t, pl, 0);
}

// y of the i-th listed entry from its logit.
__device__ __forceinline__ float ruled(const RulesArgs& a, const Table& t, int i, float z) {
  float y = z;
  const unsigned c = t.count[i], place = t.bias[i];
  if (c) {
    y = y > 0.f ? __fdiv_rn(y, t.rho) : __fmul_rn(y, t.rho);
    const unsigned made = c & ~kInPrompt;
    if (made) y = __fsub_rn(y, __fadd_rn(__fmul_rn(t.phi, (float)made), t.alpha));
  }
  if (place) {
    const int id = t.id_of(t.list[i]);
    int k = t.bias_lo + (int)place - 1;
    if (place == 0xffffu)                                    // or behind that: ids ascend
      for (int hi = t.bias_hi; k < hi;) {
        const int mid = (k + hi) >> 1;
        if (__ldg(a.bias_tok + mid) < id) k = mid + 1;
        else hi = mid;
      }
    for (; k < t.bias_hi && __ldg(a.bias_tok + k) == id; ++k) y = __fadd_rn(y, __ldg(a.bias_val + k));
  }
  return y;
}

// Calls f(i, z) for the touched entries of a row that the mask (nullable) allows, listed as the i-th, with their logits,
// each by one thread of the CTA.  More of them than there is room for are listed in turns, anew for every row.
template <typename T>
struct Touched {
  int id = 0;
  unsigned word = 0u;      // of the mask
  unsigned z = 0u;
  // fetches what the thread needs for the first of its entries
  __device__ __forceinline__ void begin(const Table& t, const Plan& pl, const unsigned* mask, const T* row) {
    if (t.total <= pl.listed) fetch(t, mask, row, threadIdx.x, t.total);
  }
  __device__ __forceinline__ void fetch(const Table& t, const unsigned* mask, const T* row, int i, int n) {
    id = t.id_of(i < n ? t.list[i] : 0);
    word = load1_if(mask + (id >> 5), i < n && mask, i < n ? 0xffffffffu : 0u);
    z = load_bits(row + id, i < n);
  }
  template <typename F>
  __device__ __forceinline__ void finish(const RulesArgs& a, const Table& t, const Plan& pl, const unsigned* mask, const T* row, F f) {
    for (int from = 0; from < t.total; from += pl.listed) {
      const int n = min(pl.listed, t.total - from);
      if (t.total > pl.listed) {
        __syncthreads();
        list_touched(a, t, pl, from);
        fetch(t, mask, row, threadIdx.x, n);
      }
      for (int i = threadIdx.x; i < n; i += kThreads) {
        if ((word >> (id & 31)) & 1u) f(i, id, from_bits(z, row));
        if (i + kThreads < n) fetch(t, mask, row, i + kThreads, n);
      }
    }
  }
};

// ---- rows ----------------------------------------------------------------------------------------------------

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

// A block of a row as vectors.  Rows at 32-byte boundaries: vectors of 32 bytes, all of it.  Others: vectors of 16 bytes
// from entry `first` of the block on; the one that would pass the block's end is not taken (unless first is 0), and the
// entries before and behind are taken one by one.  So is a vector that does not end within the vocabulary.  The vectors of
// a thread are whole blocks apart.
template <typename T, bool ALIGNED>
struct Walk {
  static constexpr int kW = ALIGNED ? 8 : 4, E = kW * 4 / sizeof(T), kSlots = kBlock / E;
  int first;
  __device__ __forceinline__ explicit Walk(const T* row)
      : first(ALIGNED ? 0 : (int)((E - (((uintptr_t)row & 15) / sizeof(T))) % E)) {}
  __device__ __forceinline__ int vectors(const Plan& pl) const { return pl.blocks * kSlots; }
  __device__ __forceinline__ int per() const { return kSlots - (first != 0); }
  // first entry of vector j of the CTA's share
  __device__ __forceinline__ int entry(int j) const { return j * E + first; }
  // the largest token with which a vector of this thread begins
  __device__ __forceinline__ int reach(const Table& t) const { return (int)(threadIdx.x & (kSlots - 1)) < per() ? t.vocab - E : -1; }
  // entry i of those taken one by one, -1: none (i < singles)
  __device__ __forceinline__ int singles(const Plan& pl, const Table& t) const {
    return first == 0 ? (t.vocab % E ? E : 0) : (pl.blocks + 1) * E;
  }
  __device__ __forceinline__ int single(const Plan& pl, const Table& t, int i) const {
    int e;
    if (i < E) {                                             // the end of the vocabulary, where it is in a vector's middle
      const int last = (t.vocab - 1) & ~(kBlock - 1);        // the block that holds it
      const int begin = last + first, id = begin + (t.vocab - begin) / E * E + i;
      if (t.vocab < begin || !t.owns(last) || id >= t.vocab || id - last >= first + per() * E) return -1;
      return t.entry_of(id);
    }
    const int k = i % E;
    e = (i / E - 1) * kBlock + (k < first ? k : per() * E + k);
    return t.id_of(e) < t.vocab ? e : -1;
  }
};

// E bits (at least) from entry e on, of the CTA's words.
template <int E, bool ALIGNED, typename F>
__device__ __forceinline__ unsigned bits_at(int e, F word) {
  const int w = e >> 5;
  if (ALIGNED) return word(w) >> (e & 31);
  return __funnelshift_r(word(w), (e & 31) > 32 - E ? word(w + 1) : 0u, e & 31);
}

__device__ __forceinline__ unsigned ordered(float m) {       // unsigned order of floats (no NaN); -0 counts as +0
  const unsigned u = __float_as_uint(__fadd_rn(m, 0.f));
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(unsigned u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
// exp(m - top) of a part's maximum, 1 where they are equal (infinities too).
__device__ __forceinline__ float weight(float m, float top) { return m == top ? 1.f : exp2_fast((m - top) * kLog2e); }

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

// ---- vectors -------------------------------------------------------------------------------------------------

template <int N>
struct Vec {
  unsigned w[N];
};
__device__ __forceinline__ void load(const void* p, Vec<4>& u) {
  asm volatile("ld.global.cs.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.w[0]), "=r"(u.w[1]), "=r"(u.w[2]), "=r"(u.w[3]) : "l"(p));
}
__device__ __forceinline__ void load(const void* p, Vec<8>& u) {
  asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(u.w[0]), "=r"(u.w[1]), "=r"(u.w[2]), "=r"(u.w[3]), "=r"(u.w[4]), "=r"(u.w[5]), "=r"(u.w[6]), "=r"(u.w[7])
               : "l"(p));
}
__device__ __forceinline__ void store(void* p, const Vec<4>& u) {
  asm volatile("st.global.cs.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(u.w[0]), "r"(u.w[1]), "r"(u.w[2]), "r"(u.w[3]) : "memory");
}
__device__ __forceinline__ void store(void* p, const Vec<8>& u) {
  asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(u.w[0]), "r"(u.w[1]), "r"(u.w[2]), "r"(u.w[3]), "r"(u.w[4]), "r"(u.w[5]), "r"(u.w[6]), "r"(u.w[7]) : "memory");
}

template <typename T>
constexpr unsigned kLeast = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;     // a word of -inf

// Entries without their bit (the lowest is the first's) become -inf.  A product puts four bits at the tops of four bytes
// (the shifted copies do not meet), from where a byte permutation spreads them over a word.
template <typename T, int N>
__device__ __forceinline__ void only(Vec<N>& u, unsigned bits) {
  constexpr int kPerWord = 4 / sizeof(T), kGroup = 4 / kPerWord;             // words that four bits decide about
#pragma unroll
  for (int g = 0; g < N / kGroup; ++g) {
    const unsigned tops = (bits >> (4 * g) & 15u) * 0x10204080u;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) {
      unsigned keep;                                         // (the permutation's selectors repeat a byte's top bit)
      asm("prmt.b32 %0, %1, %1, %2;" : "=r"(keep) : "r"(tops), "r"(sizeof(T) == 4 ? 0x8888u + 0x1111u * i : (i ? 0xbbaau : 0x9988u)));
      unsigned& w = u.w[g * kGroup + i];
      w = (w & keep) | (kLeast<T> & ~keep);
    }
  }
}
// The same with a select an entry where they are words: fewer instructions, but more registers where stores follow.
template <typename T, int N>
__device__ __forceinline__ void only_selected(Vec<N>& u, unsigned bits) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; ++i) u.w[i] = (bits >> i) & 1u ? u.w[i] : kLeast<T>;
  } else {
    only<T>(u, bits);
  }
}
// The largest entry (NaN are passed over).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
template <int N>
__device__ __forceinline__ float largest(const Vec<N>& u, const float*) {
  float m = fmaxf(__uint_as_float(u.w[0]), __uint_as_float(u.w[1]));
#pragma unroll
  for (int i = 2; i < N; i += 2) m = max3(m, __uint_as_float(u.w[i]), __uint_as_float(u.w[i + 1]));
  return m;
}
template <int N>
__device__ __forceinline__ float largest(const Vec<N>& u, const bf16*) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(u.w);
  __nv_bfloat162 m = h[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = __hmax2(m, h[i]);
  return fmaxf(__low2float(m), __high2float(m));
}
template <int N>
__device__ __forceinline__ void widen(const Vec<N>& u, float* v, const float*) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __uint_as_float(u.w[i]);
}
template <int N>
__device__ __forceinline__ void widen(const Vec<N>& u, float* v, const bf16*) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[2 * i] = __uint_as_float(u.w[i] << 16);
    v[2 * i + 1] = __uint_as_float(u.w[i] & 0xffff0000u);
  }
}
// s (two partial sums) += exp(v - ref), two entries an instruction up to the exponential.  The difference comes first: one
// product v log2(e) - ref log2(e) would leave the rounding of ref log2(e), common to all terms, in the sum.
template <int E>
__device__ __forceinline__ void add_exps(const float* v, unsigned long long minus_ref, unsigned long long log2e,
                                         unsigned long long& s) {
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    unsigned long long x;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(v[e]), "f"(v[e + 1]));
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(x), "l"(minus_ref));
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(x), "l"(log2e));
    float a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(exp2_fast(a)), "f"(exp2_fast(b)));
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(s) : "l"(s), "l"(x));
  }
}
__device__ __forceinline__ unsigned long long pair_of(float x) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(x));
  return r;
}

// ---- the confidence ------------------------------------------------------------------------------------------

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, kPerSm) k_rules_confidence(const RulesArgs a, const Plan pl, int* tok, float* conf) {
  using W = Walk<T, ALIGNED>;
  constexpr int E = W::E, kBatch = ALIGNED ? 2 : 3;          // vectors a thread has in flight (four: spills)
  constexpr unsigned kAll = (1u << E) - 1u;
  extern __shared__ __align__(16) unsigned smem[];
  __shared__ Slot parts[kRowsAtOnce * kWarps];               // of the rows that this CTA joins: [row][chunk][warp]
  __shared__ __align__(8) unsigned long long s_bar;
  __shared__ unsigned s_top[kRowsAtOnce];                    // the largest maximum that a warp has left so far, ordered
  __shared__ Row s_rows[kRowsAtOnce];
  __shared__ unsigned s_longest[kWarps];                     // the longest list so far (a copy for each warp)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) s_longest[warp] = 0u;
  if (threadIdx.x == 0) {
    tc::mbar_init(tc::smem_u32(&s_bar), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  cluster_arrive();
  pdl_wait();
  pdl_trigger();
  const int chunk = (int)cluster_rank();
  const int span = (int)blockIdx.x >> pl.lg;
  unsigned turn = 0u;
  const int r0 = (int)((long long)a.n_rows * span / pl.spans), r1 = (int)((long long)a.n_rows * (span + 1) / pl.spans);
  Table t = make_table(a, pl, chunk, smem);
  const unsigned long long log2e = pair_of(kLog2e);
  const int step = (kThreads * E) << pl.lg;                  // tokens between two vectors of a thread
  int cur = -2;
  cluster_wait();                                            // the others' barriers are there
  for (int rb = r0; rb < r1; rb += kRowsAtOnce, turn ^= 1u) {
    const int re = min(r1, rb + kRowsAtOnce);
    const int joins = (re - rb - chunk + pl.chunks - 1) >> pl.lg;                // rows that this CTA joins: chunk, chunk + chunks, ..
    if (rb > r0) {                                           // the parts of the rows before have been read everywhere
      __syncthreads();
      cluster_arrive();
      cluster_wait();
    }
    if (threadIdx.x == 0 && joins > 0) tc::mbar_expect_tx(tc::smem_u32(&s_bar), (unsigned)(joins * pl.chunks * kWarps * sizeof(Slot)));
    if (threadIdx.x < kRowsAtOnce) {
      s_top[threadIdx.x] = 0u;
      if (rb + (int)threadIdx.x < re) s_rows[threadIdx.x] = row_of(a, rb + threadIdx.x);
    }
    __syncthreads();
    for (int row = rb; row < re; ++row) {
      const Row me = s_rows[row - rb];
      const unsigned joiner = (unsigned)(row - rb) & (unsigned)(pl.chunks - 1);
      const Slot* slot = &parts[(((row - rb) >> pl.lg << pl.lg) + chunk) * kWarps + warp];
      if (!valid(a, me)) {
        if (threadIdx.x == 0 && chunk == 0) raise(a);
        if (lane == 0) send(slot, &s_bar, joiner, -INFINITY, 0.f, 0x7fffffffu);
        continue;
      }
      const T* z = static_cast<const T*>(a.logits) + (long long)row * a.ld;
      if (me.req != cur) {
        build_table(a, t, pl, me.req);
        cur = me.req;
        if (lane == 0) s_longest[warp] = max(s_longest[warp], (unsigned)(t.end - t.begin) + (unsigned)(t.bias_hi - t.bias_lo));
      }
      const unsigned* mask = me.mask < 0 ? nullptr : a.allowed + me.mask * a.allowed_ld;
      const W walk(z);
      auto usable = [&](int w) -> unsigned {
        const unsigned p = t.plain[w];
        return p & load1_if(mask + (t.id_of(w * 32) >> 5), mask && p, 0xffffffffu);
      };
      Touched<T> entries;
      entries.begin(t, pl, mask, z);
      float m = -INFINITY;
      unsigned long long s2 = 0ull;
      int best = threadIdx.x;                                // the batch that holds m: its first vector
      const int nv = t.vocab < walk.first + E ? 0 : walk.vectors(pl);
      auto dense = [&](auto masked) {
        int e0 = walk.entry(threadIdx.x), id0 = t.id_of(e0);
        const int reach = walk.reach(t);
        const unsigned shift = ALIGNED ? e0 & 31 : 0;        // (the same for all of a thread's vectors)
        const unsigned low = e0 & 31;
        const bool two = low > 32 - E;                       // its bits are in two words
        const unsigned* words = mask + (id0 >> 5);
        unsigned ahead[kBatch];                              // the mask's words of the next batch
        if (ALIGNED && masked.value) {
#pragma unroll
          for (int b = 0; b < kBatch; ++b) ahead[b] = load1_if(words + b * (step >> 5), b * step <= reach - id0, 0u);
        }
        for (int j0 = threadIdx.x; j0 < nv; j0 += kThreads * kBatch, e0 += kThreads * E * kBatch, id0 += step * kBatch, words += (step >> 5) * kBatch) {
          unsigned bits[kBatch], every = 0xffffffffu, any = 0u;
          Vec<W::kW> u[kBatch];
          const int left = reach - id0;                      // vectors that are not there lie behind the vocabulary
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
            const int e = e0 + b * kThreads * E, id = id0 + b * step;
            const bool there = b * step <= left;
            if (ALIGNED) {
              bits[b] = masked.value ? ahead[b] : 0xffffffffu;
              bits[b] &= t.plain[there ? e >> 5 : 0];        // (others lie behind the table)
              if (!masked.value && !there) bits[b] = 0u;     // (without bits: -inf)
              if (masked.value) bits[b] = bits[b] >> shift & kAll;
              // a grammar often leaves a handful of tokens: vectors without any are not read (the row's first is, instead:
              // a load under a condition would keep the registers' old values alive)
              load(z + ((masked.value ? bits[b] != 0u : there) ? id : walk.first), u[b]);
            } else {
              load(z + (there ? id : walk.first), u[b]);
              unsigned lo = there ? t.plain[e >> 5] : 0u, hi = there && two ? t.plain[(e >> 5) + 1] : 0u;
              if (masked.value) {
                lo &= load1_if(words + b * (step >> 5), there, 0u);
                hi &= load1_if(words + b * (step >> 5) + 1, there && two, 0u);
              }
              bits[b] = __funnelshift_r(lo, hi, low) & kAll;
            }
          }
          if (ALIGNED && masked.value) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
              any |= bits[b];
              ahead[b] = load1_if(words + (kBatch + b) * (step >> 5), (kBatch + b) * step <= left && j0 + (kBatch + b) * kThreads < nv, 0u);
            }
            if (!any) continue;
          }
          if (!masked.value) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) every &= bits[b];
          }
          if (masked.value || ((every >> shift) & kAll) != kAll) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) only_selected<T>(u[b], masked.value ? bits[b] : bits[b] >> shift);
          }
          float top = largest(u[0], z);
#pragma unroll
          for (int b = 1; b < kBatch; ++b) top = fmaxf(top, largest(u[b], z));
          if (top > m) {
            const unsigned long long w = pair_of(weight(m, top));
            asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(s2) : "l"(s2), "l"(w));
            m = top;
            best = j0;
          }
          if (m == INFINITY) {                               // k of them share the row
            float n = 0.f;
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
              float v[E];
              widen(u[b], v, z);
#pragma unroll
              for (int e = 0; e < E; ++e) n += v[e] == INFINITY ? 1.f : (v[e] == v[e] ? 0.f : v[e]);
            }
            unsigned long long x;
            asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(n), "f"(0.f));
            asm("add.rn.f32x2 %0, %1, %2;" : "=l"(s2) : "l"(s2), "l"(x));
          } else {
            const unsigned long long minus = pair_of(m > -INFINITY ? -m : 0.f);
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
              float v[E];
              widen(u[b], v, z);
              add_exps<E>(v, minus, log2e, s2);
            }
          }
        }
      };
      if (mask) dense(std::true_type());
      else dense(std::false_type());
      float s, s_odd;
      asm("mov.b64 {%0, %1}, %2;" : "=f"(s), "=f"(s_odd) : "l"(s2));
      s += s_odd;
      Part one{-INFINITY, 0.f, 0x7fffffff};                  // entries beside the vectors
      for (int i = threadIdx.x; i < walk.singles(pl, t); i += kThreads) {
        const int e = walk.single(pl, t, i);
        if (e >= 0 && ((usable(e >> 5) >> (e & 31)) & 1u)) {
          const int id = t.id_of(e);
          const float y = value(z + id);
          // (the end of the vocabulary comes before the blocks' ends here: equal values keep the lower entry)
          if (y == one.m) one.at = min(one.at, id);
          join_one(one, y, id);
        }
      }
      Part some{-INFINITY, 0.f, 0x7fffffff};                 // the touched entries
      entries.finish(a, t, pl, mask, z, [&](int i, int id, float v) { join_one(some, ruled(a, t, i, v), id); });
      // the warp's part: the lowest entry among the lanes that hold the maximum (where no warp has left a larger one)
      const unsigned highest = __reduce_max_sync(0xffffffffu, ordered(fmaxf(m, fmaxf(one.m, some.m))));
      const float top = unordered(highest);
      s = s * weight(m, top) + one.s * weight(one.m, top) + some.s * weight(some.m, top);
      unsigned before = 0u;
      if (lane == 0) before = atomicMax(&s_top[row - rb], highest);
      unsigned at = 0x7fffffffu;
      if (__shfl_sync(0xffffffffu, before, 0) <= highest && top > -INFINITY) {
        if (m == top) {
          for (int j = best; j < min(nv, best + kThreads * kBatch) && at == 0x7fffffffu; j += kThreads) {
            const int first = walk.entry(j), id = t.id_of(first);
            if (id > t.vocab - E) break;
            const unsigned bits = bits_at<E, ALIGNED>(first, usable);
#pragma unroll
            for (int e = E - 1; e >= 0; --e)
              if (((bits >> e) & 1u) && value(z + id + e) == top) at = (unsigned)(id + e);
          }
        }
        if (one.m == top) at = min(at, (unsigned)one.at);
        if (some.m == top) at = min(at, (unsigned)some.at);
        at = __reduce_min_sync(0xffffffffu, at);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (lane == 0) send(slot, &s_bar, joiner, top, s, at);
    }
    // join the parts of these rows: row i by CTA i mod chunks
    if (warp < joins) {
      __syncwarp();
      const bool here = wait_parts(&s_bar, turn, s_longest[warp]);
      if (!here && lane == 0 && a.error_flag) atomicMax(a.error_flag, 1);
      for (int k = warp; k < joins; k += kWarps) {
        Part p{-INFINITY, 0.f, 0x7fffffff};
        for (int i = lane; i < kWarps << pl.lg; i += 32) {
          const Part o = parts[(k << pl.lg) * kWarps + i].part;
          const float top = fmaxf(p.m, o.m);
          p.at = o.m > p.m ? o.at : (o.m == p.m ? min(p.at, o.at) : p.at);
          p.s = p.s * weight(p.m, top) + o.s * weight(o.m, top);
          p.m = top;
        }
        const float top = unordered(__reduce_max_sync(0xffffffffu, ordered(p.m)));
        const unsigned at = __reduce_min_sync(0xffffffffu, p.m == top ? (unsigned)p.at : 0x7fffffffu);
        float s = p.s * weight(p.m, top);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) {
          const int row = rb + (k << pl.lg) + chunk;
          tok[row] = here && top > -INFINITY ? (int)at : -1;
          conf[row] = !here ? __uint_as_float(0x7fffffffu) : top > -INFINITY ? __fdiv_rn(1.f, s) : (s == s ? 0.f : s);
        }
      }
    }
  }
}

// ---- the rules on the logits themselves ----------------------------------------------------------------------

// Stores y.  In place only vectors with an entry that is not allowed are written, and the touched entries.
template <typename T, bool ALIGNED, bool INPLACE>
__global__ void __launch_bounds__(kThreads, kPerSm) k_logit_rules(const RulesArgs a, const Plan pl, T* out, long long out_ld) {
  using W = Walk<T, ALIGNED>;
  constexpr int E = W::E, kBatch = ALIGNED ? 2 : 4;
  constexpr unsigned kAll = (1u << E) - 1u;
  extern __shared__ __align__(16) unsigned smem[];
  pdl_wait();
  pdl_trigger();
  const int chunk = (int)blockIdx.x & (pl.chunks - 1), span = (int)blockIdx.x >> pl.lg;
  const int r0 = (int)((long long)a.n_rows * span / pl.spans), r1 = (int)((long long)a.n_rows * (span + 1) / pl.spans);
  const int step = (kThreads * E) << pl.lg;                  // tokens between two vectors of a thread
  Table t = make_table(a, pl, chunk, smem);
  __shared__ Row s_rows[kRowsAtOnce];
  int cur = -2;
  for (int row = r0; row < r1; ++row) {
    if ((row - r0) % kRowsAtOnce == 0) {
      __syncthreads();
      if (threadIdx.x < kRowsAtOnce && row + (int)threadIdx.x < r1) s_rows[threadIdx.x] = row_of(a, row + threadIdx.x);
      __syncthreads();
    }
    const Row me = s_rows[(row - r0) % kRowsAtOnce];
    if (!valid(a, me)) {
      if (threadIdx.x == 0 && chunk == 0) raise(a);
      continue;
    }
    const T* z = static_cast<const T*>(a.logits) + (long long)row * a.ld;
    T* y = out + (long long)row * out_ld;
    const unsigned* mask = me.mask < 0 ? nullptr : a.allowed + me.mask * a.allowed_ld;
    const W walk(z);
    auto allow = [&](int w) -> unsigned {                    // entries that may stay
      const unsigned in = t.in_range(w);
      return in & load1_if(mask + (t.id_of(w * 32) >> 5), mask && in, 0xffffffffu);
    };
    const bool level = (((uintptr_t)y ^ (uintptr_t)z) & 15) == 0;              // vectors of z are vectors of y
    // All entries, the touched ones as if no rule touched them: they are written again behind a barrier.
    auto dense = [&]() {
      if (INPLACE && !mask) {
        if (threadIdx.x == 0 && (unsigned)t.mask_id < (unsigned)t.vocab && t.owns(t.mask_id)) put(y + t.mask_id, -INFINITY);
        return;
      }
      const int nv = walk.vectors(pl), reach = walk.reach(t);
      int id0 = t.id_of(walk.entry(threadIdx.x));
      const unsigned low = id0 & 31;
      const bool two = !ALIGNED && low > 32 - E;             // a vector's bits are in two words
      for (int j0 = threadIdx.x; j0 < nv; j0 += kThreads * kBatch, id0 += step * kBatch) {
        Vec<W::kW> u[kBatch];
        unsigned keep[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int id = id0 + b * step;
          const bool there = id <= reach;
          if (!INPLACE && there) load(z + id, u[b]);
          const unsigned at = (unsigned)(t.mask_id - id);
          const unsigned word = load1_if(mask + (id >> 5), mask && there, 0xffffffffu);
          const unsigned more = ALIGNED ? 0u : load1_if(mask + (id >> 5) + 1, mask && there && two, 0xffffffffu);
          keep[b] = (ALIGNED ? word >> low : __funnelshift_r(word, more, low)) & kAll;
          if (at < E) keep[b] &= ~(1u << at);
          if (!there) keep[b] = kAll;
        }
        if (INPLACE) {
#pragma unroll
          for (int b = 0; b < kBatch; ++b) {
#pragma unroll
            for (int i = 0; i < W::kW; ++i) u[b].w[i] = kLeast<T>;
            if (keep[b] && keep[b] != kAll) load(z + id0 + b * step, u[b]);
          }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int id = id0 + b * step;
          if (INPLACE ? keep[b] == kAll : id > reach) continue;
          if (keep[b] != kAll) only<T>(u[b], keep[b]);
          if (ALIGNED || INPLACE || level) {
            store(y + id, u[b]);
          } else {
            float v[E];
            widen(u[b], v, z);
#pragma unroll
            for (int e = 0; e < E; ++e) put(y + id + e, v[e]);
          }
        }
      }
      for (int i = threadIdx.x; i < walk.singles(pl, t); i += kThreads) {
        const int e = walk.single(pl, t, i);
        if (e >= 0) {
          const int id = t.id_of(e);
          if (!((allow(e >> 5) >> (e & 31)) & 1u)) put(y + id, -INFINITY);
          else if (!INPLACE) put(y + id, value(z + id));
        }
      }
    };
    Touched<T> entries;
    // Where a table is to be built, half of the CTAs build it after the pass over all entries: while some wait for context
    // tokens, the others keep memory busy.
    const bool build = me.req != cur, later = build && (span & 1);
    cur = me.req;
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
      if ((part != 0) == later) {
        if (build) build_table(a, t, pl, me.req);
        if (!later) entries.begin(t, pl, mask, z);
      } else {
        dense();
      }
    }
    if (later) entries.begin(t, pl, mask, z);
    if (t.total > 0) __syncthreads();                        // the pass has written its entries
    entries.finish(a, t, pl, mask, z, [&](int i, int id, float v) { put(y + id, ruled(a, t, i, v)); });
  }
}

// ---- launches ------------------------------------------------------------------------------------------------

using ConfKernel = void (*)(const RulesArgs, const Plan, int*, float*);
template <typename T>
ConfKernel conf_kernel(bool aligned) { return aligned ? k_rules_confidence<T, true> : k_rules_confidence<T, false>; }
template <typename T>
using RuleKernel = void (*)(const RulesArgs, const Plan, T*, long long);

// One-time set-up per device; how many spans the device holds at once, by cluster size and by the table's size (in steps of
// 1 KB), asked when first needed.
constexpr int kMaxSmem = 64 * 1024;
struct DevInfo {
  int num_sms;
  int ok;
  int spans[4][kMaxSmem / 1024 + 1];
};
DevInfo g_dev[kMaxDevices];
std::mutex g_mutex;

template <typename T>
bool allow_smem() {
  bool ok = true;
  for (ConfKernel k : {conf_kernel<T>(true), conf_kernel<T>(false)})
    ok = ok && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) == cudaSuccess;
  for (RuleKernel<T> k : {k_logit_rules<T, true, true>, k_logit_rules<T, true, false>, k_logit_rules<T, false, true>, k_logit_rules<T, false, false>})
    ok = ok && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) == cudaSuccess;
  return ok;
}

void cluster_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* at, int ctas, int chunks, size_t smem, bool early, cudaStream_t s) {
  cfg->gridDim = dim3((unsigned)ctas);
  cfg->blockDim = dim3(kThreads);
  cfg->dynamicSmemBytes = smem;
  cfg->stream = s;
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)chunks; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg->attrs = at;
  cfg->numAttrs = early && !pdl_disabled() ? 2 : 1;
}

size_t smem_of(const Plan& pl) { return (size_t)pl.listed * 8 + (size_t)pl.blocks * kBlockWords * 10 + kWarps * kQueue * 4; }

// The plan of a call, spans excepted.  Shares of at least 32 blocks: with fewer the join would cost more than the row.
Plan plan_of(const RulesArgs& a) {
  Plan pl;
  const int blocks = (a.vocab + kBlock - 1) / kBlock;
  pl.lg = 0;
  while ((1 << pl.lg) < kMaxChunks && blocks > 32 << pl.lg) ++pl.lg;
  pl.chunks = 1 << pl.lg;
  pl.blocks = (blocks + pl.chunks - 1) >> pl.lg;
  pl.listed = pl.blocks * kBlock < kListed ? pl.blocks * kBlock : kListed;
  return pl;
}

// Sets pl->spans: as many as the device holds at once, since a second round of them would double the time.  False: the
// device cannot be asked.
bool plan_spans(const RulesArgs& a, Plan* pl) {
  DevInfo* d = device_slot(g_dev);
  if (!d) return false;
  const size_t smem = smem_of(*pl);
  std::lock_guard<std::mutex> lock(g_mutex);
  if (!d->num_sms) {
    int dev = 0, n = 0;
    cudaGetDevice(&dev);
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return false;
    d->ok = allow_smem<float>() && allow_smem<bf16>();
    if (!d->ok) cudaGetLastError();
    d->num_sms = n;
  }
  if (!d->ok || smem > kMaxSmem) return false;
  int& spans = d->spans[pl->lg][smem / 1024];
  if (spans == 0) {
    spans = d->num_sms * kPerSm >> pl->lg;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    cluster_config(&cfg, at, spans << pl->lg, pl->chunks, (smem + 1023) / 1024 * 1024, false, nullptr);
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, conf_kernel<float>(true), &cfg) == cudaSuccess && n > 0) spans = n;
    else cudaGetLastError();
  }
  pl->spans = spans < a.n_rows ? spans : a.n_rows;
  pl->early = 2 * pl->spans <= spans;
  return true;
}

template <typename T>
cudaError_t launch_rules(const RulesArgs& a, const Plan& pl, T* out, long long out_ld, cudaStream_t s) {
  const bool aligned = (((uintptr_t)a.logits | (uintptr_t)out | (uintptr_t)(a.ld * sizeof(T)) | (uintptr_t)(out_ld * sizeof(T))) & 31) == 0;
  const bool inplace = out == a.logits;
  RuleKernel<T> k = inplace ? (aligned ? k_logit_rules<T, true, true> : k_logit_rules<T, false, true>)
                            : (aligned ? k_logit_rules<T, true, false> : k_logit_rules<T, false, false>);
  return launch_pdl(k, dim3((unsigned)(pl.spans * pl.chunks)), dim3(kThreads), smem_of(pl), s, a, pl, out, out_ld);
}

}  // namespace

cudaError_t launch_rules_confidence(const RulesArgs& a, int* tok, float* conf, cudaStream_t s) {
  if (a.n_rows <= 0) return cudaSuccess;
  Plan pl = plan_of(a);
  if (!plan_spans(a, &pl)) return cudaErrorInitializationError;
  const bool aligned = (((uintptr_t)a.logits | (uintptr_t)(a.ld * (a.bf16_logits ? 2 : 4))) & 31) == 0;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  cluster_config(&cfg, at, pl.spans * pl.chunks, pl.chunks, smem_of(pl), pl.early, s);
  return cudaLaunchKernelEx(&cfg, a.bf16_logits ? conf_kernel<bf16>(aligned) : conf_kernel<float>(aligned), a, pl, tok, conf);
}

cudaError_t launch_logit_rules(const RulesArgs& a, void* out, long long out_ld, cudaStream_t s) {
  if (a.n_rows <= 0) return cudaSuccess;
  Plan pl = plan_of(a);
  if (!plan_spans(a, &pl)) return cudaErrorInitializationError;
  return a.bf16_logits ? launch_rules<bf16>(a, pl, (bf16*)out, out_ld, s) : launch_rules<float>(a, pl, (float*)out, out_ld, s);
}

}  // namespace bs
