// The 8-bit paged cache: what the append and the attention kernels share.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <stdint.h>

#include "rope.cuh"

namespace hsa {

// Scales are 2^kScaleMin .. 2^kScaleMax: values up to 2^60 fit, and the scales of two pages are never further apart than
// fp32 can hold beside the weights of a softmax (2^100).
constexpr int kScaleMin = -48, kScaleMax = 52;
constexpr float kTop8 = 1.152921504606846976e18f;  // 2^60, the largest magnitude that is stored
constexpr int kDevNonfinite = HSA_ERR_DEVICE_NONFINITE;
constexpr uint32_t kMaxPolls = 1u << 17, kPollNs = 20000;  // polls of a barrier before a wait runs out, and what one may sleep

// The rows of each sequence in a call's tensors
struct Kv8Rows {
  const int32_t* start;  // [batch + 1] or null: even shares
  int n_tokens, batch, max_rows, share;
  // first row and number of rows of sequence s; false: they do not fit
  __device__ __forceinline__ bool get(int s, int* first, int* n) const {
    if (!start) {
      *first = s * share;
      *n = share;
      return true;
    }
    const int s0 = __ldg(start + s), s1 = __ldg(start + s + 1);
    *first = s0;
    *n = s1 - s0;
    return s0 >= 0 && s1 >= s0 && s1 <= n_tokens && *n <= max_rows;
  }
};

struct Kv8AppendArgs {
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  int64_t ts, hs;
  Kv8Rows rows;
  const int32_t* held;
  int H, max_pages, max_blocks;
  int heads;          // key heads of a CTA
  int blocks_per_seq; // blocks a sequence's rows can reach
  int has_rope;
  RopeDev rope;
  const int32_t* table;
  uint8_t* k_pool;
  uint8_t* v_pool;
  float* k_scale;
  float* v_scale;
  float* ksum;
  int32_t* status;
};
cudaError_t kv8_append_init(int D);
cudaError_t launch_kv8_append(const Kv8AppendArgs& a, int D, int nsm, cudaStream_t st);

struct Kv8AttendArgs {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  float* lse;          // [n_tokens][Hq] or null
  int64_t ts, hs, ots, ohs;
  Kv8Rows rows;
  const int32_t* lengths;
  int Hq, Hkv, group;  // group = Hq / Hkv
  int max_pages, max_blocks;
  int causal;
  const int32_t* sel_idx;
  const int32_t* sel_cnt;
  int max_topk;
  float scale_log2;    // softmax scale * log2(e)
  const int32_t* table;
  const uint8_t* k_pool;
  const uint8_t* v_pool;
  const float* k_scale;
  const float* v_scale;
  int32_t* status;
};
// How the attention kernels share their work out.  An item is a tile of query rows of one (sequence, key head): row r is
// token r / group of the sequence and query head h * group + r % group, so that query heads of one key head read its pages
// once.  An item has as many steps as it has pages to read (times kv8 pages a step).  The steps of all items, in order,
// are cut into equal runs, one for each CTA, from the lengths as they stand in device memory: whatever the batch holds,
// every SM gets the same share and a captured graph serves any lengths.  (Where there are CTAs for it, each item is cut by
// itself into parts of 2^part_log steps at least: a run that crosses items would make some wait for others.)  An item that lies in one CTA's run is written by
// it; of one that is cut, each CTA leaves an unnormalised part in the workspace and the last to take a ticket joins them in
// the order of the runs, which makes the result independent of which CTA that is.  Nobody waits.
struct Kv8Work {
  int tile_rows;       // query rows of an item
  int tiles;           // tiles of a sequence with max_rows rows
  int step_log;        // an item takes 2^step_log pages in a step
  int half_rows;       // items of at most so many rows take twice the pages in a step
  int part_log;        // an item is not cut into parts of less than 2^part_log steps while there is a CTA for each part
  int item_steps;      // steps that an item costs beside its own: runs are cut as if they came before them
  int64_t items;       // batch * Hkv * tiles
  float* parts;        // [2 * CTAs][slot_floats]
  int64_t slot_floats;
  int32_t* tickets;    // [2 * CTAs], zero between calls
  uint32_t first_try;  // where the count of a wait's polls begins: 0, or a later one for less patience
  uint32_t look;       // cycles that a wait looks for, where that is less than a poll's sleep; else 0
};

int kv8_decode_rows(int D);                                   // rows up to which the kernel for few rows takes a call
size_t kv8_decode_slot(int D);                                // floats of a part
cudaError_t kv8_decode_init(int D);
cudaError_t launch_kv8_decode(const Kv8AttendArgs& a, Kv8Work w, int D, int nsm, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                              cudaStream_t st);
size_t kv8_chunk_slot(int D);
cudaError_t kv8_chunk_init(int D);
cudaError_t launch_kv8_chunk(const Kv8AttendArgs& a, Kv8Work w, int D, int nsm, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                             cudaStream_t st);

__device__ __forceinline__ void kv8_flag(int32_t* status, int code) { atomicCAS(status, 0, code); }

struct Kv8Item {
  int b, h, tile;
  int first, n, len;   // rows and tokens of the sequence
  int row0, rows;      // rows of the item: row0 .. row0 + rows of the sequence's n * group
  int pages;           // pages to read
  const int32_t* list; // block list or null: blocks 0, 1, ...
  int steps;           // 0: nothing to do (no rows, or the sequence does not fit)
  // tokens that row r (of the item) sees
  __device__ __forceinline__ int limit(const Kv8AttendArgs& a, int r) const {
    return a.causal ? max(0, min(len, len - n + (row0 + r) / a.group + 1)) : len;
  }
};

// Where an item lies: needs no memory.
__device__ __forceinline__ void kv8_place(const Kv8AttendArgs& a, const Kv8Work& w, int64_t i, Kv8Item* it) {
  const uint32_t at = static_cast<uint32_t>(i);  // (launches with 2^31 items are refused)
  const uint32_t bh = w.tiles == 1 ? at : at / static_cast<uint32_t>(w.tiles), b = bh / static_cast<uint32_t>(a.Hkv);
  it->tile = static_cast<int>(at - bh * static_cast<uint32_t>(w.tiles));
  it->b = static_cast<int>(b);
  it->h = static_cast<int>(bh - b * static_cast<uint32_t>(a.Hkv));
  it->row0 = it->tile * w.tile_rows;
}

// What there is to do in it.
__device__ __forceinline__ void kv8_fill(const Kv8AttendArgs& a, const Kv8Work& w, Kv8Item* it) {
  const int64_t bh = static_cast<int64_t>(it->b) * a.Hkv + it->h;
  // (all that has to be read, at once)
  const int count = a.sel_idx ? __ldg(a.sel_cnt + bh) : 0;
  it->len = __ldg(a.lengths + it->b);
  const bool fits = a.rows.get(it->b, &it->first, &it->n);
  it->steps = it->pages = it->rows = 0;
  it->list = nullptr;
  if (!fits || it->len < 0 || it->len > static_cast<int64_t>(a.max_blocks) * kBlock) {
    if (it->h == 0 && it->tile == 0 && blockIdx.x == 0) kv8_flag(a.status, kDevBounds);
    return;
  }
  it->rows = min(w.tile_rows, it->n * a.group - it->row0);
  if (it->rows <= 0) return;
  if (a.sel_idx) {
    it->list = a.sel_idx + bh * a.max_topk;
    it->pages = min(max(count, 0), a.max_topk);
  } else {
    it->pages = (it->limit(a, it->rows - 1) + kBlock - 1) / kBlock;
  }
  const int log = w.step_log + (it->rows <= w.half_rows ? 1 : 0);
  it->steps = max(1u, (static_cast<uint32_t>(it->pages) + (1u << log) - 1) >> log);
}

// (Not inlined: the roles' walks call it, behind the segments of the plan, and they share the instruction caches of an SM.  So does
// the plan of a launch with more items than threads, twice for each of a thread's items, empty ones too: one row of 49 sequences of
// 8 key heads, 392 items of 384 threads, takes 50.7 us where 48 sequences take 48.0.)
__device__ __noinline__ static Kv8Item kv8_item(const Kv8AttendArgs& a, const Kv8Work& w, int64_t i) {
  Kv8Item it;
  kv8_place(a, w, i, &it);
  kv8_fill(a, w, &it);
  return it;
}

// A stretch of an item that one CTA does.
struct Kv8Segment {
  Kv8Item it;
  int s0, s1;                   // steps of the item
  int first_cta, last_cta;      // CTAs that the item is shared by
  __device__ __forceinline__ bool whole() const { return first_cta == last_cta; }
  // where this CTA's part of the item goes: each has at most one item that began earlier and one that goes on
  __device__ __forceinline__ int64_t slot() const { return 2 * static_cast<int64_t>(blockIdx.x) + (s0 == 0 ? 1 : 0); }
  __device__ __forceinline__ static int64_t slot_of(int cta, int first) { return 2 * static_cast<int64_t>(cta) + (cta == first ? 1 : 0); }
};

constexpr int kSegments = 32;   // of a CTA, worked out in advance; what goes beyond is worked out by each role as it gets there

// The CTA's run, in shared memory.
struct Kv8Plan {
  int64_t hi, share;            // behind the CTA's last step; steps of a CTA (those that items cost beside their own included)
  int n;                        // segments below
  bool more;                    // further ones follow, from item more_item on, whose steps begin at more_start
  int64_t more_item, more_start;
  Kv8Segment seg[kSegments];
};

// Quotients of what is seldom past 32 bits
__device__ __forceinline__ int64_t kv8_div(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? static_cast<int64_t>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}

__device__ __forceinline__ void kv8_cut(Kv8Segment* g, int64_t start, int64_t lo, int64_t hi, int64_t share) {
  const int64_t end = start + g->it.steps;
  g->s0 = static_cast<int>(max(lo - start, static_cast<int64_t>(0)));
  g->s1 = static_cast<int>(min(end, hi) - start);
  g->first_cta = start >= lo && start < hi ? static_cast<int>(blockIdx.x) : static_cast<int>(kv8_div(start, share));
  g->last_cta = end <= hi ? static_cast<int>(blockIdx.x) : static_cast<int>(kv8_div(end - 1, share));
}

// Sums over a warp's lanes up to each
template <typename T>
__device__ __forceinline__ T kv8_scan(T sum, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  return sum;
}

// Waits for the kernel before and fills the plan; all THREADS threads call it, and meet at its end.  (A launch begins with cold
// caches, and everything waits for this.  With items looked up by a call, which reads the kernel's arguments past the constant
// cache, with their places worked out behind the wait and with two scans in turn, one query row against 777 tokens took 8.7 us
// instead of 7.4, and one row each of 48 sequences of 300 to 8000 tokens 49.6 instead of 48.0.)
template <int THREADS>
__device__ void kv8_plan(const Kv8AttendArgs& a, const Kv8Work& w, Kv8Plan* plan) {
  constexpr int W = THREADS / 32;
  __shared__ int64_t sums[W];
  __shared__ int counts[W], parts_of[W];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  const bool one = w.items <= THREADS;  // every thread has one item at most: once is enough
  int64_t total = 0, sum = 0;
  Kv8Segment g{};
  if (one) kv8_place(a, w, tid, &g.it);
  if (tid == 0) {
    plan->n = 0;
    plan->more = false;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (one) {
    if (tid < w.items) kv8_fill(a, w, &g.it);
    // a part of an item for each CTA?  (counted up to more than there can be CTAs)
    const int parts = min((static_cast<uint32_t>(g.it.steps) + (1u << w.part_log) - 1) >> w.part_log, 1024u);
    const int upto = kv8_scan(parts, lane);
    sum = kv8_scan(g.it.steps ? static_cast<int64_t>(g.it.steps) + w.item_steps : 0, lane);
    if (lane == 31) {
      parts_of[warp] = upto;
      sums[warp] = sum;
    }
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      if (j < warp) before += parts_of[j];
      all += parts_of[j];
    }
    if (all <= static_cast<int>(gridDim.x)) {  // (each count is right then, and steps are few)
      const int first = before + upto - parts, cta = static_cast<int>(blockIdx.x);
      if (cta >= first && cta < first + parts) {
        g.s0 = static_cast<int>(static_cast<uint32_t>(g.it.steps * (cta - first)) / static_cast<uint32_t>(parts));
        g.s1 = static_cast<int>(static_cast<uint32_t>(g.it.steps * (cta - first + 1)) / static_cast<uint32_t>(parts));
        g.first_cta = first;
        g.last_cta = first + parts - 1;
        plan->seg[0] = g;
        plan->n = 1;
      }
      __syncthreads();
      return;
    }
  } else {
    int64_t mine = 0;
#pragma unroll 1
    for (int64_t i = tid; i < w.items; i += THREADS) {
      const int steps = kv8_item(a, w, i).steps;
      mine += steps ? static_cast<int64_t>(steps) + w.item_steps : 0;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (lane == 0) sums[warp] = mine;
    __syncthreads();
#pragma unroll 4
    for (int i = 0; i < W; ++i) total += sums[i];
    __syncthreads();
  }
  int64_t carry = 0, lo = 0, hi = 0, share = 1;
  int carried = 0;  // segments so far
#pragma unroll 1
  for (int64_t base = 0; base < w.items; base += THREADS) {
    const int64_t i = base + tid;
    if (!one) {
      g.it.steps = 0;
      if (i < w.items) g.it = kv8_item(a, w, i);
      sum = kv8_scan(g.it.steps ? static_cast<int64_t>(g.it.steps) + w.item_steps : 0, lane);
      if (lane == 31) sums[warp] = sum;
      __syncthreads();
    }
    int64_t before = carry, all = 0;
#pragma unroll 4
    for (int j = 0; j < W; ++j) {
      if (j < warp) before += sums[j];
      all += sums[j];
    }
    if (one) total = all;
    share = max(static_cast<int64_t>(1), kv8_div(total + gridDim.x - 1, gridDim.x));
    lo = min(total, share * blockIdx.x);
    hi = min(total, lo + share);
    const int64_t end = before + sum, start = end - g.it.steps;  // of its own steps
    const bool mine = g.it.steps > 0 && start < hi && end > lo;
    const uint32_t those = __ballot_sync(0xffffffffu, mine);
    if (lane == 0) counts[warp] = __popc(those);
    __syncthreads();
    int at = carried + __popc(those & ((1u << lane) - 1));
#pragma unroll 4
    for (int j = 0; j < W; ++j) {
      if (j < warp) at += counts[j];
      carried += counts[j];
    }
    if (mine && at < kSegments) {
      kv8_cut(&g, start, lo, hi, share);
      plan->seg[at] = g;
    }
    if (mine && at == kSegments) {
      plan->more = true;
      plan->more_item = i;
      plan->more_start = start;
    }
    carry += all;
    if (carry >= hi) break;  // (the same for the whole CTA)
    __syncthreads();
  }
  if (tid == 0) {
    plan->n = min(carried, kSegments);
    plan->hi = hi;
    plan->share = share;
  }
  __syncthreads();
}

// Walks over the segments of the plan: every role of a CTA has a walk of its own.
struct Kv8Walk {
  int i = 0;
  int64_t item, start;
  Kv8Segment g;
  __device__ __forceinline__ bool next(const Kv8AttendArgs& a, const Kv8Work& w, const Kv8Plan& plan) {
    if (i < plan.n) {
      g = plan.seg[i++];
      return true;
    }
    if (!plan.more) return false;
    if (i++ == kSegments) {
      item = plan.more_item;
      start = plan.more_start;
    }
    if (start >= plan.hi) return false;
    for (;; ++item) {
      g.it = kv8_item(a, w, item);
      if (g.it.steps) break;
    }
    kv8_cut(&g, start, plan.share * blockIdx.x, plan.hi, plan.share);
    start += g.it.steps + w.item_steps;
    ++item;
    return true;
  }
};

// A page of an item: its number in the pools, or -1 where there is none to be seen.
__device__ __forceinline__ int kv8_page(const Kv8AttendArgs& a, const Kv8Item& it, int nth, int* blk_out) {
  *blk_out = 0;
  if (nth >= it.pages) return -1;
  const int blk = it.list ? __ldg(it.list + nth) : nth;
  if (blk < 0 || blk >= a.max_blocks) {
    kv8_flag(a.status, kDevBounds);
    return -1;
  }
  *blk_out = blk;
  if (static_cast<int64_t>(blk) * kBlock >= it.limit(a, it.rows - 1)) return -1;
  const int page = __ldg(a.table + static_cast<int64_t>(it.b) * a.max_blocks + blk);
  if (page < 0 || page >= a.max_pages) {
    kv8_flag(a.status, kDevBounds);
    return -1;
  }
  return page;
}

}  // namespace hsa
