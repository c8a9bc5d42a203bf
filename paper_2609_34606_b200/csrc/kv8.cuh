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
// every SM gets the same share and a captured graph serves any lengths.  An item that lies in one CTA's run is written by
// it; of one that is cut, each CTA leaves an unnormalised part in the workspace and the last to take a ticket joins them in
// the order of the runs, which makes the result independent of which CTA that is.  Nobody waits.
struct Kv8Work {
  int tile_rows;       // query rows of an item
  int tiles;           // tiles of a sequence with max_rows rows
  int step_pages;
  int min_steps;       // no run is shorter
  int64_t items;       // batch * Hkv * tiles
  float* parts;        // [2 * CTAs][slot_floats]
  int64_t slot_floats;
  int32_t* tickets;    // [CTAs], zero between calls
};

int kv8_decode_rows(int D);                                   // rows up to which the kernel for few rows takes a call
size_t kv8_decode_slot(int D);                                // floats of a part
cudaError_t kv8_decode_init(int D);
cudaError_t launch_kv8_decode(const Kv8AttendArgs& a, Kv8Work w, int D, int nsm, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                              cudaStream_t st);
cudaError_t launch_kv8_attend_plain(const Kv8AttendArgs& a, int D, cudaStream_t st);

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

__device__ __forceinline__ Kv8Item kv8_item(const Kv8AttendArgs& a, const Kv8Work& w, int64_t i) {
  Kv8Item it;
  it.tile = static_cast<int>(i % w.tiles);
  const int bh = static_cast<int>(i / w.tiles);
  it.b = bh / a.Hkv;
  it.h = bh % a.Hkv;
  it.steps = it.pages = 0;
  it.list = nullptr;
  const bool fits = a.rows.get(it.b, &it.first, &it.n);
  it.len = __ldg(a.lengths + it.b);
  it.row0 = it.tile * w.tile_rows;
  it.rows = 0;
  if (!fits || it.len < 0 || it.len > static_cast<int64_t>(a.max_blocks) * kBlock) {
    if (it.h == 0 && it.tile == 0 && blockIdx.x == 0) kv8_flag(a.status, kDevBounds);
    return it;
  }
  it.rows = min(w.tile_rows, it.n * a.group - it.row0);
  if (it.rows <= 0) return it;
  if (a.sel_idx) {
    it.list = a.sel_idx + static_cast<int64_t>(bh) * a.max_topk;
    it.pages = min(max(__ldg(a.sel_cnt + bh), 0), a.max_topk);
  } else {
    it.pages = (it.limit(a, it.rows - 1) + kBlock - 1) / kBlock;
  }
  it.steps = max(1, (it.pages + w.step_pages - 1) / w.step_pages);
  return it;
}

struct Kv8Run {
  int64_t lo, hi;      // the CTA's steps
  int64_t share;
  int64_t item, start; // the item that `lo` lies in, and where its steps begin
};

// The CTA's run; all THREADS threads call it.  lo >= hi: nothing to do.
template <int THREADS>
__device__ Kv8Run kv8_run(const Kv8AttendArgs& a, const Kv8Work& w) {
  constexpr int W = THREADS / 32;
  __shared__ int64_t sums[W + 1];
  __shared__ int64_t found[2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  int64_t mine = 0;
  for (int64_t i = tid; i < w.items; i += THREADS) mine += kv8_item(a, w, i).steps;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  if (lane == 0) sums[warp] = mine;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int i = 0; i < W; ++i) total += sums[i];
  Kv8Run r;
  r.share = max(static_cast<int64_t>(w.min_steps), (total + gridDim.x - 1) / gridDim.x);
  r.lo = min(total, r.share * blockIdx.x);
  r.hi = min(total, r.lo + r.share);
  r.item = r.start = 0;
  if (r.lo >= r.hi) return r;  // (the same for the whole CTA)
  int64_t carry = 0;
  for (int64_t base = 0; base < w.items; base += THREADS) {
    __syncthreads();
    const int64_t i = base + tid;
    const int64_t steps = i < w.items ? kv8_item(a, w, i).steps : 0;
    int64_t sum = steps;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    if (lane == 31) sums[warp] = sum;
    __syncthreads();
    int64_t before = carry, all = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      if (j < warp) before += sums[j];
      all += sums[j];
    }
    const int64_t end = before + sum, begin = end - steps;
    if (r.lo >= begin && r.lo < end) {
      found[0] = i;
      found[1] = begin;
    }
    carry += all;
    if (carry > r.lo) break;  // (the same for the whole CTA)
  }
  __syncthreads();
  r.item = found[0];
  r.start = found[1];
  return r;
}

// Walks over the segments of a run: every role of a CTA has a walk of its own.
struct Kv8Walk {
  int64_t at, start, item;
  Kv8Item it;
  int s0, s1;          // steps of the item that this CTA does
  int64_t first_cta, last_cta;  // CTAs that the item is shared by
  __device__ __forceinline__ explicit Kv8Walk(const Kv8Run& r) : at(r.lo), start(r.start), item(r.item) {}
  __device__ __forceinline__ bool next(const Kv8AttendArgs& a, const Kv8Work& w, const Kv8Run& r) {
    if (at >= r.hi) return false;
    for (;; ++item) {
      it = kv8_item(a, w, item);
      if (it.steps) break;
    }
    s0 = static_cast<int>(at - start);
    s1 = static_cast<int>(min(static_cast<int64_t>(it.steps), r.hi - start));
    first_cta = start / r.share;
    last_cta = (start + it.steps - 1) / r.share;
    at = start + s1;
    start += it.steps;
    ++item;
    return true;
  }
  __device__ __forceinline__ bool whole() const { return first_cta == last_cta; }
  // where this CTA's part of the item goes: each has at most one item that began earlier and one that goes on
  __device__ __forceinline__ int64_t slot() const { return 2 * static_cast<int64_t>(blockIdx.x) + (s0 == 0 ? 1 : 0); }
  __device__ __forceinline__ static int64_t slot_of(int64_t cta, int64_t first) { return 2 * cta + (cta == first ? 1 : 0); }
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
