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
cudaError_t launch_kv8_attend_plain(const Kv8AttendArgs& a, int D, cudaStream_t st);

__device__ __forceinline__ void kv8_flag(int32_t* status, int code) { atomicCAS(status, 0, code); }

}  // namespace hsa
