// Attention over the 8-bit paged cache: one warp per query and head, keys one after another.
#include <cuda_fp8.h>

#include "kv8.cuh"

namespace hsa {

namespace {

__device__ __forceinline__ float2 from_e4m3x2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

template <int D>
__global__ void __launch_bounds__(128) kv8_attend_plain_kernel(const Kv8AttendArgs a) {
  constexpr int N = D / 32;  // dims of a lane
  const int lane = threadIdx.x & 31;
  const int b = blockIdx.z, i = blockIdx.y, h = blockIdx.x * 4 + threadIdx.x / 32;
  int first, n;
  const bool fits = a.rows.get(b, &first, &n);
  const int len = __ldg(a.lengths + b);
  if (!fits || len < 0 || len > static_cast<int64_t>(a.max_blocks) * kBlock) {
    if (lane == 0) kv8_flag(a.status, kDevBounds);
    return;
  }
  if (i >= n || h >= a.Hq) return;
  const int kvh = h / a.group;
  const int64_t row = first + i;
  const int seen = a.causal ? min(len, len - n + i + 1) : len;  // keys before this one are seen
  float q[N], o[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    q[j] = __bfloat162float(a.q[row * a.ts + h * a.hs + lane * N + j]) * a.scale_log2;
    o[j] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  int count = (seen + kBlock - 1) / kBlock;
  const int32_t* list = nullptr;
  if (a.sel_idx) {
    const int64_t at = static_cast<int64_t>(b) * a.Hkv + kvh;
    list = a.sel_idx + at * a.max_topk;
    count = min(max(a.sel_cnt[at], 0), a.max_topk);
  }
  for (int e = 0; e < count; ++e) {
    const int blk = list ? list[e] : e;
    if (blk < 0 || blk >= a.max_blocks) {
      if (lane == 0) kv8_flag(a.status, kDevBounds);
      continue;
    }
    const int64_t left = seen - static_cast<int64_t>(blk) * kBlock;
    if (left <= 0) continue;
    const int page = a.table[static_cast<int64_t>(b) * a.max_blocks + blk];
    if (page < 0 || page >= a.max_pages) {
      if (lane == 0) kv8_flag(a.status, kDevBounds);
      continue;
    }
    const int64_t ph = static_cast<int64_t>(page) * a.Hkv + kvh;
    const float ks = a.k_scale[ph], vs = a.v_scale[ph];
    const int rows = left < kBlock ? static_cast<int>(left) : kBlock;
    for (int r = 0; r < rows; ++r) {
      const uint8_t* kp = a.k_pool + (ph * kBlock + r) * D + lane * N;
      const uint8_t* vp = a.v_pool + (ph * kBlock + r) * D + lane * N;
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const float2 k = from_e4m3x2(*reinterpret_cast<const uint16_t*>(kp + j));
        s = fmaf(q[j], k.x, fmaf(q[j + 1], k.y, s));
      }
#pragma unroll
      for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
      s *= ks;
      const float top = fmaxf(m, s);
      const float keep = exp2f(m - top), p = exp2f(s - top);
      m = top;
      l = fmaf(l, keep, p);
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        const float2 v = from_e4m3x2(*reinterpret_cast<const uint16_t*>(vp + j));
        o[j] = fmaf(o[j], keep, p * v.x * vs);
        o[j + 1] = fmaf(o[j + 1], keep, p * v.y * vs);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) a.out[row * a.ots + h * a.ohs + lane * N + j] = __float2bfloat16_rn(l == 0.f ? 0.f : o[j] / l);
  if (a.lse && lane == 0) a.lse[row * a.Hq + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

}  // namespace

cudaError_t launch_kv8_attend_plain(const Kv8AttendArgs& a, int D, cudaStream_t st) {
  const dim3 grid((a.Hq + 3) / 4, a.rows.max_rows, a.rows.batch);
  if (D == 128) kv8_attend_plain_kernel<128><<<grid, 128, 0, st>>>(a);
  else kv8_attend_plain_kernel<64><<<grid, 128, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace hsa
