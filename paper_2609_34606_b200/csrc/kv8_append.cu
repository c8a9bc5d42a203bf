// Append to the 8-bit paged cache.
//
// For the 64 rows of one (block, key head): x = rotated key or value, scale = 2^s with s least such that
// max |x| <= 448 * 2^s, code = e4m3(x / scale).  Dividing by a power of two is exact, so a value is rounded once.
//
// It has to read 2 bytes and write 1 for every value; everything between stays on the SM.  One CTA takes a block and a
// few heads: the sines of the block's 64 positions are worked out once, into shared memory, and serve all of them.
#include <cuda_fp8.h>

#include "kv8.cuh"

namespace hsa {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// exponent of the least scale that holds values up to `top` (448 = 1.75 * 2^8)
__device__ __forceinline__ int scale_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = static_cast<int>(u >> 23) - 127;
  const int s = e - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return s < kScaleMin ? kScaleMin : s;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// What is stored of a value: NaN as 0, what passes 2^60 as 2^60.
__device__ __forceinline__ float storable(float x, bool* bad) {
  if (!(fabsf(x) <= kTop8)) {
    *bad = true;
    return x != x ? 0.f : copysignf(kTop8, x);
  }
  return x;
}

template <int D>
struct AppendSmem {
  float2 cs[kBlock][D / 2];        // cos, sin of the rows' pairs
  uint4 raw[kBlock][D / 8];        // the keys as they came (partners of the half layout)
  float sum[kThreads / (D / 8)][D];
  float top[kThreads / 32];
};

// One thread: a vector of 8 dims of every (256 / (D / 8))-th row.
template <int D>
__global__ void __launch_bounds__(kThreads) kv8_append_kernel(const Kv8AppendArgs a) {
  constexpr int U = D / 8;             // vectors of a row
  constexpr int R = kThreads / U;      // rows at a time
  constexpr int I = kBlock / R;        // rows of a thread
  extern __shared__ __align__(16) uint8_t smem_raw[];
  AppendSmem<D>& sm = *reinterpret_cast<AppendSmem<D>*>(smem_raw);
  const int tid = threadIdx.x, u = tid % U, row0 = tid / U;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // which block of which sequence
  const int b = static_cast<int>(blockIdx.x) / a.blocks_per_seq;
  const int nth = static_cast<int>(blockIdx.x) % a.blocks_per_seq;
  int first, n;
  const bool fits = a.rows.get(b, &first, &n);
  const int held = __ldg(a.held + b);
  if (!fits || held < 0 || static_cast<int64_t>(held) + n > static_cast<int64_t>(a.max_blocks) * kBlock) {
    if (tid == 0 && nth == 0) kv8_flag(a.status, kDevBounds);
    return;
  }
  const int blk = held / kBlock + nth;
  const int64_t t0 = static_cast<int64_t>(blk) * kBlock;
  const int end = held + n;
  if (t0 >= end || n == 0) return;
  const int r0 = held > t0 ? static_cast<int>(held - t0) : 0;                       // first row of this call
  const int r1 = end - t0 < kBlock ? static_cast<int>(end - t0) : kBlock;           // behind its last
  const int page = __ldg(a.table + static_cast<int64_t>(b) * a.max_blocks + blk);
  if (page < 0 || page >= a.max_pages) {
    if (tid == 0) kv8_flag(a.status, kDevBounds);
    return;
  }
  const int64_t src0 = first + (t0 - held);  // row of the tensors at row 0 of the block (rows r0.. are there)
  if (a.has_rope) {
    // A row's pairs side by side in threads: one position, consecutive frequencies.
    for (int i = tid; i < (r1 - r0) * a.rope.half; i += kThreads) {
      const int r = r0 + i / a.rope.half, p = i % a.rope.half;
      sm.cs[r][p] = rope_cos_sin(a.rope, p, src0 + r, static_cast<int32_t>(t0 + r));
    }
  }
  bool bad = false;
  const int h_end = min(static_cast<int>(blockIdx.y + 1) * a.heads, a.H);
  for (int h = blockIdx.y * a.heads; h < h_end; ++h) {
    const int64_t ph = static_cast<int64_t>(page) * a.H + h;
    const __nv_bfloat16* ksrc = a.k + src0 * a.ts + h * a.hs + u * 8;
    const __nv_bfloat16* vsrc = a.v + src0 * a.ts + h * a.hs + u * 8;
    uint4 kx[I], vx[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int r = row0 + i * R;
      kx[i] = vx[i] = make_uint4(0, 0, 0, 0);
      if (r >= r0 && r < r1) {
        kx[i] = __ldg(reinterpret_cast<const uint4*>(ksrc + r * a.ts));
        vx[i] = __ldg(reinterpret_cast<const uint4*>(vsrc + r * a.ts));
      }
    }
    if (a.has_rope && !a.rope.interleaved) {
#pragma unroll
      for (int i = 0; i < I; ++i) sm.raw[row0 + i * R][u] = kx[i];
    }
    __syncthreads();  // (sines and raw keys are there)
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
      const bool is_k = which == 0;
      float x[I][8];
      float top = 0.f;
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const int r = row0 + i * R;
        const uint4 w = is_k ? kx[i] : vx[i];
        x[i][0] = bf_lo(w.x); x[i][1] = bf_hi(w.x); x[i][2] = bf_lo(w.y); x[i][3] = bf_hi(w.y);
        x[i][4] = bf_lo(w.z); x[i][5] = bf_hi(w.z); x[i][6] = bf_lo(w.w); x[i][7] = bf_hi(w.w);
        if (is_k && a.has_rope && r >= r0 && r < r1) {
          if (a.rope.interleaved) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (u * 4 + j < a.rope.half) {
                const float2 cs = sm.cs[r][u * 4 + j];
                const float va = x[i][2 * j], vb = x[i][2 * j + 1];
                x[i][2 * j] = fmaf(va, cs.x, -(vb * cs.y));
                x[i][2 * j + 1] = fmaf(vb, cs.x, va * cs.y);
              }
          } else {
            const __nv_bfloat16* raw = reinterpret_cast<const __nv_bfloat16*>(&sm.raw[r][0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int dim = u * 8 + j;
              if (dim < a.rope.half) {
                const float2 cs = sm.cs[r][dim];
                x[i][j] = fmaf(x[i][j], cs.x, -(__bfloat162float(raw[dim + a.rope.half]) * cs.y));
              } else if (dim < 2 * a.rope.half) {
                const float2 cs = sm.cs[r][dim - a.rope.half];
                x[i][j] = fmaf(x[i][j], cs.x, __bfloat162float(raw[dim - a.rope.half]) * cs.y);
              }
            }
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[i][j] = storable(x[i][j], &bad);
          top = fmaxf(top, fabsf(x[i][j]));
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      if ((tid & 31) == 0) sm.top[tid / 32] = top;
      uint8_t* codes = (is_k ? a.k_pool : a.v_pool) + ph * (kBlock * D) + u * 8;
      float* scale_at = (is_k ? a.k_scale : a.v_scale) + ph;
      const float old_scale = r0 > 0 ? *scale_at : 0.f;
      __syncthreads();  // (also: everybody has read the old scale)
#pragma unroll
      for (int i = 0; i < kThreads / 32; ++i) top = fmaxf(top, sm.top[i]);
      const float scale = fmaxf(pow2(scale_exponent(top)), old_scale), inv = 1.f / scale;
      if (tid == 0) *scale_at = scale;
      const bool grown = r0 > 0 && scale > old_scale;
      const float shrink = r0 > 0 ? old_scale * inv : 0.f;
      const bool sums = is_k && a.ksum != nullptr;
      float sum[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] = 0.f;
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const int r = row0 + i * R;
        uint2* at = reinterpret_cast<uint2*>(codes + r * D);
        if ((r >= r0 && r < r1) || r0 == 0) {
          uint2 c;
          c.x = e4m3x2(x[i][0] * inv, x[i][1] * inv) | e4m3x2(x[i][2] * inv, x[i][3] * inv) << 16;
          c.y = e4m3x2(x[i][4] * inv, x[i][5] * inv) | e4m3x2(x[i][6] * inv, x[i][7] * inv) << 16;
          *at = c;
          if (sums)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += x[i][j];
        } else if (grown || (sums && r < r0)) {
          // rows of earlier calls: their codes follow a grown scale
          const uint2 c = *at;
          const uint32_t w[2] = {c.x, c.y};
          uint32_t y[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 lo = from_e4m3x2(w[j] & 0xffffu), hi = from_e4m3x2(w[j] >> 16);
            y[j] = e4m3x2(lo.x * shrink, lo.y * shrink) | e4m3x2(hi.x * shrink, hi.y * shrink) << 16;
            if (sums && r < r0) {
              const float2 l2 = from_e4m3x2(y[j] & 0xffffu), h2 = from_e4m3x2(y[j] >> 16);
              sum[4 * j] = fmaf(l2.x, scale, sum[4 * j]);
              sum[4 * j + 1] = fmaf(l2.y, scale, sum[4 * j + 1]);
              sum[4 * j + 2] = fmaf(h2.x, scale, sum[4 * j + 2]);
              sum[4 * j + 3] = fmaf(h2.y, scale, sum[4 * j + 3]);
            }
          }
          if (grown) *at = make_uint2(y[0], y[1]);
        }
      }
      if (sums) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sm.sum[row0][u * 8 + j] = sum[j];
        __syncthreads();
        if (tid < D) {
          float s = 0.f;
#pragma unroll
          for (int i = 0; i < R; ++i) s += sm.sum[i][tid];
          a.ksum[((static_cast<int64_t>(b) * a.H + h) * a.max_blocks + blk) * D + tid] = s;
        }
      }
      __syncthreads();  // (sm.top, sm.sum and, behind the keys, sm.raw are free again)
    }
  }
  if (bad) kv8_flag(a.status, kDevNonfinite);
}

}  // namespace

cudaError_t kv8_append_init(int D) {
  return D == 128 ? cudaFuncSetAttribute(kv8_append_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(AppendSmem<128>))
                  : cudaFuncSetAttribute(kv8_append_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(AppendSmem<64>));
}

cudaError_t launch_kv8_append(const Kv8AppendArgs& args, int D, int nsm, cudaStream_t st) {
  Kv8AppendArgs a = args;
  a.blocks_per_seq = (a.rows.max_rows + 2 * kBlock - 2) / kBlock;
  const int64_t blocks = static_cast<int64_t>(a.rows.batch) * a.blocks_per_seq;
  // heads of a CTA: enough to share the sines, while three CTAs to an SM are left
  int64_t heads = a.has_rope ? blocks * a.H / (3 * static_cast<int64_t>(nsm)) : 1;
  a.heads = static_cast<int>(heads < 1 ? 1 : heads > 4 ? 4 : heads);
  if (a.heads > a.H) a.heads = a.H;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks), (a.H + a.heads - 1) / a.heads);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = D == 128 ? sizeof(AppendSmem<128>) : sizeof(AppendSmem<64>);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, D == 128 ? kv8_append_kernel<128> : kv8_append_kernel<64>, a);
}

}  // namespace hsa
