// Append to the 8-bit paged cache.
//
// For the 64 rows of one (block, key head): x = rotated key or value, scale = 2^s with s least such that
// max |x| <= 448 * 2^s, code = e4m3(x / scale).  Dividing by a power of two is exact, so a value is rounded once.
//
// It has to read 2 bytes and write 1 for every value; everything between stays on the SM.  One CTA takes a block and a few
// heads.  The sines of the block's 64 positions are worked out once, into shared memory, while the first head's rows are on their
// way, and serve all heads; a head's rows are loaded while those of the head before it are turned and rounded, in registers; and
// one barrier a head does for the maxima of keys and values, the partners of the next head's half layout, and the sums of the last
// head's keys.  (With four barriers a head and nothing in flight across them 31 us instead of 18 for 4680 tokens, 12 heads of 128.)
// Measured: 4680 tokens, 12 heads of 128 with positions and sums, 43 MB: 17 us (2.5 TB/s: 74 blocks in four groups of heads, two CTAs
// to an SM, each with a start, the block's sines and three heads in turn); 30,000 tokens of 8 heads without positions 36 us (5.1 TB/s),
// with them 59 (the rotation's instructions: the schedulers issue two cycles of three); ragged prompts, heads of 64, 270 MB: 52 us (5.2 TB/s); a token of 48 sequences 5.9 us, of which the
// launch is 3 and the rest loads that wait for one another.
#include <cuda_fp8.h>

#include "kv8.cuh"

namespace hsa {

namespace {

// 512 for heads of 128, 256 for 64: two rows to a thread.  (More rows to a thread make more code, whose way from memory is most of
// a small call's time; with one row to a thread too little is in flight.)
template <int D>
constexpr int kThreads = 4 * D;

// what keys become; kHalfOdd: halves that are no whole vectors
enum { kPlain, kInterleaved, kHalf, kHalfOdd };

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

__device__ __forceinline__ float inverse(float scale) { return __uint_as_float((254u << 23) - __float_as_uint(scale)); }  // of a power of two

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// What is stored of a value: NaN as 0, what passes 2^60 as 2^60.
__device__ __forceinline__ float storable(float x) { return x != x ? 0.f : fminf(fmaxf(x, -kTop8), kTop8); }

// Where a pair's cosine and sine stand in its row.  Lanes next to each other, which have vectors next to each other, read 16 bytes
// next to each other: the half layout has four cosines of a vector, then the same four of the next, and the sines behind; the
// interleaved one two cosines and sines.  (A vector's in a row: four lanes of eight meet in a bank.)
template <int D, int MODE>
__device__ __forceinline__ int cos_at(int pair) {
  if (MODE == kHalf) return pair % 8 / 4 * (D / 4) + pair / 8 * 4 + pair % 4;
  if (MODE == kInterleaved) return pair % 4 / 2 * D / 2 + pair / 4 * 4 + pair % 2 * 2;
  return 2 * pair;
}
template <int D, int MODE>
__device__ __forceinline__ int sin_at(int pair) { return cos_at<D, MODE>(pair) + (MODE == kHalf ? D / 2 : 1); }

// two fp32 at a time
__device__ __forceinline__ void mul2(float& a, float& b, float c, float d) {
  asm("{\n.reg .b64 x, y;\nmov.b64 x, {%0, %1};\nmov.b64 y, {%2, %3};\nmul.rn.f32x2 x, x, y;\nmov.b64 {%0, %1}, x;\n}\n" : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
__device__ __forceinline__ void fma2(float& a, float& b, float c, float d, float e, float f) {
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%0, %1};\nmov.b64 y, {%2, %3};\nmov.b64 z, {%4, %5};\nfma.rn.f32x2 x, x, y, z;\nmov.b64 {%0, %1}, x;\n}\n"
      : "+f"(a), "+f"(b)
      : "f"(c), "f"(d), "f"(e), "f"(f));
}
__device__ __forceinline__ uint2 codes(const float (&x)[8], float inv) {
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    y[j] = x[j];
    y[j + 1] = x[j + 1];
    mul2(y[j], y[j + 1], inv, inv);
  }
  return make_uint2(e4m3x2(y[0], y[1]) | e4m3x2(y[2], y[3]) << 16, e4m3x2(y[4], y[5]) | e4m3x2(y[6], y[7]) << 16);
}
__device__ __forceinline__ void values(uint2 c, float (&x)[8]) {
  const float2 a = from_e4m3x2(c.x & 0xffffu), b = from_e4m3x2(c.x >> 16), d = from_e4m3x2(c.y & 0xffffu), e = from_e4m3x2(c.y >> 16);
  x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = d.x; x[5] = d.y; x[6] = e.x; x[7] = e.y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) { return __float_as_uint(lo) >> 16 | (__float_as_uint(hi) & 0xffff0000u); }

template <int D>
struct AppendSmem {
  float cs[kBlock][D];                    // cos, sin of the rows' pairs
  uint4 raw[2][kBlock][D / 8];            // the keys as they came (partners of the half layout), of this head and the next
  float sum[2][kThreads<D> / 32][D];         // a warp's rows
  float top[2][2][kThreads<D> / 32];         // [head parity][keys, values]
};

__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void unpack(uint4 w, float (&x)[8]) {
  x[0] = bf_lo(w.x); x[1] = bf_hi(w.x); x[2] = bf_lo(w.y); x[3] = bf_hi(w.y);
  x[4] = bf_lo(w.z); x[5] = bf_hi(w.z); x[6] = bf_lo(w.w); x[7] = bf_hi(w.w);
}

// One thread: a vector of 8 dims of every 32nd row.
template <int D, int MODE>
__global__ void __launch_bounds__(kThreads<D>, D == 128 ? 2 : 4) kv8_append_kernel(const Kv8AppendArgs a) {
  constexpr int U = D / 8;             // vectors of a row
  constexpr int R = kThreads<D> / U;      // rows at a time
  constexpr int I = kBlock / R;        // rows of a thread
  extern __shared__ __align__(16) uint8_t smem_raw[];
  AppendSmem<D>& sm = *reinterpret_cast<AppendSmem<D>*>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32, u = tid % U, row0 = tid / U;
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
  const int64_t src0 = first + (t0 - held);  // row of the tensors at row 0 of the block (rows r0.. are there)
  const int h0 = blockIdx.y * a.heads, h_end = min(h0 + a.heads, a.H);
  constexpr bool swaps = MODE == kHalf || MODE == kHalfOdd;  // partners are in other threads' vectors
  const auto is_new = [&](int i) { return row0 + i * R >= r0 && row0 + i * R < r1; };
  uint4 kx[I], vx[I];
  const int64_t base = (src0 + row0) * a.ts + u * 8, step = R * a.ts;
  const auto load = [&](int h) {
    const int64_t at = base + h * a.hs;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      kx[i] = vx[i] = make_uint4(0, 0, 0, 0);
      if (is_new(i)) {
        kx[i] = __ldg(reinterpret_cast<const uint4*>(a.k + at + i * step));
        vx[i] = __ldg(reinterpret_cast<const uint4*>(a.v + at + i * step));
      }
    }
  };
  load(h0);
  const int page = __ldg(a.table + static_cast<int64_t>(b) * a.max_blocks + blk);
  if constexpr (MODE != kPlain) {
    // A row to a warp, its pairs side by side in lanes: one position, consecutive frequencies.
    for (int r = r0 + warp; r < r1; r += kThreads<D> / 32) {
      for (int p = lane; p < a.rope.half; p += 32) {
        const float2 cs = rope_cos_sin(a.rope, p, src0 + r, static_cast<int32_t>(t0 + r));
        sm.cs[r][cos_at<D, MODE>(p)] = cs.x;
        sm.cs[r][sin_at<D, MODE>(p)] = cs.y;
      }
    }
    if constexpr (swaps) {
#pragma unroll
      for (int i = 0; i < I; ++i) sm.raw[0][row0 + i * R][u] = kx[i];
    }
    __syncthreads();
  }
  if (page < 0 || page >= a.max_pages) {
    if (tid == 0) kv8_flag(a.status, kDevBounds);
    return;
  }
  bool bad = false;
  const bool sums = a.ksum != nullptr;
  // the sum of the keys of the head before h, whose warps' sums a barrier has let through
  const auto put_sum = [&](int h) {
    if (tid < D) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < kThreads<D> / 32; ++i) s += sm.sum[(h - h0) & 1][i][tid];
      a.ksum[((static_cast<int64_t>(b) * a.H + h) * a.max_blocks + blk) * D + tid] = s;
    }
  };
#pragma unroll 1
  for (int h = h0; h < h_end; ++h) {
    const int par = (h - h0) & 1;
    const int64_t ph = static_cast<int64_t>(page) * a.H + h;
    const float old_k = r0 > 0 ? a.k_scale[ph] : 0.f, old_v = r0 > 0 ? a.v_scale[ph] : 0.f;
    float x[I][8];                     // keys as they are stored
    uint4 v[I];
    float top_k = 0.f, top_v = 0.f;
    uint32_t most = 0;                 // of the values, as pairs of bf16
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int r = row0 + i * R;
      unpack(kx[i], x[i]);
      v[i] = vx[i];
      if (MODE != kPlain && is_new(i)) {
        if constexpr (MODE == kInterleaved) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (u * 4 + j < a.rope.half) {
              const float2 cs = *reinterpret_cast<const float2*>(&sm.cs[r][cos_at<D, MODE>(u * 4 + j)]);
              const float va = x[i][2 * j], vb = x[i][2 * j + 1];
              x[i][2 * j] = fmaf(va, cs.x, -(vb * cs.y));
              x[i][2 * j + 1] = fmaf(vb, cs.x, va * cs.y);
            }
        } else if constexpr (MODE == kHalf) {
          const int hv = a.rope.half / 8;
          if (u < 2 * hv) {
            float y[8];
            unpack(sm.raw[par][r][u < hv ? u + hv : u - hv], y);
            const float sign = u < hv ? -1.f : 1.f;
            const int w = (u < hv ? u : u - hv) * 8;
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
              const float4 c = *reinterpret_cast<const float4*>(&sm.cs[r][cos_at<D, MODE>(w + j)]);
              const float4 d = *reinterpret_cast<const float4*>(&sm.cs[r][sin_at<D, MODE>(w + j)]);
              mul2(y[j], y[j + 1], sign, sign);
              mul2(y[j + 2], y[j + 3], sign, sign);
              mul2(y[j], y[j + 1], d.x, d.y);
              mul2(y[j + 2], y[j + 3], d.z, d.w);
              fma2(x[i][j], x[i][j + 1], c.x, c.y, y[j], y[j + 1]);
              fma2(x[i][j + 2], x[i][j + 3], c.z, c.w, y[j + 2], y[j + 3]);
            }
          }
        } else {
          const __nv_bfloat16* raw = reinterpret_cast<const __nv_bfloat16*>(&sm.raw[par][r][0]);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int dim = u * 8 + j;
            if (dim < 2 * a.rope.half) {
              const bool first = dim < a.rope.half;
              const float2 cs = *reinterpret_cast<const float2*>(&sm.cs[r][cos_at<D, MODE>(first ? dim : dim - a.rope.half)]);
              const float y = __bfloat162float(raw[first ? dim + a.rope.half : dim - a.rope.half]);
              x[i][j] = fmaf(x[i][j], cs.x, (first ? -1.f : 1.f) * (y * cs.y));
            }
          }
        }
      }
      // (maxima that keep NaN)
#pragma unroll
      for (int j = 0; j < 8; j += 2) asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(top_k) : "f"(x[i][j]), "f"(x[i][j + 1]));
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(most) : "r"(w[j] & 0x7fff7fffu));
    }
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(top_v) : "f"(bf_lo(most)), "f"(bf_hi(most)));
    if (h + 1 < h_end) {
      load(h + 1);
      if constexpr (swaps) {
#pragma unroll
        for (int i = 0; i < I; ++i) sm.raw[par ^ 1][row0 + i * R][u] = kx[i];
      }
    }
    const auto meet = [&]() {  // the maxima of the CTA
      top_k = warp_max(top_k);
      top_v = warp_max(top_v);
      if (lane == 0) {
        sm.top[par][0][warp] = top_k;
        sm.top[par][1][warp] = top_v;
      }
      __syncthreads();  // (also: everybody has read the old scales, and the last head's sums are there)
      top_k = warp_max(sm.top[par][0][lane % (kThreads<D> / 32)]);
      top_v = warp_max(sm.top[par][1][lane % (kThreads<D> / 32)]);
    };
    meet();
    if (__builtin_expect(!(top_k <= kTop8) || !(top_v <= kTop8), 0)) {
      // something that cannot be stored as it is
      __syncthreads();  // (the maxima have been read)
      top_k = top_v = 0.f;
      bad = true;
#pragma unroll
      for (int i = 0; i < I; ++i) {
        float y[8];
        unpack(v[i], y);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[i][j] = storable(x[i][j]);
          y[j] = storable(y[j]);
          top_k = fmaxf(top_k, fabsf(x[i][j]));
          top_v = fmaxf(top_v, fabsf(y[j]));
        }
        v[i] = make_uint4(pack(y[0], y[1]), pack(y[2], y[3]), pack(y[4], y[5]), pack(y[6], y[7]));  // (exact)
      }
      meet();
    }
    if (sums && h > h0) put_sum(h - 1);
    const float scale_k = fmaxf(pow2(scale_exponent(top_k)), old_k), scale_v = fmaxf(pow2(scale_exponent(top_v)), old_v);
    const float inv_k = inverse(scale_k), inv_v = inverse(scale_v);
    if (tid == 0) {
      a.k_scale[ph] = scale_k;
      a.v_scale[ph] = scale_v;
    }
    const int64_t to = ph * (kBlock * D) + row0 * D + u * 8;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      if (!is_new(i) && r0 > 0) continue;  // (rows behind the last one of a block that begins here: zeros)
      float y[8];
      unpack(v[i], y);
      *reinterpret_cast<uint2*>(a.k_pool + to + i * (R * D)) = codes(x[i], inv_k);
      *reinterpret_cast<uint2*>(a.v_pool + to + i * (R * D)) = codes(y, inv_v);
      if (sums) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += x[i][j];
      }
    }
    if (r0 > 0 && (scale_k > old_k || scale_v > old_v || sums)) {
      // rows of earlier calls, and those behind the last: their codes follow a scale that has grown
#pragma unroll 1
      for (int job = 0; job < 2 * I; ++job) {
        const bool is_k = job < I;
        const int i = is_k ? job : job - I, r = row0 + i * R;
        const float old_scale = is_k ? old_k : old_v, scale = is_k ? scale_k : scale_v;
        const bool summed = is_k && sums && r < r0;
        if ((r >= r0 && r < r1) || !(scale > old_scale || summed)) continue;
        const float shrink = old_scale * (is_k ? inv_k : inv_v);
        uint2* at = reinterpret_cast<uint2*>((is_k ? a.k_pool : a.v_pool) + to + i * (R * D));
        const uint2 c = *at;
        float y[8];
        values(c, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= shrink;
        const uint2 now = codes(y, 1.f);
        if (scale > old_scale) *at = now;
        if (summed) {
          values(now, y);
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[j] = fmaf(y[j], scale, sum[j]);
        }
      }
    }
    if (sums) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int o = U; o < 32; o <<= 1) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
        if (lane < U) sm.sum[par][warp][u * 8 + j] = sum[j];
      }
    }
  }
  if (sums) {
    __syncthreads();
    put_sum(h_end - 1);
  }
  if (bad && tid == 0) kv8_flag(a.status, kDevNonfinite);
}

}  // namespace

namespace {

using AppendKernel = void (*)(Kv8AppendArgs);
template <int D>
constexpr AppendKernel kKernels[4] = {kv8_append_kernel<D, kPlain>, kv8_append_kernel<D, kInterleaved>, kv8_append_kernel<D, kHalf>,
                                      kv8_append_kernel<D, kHalfOdd>};

}  // namespace

cudaError_t kv8_append_init(int D) {
  cudaError_t e = cudaSuccess;
  for (int mode = 0; mode < 4 && e == cudaSuccess; ++mode)
    e = cudaFuncSetAttribute(D == 128 ? kKernels<128>[mode] : kKernels<64>[mode], cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(D == 128 ? sizeof(AppendSmem<128>) : sizeof(AppendSmem<64>)));
  return e;
}

cudaError_t launch_kv8_append(const Kv8AppendArgs& args, int D, int nsm, cudaStream_t st) {
  Kv8AppendArgs a = args;
  a.blocks_per_seq = (a.rows.max_rows + 2 * kBlock - 2) / kBlock;
  const int64_t blocks = static_cast<int64_t>(a.rows.batch) * a.blocks_per_seq;
  // Heads of a CTA: as many as leave two CTAs to an SM, at most 6, in even shares: with positions they share the sines, and all share a
  // CTA's start.  (At most 16: ragged prompts of 16 heads of 64 61 us instead of 52, for want of CTAs to even out the last ones.)
  int64_t heads = blocks * a.H / (2 * static_cast<int64_t>(nsm));
  heads = heads < 1 ? 1 : heads > 6 ? 6 : heads > a.H ? a.H : heads;
  const int groups = static_cast<int>((a.H + heads - 1) / heads);
  a.heads = (a.H + groups - 1) / groups;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks), groups);
  cfg.blockDim = dim3(D == 128 ? kThreads<128> : kThreads<64>);
  cfg.dynamicSmemBytes = D == 128 ? sizeof(AppendSmem<128>) : sizeof(AppendSmem<64>);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const int mode = !a.has_rope ? kPlain : a.rope.interleaved ? kInterleaved : a.rope.half % 8 ? kHalfOdd : kHalf;
  return cudaLaunchKernelEx(&cfg, D == 128 ? kKernels<128>[mode] : kKernels<64>[mode], a);
}

}  // namespace hsa
