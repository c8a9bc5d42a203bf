// Rotary positions: out = amplitude * R(position * frequency) x for the pairs of each row.
//
// What it needs: every value read once and written once; the arithmetic (three operations a value, a sine and a cosine a
// pair and token) hides behind that if the sines are not worked out again for every head.  So a thread owns a few pairs
// of a token and walks over heads with them.
// Measured: 20,011 tokens x 8 heads of 128 in fp32 26.4 us (6.2 TB/s; a plain copy 6.54), 20,011 x 12 in bf16 27.4 us (4.5 TB/s:
// eight sines to 32 bytes of a row), 4680 x 12 7.0 us, one token 3 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "rope.cuh"

namespace hsa {

namespace {

constexpr int kRows = 4;  // heads in flight

template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__half* p, float x) { *p = __float2half_rn(x); }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// n / d for n < 2^31 as a product: with 2^(s - 1) < d <= 2^s and m = floor(2^(31 + s) / d) + 1, n m / 2^(31 + s) is above n / d by
// at most n / 2^(31 + s) < 1 / d, and m is below 2^32.
struct Divide {
  uint32_t m;
  int s;
  int d;
  __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return static_cast<uint32_t>(static_cast<uint64_t>(n) * m >> s); }
};
Divide divide_by(int d) {
  int s = 0;
  while ((1ll << s) < d) ++s;
  return Divide{static_cast<uint32_t>((1ull << (31 + s)) / d + 1), 31 + s, d};
}

struct RopeArgs {
  const void* x;
  void* out;
  int64_t ts, hs, ots, ohs;
  int H, D, heads_per_thread, head_groups;
  uint32_t threads;   // of a slab of tokens: tokens * head_groups * units
  int64_t tokens, slab;
  int units;
  Divide by_units, by_groups;
  RopeDev rope;
};

// MODE 0, interleaved: a unit is a 16-byte vector, which holds whole pairs; pairs behind the rotated ones get the identity.
// MODE 1, halves whose length is a multiple of a vector: a unit is a vector of the first half with its partner, units
//         behind those are vectors that pass through.
// MODE 2, other halves: a unit is one pair, or one value that passes through.
template <typename T, int MODE>
__global__ void __launch_bounds__(256, sizeof(T) == 4 ? 4 : 3) rope_kernel(const RopeArgs a) {
  constexpr int N = Vec<T>::N;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t idx = blockIdx.x * 256 + threadIdx.x;
  if (idx >= a.threads) return;
  const uint32_t rest = a.by_units(idx), in_slab = a.by_groups(rest);
  const int u = static_cast<int>(idx - rest * a.units), hg = static_cast<int>(rest - in_slab * a.head_groups);
  const int64_t t = blockIdx.y * a.slab + in_slab;
  if (t >= a.tokens) return;
  const int h0 = hg * a.heads_per_thread, h1 = h0 + a.heads_per_thread < a.H ? h0 + a.heads_per_thread : a.H;
  const T* x = static_cast<const T*>(a.x) + t * a.ts;
  T* out = static_cast<T*>(a.out) + t * a.ots;
  const RopeDev& r = a.rope;
  if constexpr (MODE == 2) {
    const bool turn = u < r.half;
    const int d0 = turn ? u : u + r.half;
    const float2 cs = turn ? rope_cos_sin(r, u, t, static_cast<int32_t>(t)) : make_float2(1.f, 0.f);
    for (int h = h0; h < h1; h += kRows) {
      T va[kRows], vb[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (h + i < h1) {
          const T* p = x + (h + i) * a.hs + d0;
          va[i] = p[0];
          if (turn) vb[i] = p[r.half];
        }
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (h + i < h1) {
          T* o = out + (h + i) * a.ohs + d0;
          if (turn) {
            const float v0 = to_f(va[i]), v1 = to_f(vb[i]);
            put(&va[i], fmaf(v0, cs.x, -(v1 * cs.y)));
            put(o + r.half, fmaf(v1, cs.x, v0 * cs.y));
          }
          o[0] = va[i];
        }
    }
    return;
  } else {
    constexpr int P = MODE == 0 ? N / 2 : N;  // pairs of a unit
    const bool turn = MODE == 0 || u * N < r.half;
    const int d0 = turn ? u * N : u * N + r.half;
    uint4 va[kRows], vb[kRows];
    const auto load = [&](int h) {
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (h + i < h1) {
          const T* p = x + (h + i) * a.hs + d0;
          va[i] = *reinterpret_cast<const uint4*>(p);
          if (MODE == 1 && turn) vb[i] = *reinterpret_cast<const uint4*>(p + r.half);
        }
    };
    load(h0);  // (on their way while the sines are worked out)
    float2 cs[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int pair = MODE == 0 ? u * P + i : u * N + i;
      cs[i] = make_float2(1.f, 0.f);
      if (pair < r.half) cs[i] = rope_cos_sin(r, pair, t, static_cast<int32_t>(t));
    }
    for (int h = h0; h < h1; h += kRows) {
      if (h > h0) load(h);
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (h + i < h1) {
          T* o = out + (h + i) * a.ohs + d0;
          if (turn) {
            T* ea = reinterpret_cast<T*>(&va[i]);
            T* eb = reinterpret_cast<T*>(&vb[i]);
#pragma unroll
            for (int j = 0; j < P; ++j) {
              T* p0 = MODE == 0 ? ea + 2 * j : ea + j;
              T* p1 = MODE == 0 ? ea + 2 * j + 1 : eb + j;
              const float v0 = to_f(*p0), v1 = to_f(*p1);
              if (MODE == 1 || u * P + j < r.half) {  // (values that pass through keep their bits)
                put(p0, fmaf(v0, cs[j].x, -(v1 * cs[j].y)));
                put(p1, fmaf(v1, cs[j].x, v0 * cs[j].y));
              }
            }
            if (MODE == 1) *reinterpret_cast<uint4*>(o + r.half) = vb[i];
          }
          *reinterpret_cast<uint4*>(o) = va[i];
        }
    }
  }
}

template <typename T>
cudaError_t launch_rope(RopeArgs a, int64_t tokens, int nsm, cudaStream_t st) {
  constexpr int N = Vec<T>::N;
  const int rest = a.D - 2 * a.rope.half;
  const int mode = a.rope.interleaved ? 0 : a.rope.half % N == 0 ? 1 : 2;
  a.units = mode == 0 ? a.D / N : mode == 1 ? (a.rope.half + rest) / N : a.rope.half + rest;
  // As many heads to a thread as leave 1024 threads to an SM, at most 4, whose loads are in flight at once: the sines are shared
  // by them.  (At most 16: 20,011 tokens, 12 heads of 128 in bf16 32 us, for want of threads.)
  int64_t per = tokens * a.H * a.units / (static_cast<int64_t>(nsm) * 1024);
  a.heads_per_thread = static_cast<int>(per < 1 ? 1 : per > kRows ? kRows : per);
  if (a.heads_per_thread > a.H) a.heads_per_thread = a.H;
  a.head_groups = (a.H + a.heads_per_thread - 1) / a.heads_per_thread;
  a.heads_per_thread = (a.H + a.head_groups - 1) / a.head_groups;  // even shares
  // threads are counted in 31 bits: more tokens than that go into slabs
  const int64_t per_token = static_cast<int64_t>(a.head_groups) * a.units;
  a.tokens = tokens;
  a.slab = std::min(tokens, static_cast<int64_t>((1ll << 31) - 256) / per_token);
  a.threads = static_cast<uint32_t>(a.slab * per_token);
  a.by_units = divide_by(a.units);
  a.by_groups = divide_by(a.head_groups);
  const int64_t slabs = (tokens + a.slab - 1) / a.slab;
  if (slabs > 65535) return cudaErrorInvalidValue;  // (more than any memory holds)
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((a.threads + 255) / 256, static_cast<unsigned>(slabs));
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, mode == 0 ? rope_kernel<T, 0> : mode == 1 ? rope_kernel<T, 1> : rope_kernel<T, 2>, a);
}

}  // namespace

bool rope_args(const hsa_rope_args* r, int head_dim, int64_t tokens, bool transpose, RopeDev* out) {
  if (!r || !r->turns_dev || (reinterpret_cast<uintptr_t>(r->turns_dev) & 7) || (reinterpret_cast<uintptr_t>(r->positions_dev) & 3))
    return false;
  if (r->rot_dim < 2 || (r->rot_dim & 1) || r->rot_dim > head_dim) return false;
  if (r->layout != HSA_ROPE_HALF && r->layout != HSA_ROPE_INTERLEAVED) return false;
  if (r->n_axes < 1 || r->n_axes > 3) return false;
  int64_t sum = 0;
  for (int i = 0; i < r->n_axes; ++i) {
    if (r->axis_pairs[i] < 0) return false;
    sum += r->axis_pairs[i];
  }
  if (sum != r->rot_dim / 2) return false;
  if (r->positions_dev && r->n_axes > 1 && r->axis_stride < tokens) return false;
  if (!std::isfinite(r->amplitude)) return false;
  out->turns = r->turns_dev;
  out->pos = r->positions_dev;
  out->axis_stride = r->axis_stride;
  out->half = r->rot_dim / 2;
  out->interleaved = r->layout == HSA_ROPE_INTERLEAVED;
  out->end0 = r->axis_pairs[0];
  out->end1 = r->n_axes > 1 ? r->axis_pairs[0] + r->axis_pairs[1] : out->half;
  if (r->n_axes == 1) out->end0 = out->half;
  out->amplitude = r->amplitude;
  out->sign = transpose ? -1.f : 1.f;
  return true;
}

}  // namespace hsa

using namespace hsa;

extern "C" {

int hsa_rope_table(const hsa_rope_config* c, uint64_t* turns_host, float* amplitude_host) {
  if (!c || !turns_host || !amplitude_host) return HSA_ERR_INVALID_ARG;
  if (c->head_dim < 8 || c->head_dim > 512 || (c->head_dim % 8)) return HSA_ERR_INVALID_ARG;
  if (c->rot_dim < 2 || (c->rot_dim & 1) || c->rot_dim > c->head_dim) return HSA_ERR_INVALID_ARG;
  if (c->layout != HSA_ROPE_HALF && c->layout != HSA_ROPE_INTERLEAVED) return HSA_ERR_INVALID_ARG;
  if (c->n_axes < 1 || c->n_axes > 3) return HSA_ERR_INVALID_ARG;
  int64_t sum = 0;
  for (int i = 0; i < c->n_axes; ++i) {
    if (c->axis_pairs[i] < 0) return HSA_ERR_INVALID_ARG;
    sum += c->axis_pairs[i];
  }
  if (sum != c->rot_dim / 2) return HSA_ERR_INVALID_ARG;
  if (!(c->base > 1.0) || !std::isfinite(c->base)) return HSA_ERR_INVALID_ARG;
  if (c->scaling < HSA_ROPE_SCALE_NONE || c->scaling > HSA_ROPE_SCALE_BANDS) return HSA_ERR_INVALID_ARG;
  if (c->scaling != HSA_ROPE_SCALE_NONE && (!(c->factor >= 1.0) || !std::isfinite(c->factor))) return HSA_ERR_INVALID_ARG;
  if (c->scaling == HSA_ROPE_SCALE_BANDS &&
      (!(c->trained_tokens > 0.0) || !std::isfinite(c->trained_tokens) || !(c->beta_slow >= 0.0) ||
       !(c->beta_fast > c->beta_slow) || !std::isfinite(c->beta_fast)))
    return HSA_ERR_INVALID_ARG;
  const long double two_pi = 6.283185307179586476925286766559L;
  int p = 0;
  for (int a = 0; a < c->n_axes; ++a) {
    const int n = c->axis_pairs[a];
    long double base = c->base;
    if (c->scaling == HSA_ROPE_SCALE_BASE && n > 1)
      base *= powl(static_cast<long double>(c->factor), static_cast<long double>(n) / (n - 1));
    for (int i = 0; i < n; ++i, ++p) {
      long double f = powl(base, -static_cast<long double>(i) / n);
      if (c->scaling == HSA_ROPE_SCALE_LINEAR) f /= c->factor;
      if (c->scaling == HSA_ROPE_SCALE_BANDS) {
        long double g = (c->trained_tokens * f / two_pi - c->beta_slow) / (c->beta_fast - c->beta_slow);
        g = g < 0 ? 0 : g > 1 ? 1 : g;
        f *= g + (1 - g) / c->factor;
      }
      turns_host[p] = static_cast<uint64_t>(roundl(f / two_pi * 18446744073709551616.0L));
    }
  }
  *amplitude_host = c->scaling == HSA_ROPE_SCALE_BANDS ? static_cast<float>(0.1 * std::log(c->factor) + 1.0) : 1.0f;
  return HSA_OK;
}

int hsa_rope(const void* x, void* out, int32_t type, int32_t n_tokens, int32_t num_heads, int32_t head_dim,
             int64_t tok_stride, int64_t head_stride, int64_t out_tok_stride, int64_t out_head_stride,
             const hsa_rope_args* rope, uint32_t flags, void* stream) {
  if (type != HSA_TYPE_BF16 && type != HSA_TYPE_FP16 && type != HSA_TYPE_FP32) return HSA_ERR_INVALID_ARG;
  if (n_tokens < 0 || num_heads < 1 || num_heads > 4096) return HSA_ERR_INVALID_ARG;
  if (head_dim < 8 || head_dim > 512 || (head_dim % 8)) return HSA_ERR_INVALID_ARG;
  if (flags & ~HSA_ROPE_TRANSPOSE) return HSA_ERR_INVALID_ARG;
  RopeArgs a{};
  if (!rope_args(rope, head_dim, n_tokens, flags & HSA_ROPE_TRANSPOSE, &a.rope)) return HSA_ERR_INVALID_ARG;
  if (n_tokens == 0) return HSA_OK;
  const int vec = type == HSA_TYPE_FP32 ? 4 : 8;
  const int64_t strides[4] = {tok_stride, head_stride, out_tok_stride, out_head_stride};
  for (int64_t s : strides)
    if (s < head_dim || (s % vec)) return HSA_ERR_INVALID_ARG;
  if (!x || !out || (reinterpret_cast<uintptr_t>(x) & 15) || (reinterpret_cast<uintptr_t>(out) & 15)) return HSA_ERR_INVALID_ARG;
  if (x == out && (tok_stride != out_tok_stride || head_stride != out_head_stride)) return HSA_ERR_INVALID_ARG;
  int dev = 0, nsm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return HSA_ERR_CUDA;
  if (cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return HSA_ERR_CUDA;
  a.x = x;
  a.out = out;
  a.ts = tok_stride;
  a.hs = head_stride;
  a.ots = out_tok_stride;
  a.ohs = out_head_stride;
  a.H = num_heads;
  a.D = head_dim;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = type == HSA_TYPE_BF16   ? launch_rope<__nv_bfloat16>(a, n_tokens, nsm, st)
                        : type == HSA_TYPE_FP16 ? launch_rope<__half>(a, n_tokens, nsm, st)
                                                : launch_rope<float>(a, n_tokens, nsm, st);
  return e == cudaSuccess ? HSA_OK : HSA_ERR_CUDA;
}

}  // extern "C"
