// Attention over the 8-bit paged cache for few query rows of a key head (a token of each sequence, a few drafted ones).
//
// Such a call reads every key and value once and does little with it: the bytes bound it.  So one warp of a CTA does
// nothing but keep TMA loads in flight, a ring of page tiles ahead, and eight warps take pages in turn, each on its own:
//   S = Q K^T        16 rows x 64 keys, codes of K turned into fp16 (exact) in registers, fp32 sums
//   y = S * scales + ev,  ev the exponent of the page's value scale: the weights 2^(y - m) carry it, so that codes of V are
//                    all that the second product sees, and the sum of weights takes it out again
//   O += P V         P in fp16 (11 bits)
// with running maxima per warp.  Rows of Q are scaled by a power of two into fp16's range (their 8 bits stay).  At the end of
// an item the warps' parts are added up in shared memory.
#include <cuda_fp8.h>
#include <cuda_fp16.h>

#include "kv8.cuh"
#include "ptx.cuh"

namespace hsa {

namespace {

constexpr int kWarps = 8;                        // warps that take pages; one more loads
constexpr int kThreads = (kWarps + 1) * 32;
constexpr int kMaxRows = 64;                     // rows of an item: up to four tiles of 16
constexpr float kShift = 8.f;                    // the largest weight is 2^8 when the reference is set ...
constexpr float kSlack = 6.f;                    // ... and may grow to 2^14 before it is set anew

struct PageMeta {
  int pos;      // position of the page's first token; < 0: nothing to see
  float ks;     // scale of the keys
  float ev;     // exponent of the values' scale
  float inv;    // 2^-ev
};

template <int D>
struct DecodeSmem {
  static constexpr int kStages = D == 128 ? 8 : 12;
  static constexpr int kTile = kBlock * D;
  uint8_t kv[kStages][2][kTile];
  float o[kWarps][16 * D];
  __half q[kMaxRows][D + 8];
  float qscale[kMaxRows];
  float m[kWarps][16], l[kWarps][16];
  PageMeta meta[kStages];
  uint64_t full[kStages], empty[kStages];
  int last;
};

__device__ __forceinline__ uint32_t half2_of(uint32_t two) {  // two e4m3 codes (low 16 bits) -> f16x2
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory"); }

// The place of four floats of a warp's part in shared memory: row, fourth of 4 dims.  A thread of the product holds D / 4
// dims in a row; the exclusive-or keeps the eight threads of a store apart.
template <int D>
__device__ __forceinline__ int o_at(int row, int four) {
  constexpr int kPer = D / 16;  // fours of a thread
  const int t = four / kPer, f = four % kPer;
  return row * D + (t * kPer + (f ^ (((row & 1) * 4 + t) & (kPer - 1)))) * 4;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) kv8_decode_kernel(const Kv8AttendArgs a, const Kv8Work w,
                                                                 const __grid_constant__ CUtensorMap tm_k,
                                                                 const __grid_constant__ CUtensorMap tm_v) {
  using Smem = DecodeSmem<D>;
  constexpr int kStages = Smem::kStages;
  constexpr int KS = D / 16;       // steps of the first product, columns of 8 / 8 ... of the second: D / 8 tiles
  constexpr int NT = D / 8;
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  const int tiles = w.tile_rows / 16;            // row tiles of an item: as many warps share a page
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], tiles);
    }
    fence_mbar_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Kv8Run run = kv8_run<kThreads>(a, w);
  __syncthreads();
  if (run.lo >= run.hi) return;
  Kv8Walk walk(run);

  if (warp == kWarps) {
    // ---- loads.  The lanes look up 32 pages at a time; lane by lane they are then sent for.
    uint32_t n = 0;
    bool ok = true;
    while (ok && walk.next(a, w, run)) {
      const Kv8Item& it = walk.it;
      for (int s = walk.s0; s < walk.s1; s += 32) {
        int blk = 0, page = -1;
        PageMeta meta{-1, 0.f, 0.f, 0.f};
        if (s + lane < walk.s1) page = kv8_page(a, it, s + lane, &blk);
        if (page >= 0) {
          const int64_t ph = static_cast<int64_t>(page) * a.Hkv + it.h;
          const float vs = __ldg(a.v_scale + ph);
          meta.pos = blk * kBlock;
          meta.ks = __ldg(a.k_scale + ph);
          meta.ev = static_cast<float>(static_cast<int>((__float_as_uint(vs) >> 23) & 255u) - 127);
          meta.inv = 1.f / vs;
        }
        const int count = min(32, walk.s1 - s);
        for (int i = 0; i < count && ok; ++i, ++n) {
          if (lane == i) {
            const uint32_t st = n % kStages;
            ok = mbar_wait(&sm.empty[st], ((n / kStages) & 1) ^ 1);
            sm.meta[st] = meta;
            if (!ok) {
              kv8_flag(a.status, kDevTimeout);
            } else if (page >= 0) {
              const int row = static_cast<int>((static_cast<int64_t>(page) * a.Hkv + it.h) * kBlock);
              mbar_expect_tx(&sm.full[st], 2 * Smem::kTile);
              tma_load_2d(sm.kv[st][0], &tm_k, &sm.full[st], 0, row);
              tma_load_2d(sm.kv[st][1], &tm_v, &sm.full[st], 0, row);
            } else {
              mbar_arrive(&sm.full[st]);
            }
          }
          ok = __shfl_sync(0xffffffffu, ok, i);
        }
      }
    }
    if (!ok)  // pages that nobody took: their loads must not outlive the CTA
      for (uint32_t i = 2; i <= kStages + 1 && i <= n; ++i) mbar_wait(&sm.full[(n - i) % kStages], ((n - i) / kStages) & 1);
    return;
  }

  // ---- pages
  const int g = lane >> 2, t = lane & 3;
  const int tile = warp % tiles, turn = warp / tiles, turns = kWarps / tiles;
  uint32_t n = 0;  // pages of the CTA so far
  bool ok = true;  // false: a wait ran out; nothing more is waited for
  while (walk.next(a, w, run)) {
    const Kv8Item& it = walk.it;
    // rows of Q in fp16, each scaled so that its largest value lies in [2^12, 2^13)
    consumers_sync();  // (the last item's parts and rows have been read)
    for (int r = warp; r < w.tile_rows; r += kWarps) {
      constexpr int N = D / 32;
      float x[N];
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = 0.f;
      if (r < it.rows) {
        const int at = it.row0 + r;
        const __nv_bfloat16* src = a.q + (it.first + at / a.group) * a.ts + (it.h * a.group + at % a.group) * a.hs + lane * N;
#pragma unroll
        for (int j = 0; j < N; ++j) {
          x[j] = __bfloat162float(src[j]);
          top = fmaxf(top, fabsf(x[j]));
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      // (zero, subnormal and infinite rows: an exponent that leaves the factors normal)
      const int e = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100), 127) - 12;
      const float up = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
      for (int j = 0; j < N; ++j) sm.q[r][lane * N + j] = __float2half_rn(x[j] * up);
      if (lane == 0) sm.qscale[r] = __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * a.scale_log2;
    }
    consumers_sync();
    uint32_t qf[KS][4];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const uint2 lo = *reinterpret_cast<const uint2*>(&sm.q[tile * 16 + g][t * (D / 4) + 4 * i]);
      const uint2 hi = *reinterpret_cast<const uint2*>(&sm.q[tile * 16 + g + 8][t * (D / 4) + 4 * i]);
      qf[i][0] = lo.x;
      qf[i][1] = hi.x;
      qf[i][2] = lo.y;
      qf[i][3] = hi.y;
    }
    const int rows = it.rows - tile * 16;        // rows of the tile (may be none)
    const bool upper = rows > 8;
    const float qs0 = sm.qscale[tile * 16 + g], qs1 = sm.qscale[tile * 16 + g + 8];
    const int lim0 = it.limit(a, min(tile * 16 + g, it.rows - 1)), lim1 = it.limit(a, min(tile * 16 + g + 8, it.rows - 1));
    const int lim_low = it.limit(a, min(tile * 16, it.rows - 1));
    float m0 = -1e30f, m1 = -1e30f, l0 = 0.f, l1 = 0.f;
    float o[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;

    const int count = walk.s1 - walk.s0;
    for (int i = (turn + turns - static_cast<int>(n % turns)) % turns; i < count; i += turns) {
      const uint32_t st = (n + i) % kStages;
      if (ok && !mbar_wait(&sm.full[st], ((n + i) / kStages) & 1)) {
        ok = false;
        kv8_flag(a.status, kDevTimeout);
      }
      const PageMeta meta = sm.meta[st];
      if (ok && meta.pos >= 0 && rows > 0) {
        const uint8_t* kt = sm.kv[st][0];
        const uint8_t* vt = sm.kv[st][1];
        float sum0 = 0.f, sum1 = 0.f;
        // half a page at a time: the scores of all of it do not fit the registers beside O and Q
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          float s[4][4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
            uint32_t x[KS];
            if constexpr (D == 128) {
              *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(kt + (half * 32 + j * 8 + g) * 128 + (((2 * t) ^ g) << 4));
              *reinterpret_cast<uint4*>(x + 4) = *reinterpret_cast<const uint4*>(kt + (half * 32 + j * 8 + g) * 128 + (((2 * t + 1) ^ g) << 4));
            } else {
              *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(kt + (half * 32 + j * 8 + g) * 64 + ((t ^ ((g >> 1) & 3)) << 4));
            }
#pragma unroll
            for (int k = 0; k < KS; ++k) mma16816(s[j], qf[k], half2_of(x[k] & 0xffffu), half2_of(x[k] >> 16));
          }
          const float f0 = qs0 * meta.ks, f1 = qs1 * meta.ks;
          float t0 = -INFINITY, t1 = -INFINITY;
          const int pos = meta.pos + half * 32;
          const bool cut = pos + 32 > lim_low;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              s[j][e] = fmaf(s[j][e], f0, meta.ev);
              if (cut && pos + j * 8 + 2 * t + e >= lim0) s[j][e] = -INFINITY;
              t0 = fmaxf(t0, s[j][e]);
            }
            if (upper) {
#pragma unroll
              for (int e = 2; e < 4; ++e) {
                s[j][e] = fmaf(s[j][e], f1, meta.ev);
                if (cut && pos + j * 8 + 2 * t + e - 2 >= lim1) s[j][e] = -INFINITY;
                t1 = fmaxf(t1, s[j][e]);
              }
            }
          }
          t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, 1));
          t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, 2));
          if (upper) {
            t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, 1));
            t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, 2));
          }
          if (__any_sync(0xffffffffu, t0 > m0 + kSlack || t1 > m1 + kSlack)) {
            const float n0 = t0 > m0 + kSlack ? t0 : m0, n1 = t1 > m1 + kSlack ? t1 : m1;
            const float c0 = ex2(m0 - n0), c1 = ex2(m1 - n1);
            m0 = n0;
            m1 = n1;
            l0 *= c0;
            l1 *= c1;
            sum0 *= c0;
            sum1 *= c1;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              o[j][0] *= c0;
              o[j][1] *= c0;
              o[j][2] *= c1;
              o[j][3] *= c1;
            }
          }
          const float r0 = kShift - m0, r1 = kShift - m1;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t p[4] = {0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float x0 = ex2(s[2 * k + e][0] + r0), x1 = ex2(s[2 * k + e][1] + r0);
              sum0 += x0 + x1;
              p[2 * e] = pack_half(x0, x1);
              if (upper) {
                const float y0 = ex2(s[2 * k + e][2] + r1), y1 = ex2(s[2 * k + e][3] + r1);
                sum1 += y0 + y1;
                p[2 * e + 1] = pack_half(y0, y1);
              }
            }
            const int row = half * 32 + 16 * k + 2 * t;  // and row + 1, + 8, + 9: their last three bits are 2t, 2t + 1
            constexpr int WORDS = D / 32;    // 4-byte words of a thread's dims: 16 of 128, 8 of 64
            uint32_t x[4][WORDS];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = row + (e & 1) + (e >> 1) * 8;
              if constexpr (D == 128)
                *reinterpret_cast<uint4*>(x[e]) = *reinterpret_cast<const uint4*>(vt + r * 128 + ((g ^ (2 * t + (e & 1))) << 4));
              else
                *reinterpret_cast<uint2*>(x[e]) = *reinterpret_cast<const uint2*>(vt + r * 64 + (((g >> 1) ^ t) << 4) + (g & 1) * 8);
            }
#pragma unroll
            for (int i2 = 0; i2 < WORDS; ++i2) {
              const uint32_t a_lo = __byte_perm(x[0][i2], x[1][i2], 0x5140), a_hi = __byte_perm(x[0][i2], x[1][i2], 0x7362);
              const uint32_t b_lo = __byte_perm(x[2][i2], x[3][i2], 0x5140), b_hi = __byte_perm(x[2][i2], x[3][i2], 0x7362);
              mma16816(o[4 * i2], p, half2_of(a_lo & 0xffffu), half2_of(b_lo & 0xffffu));
              mma16816(o[4 * i2 + 1], p, half2_of(a_lo >> 16), half2_of(b_lo >> 16));
              mma16816(o[4 * i2 + 2], p, half2_of(a_hi & 0xffffu), half2_of(b_hi & 0xffffu));
              mma16816(o[4 * i2 + 3], p, half2_of(a_hi >> 16), half2_of(b_hi >> 16));
            }
          }
        }
        l0 = fmaf(sum0, meta.inv, l0);
        l1 = fmaf(sum1, meta.inv, l1);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.empty[st]);
    }
    n += static_cast<uint32_t>(count);

    // ---- the warps' parts
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
    l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    if (t == 0) {
      sm.m[warp][g] = m0;
      sm.m[warp][g + 8] = m1;
      sm.l[warp][g] = l0;
      sm.l[warp][g + 8] = l1;
    }
    {
      // columns 2t and 2t + 1 of tile j are dims (D / 8) (2t) + j and (D / 8) (2t + 1) + j: D / 4 dims in a row
      constexpr int kPer = D / 16;
#pragma unroll
      for (int f = 0; f < kPer; ++f) {
        const int e = f >= kPer / 2 ? 1 : 0, j = (f - e * (kPer / 2)) * 4;
        if (g < rows)
          *reinterpret_cast<float4*>(&sm.o[warp][o_at<D>(g, t * kPer + f)]) = make_float4(o[j][e], o[j + 1][e], o[j + 2][e], o[j + 3][e]);
        if (g + 8 < rows)
          *reinterpret_cast<float4*>(&sm.o[warp][o_at<D>(g + 8, t * kPer + f)]) =
              make_float4(o[j][2 + e], o[j + 1][2 + e], o[j + 2][2 + e], o[j + 3][2 + e]);
      }
    }
    consumers_sync();
    constexpr int F = D / 4;
    const bool whole = walk.whole();
    float* part = w.parts + walk.slot() * w.slot_floats;
    for (int i = tid; i < it.rows * F; i += kWarps * 32) {
      const int r = i / F, f = i % F, rt = r / 16, rr = r % 16;
      float m = -1e30f;
      for (int c = rt; c < kWarps; c += tiles) m = fmaxf(m, sm.m[c][rr]);
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      float l = 0.f;
      for (int c = rt; c < kWarps; c += tiles) {
        const float k = ex2(sm.m[c][rr] - m);
        const float4 v = *reinterpret_cast<const float4*>(&sm.o[c][o_at<D>(rr, f)]);
        sum.x = fmaf(v.x, k, sum.x);
        sum.y = fmaf(v.y, k, sum.y);
        sum.z = fmaf(v.z, k, sum.z);
        sum.w = fmaf(v.w, k, sum.w);
        l = fmaf(sm.l[c][rr], k, l);
      }
      if (whole) {
        const int at = it.row0 + r;
        const int64_t tok = it.first + at / a.group;
        const int head = it.h * a.group + at % a.group;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        *reinterpret_cast<uint2*>(a.out + tok * a.ots + head * a.ohs + f * 4) =
            make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
        if (a.lse && f == 0) a.lse[tok * a.Hq + head] = l == 0.f ? -INFINITY : (m - kShift + log2f(l)) * 0.69314718055994531f;
      } else {
        *reinterpret_cast<float4*>(part + r * D + f * 4) = sum;
        if (f == 0) {
          part[kMaxRows * D + r] = m;
          part[kMaxRows * D + kMaxRows + r] = l;
        }
      }
    }
    if (!whole) {
      // the last CTA of the item to get here joins all parts
      __threadfence();
      consumers_sync();
      if (tid == 0) {
        const int32_t others = static_cast<int32_t>(walk.last_cta - walk.first_cta);
        sm.last = atomicAdd(w.tickets + walk.first_cta, 1) == others;
        __threadfence();
        if (sm.last) w.tickets[walk.first_cta] = 0;
      }
      consumers_sync();
      if (sm.last) {
        for (int i = tid; i < it.rows * F; i += kWarps * 32) {
          const int r = i / F, f = i % F;
          float m = -1e30f;
          for (int64_t c = walk.first_cta; c <= walk.last_cta; ++c)
            m = fmaxf(m, __ldcg(w.parts + Kv8Walk::slot_of(c, walk.first_cta) * w.slot_floats + kMaxRows * D + r));
          float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
          float l = 0.f;
#pragma unroll 4
          for (int64_t c = walk.first_cta; c <= walk.last_cta; ++c) {
            const float* p = w.parts + Kv8Walk::slot_of(c, walk.first_cta) * w.slot_floats;
            const float k = ex2(__ldcg(p + kMaxRows * D + r) - m);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p + r * D + f * 4));
            sum.x = fmaf(v.x, k, sum.x);
            sum.y = fmaf(v.y, k, sum.y);
            sum.z = fmaf(v.z, k, sum.z);
            sum.w = fmaf(v.w, k, sum.w);
            l = fmaf(__ldcg(p + kMaxRows * D + kMaxRows + r), k, l);
          }
          const int at = it.row0 + r;
          const int64_t tok = it.first + at / a.group;
          const int head = it.h * a.group + at % a.group;
          const float inv = l == 0.f ? 0.f : 1.f / l;
          *reinterpret_cast<uint2*>(a.out + tok * a.ots + head * a.ohs + f * 4) =
              make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
          if (a.lse && f == 0) a.lse[tok * a.Hq + head] = l == 0.f ? -INFINITY : (m - kShift + log2f(l)) * 0.69314718055994531f;
        }
      }
    }
  }
}

}  // namespace

int kv8_decode_rows(int) { return kMaxRows; }
size_t kv8_decode_slot(int D) { return static_cast<size_t>(kMaxRows) * (D + 2); }

cudaError_t kv8_decode_init(int D) {
  return D == 128 ? cudaFuncSetAttribute(kv8_decode_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(DecodeSmem<128>) + 1024)
                  : cudaFuncSetAttribute(kv8_decode_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(DecodeSmem<64>) + 1024);
}

cudaError_t launch_kv8_decode(const Kv8AttendArgs& a, Kv8Work w, int D, int nsm, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                              cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(a.rows.max_rows) * a.group;
  w.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  w.tiles = static_cast<int>((rows + w.tile_rows - 1) / w.tile_rows);
  w.items = static_cast<int64_t>(a.rows.batch) * a.Hkv * w.tiles;
  w.step_pages = 1;
  w.min_steps = 16;
  w.slot_floats = static_cast<int64_t>(kv8_decode_slot(D));
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(nsm);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (D == 128 ? sizeof(DecodeSmem<128>) : sizeof(DecodeSmem<64>)) + 1024;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, D == 128 ? kv8_decode_kernel<128> : kv8_decode_kernel<64>, a, w, tm_k, tm_v);
}

}  // namespace hsa
