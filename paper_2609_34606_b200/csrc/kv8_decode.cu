// Attention over the 8-bit paged cache for few query rows of a key head (a token of each sequence, a few drafted ones).
//
// Such a call reads every key and value once and does little with it: the bytes bound it.  So the codes go from memory to
// the tensor cores as they are -- no thread ever touches a key or a value -- and the products are turned round to have
// keys, or dims of the values, in their long dimension:
//     S^T [128 keys x 2R] = K [128 x d] (Qhi | Qlo)^T         K tiles as TMA leaves them, K-major
//     O^T [d x 3R]        = V^T [d x 64 keys] (P0 | P1 | P2)^T   V tiles as TMA leaves them, M-major, a page at a time
// Both products need the other operand in 8 bits too.  It is given in terms side by side, as columns of their own, which are
// added up in fp32.
//   Queries: x = hi + lo / 16 with hi = e4m3(x), lo = e4m3(16 (x - hi)).  With the largest value of a row between 2^7 and 2^8
// that keeps 8 bits of every value, or 2^-21 of the largest (x - hi is at most 2^4; the last step of e4m3 is 2^-9).  So the bf16
// queries stay exact unless they are below 2^-13 of their row's largest.
//   Weights: w = t0 + t1 / 8 + t2 / 64, each the e5m2 nearest to what those before it leave (at most an eighth of it): 9 bits of
// every weight down to 2^-14, 2^-23 below that.  The largest is 2^12 when the reference is set and stays below 2^15.8, so that 9
// bits are left 2^-26 below it, and 2^-35 of it is the least that counts.  (Two e4m3 terms, whose weights ended at 2^-21
// of the largest: behind a key 15 nats above 1500 others the result lost a quarter, and an error of 2^-21 a key adds up.)
//
// One thread holds one key: y = S * scales, weight 2^(y - ref).  ref[row] is what the largest y was when it was set; as long as
// no y passes it by kSlack nothing but a vote is needed, else the maxima are taken anew.  The same thread then holds one
// dim: what comes out of a page's second product is multiplied by the page's value scale and added up in its registers, in
// fp32, while the next step's products run.  (Summed over pages on the tensor core, the weights would have to carry the
// scales, and one page with a large value would cost the weights of all others their low bits.)
//
// Warps: 0 loads pages, 1 issues the first products and 3 the second ones (one thread for both spends 1600 cycles a step on
// looking at barriers and issuing, the loads of a step take 1400), 2 prepares the rows of Q of the next item, then two
// groups of four for softmax and output, which take the steps in turn, each with sums and references of its own, which they bring
// together at an item's end; the group that had the item's last step writes it, while the other goes on.
//
// Measured: a token against 280,800 tokens of 12 heads of 128, 862 MB: 138 us, 6.25 TB/s (a plain copy: 6.54); a token of each of 48
// sequences of 300 to 8000, four query heads to a key head, 233 MB: 48 us, 4.85 TB/s, where runs of unequal items begin and end
// at different times (sixteen rows of each: 86 us, of which the third term of the weights is 2); 777 tokens: 7.2 us, of which the
// launch is 3.  Up to 16 rows of a key head come here; with 32 the columns of
// both products and the registers of the softmax cost more than the kernel for many rows does (106 against 68 us for 8 sequences of
// 9000 tokens).
#include "kv8.cuh"
#include "kv8_mma.cuh"

namespace hsa {

namespace {

constexpr float kShift = 12.f;  // the largest weight is 2^12 when the reference is set ...
constexpr float kSlack = 3.75f; // ... and may grow to 2^15.75 < 57344, the largest e5m2, before it is set anew

// R: rows of an item.  A step is a tile of 128 keys, two pages.
template <int D, int R>
struct DecodeShape {
  static constexpr int N = R < 8 ? 16 : 2 * R;           // columns of the first products: first terms, then second ones (16 at least)
  static constexpr int NP = R < 8 ? 16 : R == 8 ? 32 : 3 * R;  // of the second ones: three terms (a multiple of 16)
  static constexpr int kGroups = 2;
  static constexpr int kThreads = 128 + 128 * kGroups;
  static constexpr int kPage = kBlock * D;               // bytes of a page tile
  static constexpr int kStage = 2 * kPage;               // of K or of V of a step
  static constexpr int kStages = D == 64 ? 12 : 6;
  static constexpr uint32_t kS = 0;                      // TMEM columns: S of two steps, then O of their pages
  static constexpr uint32_t kO = 2 * N;
  static constexpr uint32_t kCols = 2 * N + 4 * NP <= 128 ? 128 : 256;
  static_assert(2 * N + 4 * NP <= 256);
};

template <int D, int R>
struct DecodeSmem {
  using Sh = DecodeShape<D, R>;
  uint8_t k[Sh::kStages][Sh::kStage];
  uint8_t v[Sh::kStages][Sh::kStage];
  uint8_t p[2][Sh::NP * 128];              // weights: [rows of a term, three times][128 keys]
  uint8_t q[2][Sh::N * D];
  float other[R * (D + 2)];  // sums of the group that does not write the item: [R][D], references, sums of weights
  float qscale[2][R];
  int limit[2][R];                         // tokens that a row sees
  PageMeta meta[Sh::kStages][2];
  float red[Sh::kGroups][4][R];
  uint64_t k_full[Sh::kStages], v_full[Sh::kStages], empty[Sh::kStages];
  uint64_t s_full[2], s_free[2], p_full[2], p_free[2], q_full[2], q_free[2], other_full, other_free, done[2];
  uint32_t tmem;
  Kv8Plan plan;
};

// The four warps of a group meet; `any`: whether x holds for one of them.
__device__ __forceinline__ void group_sync(int group) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(1 + group) : "memory"); }
__device__ __forceinline__ bool group_any(int group, bool x) {
  uint32_t r;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %2, 0;\n"
      "barrier.cta.red.or.pred q, %1, 128, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(r)
      : "r"(1 + group), "r"(static_cast<uint32_t>(x))
      : "memory");
  return r != 0;
}

__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}

constexpr float kLow = 1.f / 16.f;  // what the second term counts

// Two values as e4m3 hi and lo terms: bytes 0, 1 of each result.
__device__ __forceinline__ void two_terms(float a, float b, uint32_t* hi, uint32_t* lo) {
  const uint32_t h = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const __half2_raw back = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(h), __NV_E4M3);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&back));
  *hi = h;
  *lo = __nv_cvt_float2_to_fp8x2(make_float2((a - f.x) * 16.f, (b - f.y) * 16.f), __NV_SATFINITE, __NV_E4M3);
}

// Two weights (below 65504) as three e5m2 terms each: bytes 0, 1 of each result.  The 11 bits of fp16 are more than the terms hold,
// and so is its last step of 2^-24; what is left behind a term, and eight times that, is exact in it.
__device__ __forceinline__ void three_terms(float a, float b, uint32_t* t0, uint32_t* t1, uint32_t* t2) {
  asm("{\n"
      ".reg .b32 x, z, e;\n"
      ".reg .b16 t;\n"
      "mov.b32 e, 0x48004800;\n"
      "cvt.rn.f16x2.f32 x, %4, %3;\n"
      "cvt.rn.satfinite.e5m2x2.f16x2 t, x;\n"
      "cvt.u32.u16 %0, t;\n"
      "cvt.rn.f16x2.e5m2x2 z, t;\n"
      "sub.rn.f16x2 x, x, z;\n"
      "mul.rn.f16x2 x, x, e;\n"
      "cvt.rn.satfinite.e5m2x2.f16x2 t, x;\n"
      "cvt.u32.u16 %1, t;\n"
      "cvt.rn.f16x2.e5m2x2 z, t;\n"
      "sub.rn.f16x2 x, x, z;\n"
      "mul.rn.f16x2 x, x, e;\n"
      "cvt.rn.satfinite.e5m2x2.f16x2 t, x;\n"
      "cvt.u32.u16 %2, t;\n"
      "}\n"
      : "=r"(*t0), "=r"(*t1), "=r"(*t2)
      : "f"(a), "f"(b));
}

template <int COLS>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t* r) {
  if constexpr (COLS == 16) tmem_ld16(addr, *reinterpret_cast<uint32_t(*)[16]>(r));
  else if constexpr (COLS == 32) tmem_ld32(addr, *reinterpret_cast<uint32_t(*)[32]>(r));
  else {
    tmem_ld32(addr, *reinterpret_cast<uint32_t(*)[32]>(r));
    tmem_ld32(addr + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
  }
}

// The three terms of R rows, added up.
template <int R>
__device__ __forceinline__ void tmem_load_terms(uint32_t addr, float (&sum)[R]) {
  if constexpr (R <= 4) {
    uint32_t x[16];
    tmem_ld16(addr, x);
    tc_wait_ld();
#pragma unroll
    for (int r = 0; r < R; ++r) sum[r] = fmaf(fmaf(__uint_as_float(x[2 * R + r]), 0.125f, __uint_as_float(x[R + r])), 0.125f, __uint_as_float(x[r]));
  } else if constexpr (R == 8) {
    uint32_t x[16], y[8];
    tmem_ld16(addr, x);
    tmem_ld8(addr + 16, y);
    tc_wait_ld();
#pragma unroll
    for (int r = 0; r < 8; ++r) sum[r] = fmaf(fmaf(__uint_as_float(y[r]), 0.125f, __uint_as_float(x[8 + r])), 0.125f, __uint_as_float(x[r]));
  } else {  // (one after the other: the registers are few)
    static_assert(R == 16);
#pragma unroll
    for (int t = 2; t >= 0; --t) {
      uint32_t x[16];
      tmem_ld16(addr + t * 16, x);
      tc_wait_ld();
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[r] = t == 2 ? __uint_as_float(x[r]) : fmaf(sum[r], 0.125f, __uint_as_float(x[r]));
    }
  }
}

// Adds the parts of an item up, in the order of the CTAs, and writes its rows: 128 threads, four dims of a row at a time.
template <int D, int R>
__device__ __forceinline__ void join_parts(const Kv8AttendArgs& a, const Kv8Work& w, const Kv8Segment& g, int tid) {
  constexpr int F = D / 4, kAtOnce = 8;
  for (int i = tid; i < g.it.rows * F; i += 128) {
    const int r = i / F, f = i % F;
    float m = kNone, tot = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = g.first_cta; c0 <= g.last_cta; c0 += kAtOnce) {
      float pm[kAtOnce], pl[kAtOnce];
      float4 pv[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        pm[j] = kNone;
        pl[j] = 0.f;
        pv[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c0 + j <= g.last_cta) {
          const float* p = w.parts + Kv8Segment::slot_of(c0 + j, g.first_cta) * w.slot_floats;
          pm[j] = __ldcg(p + R * D + r);
          pl[j] = __ldcg(p + R * D + R + r);
          pv[j] = __ldcg(reinterpret_cast<const float4*>(p + r * D + f * 4));
        }
      }
      float to = m;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) to = fmaxf(to, pm[j]);
      const float c = ex2(m - to);
      m = to;
      sum.x *= c;
      sum.y *= c;
      sum.z *= c;
      sum.w *= c;
      tot *= c;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const float k = ex2(pm[j] - to);
        sum.x = fmaf(pv[j].x, k, sum.x);
        sum.y = fmaf(pv[j].y, k, sum.y);
        sum.z = fmaf(pv[j].z, k, sum.z);
        sum.w = fmaf(pv[j].w, k, sum.w);
        tot = fmaf(pl[j], k, tot);
      }
    }
    const int at = g.it.row0 + r;
    const int64_t tok = g.it.first + at / a.group;
    const int head = g.it.h * a.group + at % a.group;
    const float down = tot == 0.f ? 0.f : 1.f / tot;
    *reinterpret_cast<uint2*>(a.out + tok * a.ots + head * a.ohs + f * 4) =
        make_uint2(pack_bf16(sum.x * down, sum.y * down), pack_bf16(sum.z * down, sum.w * down));
    if (a.lse && f == 0) a.lse[tok * a.Hq + head] = tot == 0.f ? -INFINITY : (m + (log2f(tot) - kShift)) * 0.69314718055994531f;
  }
}

// LOOK: waits of less than a poll's sleep
template <int D, int R, bool LOOK>
__global__ void __launch_bounds__((DecodeShape<D, R>::kThreads), 1)
kv8_decode_kernel(const __grid_constant__ Kv8AttendArgs a, const __grid_constant__ Kv8Work w, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  using Sh = DecodeShape<D, R>;
  using Smem = DecodeSmem<D, R>;
  constexpr int N = Sh::N, NP = Sh::NP, kStages = Sh::kStages, kGroups = Sh::kGroups;
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sm.k_full[i], 1);
      mbar_init(&sm.v_full[i], 1);
      mbar_init(&sm.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.s_full[i], 1);
      mbar_init(&sm.s_free[i], 128);
      mbar_init(&sm.p_full[i], 128);
      mbar_init(&sm.p_free[i], 1);
      mbar_init(&sm.done[i], 1);
      mbar_init(&sm.q_full[i], 32);
      mbar_init(&sm.q_free[i], 1 + 4 * kGroups);  // its products, and the softmax warps (its scales)
    }
    mbar_init(&sm.other_full, 128);
    mbar_init(&sm.other_free, 128);
    fence_mbar_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem, Sh::kCols);
    tmem_relinquish();
  }
  kv8_plan<Sh::kThreads>(a, w, &sm.plan);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  Kv8Walk walk;
  uint32_t tries = w.first_try;
  bool ok = true;  // false: a wait ran out; nothing more is waited for or handed on
  const auto wait = [&](uint64_t* bar, uint32_t parity) {
    tries = LOOK ? mbar_look(bar, parity, tries, w.look) : mbar_poll(bar, parity, tries);
    return ok = tries != kMaxPolls;
  };
  // the same for a whole warp that stays together
  const auto warp_wait = [&](uint64_t* bar, uint32_t parity) { return ok = __all_sync(0xffffffffu, wait(bar, parity)); };

  if (warp == 0) {
    // ---- loads.  The lanes look up the pages of 16 steps at once.
    uint32_t n = 0;
    while (ok && walk.next(a, w, sm.plan)) {
      const Kv8Item& it = walk.g.it;
      for (int s = walk.g.s0; s < walk.g.s1 && ok; s += 16) {
        int blk = 0, page = -1;
        PageMeta meta{-1, 0.f, 0.f};
        if (s + lane / 2 < walk.g.s1) page = kv8_page(a, it, s * 2 + lane, &blk);
        if (page >= 0) {
          const int64_t ph = static_cast<int64_t>(page) * a.Hkv + it.h;
          meta.pos = blk * kBlock;
          meta.ks = __ldg(a.k_scale + ph);
          meta.vs = __ldg(a.v_scale + ph);
        }
        const int count = min(16, walk.g.s1 - s);
#pragma unroll 1
        for (int i = 0; i < count; ++i, ++n) {
          const uint32_t st = n % kStages;
          if (!warp_wait(&sm.empty[st], ((n / kStages) & 1) ^ 1)) break;
          int pages[2], bytes = 0;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            pages[j] = __shfl_sync(0xffffffffu, page, i * 2 + j);
            if (pages[j] >= 0) bytes += Sh::kPage;
          }
          // the loads go out before the scales are there; the keys' barrier is arrived at behind them
          if (elect_one_sync()) {
            if (bytes) mbar_expect_tx_only(&sm.k_full[st], bytes);
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (pages[j] >= 0)
                tma_load_2d(sm.k[st] + j * Sh::kPage, &tm_k, &sm.k_full[st], 0,
                            static_cast<int>((static_cast<int64_t>(pages[j]) * a.Hkv + it.h) * kBlock));
            if (bytes) mbar_expect_tx(&sm.v_full[st], bytes);
            else mbar_arrive(&sm.v_full[st]);
#pragma unroll
            for (int j = 0; j < 2; ++j)
              if (pages[j] >= 0)
                tma_load_2d(sm.v[st] + j * Sh::kPage, &tm_v, &sm.v_full[st], 0,
                            static_cast<int>((static_cast<int64_t>(pages[j]) * a.Hkv + it.h) * kBlock));
          }
          if (lane / 2 == i) sm.meta[st][lane % 2] = meta;
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.k_full[st]);
        }
      }
    }
    // the last pages, a lane each, whether somebody takes them or not
    static_assert(kStages <= 16);
    const uint32_t back = lane % 16 + 1;
    if (back <= kStages && back <= n) {
      const uint32_t st = (n - back) % kStages;
      if (!mbar_drain(lane < 16 ? &sm.k_full[st] : &sm.v_full[st], ((n - back) / kStages) & 1)) ok = false;
    }
  } else if (warp == 1) {
    // ---- first products.  (The warps that issue products stay together and choose a lane at the last moment, so that the operands
    // are in uniform registers.)
    constexpr uint32_t id = idesc_e4m3(128, N, 0, 0);
    const uint32_t k0 = row_desc_lo(smem_u32(sm.k)), q0 = row_desc_lo(smem_u32(sm.q)), tm = warp_uniform(tmem);
    uint32_t n = 0, items = 0, st = 0, round = 0;
    while (warp_uniform(walk.next(a, w, sm.plan))) {
      const uint32_t qb = items & 1, steps = warp_uniform(walk.g.s1 - walk.g.s0);
      wait(&sm.q_full[qb], (items / 2) & 1);
#pragma unroll 1
      for (uint32_t s = 0; s < steps; ++s, ++n) {
        const uint32_t b = n & 1, k = k0 + st * (Sh::kStage / 16), q = q0 + qb * (N * D / 16);
        wait(&sm.k_full[st], round & 1);
        wait(&sm.s_free[b], ((n / 2) & 1) ^ 1);
        tc_fence_after();
        if (elect_one_sync() && ok) {
#pragma unroll
          for (int kk = 0; kk < D / 32; ++kk)  // (descriptors count in 16 bytes)
            mma_f8_lo(tm + Sh::kS + b * N, k + kk * 2, q + kk * 2, row_desc_hi<D>(), row_desc_hi<D>(), id, kk > 0);
          tc_commit(&sm.s_full[b]);
          if (s + 1 == steps) tc_commit(&sm.q_free[qb]);
        }
        __syncwarp();
        if (++st == kStages) {
          st = 0;
          ++round;
        }
      }
      ++items;
    }
    if (elect_one_sync()) tc_commit(&sm.done[0]);
    __syncwarp();
    if (!mbar_drain(&sm.done[0], 0)) ok = false;  // (whatever ran out before: products in flight must not outlive the CTA)
  } else if (warp == 3) {
    // ---- second products, a page at a time (of pages that are not there too: nobody looks at what they give)
    constexpr uint32_t id = idesc_e4m3(128, NP, 1, 0) | 1u << 10;  // (B: e5m2)
    // (head_dim 64: the upper half of M reads what lies a page further, whatever that is; those lanes of the accumulator
    // are not looked at)
    const uint32_t v0 = row_desc_lo(smem_u32(sm.v)) | (D == 128 ? 0u : static_cast<uint32_t>(Sh::kPage >> 4) << 16),
                   p0 = row_desc_lo(smem_u32(sm.p)), tm = warp_uniform(tmem);
    uint32_t n = 0, st = 0, round = 0;
    while (warp_uniform(walk.next(a, w, sm.plan))) {
      const uint32_t steps = warp_uniform(walk.g.s1 - walk.g.s0);
#pragma unroll 1
      for (uint32_t s = 0; s < steps; ++s, ++n) {
        const uint32_t b = n & 1, v = v0 + st * (Sh::kStage / 16), p = p0 + b * (NP * 128 / 16);
        wait(&sm.v_full[st], round & 1);
        wait(&sm.p_full[b], (n / 2) & 1);
        tc_fence_after();
        if (elect_one_sync() && ok) {
#pragma unroll
          for (int pg = 0; pg < 2; ++pg)
#pragma unroll
            for (int half = 0; half < 2; ++half)  // 32 keys: rows of V, bytes of a row of P
              mma_f8_lo(tm + Sh::kO + (b * 2 + pg) * NP, v + (pg * Sh::kPage + half * 32 * D) / 16, p + (pg * 64 + half * 32) / 16,
                        row_desc_hi<D>(), row_desc_hi<128>(), id, half);
          tc_commit(&sm.empty[st]);
          tc_commit(&sm.p_free[b]);
        }
        __syncwarp();
        if (++st == kStages) {
          st = 0;
          ++round;
        }
      }
    }
    if (elect_one_sync()) tc_commit(&sm.done[1]);
    __syncwarp();
    if (!mbar_drain(&sm.done[1], 0)) ok = false;  // (whatever ran out before: products in flight must not outlive the CTA)
  } else if (warp == 2) {
    // ---- rows of Q, an item ahead: a thread takes 8 dims of a row
    uint32_t items = 0;
    while (ok && walk.next(a, w, sm.plan)) {
      const Kv8Item& it = walk.g.it;
      const uint32_t qb = items & 1;
      constexpr int V = D / 8, kRows = 32 / V;     // vectors of a row, rows at a time
      constexpr int kTimes = (R + kRows - 1) / kRows;
      const int r0 = lane / V, c = lane % V;
      uint4 in[kTimes];
#pragma unroll
      for (int i = 0; i < kTimes; ++i) {
        const int r = r0 + i * kRows;
        in[i] = make_uint4(0, 0, 0, 0);
        if (r < it.rows) {
          const int at = it.row0 + r;
          in[i] = __ldg(reinterpret_cast<const uint4*>(a.q + (it.first + at / a.group) * a.ts + (it.h * a.group + at % a.group) * a.hs + c * 8));
        }
      }
      if (!warp_wait(&sm.q_free[qb], ((items / 2) & 1) ^ 1)) break;
      uint8_t* q = sm.q[qb];
      if (lane < R) sm.limit[qb][lane] = it.limit(a, min(lane, it.rows - 1));
#pragma unroll
      for (int i = 0; i < kTimes; ++i) {
        const int r = r0 + i * kRows;
        const uint32_t words[4] = {in[i].x, in[i].y, in[i].z, in[i].w};
        float x[8];
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = __uint_as_float(j & 1 ? words[j / 2] & 0xffff0000u : words[j / 2] << 16);
          // (what is not finite: NaN, which spoils the row and no other)
          if (fabsf(x[j]) < INFINITY) top = fmaxf(top, fabsf(x[j]));
          else x[j] = NAN;
        }
#pragma unroll
        for (int o = V / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int e = max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100) - 7;  // (rows of zeros: any will do)
        const float up = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) two_terms(x[2 * j] * up, x[2 * j + 1] * up, &hi[j], &lo[j]);
        if (R % kRows == 0 || r < R) {
          *reinterpret_cast<uint2*>(q + swizzled<D>(r, c * 8)) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
          *reinterpret_cast<uint2*>(q + swizzled<D>(N / 2 + r, c * 8)) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
          if (c == 0) sm.qscale[qb][r] = __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * a.scale_log2;
        }
      }
      fence_proxy_async_smem();
      mbar_arrive(&sm.q_full[qb]);
      ++items;
    }
  } else {
    // ---- softmax: a thread is a key of the tile, and a dim of the output.  After a wait that ran out the threads go on
    // with whatever is there, because they meet at barriers; the status word says that the result is none.
    const int group = (warp - 4) / 4;
    const int w4 = warp & 3, key = w4 * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(w4 * 32) << 16;
    uint32_t n = 0, items = 0, merges = 0;
    Kv8Segment shared[2];
    int n_shared = 0;
    while (walk.next(a, w, sm.plan)) {
      const Kv8Item& it = walk.g.it;
      const int steps = walk.g.s1 - walk.g.s0;
      const uint32_t qb = items & 1;
      ++items;
      // steps n, n + 1, ... are this item's; every kGroups-th one is this group's
      uint32_t j = n + ((n + group) & 1);
      const uint32_t end = n + steps;
      n = end;
      const bool writes = ((end - 1) & 1) == static_cast<uint32_t>(group);
      const bool both = steps > 1;
      float ref[R], l[R], o[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        ref[r] = kNone;
        l[r] = o[r] = 0.f;
      }
      const int lim_low = it.limit(a, 0), rows = it.rows;
      float vs0 = 0.f, vs1 = 0.f;       // scales of the step whose second product has not been added yet
      uint32_t added = j;               // steps up to here have been
      // adds what the second product of step i gave
      const auto add = [&](uint32_t i) {
        wait(&sm.p_free[i & 1], (i / 2) & 1);
        __syncwarp();
        tc_fence_after();
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
          const float vs = pg ? vs1 : vs0;
          float x[R];
          tmem_load_terms<R>(tmem + lanes + Sh::kO + ((i & 1) * 2 + pg) * NP, x);
#pragma unroll
          for (int r = 0; r < R; ++r) o[r] = vs > 0.f ? fmaf(x[r], vs, o[r]) : o[r];  // (0: a page that is not there)
        }
        tc_fence_before();
        added = i + kGroups;
      };
      wait(&sm.q_full[qb], ((items - 1) / 2) & 1);
#pragma unroll 1
      for (; j < end; j += kGroups) {
        const uint32_t st = j % kStages, b = j & 1;
        wait(&sm.s_full[b], (j / 2) & 1);
        __syncwarp();
        tc_fence_after();
        float y[R];
        bool over = false;
        {
          uint32_t x[N];
          tmem_load<N>(tmem + lanes + Sh::kS + b * N, x);
          const PageMeta meta = sm.meta[st][key / kBlock];
          const int pos = meta.pos + key % kBlock;
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < R; ++r) y[r] = fmaf(__uint_as_float(x[N / 2 + r]), kLow, __uint_as_float(x[r])) * (sm.qscale[qb][r] * meta.ks);
          if (meta.pos < 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) y[r] = -INFINITY;
          } else if (pos >= lim_low) {
#pragma unroll
            for (int r = 0; r < R; ++r)
              if (pos >= sm.limit[qb][r]) y[r] = -INFINITY;
          }
#pragma unroll
          for (int r = 0; r < R; ++r) over |= y[r] - ref[r] > kSlack;  // (ref + kSlack would be rounded where scores pass 2^22)
        }
        const float vs0_now = sm.meta[st][0].vs, vs1_now = sm.meta[st][1].vs;
        tc_fence_before();
        mbar_arrive_if(&sm.s_free[b], ok);
        if (__builtin_expect(group_any(group, over), 0)) {
          // the maxima anew
          if (added < j) add(added);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float top = warp_max(y[r]);
            if (lane == 0) sm.red[group][w4][r] = top;
          }
          group_sync(group);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float* red = &sm.red[group][0][r];
            const float top = fmaxf(fmaxf(red[0], red[R]), fmaxf(red[2 * R], red[3 * R]));
            const float to = top - ref[r] > kSlack ? top : ref[r], c = ex2(ref[r] - to);
            ref[r] = to;
            l[r] *= c;
            o[r] *= c;
          }
          group_sync(group);  // (red is free again)
        }
        // (the buffer of P: what it held two steps ago has been multiplied before that could be added)
        if (added < j) add(added);
        uint8_t* p = sm.p[b];
#pragma unroll
        for (int r = 0; r < R; r += 2) {
          const float p0 = ex2((y[r] - ref[r]) + kShift), p1 = ex2((y[r + 1] - ref[r + 1]) + kShift);
          l[r] += p0;
          l[r + 1] += p1;
          uint32_t t[3];
          three_terms(p0, p1, &t[0], &t[1], &t[2]);
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            p[swizzled<128>(i * R + r, key)] = static_cast<uint8_t>(t[i]);
            p[swizzled<128>(i * R + r + 1, key)] = static_cast<uint8_t>(t[i] >> 8);
          }
        }
        fence_proxy_async_smem();
        mbar_arrive_if(&sm.p_full[b], ok);
        vs0 = vs0_now;
        vs1 = vs1_now;
      }
      mbar_arrive_if(&sm.q_free[qb], ok && lane == 0);
      if (!writes && !both) continue;  // the item's one step was the other group's

      // ---- the item's sums: of weights over the keys, then a dim of every row
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], s);
        if (lane == 0) sm.red[group][w4][r] = l[r];
      }
      add(added);
      group_sync(group);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float* red = &sm.red[group][0][r];
        l[r] = (red[0] + red[R]) + (red[2 * R] + red[3 * R]);
      }
      if (both) {
        if (!writes) {
          wait(&sm.other_free, (merges & 1) ^ 1);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (key < D) sm.other[r * D + key] = o[r];
            if (key == r) {
              sm.other[R * D + r] = ref[r];
              sm.other[R * D + R + r] = l[r];
            }
          }
          mbar_arrive_if(&sm.other_full, ok);
        } else {
          wait(&sm.other_full, merges & 1);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float m = sm.other[R * D + r], to = fmaxf(ref[r], m), c = ex2(ref[r] - to), k = ex2(m - to);
            o[r] *= c;
            if (key < D) o[r] = fmaf(sm.other[r * D + key], k, o[r]);
            l[r] = fmaf(sm.other[R * D + R + r], k, l[r] * c);
            ref[r] = to;
          }
          mbar_arrive_if(&sm.other_free, ok);
        }
        ++merges;
      }
      if (writes) {
        const bool whole = walk.g.whole();
        float* part = w.parts + walk.g.slot() * w.slot_floats;
        int tok = it.first + it.row0 / a.group, head = it.row0 % a.group;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r < rows && ok) {
            if (whole) {
              const int h = it.h * a.group + head;
              if (key < D) a.out[tok * a.ots + h * a.ohs + key] = __float2bfloat16_rn(l[r] == 0.f ? 0.f : o[r] / l[r]);
              if (a.lse && key == 0)
                a.lse[static_cast<int64_t>(tok) * a.Hq + h] = l[r] == 0.f ? -INFINITY : (ref[r] + (log2f(l[r]) - kShift)) * 0.69314718055994531f;
            } else {
              if (key < D) part[r * D + key] = o[r];
              if (key == 0) {
                part[R * D + r] = ref[r];
                part[R * D + R + r] = l[r];
              }
            }
          }
          if (++head == a.group) {
            head = 0;
            ++tok;
          }
        }
        if (!whole) shared[n_shared++ & 1] = walk.g;  // (two at most: the run's first and its last)
      }
      group_sync(group);  // (red is free again)
    }
    // ---- items that other CTAs have parts of: the last one to get here joins them
    for (int i = 0; i < n_shared; ++i) {
      const Kv8Segment g = shared[i];
      group_sync(group);
      if (key == 0) {
        bool last = false;
        if (ok) {  // (what the group has written before the barrier goes before, what it reads behind it comes after)
          int32_t ticket;
          asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(ticket) : "l"(w.tickets + g.first_cta) : "memory");
          last = ticket == g.last_cta - g.first_cta;
        }
        if (last) w.tickets[g.first_cta] = 0;
        sm.red[group][0][0] = last ? 1.f : 0.f;
      }
      group_sync(group);
      const bool last = sm.red[group][0][0] != 0.f;
      if (last) join_parts<D, R>(a, w, g, key);
      group_sync(group);
    }
  }
  if (!ok) kv8_flag(a.status, kDevTimeout);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, Sh::kCols);
}

template <int D, int R>
constexpr size_t smem_bytes() {
  static_assert(sizeof(DecodeSmem<D, R>) + 1024 <= 232448, "shared memory of an SM");
  return sizeof(DecodeSmem<D, R>) + 1024;
}
template <int D, int R, bool LOOK = false>
cudaError_t init_one() {
  return cudaFuncSetAttribute(kv8_decode_kernel<D, R, LOOK>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem_bytes<D, R>()));
}
template <int D, int R, bool LOOK = false>
cudaError_t launch_one(const Kv8AttendArgs& a, Kv8Work w, int64_t rows, int ctas, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                       cudaStream_t st) {
  w.tile_rows = R;
  w.tiles = static_cast<int>((rows + R - 1) / R);
  w.items = static_cast<int64_t>(a.rows.batch) * a.Hkv * w.tiles;
  w.step_log = 1;
  w.half_rows = 0;
  w.part_log = 4;
  w.item_steps = 4;
  w.slot_floats = static_cast<int64_t>(kv8_decode_slot(D));
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(DecodeShape<D, R>::kThreads);
  cfg.dynamicSmemBytes = smem_bytes<D, R>();
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kv8_decode_kernel<D, R, LOOK>, a, w, tm_k, tm_v);
}
template <int D>
cudaError_t launch_dim(const Kv8AttendArgs& a, const Kv8Work& w, int ctas, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(a.rows.max_rows) * a.group;
  if (w.look) return launch_one<D, 16, true>(a, w, rows, ctas, tm_k, tm_v, st);
  return rows <= 2    ? launch_one<D, 2>(a, w, rows, ctas, tm_k, tm_v, st)
         : rows <= 4  ? launch_one<D, 4>(a, w, rows, ctas, tm_k, tm_v, st)
         : rows <= 8  ? launch_one<D, 8>(a, w, rows, ctas, tm_k, tm_v, st)
                      : launch_one<D, 16>(a, w, rows, ctas, tm_k, tm_v, st);
}

}  // namespace

int kv8_decode_rows(int) { return 16; }
size_t kv8_decode_slot(int D) { return static_cast<size_t>(16) * (D + 2); }

cudaError_t kv8_decode_init(int D) {
  cudaError_t e = D == 128 ? init_one<128, 2>() : init_one<64, 2>();
  if (e == cudaSuccess) e = D == 128 ? init_one<128, 4>() : init_one<64, 4>();
  if (e == cudaSuccess) e = D == 128 ? init_one<128, 8>() : init_one<64, 8>();
  if (e == cudaSuccess) e = D == 128 ? init_one<128, 16>() : init_one<64, 16>();
  if (e == cudaSuccess) e = D == 128 ? init_one<128, 16, true>() : init_one<64, 16, true>();
  return e;
}

cudaError_t launch_kv8_decode(const Kv8AttendArgs& a, Kv8Work w, int D, int ctas, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                              cudaStream_t st) {
  return D == 128 ? launch_dim<128>(a, w, ctas, tm_k, tm_v, st) : launch_dim<64>(a, w, ctas, tm_k, tm_v, st);
}

}  // namespace hsa
