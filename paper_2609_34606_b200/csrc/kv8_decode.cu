// Attention over the 8-bit paged cache for few query rows of a key head (a token of each sequence, a few drafted ones).
//
// Such a call reads every key and value once and does little with it: the bytes bound it.  So the codes go from memory to
// the tensor cores as they are -- no thread ever touches a key or a value -- and the products are turned round to have
// keys, or dims of the values, in their long dimension:
//     S^T [128 keys x 2R] = K [128 x d] (Qhi | Qlo)^T         K tiles as TMA leaves them, K-major
//     O^T [d x 2R]        = V^T [d x 64 keys] (Phi | Plo)^T   V tiles as TMA leaves them, M-major, a page at a time
// Both products need the other operand in 8 bits too.  It is given in two terms side by side, as columns of their own:
// x = hi + lo / 16 with hi = e4m3(x), lo = e4m3(16 (x - hi)).  With the largest value of a row between 2^7 and 2^8.75 that
// keeps 8 bits of every value, or 2^-21 of the largest (x - hi is at most 2^4; the last step of e4m3 is 2^-9).  So the bf16
// queries stay exact unless they are below 2^-13 of their row's largest, and weights are rounded to 8 bits.  The columns are
// added up in fp32.
//
// One thread holds one key: y = S * scales, weight 2^(y - ref).  ref[row] is what the largest y was when it was set; as long as
// no y passes it by kSlack nothing but a vote is needed, else the maxima are taken anew.  The same thread then holds one
// dim: what comes out of a page's second product is multiplied by the page's value scale and added up in its registers, in
// fp32, while the next step's products run.  (Summed over pages on the tensor core, the weights would have to carry the
// scales, and one page with a large value would cost the weights of all others their low bits.)
//
// Warps: 0 loads pages, 1 issues products, 2 and 3 prepare the rows of Q of the next item, 4 to 7 softmax and output.
#include <cuda_fp8.h>
#include <cuda_fp16.h>

#include "kv8.cuh"
#include "ptx.cuh"

namespace hsa {

namespace {

constexpr int kThreads = 256;
constexpr float kShift = 7.f;   // the largest weight is 2^7 when the reference is set ...
constexpr float kSlack = 1.75f; // ... and may grow to 2^8.75 < 448 before it is set anew
constexpr float kNone = -1e30f; // reference of a row that has seen nothing

struct PageMeta {
  int pos;      // position of the page's first token; < 0: nothing to see
  float ks, vs; // scales; vs 0: no page
};

// R: rows of an item; T: tiles of 128 keys of a step
template <int D, int R>
struct DecodeShape {
  static constexpr int T = R <= 16 ? 2 : 1;
  static constexpr int N = 2 * R;
  static constexpr int kPages = 2 * T;                   // pages of a step
  static constexpr int kPage = kBlock * D;               // bytes of a page tile
  static constexpr int kStage = kPages * kPage;          // of K or of V of a step
  static constexpr int kStages = (R == 32 ? 5 : 3) * (D == 64 ? 2 : 1);
  static constexpr uint32_t kS = 0;                      // TMEM columns: S of two steps, then O of their pages
  static constexpr uint32_t kO = 2 * T * N;
  static constexpr uint32_t kCols = kO + 2 * kPages * N <= 256 ? 256 : 512;
  static_assert(kO + 2 * kPages * N <= 512, "");
};

template <int D, int R>
struct DecodeSmem {
  using Sh = DecodeShape<D, R>;
  uint8_t k[Sh::kStages][Sh::kStage];
  uint8_t v[Sh::kStages][Sh::kStage];
  uint8_t p[2][Sh::T][Sh::N * 128];        // weights: [hi rows | lo rows][128 keys]
  uint8_t q[2][Sh::N * D];
  float qscale[2][R];
  PageMeta meta[Sh::kStages][Sh::kPages];
  float red[4][R];
  float lsum[4][R];
  uint64_t k_full[Sh::kStages], v_full[Sh::kStages], empty[Sh::kStages];
  uint64_t s_full[2], s_free[2], p_full[2], p_free[2], q_full[2], q_free[2], done;
  uint32_t tmem;
  int last;
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool softmax_any(bool x) {
  uint32_t r;
  asm volatile(
      "{\n"
      ".reg .pred p, q;\n"
      "setp.ne.u32 p, %1, 0;\n"
      "barrier.cta.red.or.pred q, 2, 128, p;\n"
      "selp.u32 %0, 1, 0, q;\n"
      "}\n"
      : "=r"(r)
      : "r"(static_cast<uint32_t>(x))
      : "memory");
  return r != 0;
}

__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// kind::f8f6f4, e4m3 operands (format 0), fp32 accumulator; bits as idesc_bf16_f32
__host__ __device__ constexpr uint32_t idesc_e4m3(uint32_t M, uint32_t N, uint32_t a_mn, uint32_t b_mn) {
  return (1u << 4) | (a_mn << 15) | (b_mn << 16) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
// Rows of D bytes in the swizzle that spans a row (128 bytes: layout 2, 64 bytes: layout 4); eight rows are 8 * D bytes.
template <int D>
__device__ __forceinline__ uint64_t row_desc(uint32_t addr, uint32_t lbo) {
  return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | static_cast<uint64_t>(lbo >> 4) << 16 |
         static_cast<uint64_t>((8 * D) >> 4) << 32 | static_cast<uint64_t>(1) << 46 |
         static_cast<uint64_t>(D == 128 ? 2 : 4) << 61;
}
// Byte of (row, byte in the row) in such a tile.
template <int D>
__device__ __forceinline__ int swizzled(int row, int byte) {
  return row * D + ((byte >> 4) ^ (D == 128 ? row & 7 : (row >> 1) & 3)) * 16 + (byte & 15);
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

template <int COLS>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t* r) {
  if constexpr (COLS == 16) tmem_ld16(addr, *reinterpret_cast<uint32_t(*)[16]>(r));
  else if constexpr (COLS == 32) tmem_ld32(addr, *reinterpret_cast<uint32_t(*)[32]>(r));
  else {
    tmem_ld32(addr, *reinterpret_cast<uint32_t(*)[32]>(r));
    tmem_ld32(addr + 32, *reinterpret_cast<uint32_t(*)[32]>(r + 32));
  }
}

template <int D, int R>
__global__ void __launch_bounds__(kThreads, 1) kv8_decode_kernel(const Kv8AttendArgs a, const Kv8Work w,
                                                                 const __grid_constant__ CUtensorMap tm_k,
                                                                 const __grid_constant__ CUtensorMap tm_v) {
  using Sh = DecodeShape<D, R>;
  using Smem = DecodeSmem<D, R>;
  constexpr int T = Sh::T, N = Sh::N, kPages = Sh::kPages, kStages = Sh::kStages;
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
      mbar_init(&sm.q_full[i], 64);
      mbar_init(&sm.q_free[i], 5);  // its products, and the softmax warps (its scales)
    }
    mbar_init(&sm.done, 1);
    fence_mbar_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem, Sh::kCols);
    tmem_relinquish();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Kv8Run run = kv8_run<kThreads>(a, w);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem;
  Kv8Walk walk(run);
  bool ok = true;  // false: a wait ran out; nothing more is waited for
  const auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (ok && !mbar_wait(bar, parity)) {
      ok = false;
      kv8_flag(a.status, kDevTimeout);
    }
    return ok;
  };
  // the same for a whole warp that stays together
  const auto warp_wait = [&](uint64_t* bar, uint32_t parity) { return ok = __all_sync(0xffffffffu, wait(bar, parity)); };

  if (warp == 0) {
    // ---- loads.  The lanes look up the pages of some steps at once.
    constexpr int kLook = 32 / kPages;
    uint32_t n = 0;
    while (ok && walk.next(a, w, run)) {
      const Kv8Item& it = walk.it;
      for (int s = walk.s0; s < walk.s1 && ok; s += kLook) {
        int blk = 0, page = -1;
        PageMeta meta{-1, 0.f, 0.f};
        if (s + lane / kPages < walk.s1) page = kv8_page(a, it, s * kPages + lane, &blk);
        if (page >= 0) {
          const int64_t ph = static_cast<int64_t>(page) * a.Hkv + it.h;
          meta.pos = blk * kBlock;
          meta.ks = __ldg(a.k_scale + ph);
          meta.vs = __ldg(a.v_scale + ph);
        }
        const int count = min(kLook, walk.s1 - s);
        for (int i = 0; i < count; ++i, ++n) {
          const uint32_t st = n % kStages;
          if (!warp_wait(&sm.empty[st], ((n / kStages) & 1) ^ 1)) break;
          if (lane / kPages == i) sm.meta[st][lane % kPages] = meta;
          int pages[kPages], bytes = 0;
#pragma unroll
          for (int j = 0; j < kPages; ++j) {
            pages[j] = __shfl_sync(0xffffffffu, page, i * kPages + j);
            if (pages[j] >= 0) bytes += Sh::kPage;
          }
          __syncwarp();
          if (elect_one_sync()) {
#pragma unroll
            for (int which = 0; which < 2; ++which) {
              uint64_t* full = which ? &sm.v_full[st] : &sm.k_full[st];
              if (bytes) mbar_expect_tx(full, bytes);
              else mbar_arrive(full);
#pragma unroll
              for (int j = 0; j < kPages; ++j)
                if (pages[j] >= 0)
                  tma_load_2d((which ? sm.v[st] : sm.k[st]) + j * Sh::kPage, which ? &tm_v : &tm_k, full, 0,
                              static_cast<int>((static_cast<int64_t>(pages[j]) * a.Hkv + it.h) * kBlock));
            }
          }
          __syncwarp();
        }
      }
    }
    if (!ok)  // pages that nobody took: their loads must not outlive the CTA
      for (uint32_t i = 1; i <= kStages && i <= n; ++i) {
        mbar_wait(&sm.k_full[(n - i) % kStages], ((n - i) / kStages) & 1);
        mbar_wait(&sm.v_full[(n - i) % kStages], ((n - i) / kStages) & 1);
      }
  } else if (warp == 1) {
    // ---- products
    if (elect_one_sync()) {
      constexpr uint32_t id_s = idesc_e4m3(128, N, 0, 0), id_o = idesc_e4m3(128, N, 1, 0);
      const uint32_t k0 = smem_u32(sm.k), v0 = smem_u32(sm.v), p0 = smem_u32(sm.p), q0 = smem_u32(sm.q);
      uint32_t n = 0, items = 0;      // steps and items so far
      int pending = -1;               // pages of the step whose second product is still to come; bit j: page j is there
      // The second product of step n - 1.
      const auto second = [&]() {
        const uint32_t j = n - 1, st = j % kStages, b = j & 1;
        if (!wait(&sm.p_full[b], (j / 2) & 1) || !wait(&sm.v_full[st], (j / kStages) & 1)) return;
        tc_fence_after();
#pragma unroll
        for (int pg = 0; pg < kPages; ++pg)
          if (pending & (1 << pg)) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              // 32 keys: rows of V, bytes of a row of P.  (head_dim 64: the upper half of M reads what lies a page further,
              // whatever that is; those lanes of the accumulator are not looked at.)
              const uint64_t da = row_desc<D>(v0 + st * Sh::kStage + pg * Sh::kPage + half * 32 * D, D == 128 ? 0 : Sh::kPage);
              const uint64_t db = row_desc<128>(p0 + (b * T + pg / 2) * (N * 128) + (pg & 1) * 64 + half * 32, 0);
              mma_f8(tmem + Sh::kO + (b * kPages + pg) * N, da, db, id_o, half);
            }
          }
        tc_commit(&sm.empty[st]);
        tc_commit(&sm.p_free[b]);
      };
      while (ok && walk.next(a, w, run)) {
        const uint32_t qb = items & 1;
        if (!wait(&sm.q_full[qb], (items / 2) & 1)) break;
        for (int s = walk.s0; s < walk.s1 && ok; ++s) {
          const uint32_t st = n % kStages, b = n & 1;
          if (!wait(&sm.k_full[st], (n / kStages) & 1) || !wait(&sm.s_free[b], ((n / 2) & 1) ^ 1)) break;
          tc_fence_after();
          int there = 0;
#pragma unroll
          for (int pg = 0; pg < kPages; ++pg) there |= (sm.meta[st][pg].pos >= 0 ? 1 : 0) << pg;
#pragma unroll
          for (int tt = 0; tt < T; ++tt)
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk)
              mma_f8(tmem + Sh::kS + (b * T + tt) * N, row_desc<D>(k0 + st * Sh::kStage + tt * 2 * Sh::kPage + kk * 32, 0),
                     row_desc<D>(q0 + qb * (N * D) + kk * 32, 0), id_s, kk > 0);
          tc_commit(&sm.s_full[b]);
          if (s == walk.s1 - 1) tc_commit(&sm.q_free[qb]);
          if (pending >= 0) second();
          pending = there;
          ++n;
        }
        ++items;
      }
      if (ok && pending >= 0) second();
      tc_commit(&sm.done);
      mbar_wait(&sm.done, 0);
    }
    __syncwarp();
  } else if (warp < 4) {
    // ---- rows of Q, an item ahead: a warp takes every other row
    uint32_t items = 0;
    while (ok && walk.next(a, w, run)) {
      const Kv8Item& it = walk.it;
      const uint32_t qb = items & 1;
      if (!warp_wait(&sm.q_free[qb], ((items / 2) & 1) ^ 1)) break;
      constexpr int PER = D / 32;
#pragma unroll 4
      for (int r = warp & 1; r < R; r += 2) {
        float x[PER];
        float top = 0.f;
#pragma unroll
        for (int j = 0; j < PER; ++j) x[j] = 0.f;
        if (r < it.rows) {
          const int at = it.row0 + r;
          const __nv_bfloat16* src = a.q + (it.first + at / a.group) * a.ts + (it.h * a.group + at % a.group) * a.hs + lane * PER;
#pragma unroll
          for (int j = 0; j < PER; ++j) {
            x[j] = __bfloat162float(src[j]);
            if (fabsf(x[j]) < INFINITY) top = fmaxf(top, fabsf(x[j]));
          }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int e = max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -100) - 7;  // (rows of zeros: any will do)
        const float up = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        uint8_t* q = sm.q[qb];
#pragma unroll
        for (int j = 0; j < PER; j += 2) {
          // (what is not finite: NaN, which spoils the row and no other)
          const float c0 = fabsf(x[j]) < INFINITY ? x[j] * up : NAN, c1 = fabsf(x[j + 1]) < INFINITY ? x[j + 1] * up : NAN;
          uint32_t hi, lo;
          two_terms(c0, c1, &hi, &lo);
          *reinterpret_cast<uint16_t*>(q + swizzled<D>(r, lane * PER + j)) = static_cast<uint16_t>(hi);
          *reinterpret_cast<uint16_t*>(q + swizzled<D>(R + r, lane * PER + j)) = static_cast<uint16_t>(lo);
        }
        if (lane == 0) sm.qscale[qb][r] = __uint_as_float(static_cast<uint32_t>(127 + e) << 23) * a.scale_log2;
      }
      fence_proxy_async_smem();
      mbar_arrive(&sm.q_full[qb]);
      ++items;
    }
  } else {
    // ---- softmax: a thread is a key of each tile, and a dim of the output.  After a wait that ran out the threads go on
    // with whatever is there, because they meet at barriers; the status word says that the result is none.
    const int w4 = warp & 3, key = w4 * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>(w4 * 32) << 16;
    uint32_t n = 0, items = 0;
    while (walk.next(a, w, run)) {
      const Kv8Item& it = walk.it;
      const uint32_t qb = items & 1;
      wait(&sm.q_full[qb], (items / 2) & 1);
      float ref[R], l[R], o[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        ref[r] = kNone;
        l[r] = o[r] = 0.f;
      }
      const int lim_low = it.limit(a, 0);
      float vs[kPages];       // of the step whose second product has not been added yet
      bool pending = false;
      // adds what the second product of step j gave
      const auto add = [&](uint32_t j) {
        wait(&sm.p_free[j & 1], (j / 2) & 1);
        __syncwarp();
        tc_fence_after();
#pragma unroll
        for (int pg = 0; pg < kPages; ++pg)
          if (vs[pg] > 0.f) {
            uint32_t x[N];
            tmem_load<N>(tmem + lanes + Sh::kO + ((j & 1) * kPages + pg) * N, x);
            tc_wait_ld();
#pragma unroll
            for (int r = 0; r < R; ++r) o[r] = fmaf(fmaf(__uint_as_float(x[R + r]), kLow, __uint_as_float(x[r])), vs[pg], o[r]);
          }
        tc_fence_before();
        pending = false;
      };
      for (int s = walk.s0; s < walk.s1; ++s, ++n) {
        const uint32_t st = n % kStages, b = n & 1;
        wait(&sm.k_full[st], (n / kStages) & 1);  // (long since: for the pages' scales)
        wait(&sm.s_full[b], (n / 2) & 1);
        __syncwarp();
        tc_fence_after();
        float y[T][R];
        bool over = false;
#pragma unroll
        for (int tt = 0; tt < T; ++tt) {
          uint32_t x[N];
          tmem_load<N>(tmem + lanes + Sh::kS + (b * T + tt) * N, x);
          const PageMeta meta = sm.meta[st][tt * 2 + key / kBlock];
          const int pos = meta.pos + key % kBlock;
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < R; ++r) y[tt][r] = fmaf(__uint_as_float(x[R + r]), kLow, __uint_as_float(x[r])) * (sm.qscale[qb][r] * meta.ks);
          if (meta.pos < 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) y[tt][r] = -INFINITY;
          } else if (pos >= lim_low) {
#pragma unroll
            for (int r = 0; r < R; ++r)
              if (pos >= it.limit(a, min(r, it.rows - 1))) y[tt][r] = -INFINITY;
          }
#pragma unroll
          for (int r = 0; r < R; ++r) over |= y[tt][r] > ref[r] + kSlack;
        }
        float vs_now[kPages];
#pragma unroll
        for (int pg = 0; pg < kPages; ++pg) vs_now[pg] = sm.meta[st][pg].vs;
        tc_fence_before();
        mbar_arrive(&sm.s_free[b]);
        if (softmax_any(over)) {
          // the maxima anew
          if (pending) add(n - 1);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            float top = y[0][r];
#pragma unroll
            for (int tt = 1; tt < T; ++tt) top = fmaxf(top, y[tt][r]);
#pragma unroll
            for (int o2 = 16; o2 > 0; o2 >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o2));
            if (lane == 0) sm.red[w4][r] = top;
          }
          softmax_sync();
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float top = fmaxf(fmaxf(sm.red[0][r], sm.red[1][r]), fmaxf(sm.red[2][r], sm.red[3][r]));
            const float to = top > ref[r] + kSlack ? top : ref[r], c = ex2(ref[r] - to);
            ref[r] = to;
            l[r] *= c;
            o[r] *= c;
          }
          softmax_sync();  // (red is free again)
        }
        // (the buffer of P: what it held two steps ago has been added)
#pragma unroll
        for (int tt = 0; tt < T; ++tt) {
          uint8_t* p = sm.p[b][tt];
#pragma unroll
          for (int r = 0; r < R; r += 2) {
            const float p0 = ex2(y[tt][r] + (kShift - ref[r])), p1 = ex2(y[tt][r + 1] + (kShift - ref[r + 1]));
            l[r] += p0;
            l[r + 1] += p1;
            uint32_t hi, lo;
            two_terms(p0, p1, &hi, &lo);
            p[swizzled<128>(r, key)] = static_cast<uint8_t>(hi);
            p[swizzled<128>(r + 1, key)] = static_cast<uint8_t>(hi >> 8);
            p[swizzled<128>(R + r, key)] = static_cast<uint8_t>(lo);
            p[swizzled<128>(R + r + 1, key)] = static_cast<uint8_t>(lo >> 8);
          }
        }
        fence_proxy_async_smem();
        mbar_arrive(&sm.p_full[b]);
        if (pending) add(n - 1);
#pragma unroll
        for (int pg = 0; pg < kPages; ++pg) vs[pg] = vs_now[pg];
        pending = true;
      }
      ++items;

      // ---- output: the sums of weights over the keys, then a dim of every row
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], o);
        if (lane == 0) sm.lsum[w4][r] = l[r];
      }
      add(n - 1);
      softmax_sync();
      const bool whole = walk.whole();
      float* part = w.parts + walk.slot() * w.slot_floats;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r < it.rows && ok) {
          const float sum = (sm.lsum[0][r] + sm.lsum[1][r]) + (sm.lsum[2][r] + sm.lsum[3][r]);
          if (whole) {
            const int at = it.row0 + r;
            const int64_t tok = it.first + at / a.group;
            const int head = it.h * a.group + at % a.group;
            if (key < D) a.out[tok * a.ots + head * a.ohs + key] = __float2bfloat16_rn(sum == 0.f ? 0.f : o[r] / sum);
            if (a.lse && key == 0) a.lse[tok * a.Hq + head] = sum == 0.f ? -INFINITY : (ref[r] - kShift + log2f(sum)) * 0.69314718055994531f;
          } else {
            if (key < D) part[r * D + key] = o[r];
            if (key == 0) {
              part[R * D + r] = ref[r];
              part[R * D + R + r] = sum;
            }
          }
        }
      }
      if (!whole) {
        // the last CTA of the item to get here joins all parts
        __threadfence();
        softmax_sync();
        if (key == 0) {
          const int32_t others = static_cast<int32_t>(walk.last_cta - walk.first_cta);
          sm.last = ok && atomicAdd(w.tickets + walk.first_cta, 1) == others;
          __threadfence();
          if (sm.last) w.tickets[walk.first_cta] = 0;
        }
        softmax_sync();
        if (sm.last) {
          constexpr int F = D / 4;
          for (int i = key; i < it.rows * F; i += 128) {
            const int r = i / F, f = i % F;
            float m = kNone;
#pragma unroll 4
            for (int64_t c = walk.first_cta; c <= walk.last_cta; ++c)
              m = fmaxf(m, __ldcg(w.parts + Kv8Walk::slot_of(c, walk.first_cta) * w.slot_floats + R * D + r));
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            float tot = 0.f;
#pragma unroll 4
            for (int64_t c = walk.first_cta; c <= walk.last_cta; ++c) {
              const float* p = w.parts + Kv8Walk::slot_of(c, walk.first_cta) * w.slot_floats;
              const float k = ex2(__ldcg(p + R * D + r) - m);
              const float4 v = __ldcg(reinterpret_cast<const float4*>(p + r * D + f * 4));
              sum.x = fmaf(v.x, k, sum.x);
              sum.y = fmaf(v.y, k, sum.y);
              sum.z = fmaf(v.z, k, sum.z);
              sum.w = fmaf(v.w, k, sum.w);
              tot = fmaf(__ldcg(p + R * D + R + r), k, tot);
            }
            const int at = it.row0 + r;
            const int64_t tok = it.first + at / a.group;
            const int head = it.h * a.group + at % a.group;
            const float down = tot == 0.f ? 0.f : 1.f / tot;
            *reinterpret_cast<uint2*>(a.out + tok * a.ots + head * a.ohs + f * 4) =
                make_uint2(pack_bf16(sum.x * down, sum.y * down), pack_bf16(sum.z * down, sum.w * down));
            if (a.lse && f == 0) a.lse[tok * a.Hq + head] = tot == 0.f ? -INFINITY : (m - kShift + log2f(tot)) * 0.69314718055994531f;
          }
        }
      }
      softmax_sync();  // (lsum and last are free again)
      if (lane == 0) mbar_arrive(&sm.q_free[qb]);
    }
  }
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
template <int D, int R>
cudaError_t init_one() {
  return cudaFuncSetAttribute(kv8_decode_kernel<D, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem_bytes<D, R>()));
}
template <int D, int R>
cudaError_t launch_one(const Kv8AttendArgs& a, Kv8Work w, int64_t rows, int ctas, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                       cudaStream_t st) {
  w.tile_rows = R;
  w.tiles = static_cast<int>((rows + R - 1) / R);
  w.items = static_cast<int64_t>(a.rows.batch) * a.Hkv * w.tiles;
  w.step_pages = DecodeShape<D, R>::kPages;
  w.min_steps = 4;
  w.slot_floats = static_cast<int64_t>(kv8_decode_slot(D));
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem_bytes<D, R>();
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kv8_decode_kernel<D, R>, a, w, tm_k, tm_v);
}
template <int D>
cudaError_t launch_dim(const Kv8AttendArgs& a, const Kv8Work& w, int ctas, const CUtensorMap& tm_k, const CUtensorMap& tm_v, cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(a.rows.max_rows) * a.group;
  return rows <= 8    ? launch_one<D, 8>(a, w, rows, ctas, tm_k, tm_v, st)
         : rows <= 16 ? launch_one<D, 16>(a, w, rows, ctas, tm_k, tm_v, st)
                      : launch_one<D, 32>(a, w, rows, ctas, tm_k, tm_v, st);
}

}  // namespace

int kv8_decode_rows(int) { return 32; }
size_t kv8_decode_slot(int D) { return static_cast<size_t>(32) * (D + 2); }

cudaError_t kv8_decode_init(int D) {
  cudaError_t e = D == 128 ? init_one<128, 8>() : init_one<64, 8>();
  if (e == cudaSuccess) e = D == 128 ? init_one<128, 16>() : init_one<64, 16>();
  if (e == cudaSuccess) e = D == 128 ? init_one<128, 32>() : init_one<64, 32>();
  return e;
}

cudaError_t launch_kv8_decode(const Kv8AttendArgs& a, Kv8Work w, int D, int ctas, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                              cudaStream_t st) {
  return D == 128 ? launch_dim<128>(a, w, ctas, tm_k, tm_v, st) : launch_dim<64>(a, w, ctas, tm_k, tm_v, st);
}

}  // namespace hsa
