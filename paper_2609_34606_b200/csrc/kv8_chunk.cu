// Attention over the 8-bit paged cache for many query rows of a key head: chunks, prompts.
//
// Here the operations bound the call, 4 * D for every pair of a query and a key, and what the tensor cores do not do has to
// fit beside them: an exponential for every pair (16 a clock on an SM, which is what the products of D = 128 take as well)
// and the values' way from 8 bits to 16.
//   S [128 rows x 64 keys] = (Qhi + Qlo) [128 x D] K^T [D x 64]   e4m3 codes as TMA leaves them; the queries in two terms,
//                                                                  which together take as long as one product of 16 bits
//   O [128 rows x D]      += P [128 x 64 keys] V [64 x D]          fp16: P from tensor memory, V from shared memory
// A query is hi = e4m3(x), lo = e4m3(x - hi), x scaled by a power of two that brings its row's largest value to 2^7 .. 2^8:
// bf16 values stay exact unless they are below 2^-10 of that, which may lose 2^-18 of it.  The codes of the values become fp16,
// which is exact.  Scales are left to the softmax: a page's key scale is in the factor that scores are multiplied by anyhow, its
// value scale in what is added in the exponent (and taken out of the sum of weights again).  So P holds weight times value scale.
// It is set up to have its largest value at 2^8 and may grow to 2^15; what fp16 cannot hold beside that, below 2^-25, is less than
// 2^-33 of the largest contribution.
// A row's reference has two parts, of the scores (`top`) and of the scales (`base`): a weight is 2^((s c - top) + (lv - base)).  Up to
// 2^22 both are whole numbers, so that (lv - base) - top is exact and one fma makes the exponent.  Above that fp32 leaves scores no
// fraction, and the exact product in an fma would differ from a rounded reference by up to half a step of it, which passes what fp16
// holds from 2^27 on: there the product is rounded first, the largest score gives a difference of 0, and only then the scales'
// part is added.
//
// An item has 256 rows, two tiles of 128, so that every page that is read and turned into fp16 serves both.  A tile's S has
// two buffers of a page's 64 keys: the products of a page run while the softmax is at the page before it.  (With one buffer of
// 128 keys products take 2048 cycles for two tiles and two pages instead of 2500, but products and softmax of a tile wait for each
// other: 1543 us instead of 1237 for the chunk below.)  An item of 128 rows or fewer gives both tiles to the same rows: they take its
// pages in turn and are brought together at its end.
//
// Warps: 0 loads pages, 1 and 2 issue the products of a tile each, 3 looks ahead for them, 4 - 7 turn values into fp16, 8 - 11
// and 12 - 15 are the softmax of a tile each, a row to a thread, whose query they also bring into its two terms.
// The warps that issue products stay together and choose a lane for it at the last moment: so their operands are in uniform
// registers.  A loop of one lane alone takes some 75 cycles to issue a product, beside busy warps, more than the product's 64.
//
// Measured: 4680 queries, 46,800 tokens, 12 heads of 128: 1160 to 1220 us in short runs (1160 to 1103 TFLOP/s), 1345 in a long one, at
// the board's 1 kW (1000 TFLOP/s; a library product of bf16 alone holds 1373).  A page takes 1750 to 1900 cycles for both tiles: its
// products 1280, its exponentials, of two warps on a special function unit at the same time, 1024.  What was tried and did not
// help: turns at the exponentials (1192 us), an eighth or a quarter of them as polynomials (1185, 1196), half a row to a thread and
// twice the warps (1400 against 1319), the next page's scores asked for early (1264 against 1237).
// Heads of 64 have half the products and the same exponentials: the softmax bounds them, and 10,000 cycles an item at its ends.
// Tensor memory: four S (P, packed fp16, over their first halves), O of both tiles.
#include "kv8.cuh"
#include "kv8_mma.cuh"

namespace hsa {

namespace {

constexpr int kThreads = 512;
constexpr int kTile = 128;          // rows of a tile
constexpr float kMost = 32768.f;    // what a page's 64 keys may add up to in P before a row's reference is set anew
constexpr float kShift = 8.f;       // ... to have the largest at 2^8
constexpr float kFar = 4194304.f;   // 2^22: references up to here take part in the product's own rounding
constexpr int kMetas = 16;

template <int D>
struct ChunkSmem {
  static constexpr int kPage = kBlock * D;
  static constexpr int kKStages = D == 128 ? 6 : 12, kVStages = 4, kBStages = 4;  // pages
  union {
    uint8_t q[2][2][kTile * D];        // [tile][term]
    float other[D][kTile];             // where both tiles have the same rows: what each gives the other of O
  };
  uint8_t k[kKStages][kPage];
  uint8_t vc[kVStages][kPage];         // codes
  uint8_t vb[kBStages][kPage * 2];     // fp16, [64 dims][key][64 dims]
  float qscale[2 * kTile];
  float other_top[2][kTile], other_base[2][kTile], other_sum[2][kTile];
  PageMeta meta[kMetas];
  int last[2];
  uint64_t k_full[kKStages], k_empty[kKStages], vc_full[kVStages], vc_empty[kVStages], vb_full[kBStages], vb_empty[kBStages];
  uint64_t s_full[4], p_full[4], pv_done[4], q_full, done[2];
  uint32_t tmem;
  Kv8Plan plan;
};

constexpr uint32_t kColS = 0, kColO = 256;  // + 64 a buffer of S, + 128 a tile

// ---- two fp32 in a register pair
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float2 unpair(uint64_t d) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(d));
  return f;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float m;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
  return m;
}

// Weights of 64 keys: 2^(s * c + nref) as fp16 pairs, and their sum in fp32.  The order of the instructions is made by hand: a
// pair's exponentials come kLag pairs behind its product, its sum and rounding another kLag behind them, so that nothing waits
// for its operands (the compiler's order leaves a lone warp waiting at each of them).
constexpr int kLag = 4;
__device__ __forceinline__ float weights(uint32_t* s, float c, float nref, uint32_t* w) {
  const uint64_t c2 = pair(c, c), r2 = pair(nref, nref);
  uint64_t sum[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 32 + 2 * kLag; ++i) {
    if (i < 32)
      asm volatile("{\n.reg .b64 t;\nmov.b64 t, {%0, %1};\nfma.rn.f32x2 t, t, %2, %3;\nmov.b64 {%0, %1}, t;\n}\n" : "+r"(s[2 * i]), "+r"(s[2 * i + 1]) : "l"(c2), "l"(r2));
    const int j = i - kLag;
    if (j >= 0 && j < 32) asm volatile("ex2.approx.ftz.f32 %0, %0;\nex2.approx.ftz.f32 %1, %1;\n" : "+r"(s[2 * j]), "+r"(s[2 * j + 1]));
    const int k = i - 2 * kLag;
    if (k >= 0)
      asm volatile("{\n.reg .b64 t;\nmov.b64 t, {%2, %3};\nadd.rn.f32x2 %0, %0, t;\ncvt.rn.f16x2.f32 %1, %3, %2;\n}\n" : "+l"(sum[k & 1]), "=r"(w[k]) : "r"(s[2 * k]), "r"(s[2 * k + 1]));
  }
  const float2 a = unpair(sum[0]), b = unpair(sum[1]);
  return (a.x + a.y) + (b.x + b.y);
}

// The same where a row of the warp is far: 2^(((s * c + n1) + n2) + n3).  (Summed in the same order: rows that are not far get what
// they get from weights().)
__device__ __forceinline__ float weights_far(uint32_t* s, float c, float n1, float n2, float n3, uint32_t* w) {
  float sum[2][2] = {};
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    float e[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      e[j] = ex2((fmaf(__uint_as_float(s[2 * i + j]), c, n1) + n2) + n3);
      sum[i & 1][j] += e[j];
    }
    asm("cvt.rn.f16x2.f32 %0, %2, %1;" : "=r"(w[i]) : "f"(e[0]), "f"(e[1]));
  }
  return (sum[0][0] + sum[0][1]) + (sum[1][0] + sum[1][1]);
}

// two e4m3 codes as fp16
__device__ __forceinline__ uint32_t fp16_of(uint32_t two) {
  uint32_t d;
  asm("{\n.reg .b16 lo, hi;\nmov.b32 {lo, hi}, %1;\ncvt.rn.f16x2.e4m3x2 %0, lo;\n}\n" : "=r"(d) : "r"(two));
  return d;
}
// Rows lo .. hi of 32 rows of the queries (row r at q_in + `from` of lane r, if it is in `there`) as two e4m3 terms into the rows from
// `first` on of the tiles at q and behind it.  Lane r gets what its row has been divided by.  Lanes next to each other read a row together.
// (Short code: it runs once an item, and has to come from far each time.)
template <int D>
__device__ __forceinline__ float two_terms(const __nv_bfloat16* q_in, int64_t from, uint32_t there, uint8_t* q, int first, int lane,
                                          int lo, int hi) {
  constexpr int C = D / 8, R = 32 / C, kAtOnce = 4;  // vectors of a row, rows at a time, loads in flight (and as many behind them)
  const int e = lane % C, k0 = lane / C;
  float mine = 1.f;
  uint4 in[kAtOnce], next[kAtOnce];
  const auto load = [&](int base) {
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int k = (base + i * R + k0) & 31;
      const int64_t at = __shfl_sync(0xffffffffu, from, k);
      next[i] = there >> k & 1 ? __ldg(reinterpret_cast<const uint4*>(q_in + at) + e) : make_uint4(0, 0, 0, 0);
    }
  };
  load(lo);
#pragma unroll 1
  for (int base = lo; base < hi; base += R * kAtOnce) {
    uint32_t top[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      in[i] = next[i];
      uint32_t* x = &in[i].x;
      __nv_bfloat162 m = __float2bfloat162_rn(0.f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // what is not finite: NaN, which spoils the row and no other
        const uint32_t size = x[j] & 0x7fff7fffu;
        const uint32_t bad = __hgeu2_mask(*reinterpret_cast<const __nv_bfloat162*>(&size), __float2bfloat162_rn(INFINITY));
        const uint32_t good = size & ~bad;
        x[j] |= bad & 0x7fff7fffu;
        m = __hmax2(m, *reinterpret_cast<const __nv_bfloat162*>(&good));
      }
      const uint32_t two = *reinterpret_cast<uint32_t*>(&m);
      top[i] = max(two & 0xffffu, two >> 16);
    }
    load(base + R * kAtOnce);
#pragma unroll
    for (int o = C / 2; o > 0; o >>= 1)
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) top[i] = max(top[i], __shfl_xor_sync(0xffffffffu, top[i], o));
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const uint32_t* x = &in[i].x;
      const int k = base + i * R + k0, ex = max(static_cast<int>(top[i] >> 7) - 127, -100) - 7;  // (rows of zeros: any will do)
      const float up = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
      uint32_t big[4], small[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // (fp16 has the 8 bits of these values, down to 2^-14, far below the last one of the second term)
        asm("{\n"
            ".reg .f32 a, b;\n"
            ".reg .b32 y, z, w;\n"
            ".reg .b16 h, l;\n"
            "shl.b32 w, %2, 16;\n"
            "mul.f32 a, w, %3;\n"
            "and.b32 w, %2, 0xffff0000;\n"
            "mul.f32 b, w, %3;\n"
            "cvt.rn.f16x2.f32 y, b, a;\n"
            "cvt.rn.satfinite.e4m3x2.f16x2 h, y;\n"
            "cvt.rn.f16x2.e4m3x2 z, h;\n"
            "sub.rn.f16x2 y, y, z;\n"
            "cvt.rn.satfinite.e4m3x2.f16x2 l, y;\n"
            "cvt.u32.u16 %0, h;\n"
            "cvt.u32.u16 %1, l;\n"
            "}\n"
            : "=r"(big[j]), "=r"(small[j])
            : "r"(x[j]), "f"(up));
      }
      uint8_t* at = q + swizzled<D>(first + k, e * 8);
      *reinterpret_cast<uint2*>(at) = make_uint2(big[0] | big[1] << 16, big[2] | big[3] << 16);
      *reinterpret_cast<uint2*>(at + kTile * D) = make_uint2(small[0] | small[1] << 16, small[2] | small[3] << 16);
      // rows base + i R .. + R are in the groups of C lanes
      const uint32_t of = __shfl_sync(0xffffffffu, 127 + ex, (lane % R) * C);
      if (lane / R == base / R + i) mine = __uint_as_float(of << 23);
    }
  }
  return mine;
}

__device__ __forceinline__ void tiles_sync() { asm volatile("barrier.cta.sync 3, 256;" ::: "memory"); }
__device__ __forceinline__ void tile_sync(int tile) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(1 + tile) : "memory"); }

// A row's reference.
struct RowRef {
  float top = kNone, base = 0.f;
  __device__ __forceinline__ static RowRef load(const float* p) { return RowRef{__ldcg(p), __ldcg(p + kTile)}; }
  __device__ __forceinline__ bool far() const { return fabsf(top) > kFar && top != kNone; }
  __device__ __forceinline__ float above(const RowRef& o) const { return (top - o.top) + (base - o.base); }  // exponent of what counted by this one
  __device__ __forceinline__ void raise(const RowRef& o) {  // (in the order of the CTAs: the result is the same whoever joins)
    if (o.above(*this) > 0.f) *this = o;
  }
  // ln of a sum of weights counted by it
  __device__ __forceinline__ float lse(float l) const { return l == 0.f ? -INFINITY : (top + (base + log2f(l))) * 0.69314718055994531f; }
};

// A part: a tile's O (fp32, unnormalised) as [D / 4][row][4], both parts of the rows' references, and sums.
template <int D>
__device__ __forceinline__ float* part_of(const Kv8Work& w, int64_t slot, int tile) {
  return w.parts + slot * w.slot_floats + tile * (kTile * (D + 3));
}

// Dims d0 .. d1 of a row of an item that is shared by CTAs, from all their parts.
template <int D>
__device__ __noinline__ void join_parts(const Kv8AttendArgs& a, const Kv8Work& w, const Kv8Segment& g, int t, int r, int d0, int d1, __nv_bfloat16* out,
                                        int64_t lse_at) {
  RowRef ref;
  float l = 0.f;
  for (int j = g.first_cta; j <= g.last_cta; ++j) ref.raise(RowRef::load(part_of<D>(w, Kv8Segment::slot_of(j, g.first_cta), t) + kTile * D + r));
#pragma unroll 1
  for (int c = d0; c < d1; c += 32) {
    float4 o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    l = 0.f;
#pragma unroll 1
    for (int j = g.first_cta; j <= g.last_cta; ++j) {
      const float* p = part_of<D>(w, Kv8Segment::slot_of(j, g.first_cta), t);
      const float f = ex2(RowRef::load(p + kTile * D + r).above(ref));
      l = fmaf(__ldcg(p + kTile * D + 2 * kTile + r), f, l);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(p) + (c / 4 + k) * kTile + r);
        o[k].x = fmaf(v.x, f, o[k].x);
        o[k].y = fmaf(v.y, f, o[k].y);
        o[k].z = fmaf(v.z, f, o[k].z);
        o[k].w = fmaf(v.w, f, o[k].w);
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int k = 0; k < 8; k += 2)
      *reinterpret_cast<uint4*>(out + c + k * 4) =
          make_uint4(pack_bf16(o[k].x * inv, o[k].y * inv), pack_bf16(o[k].z * inv, o[k].w * inv),
                     pack_bf16(o[k + 1].x * inv, o[k + 1].y * inv), pack_bf16(o[k + 1].z * inv, o[k + 1].w * inv));
  }
  if (a.lse && d0 == 0) a.lse[lse_at] = ref.lse(l);
}

// LOOK: waits of less than a poll's sleep
template <int D, bool LOOK>
__global__ void __launch_bounds__(kThreads, 1)
kv8_chunk_kernel(const __grid_constant__ Kv8AttendArgs a, const __grid_constant__ Kv8Work w, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v) {
  using Smem = ChunkSmem<D>;
  constexpr int kKStages = Smem::kKStages, kVStages = Smem::kVStages, kBStages = Smem::kBStages, kPage = Smem::kPage;
  extern __shared__ uint8_t smem_raw[];
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, lane = tid & 31, warp = tid / 32;
  if (tid == 0) {
    for (int i = 0; i < kKStages; ++i) {
      mbar_init(&sm.k_full[i], 1);
      mbar_init(&sm.k_empty[i], 2);
    }
    for (int i = 0; i < kVStages; ++i) {
      mbar_init(&sm.vc_full[i], 1);
      mbar_init(&sm.vc_empty[i], 4);
    }
    for (int i = 0; i < kBStages; ++i) {
      mbar_init(&sm.vb_full[i], 4);
      mbar_init(&sm.vb_empty[i], 2);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&sm.s_full[i], 1);
      mbar_init(&sm.p_full[i], 4 + 1);  // the tile's warps, and the one that looks ahead
      mbar_init(&sm.pv_done[i], 1);
    }
    mbar_init(&sm.q_full, 8);
    mbar_init(&sm.done[0], 1);
    mbar_init(&sm.done[1], 1);
    fence_mbar_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem, 512);
    tmem_relinquish();
  }
  kv8_plan<kThreads>(a, w, &sm.plan);
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
  // both tiles of the item on the same rows?
  const auto shared_rows = [](const Kv8Item& it) { return it.rows <= kTile; };

  // The CTA is allocated 128 registers a thread.  Half of them give back 48, which the softmax warps take.
  static_assert(256 * (128 - 80) >= 256 * (176 - 128), "setmaxnreg.inc would never be satisfied");
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 0) {
      // ---- loads.  The lanes look up 32 pages at once.
      uint32_t n = 0, ahead = 0;  // pages; 1: keys whose values have not been asked for
      while (ok && walk.next(a, w, sm.plan)) {
        const Kv8Item& it = walk.g.it;
        const int per = shared_rows(it) ? 2 : 1, s1 = walk.g.s1 * per;  // pages
        for (int s = walk.g.s0 * per; s < s1 && ok; s += 32) {
          int blk = 0, page = -1;
          PageMeta meta{-1, 1.f, 1.f};
          if (s + lane < s1) page = kv8_page(a, it, s + lane, &blk);
          if (page >= 0) {
            const int64_t ph = static_cast<int64_t>(page) * a.Hkv + it.h;
            meta.pos = blk * kBlock;
            meta.ks = __ldg(a.k_scale + ph);
            meta.vs = fmaxf(__ldg(a.v_scale + ph), 0x1p-60f);  // (0 is no scale; it would leave NaN)
          }
          const int count = min(32, s1 - s);
#pragma unroll 1
          for (int i = 0; i < count; ++i, ++n) {
            const uint32_t st = n % kKStages, sv = n % kVStages;
            if (!warp_wait(&sm.k_empty[st], ((n / kKStages) & 1) ^ 1)) break;
            const int p = __shfl_sync(0xffffffffu, page, i);
            const int row = static_cast<int>((static_cast<int64_t>(p) * a.Hkv + it.h) * kBlock);
            // the loads go out before the scales are there; the barrier is arrived at behind them
            if (p >= 0 && elect_one_sync()) {
              mbar_expect_tx_only(&sm.k_full[st], kPage);
              tma_load_2d(sm.k[st], &tm_k, &sm.k_full[st], 0, row);
            }
            if (lane == i) sm.meta[n % kMetas] = meta;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.k_full[st]);
            if (!warp_wait(&sm.vc_empty[sv], ((n / kVStages) & 1) ^ 1)) {
              ahead = 1;
              break;
            }
            if (elect_one_sync()) {
              if (p >= 0) {
                mbar_expect_tx(&sm.vc_full[sv], kPage);
                tma_load_2d(sm.vc[sv], &tm_v, &sm.vc_full[sv], 0, row);
              } else {
                mbar_arrive(&sm.vc_full[sv]);
              }
            }
            __syncwarp();
          }
        }
      }
      // the last pages, a lane each, whether somebody takes them or not
      static_assert(kKStages <= 16 && kVStages <= 16);
      const uint32_t back = lane % 16 + 1, all = lane < 16 ? n + ahead : n, ring = lane < 16 ? kKStages : kVStages;
      if (back <= ring && back <= all) {
        const uint32_t i = all - back;
        if (!mbar_drain(lane < 16 ? &sm.k_full[i % kKStages] : &sm.vc_full[i % kVStages], (i / ring) & 1)) ok = false;
      }
    } else if (warp <= 2) {
      // ---- products of a tile.  A unit is a page of the item (of shared rows: every other page); scores are two units ahead, and
      // go over the weights of a page as soon as those have been issued: the products run in the order of their issue.
      constexpr uint32_t id_s = idesc_e4m3(128, kBlock, 0, 0), id_o = idesc_fp16(128, D, 0, 1), hi_v = desc_hi_sw128(1024);
      const uint32_t t = warp_uniform(warp - 1), tm = warp_uniform(tmem);
      const uint32_t q0 = row_desc_lo(smem_u32(sm.q)), k0 = row_desc_lo(smem_u32(sm.k)), v0 = desc_lo_sw128(smem_u32(sm.vb), kBlock * 128);
      const uint32_t s0 = tm + kColS + t * 64, o0 = tm + kColO + t * 128;
      uint32_t items = 0, ns = 0, n = 0, st = 0, round = 0, nv = 0;  // items; units of scores, of values; stages of K and V
      while (warp_uniform(walk.next(a, w, sm.plan))) {
        const uint32_t same = warp_uniform(shared_rows(walk.g.it)), units = warp_uniform(walk.g.s1 - walk.g.s0);
        const uint32_t q = q0 + (same ? 0 : t) * (2 * kTile * D / 16), step = 1 + same, first = same & t;
        // K's stages go round in turn
        const auto move = [&](uint32_t by) {
          st += by;
          const uint32_t over = st >= kKStages;
          round += over;
          st -= over ? kKStages : 0;
        };
        const auto scores = [&]() {
          const uint32_t k = k0 + st * (kPage / 16), d = s0 + (ns & 1) * 128, b = (ns & 1) * 2 + t;
          if (elect_one_sync() && ok) {
#pragma unroll
            for (int term = 0; term < 2; ++term)
#pragma unroll
              for (int kk = 0; kk < D / 32; ++kk)
                mma_f8_lo(d, q + (term * kTile * D + kk * 32) / 16, k + kk * 2, row_desc_hi<D>(), row_desc_hi<D>(), id_s, term + kk > 0);
            tc_commit(&sm.s_full[b]);
            tc_commit(&sm.k_empty[st]);
          }
          __syncwarp();
          move(step);
          ++ns;
        };
        wait(&sm.q_full, items & 1);
        ++items;
        move(first);
        nv += first;
        for (uint32_t u = 0; u < 2 && u < units; ++u) {
          wait(&sm.k_full[st], round & 1);
          tc_fence_after();
          scores();
        }
#pragma unroll 1
        for (uint32_t u = 0; u < units; ++u, ++n) {
          const uint32_t sv = nv % kBStages, v = v0 + sv * (kPage * 2 / 16), b = (n & 1) * 2 + t, pw = s0 + (n & 1) * 128;
          wait(&sm.p_full[b], (n / 2) & 1);
          tc_fence_after();
          if (elect_one_sync() && ok) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) tc_mma_ts_lo(o0, pw + kk * 8, v + kk * 128, hi_v, id_o, u > 0 || kk > 0);
            tc_commit(&sm.pv_done[b]);
            tc_commit(&sm.vb_empty[sv]);
          }
          __syncwarp();
          nv += step;
          if (u + 2 < units) scores();
        }
        // (behind the item's last page)
        nv -= first;
        if (first) {
          round -= st == 0;
          st = st == 0 ? kKStages - 1 : st - 1;
        }
      }
      if (elect_one_sync()) tc_commit(&sm.done[t]);
      __syncwarp();
      if (!mbar_drain(&sm.done[t], 0)) ok = false;  // (whatever ran out before: products in flight must not outlive the CTA)
    } else {
      // ---- looks ahead for warps 1 and 2, who would otherwise poll three barriers for a page (each some 250 cycles beside busy
      // warps): arrives with the weights of a page where its values and the keys of the scores behind it are there.  Where the
      // tiles share rows, gives pages back for the tile that does not use them.
      uint32_t n = 0, ks = 0, kr = 0, nv = 0;  // units of a tile before the item; stage of K, rounds; pages of V
      const auto keys = [&](bool same) {
        wait(&sm.k_full[ks], kr & 1);
        mbar_arrive_if(&sm.k_empty[ks], same && lane == 0 && ok);
        ++ks;
        kr += ks == kKStages;
        ks = ks == kKStages ? 0 : ks;
      };
      while (walk.next(a, w, sm.plan)) {
        const bool same = shared_rows(walk.g.it);
        const int pages = (walk.g.s1 - walk.g.s0) * (same ? 2 : 1), first = same ? 4 : 2;  // pages of the scores ahead
        for (int m = 0; m < first && m < pages; ++m) keys(same);
#pragma unroll 1
        for (int m = 0; m < pages; ++m, ++nv) {
          wait(&sm.vb_full[nv % kBStages], (nv / kBStages) & 1);
          mbar_arrive_if(&sm.vb_empty[nv % kBStages], same && lane == 0 && ok);
          if (m + first < pages) keys(same);
          const uint32_t at = n + (same ? m / 2 : m), b = (at & 1) * 2;
          for (int t = 0; t < 2; ++t) {
            if (same && t != (m & 1)) continue;
            if (at >= 2) wait(&sm.p_full[b + t], (at / 2 + 1) & 1);  // (the weights before these are complete)
            mbar_arrive_if(&sm.p_full[b + t], lane == 0 && ok);
          }
        }
        n += walk.g.s1 - walk.g.s0;
      }
    }
  } else if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    // ---- values into fp16
    const int c = tid - 128;
    uint32_t n = 0;
    while (walk.next(a, w, sm.plan)) {
      const int pages = (walk.g.s1 - walk.g.s0) * (shared_rows(walk.g.it) ? 2 : 1);
      constexpr int C = D / 8, R = 128 / C;  // 8 dims of a row, rows at a time
      const int r0 = c / C, e = c % C;
      // (row & 7 and the bits of the swizzle are the same for all of a thread's rows, R apart)
      const int from = swizzled<D>(r0, e * 8), to = (e / 8) * (kBlock * 128) + r0 * 128 + (((e & 7) ^ (r0 & 7)) << 4);
#pragma unroll 1
      for (int s = 0; s < pages; ++s, ++n) {
        const uint32_t sv = n % kVStages, b = n % kBStages;
        warp_wait(&sm.vc_full[sv], (n / kVStages) & 1);
        const bool there = sm.meta[n % kMetas].pos >= 0;  // (else: zeros, which is what weights of 0 can bear)
        uint2 in[kBlock / R];
#pragma unroll
        for (int i = 0; i < kBlock / R; ++i) in[i] = *reinterpret_cast<const uint2*>(sm.vc[sv] + from + i * R * D);
        warp_wait(&sm.vb_empty[b], ((n / kBStages) & 1) ^ 1);
#pragma unroll
        for (int i = 0; i < kBlock / R; ++i) {
          if (!there) in[i] = make_uint2(0, 0);
          *reinterpret_cast<uint4*>(sm.vb[b] + to + i * R * 128) =
              make_uint4(fp16_of(in[i].x), fp16_of(in[i].x >> 16), fp16_of(in[i].y), fp16_of(in[i].y >> 16));
        }
        fence_proxy_async_smem();
        __syncwarp();
        mbar_arrive_if(&sm.vb_full[b], lane == 0 && ok);
        mbar_arrive_if(&sm.vc_empty[sv], lane == 0 && ok);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
    // ---- softmax: a thread is a row of the tile.  After a wait that ran out the threads go on with whatever is there,
    // because they meet at barriers; the status word says that the result is none.
    const int t = (warp - 8) / 4, r = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t col_o = tmem + lanes + kColO + t * 128;
    uint32_t items = 0, n = 0, kn = 0;  // items, units of this tile, pages before the item's first
    while (walk.next(a, w, sm.plan)) {
      const Kv8Item& it = walk.g.it;
      const bool same = shared_rows(it);
      const int units = walk.g.s1 - walk.g.s0;
      const int row = same ? r : t * kTile + r;  // of the item
      const int lim = it.limit(a, min(row, it.rows - 1)), lim_low = it.limit(a, same ? 0 : t * kTile);
      const bool mine = row < it.rows;
      const int at = it.row0 + min(row, it.rows - 1), head = it.h * a.group + at % a.group;
      const int64_t tok = it.first + at / a.group;
      // The rows into their two terms; of shared ones each tile's warps do half.  (Nobody reads what was there: the scores of the
      // last item have been seen, and with this barrier all its rows have been written out.)
      if (same) tiles_sync();
      else tile_sync(t);
      const int lo = same ? t * 16 : 0, hi = same ? lo + 16 : 32;
      const float e = two_terms<D>(a.q, tok * a.ts + head * a.hs, __ballot_sync(0xffffffffu, mine), sm.q[same ? 0 : t][0], r - lane, lane, lo, hi);
      if (lane >= lo && lane < hi) sm.qscale[row] = e * a.scale_log2;
      fence_proxy_async_smem();
      __syncwarp();
      mbar_arrive_if(&sm.q_full, lane == 0 && ok);
      if (same) {
        wait(&sm.q_full, items & 1);
        __syncwarp();
      }
      const float qs = sm.qscale[row];
      RowRef ref;
      float l = 0.f;
      bool far = false;
#pragma unroll 1
      for (int u = 0; u < units; ++u, ++n) {
        const uint32_t b = (n & 1) * 2 + t, col_s = tmem + lanes + kColS + b * 64;
        wait(&sm.s_full[b], (n / 2) & 1);
        __syncwarp();
        tc_fence_after();
        uint32_t x[64], p[32];
        const auto load = [&]() {
          tmem_ld32(col_s, *reinterpret_cast<uint32_t(*)[32]>(x));
          tmem_ld32(col_s + 32, *reinterpret_cast<uint32_t(*)[32]>(x + 32));
        };
        load();
        const PageMeta meta = sm.meta[(kn + (same ? 2 * u + t : u)) % kMetas];
        const float c = fmaxf(qs * meta.ks, 0x1p-126f);  // (never 0: scores may be -inf)
        const float lv = static_cast<float>(static_cast<int>(__float_as_uint(meta.vs) >> 23) - 127);
        const bool masked = meta.pos < 0 || meta.pos + kBlock > lim_low;
        const auto mask = [&]() {
          const int lim0 = meta.pos < 0 ? 0 : lim - meta.pos;
#pragma unroll
          for (int i = 0; i < 64; ++i)
            if (i >= lim0) x[i] = 0xff800000u;
        };
        tc_wait_ld();
        if (__builtin_expect(masked, 0)) mask();
        float more = weights(x, c, (lv - ref.base) - ref.top, p);
        // The sum tells whether the reference is still good (at an item's begin it is not: the sum is infinite).  The maximum of the
        // scores is looked for only where it is not, and for rows that are far.
        if (__builtin_expect(__any_sync(0xffffffffu, more > kMost || far), 0)) {
          load();
          tc_wait_ld();
          if (masked) mask();
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < 64; i += 2) top = max3(top, __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
          top *= c;
          const bool up = far ? (top - ref.top) + (lv - ref.base) > kShift : more > kMost;
          const RowRef to{up ? rintf(top) : ref.top, up ? lv - kShift : ref.base};
          if (__any_sync(0xffffffffu, up)) {
            const float f = up ? ex2(ref.above(to)) : 1.f;
            l *= f;
            if (u > 0) {
              wait(&sm.pv_done[((n - 1) & 1) * 2 + t], ((n - 1) / 2) & 1);  // (those before have been, or these scores were not there)
              __syncwarp();
              tc_fence_after();
#pragma unroll 1
              for (int i = 0; i < D; i += 16) {
                uint32_t o[16];
                tmem_ld16(col_o + i, o);
                tc_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                tmem_st16(col_o + i, o);
              }
            }
          }
          ref = to;
          far = ref.far();
          // (rows whose reference stays get the weights they had)
          const float scales = lv - ref.base;
          if (__any_sync(0xffffffffu, far)) more = weights_far(x, c, far ? -0.f : scales - ref.top, far ? -ref.top : 0.f, far ? scales : 0.f, p);
          else more = weights(x, c, scales - ref.top, p);
        }
        tmem_st32(col_s, p);
        l = fmaf(more, __uint_as_float((254u << 23) - (__float_as_uint(meta.vs) & 0x7f800000u)), l);  // 1 / vs
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        mbar_arrive_if(&sm.p_full[b], lane == 0 && ok);
      }
      kn += units * (same ? 2 : 1);
      wait(&sm.pv_done[((n - 1) & 1) * 2 + t], ((n - 1) / 2) & 1);
      __syncwarp();
      tc_fence_after();
      ++items;
      if (same) tiles_sync();  // (`other` lies where the queries are: both tiles have all their scores)
      // Of shared rows each tile brings half of the dims to their end: it gives its sums of the other half.
      float down = 1.f, take = 0.f;  // what this tile's O counts, and the other's
      const int d0 = same ? t * (D / 2) : 0, d1 = same ? d0 + D / 2 : D;
      if (same) {
        const int give = D / 2 - d0;
#pragma unroll 1
        for (int i = give; i < give + D / 2; i += 32) {
          uint32_t o[32];
          tmem_ld32(col_o + i, o);
          tc_wait_ld();
#pragma unroll
          for (int j = 0; j < 32; ++j) sm.other[i + j][r] = __uint_as_float(o[j]);
        }
        sm.other_top[t][r] = ref.top;
        sm.other_base[t][r] = ref.base;
        sm.other_sum[t][r] = l;
        tiles_sync();
        const RowRef r0{sm.other_top[0][r], sm.other_base[0][r]}, r1{sm.other_top[1][r], sm.other_base[1][r]};
        const float above = r1.above(r0), f0 = above > 0.f ? ex2(-above) : 1.f, f1 = above > 0.f ? 1.f : ex2(above);
        down = t == 0 ? f0 : f1;
        take = t == 0 ? f1 : f0;
        l = fmaf(sm.other_sum[1][r], f1, sm.other_sum[0][r] * f0);
        ref = above > 0.f ? r1 : r0;
      }
      // Is the item shared with other CTAs, then the last one of them joins the parts, in the order of the CTAs whoever that is, its
      // own from where it is.  The others leave theirs in the workspace.
      const Kv8Segment& g = walk.g;
      const bool real = mine && ok;
      const int others = g.last_cta - g.first_cta;
      int32_t* ticket = w.tickets + 2 * g.first_cta + t;
      bool joins = false;
      if (others) {
        if (r == 0) {
          int32_t there;
          asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(there) : "l"(ticket) : "memory");
          if (there == others) *ticket = 0;
          sm.last[t] = there == others;
        }
        tile_sync(t);
        joins = sm.last[t];
      }
      const bool writes = !others || joins;  // the item's rows, else a part
      float own = 1.f;                       // what this CTA's O counts
      if (joins) {
        RowRef m;
#pragma unroll 4
        for (int j = g.first_cta; j <= g.last_cta; ++j)
          m.raise(j == static_cast<int>(blockIdx.x) ? ref : RowRef::load(part_of<D>(w, Kv8Segment::slot_of(j, g.first_cta), t) + kTile * D + r));
        own = ex2(ref.above(m));
        float sum = 0.f;
#pragma unroll 1
        for (int j = g.first_cta; j <= g.last_cta; ++j) {
          const float* p = part_of<D>(w, Kv8Segment::slot_of(j, g.first_cta), t) + kTile * D + r;
          const bool here = j == static_cast<int>(blockIdx.x);
          sum = fmaf(here ? l : __ldcg(p + 2 * kTile), here ? own : ex2(RowRef::load(p).above(m)), sum);
        }
        l = sum;
        ref = m;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      float* part = part_of<D>(w, g.slot(), t);
      __nv_bfloat16* out = a.out + tok * a.ots + head * a.ohs;
      // Whole rows go through shared memory, where the tile's queries were, so that lanes next to each other write next to each
      // other (`other` leaves no place for that).
      uint8_t* rows = sm.q[t][0] + (warp & 3) * (32 * D * 2);
#pragma unroll 1
      for (int i = d0; i < d1; i += 32) {
        uint32_t o[32];
        tmem_ld32(col_o + i, o);
        tc_wait_ld();
        if (same) {
#pragma unroll
          for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(fmaf(sm.other[i + j][r], take, __uint_as_float(o[j]) * down));
        }
        if (joins) {
          float sum[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) sum[k] = 0.f;
#pragma unroll 1
          for (int j = g.first_cta; j <= g.last_cta; ++j) {
            if (j == static_cast<int>(blockIdx.x)) {
#pragma unroll
              for (int k = 0; k < 32; ++k) sum[k] = fmaf(__uint_as_float(o[k]), own, sum[k]);
              continue;
            }
            const float* p = part_of<D>(w, Kv8Segment::slot_of(j, g.first_cta), t);
            float4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __ldcg(reinterpret_cast<const float4*>(p) + (i / 4 + k) * kTile + r);
            const float f = ex2(RowRef::load(p + kTile * D + r).above(ref));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              sum[4 * k] = fmaf(v[k].x, f, sum[4 * k]);
              sum[4 * k + 1] = fmaf(v[k].y, f, sum[4 * k + 1]);
              sum[4 * k + 2] = fmaf(v[k].z, f, sum[4 * k + 2]);
              sum[4 * k + 3] = fmaf(v[k].w, f, sum[4 * k + 3]);
            }
          }
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(sum[k]);
        }
        if (writes) {
#pragma unroll
          for (int j = 0; j < 32; j += 8) {
            uint32_t y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              y[k] = pack_bf16(__uint_as_float(o[j + 2 * k]) * inv, __uint_as_float(o[j + 2 * k + 1]) * inv);
            const uint4 v = make_uint4(y[0], y[1], y[2], y[3]);
            if (!same) *reinterpret_cast<uint4*>(rows + lane * (D * 2) + ((((i + j) / 8) ^ (lane & 7)) << 4)) = v;
            else if (real) *reinterpret_cast<uint4*>(out + i + j) = v;
          }
        } else if (real) {
#pragma unroll
          for (int j = 0; j < 32; j += 4)
            __stcg(reinterpret_cast<uint4*>(part) + ((i + j) / 4) * kTile + r, make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]));
        }
        __syncwarp();
      }
      if (writes && !same) {
        constexpr int C = D / 8, R = 32 / C;  // vectors of a row, rows at a time
        const uint32_t reals = __ballot_sync(0xffffffffu, real);
        const int64_t from = tok * a.ots + head * a.ohs;
#pragma unroll 4
        for (int i = 0; i < 32; i += R) {
          const int k = i + lane / C, v = lane % C;
          const int64_t to = __shfl_sync(0xffffffffu, from, k);
          if (reals >> k & 1) *reinterpret_cast<uint4*>(a.out + to + v * 8) = *reinterpret_cast<const uint4*>(rows + k * (D * 2) + ((v ^ (k & 7)) << 4));
        }
        __syncwarp();
      }
      if (real) {
        if (writes) {
          if (a.lse && d0 == 0) a.lse[tok * a.Hq + head] = ref.lse(l);
        } else {
          __stcg(part + kTile * D + r, ref.top);
          __stcg(part + kTile * D + kTile + r, ref.base);
          __stcg(part + kTile * D + 2 * kTile + r, l);
        }
      }
      if (same) tiles_sync();
      if (!writes) {
        tile_sync(t);
        if (r == 0) {
          bool last = false;
          if (ok) {  // (what the tile has written before the barrier goes before, what it reads behind it comes after)
            int32_t before;
            asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(ticket) : "memory");
            last = before == others;
            if (last) *ticket = 0;
          }
          sm.last[t] = last;
        }
        tile_sync(t);
        if (sm.last[t] && real) join_parts<D>(a, w, g, t, r, d0, d1, out, tok * a.Hq + head);  // (the last of the others came meanwhile)
      }
    }
  }
  if (!ok) kv8_flag(a.status, kDevTimeout);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) tmem_dealloc(tmem, 512);
}

template <int D>
constexpr size_t smem_bytes() {
  static_assert(sizeof(ChunkSmem<D>) + 1024 <= 232448, "shared memory of an SM");
  return sizeof(ChunkSmem<D>) + 1024;
}
using ChunkKernel = void (*)(Kv8AttendArgs, Kv8Work, CUtensorMap, CUtensorMap);
ChunkKernel kernel_of(int D, bool look) {
  return D == 128 ? look ? kv8_chunk_kernel<128, true> : kv8_chunk_kernel<128, false> : look ? kv8_chunk_kernel<64, true> : kv8_chunk_kernel<64, false>;
}

}  // namespace

size_t kv8_chunk_slot(int D) { return static_cast<size_t>(2 * kTile) * (D + 3); }

cudaError_t kv8_chunk_init(int D) {
  const int bytes = static_cast<int>(D == 128 ? smem_bytes<128>() : smem_bytes<64>());
  const cudaError_t e = cudaFuncSetAttribute(kernel_of(D, false), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  return e == cudaSuccess ? cudaFuncSetAttribute(kernel_of(D, true), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) : e;
}

cudaError_t launch_kv8_chunk(const Kv8AttendArgs& a, Kv8Work w, int D, int ctas, const CUtensorMap& tm_k, const CUtensorMap& tm_v,
                             cudaStream_t st) {
  const int64_t rows = static_cast<int64_t>(a.rows.max_rows) * a.group;
  w.tile_rows = 2 * kTile;
  w.tiles = static_cast<int>((rows + 2 * kTile - 1) / (2 * kTile));
  w.items = static_cast<int64_t>(a.rows.batch) * a.Hkv * w.tiles;
  w.step_log = 0;
  w.half_rows = kTile;
  w.part_log = 3;
  w.item_steps = 8;
  w.slot_floats = static_cast<int64_t>(kv8_chunk_slot(D));
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = D == 128 ? smem_bytes<128>() : smem_bytes<64>();
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel_of(D, w.look != 0), a, w, tm_k, tm_v);
}

}  // namespace hsa
