// C-ABI layer of the 8-bit paged cache: context, argument checks, launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <cmath>
#include <new>

#include "kv8.cuh"

using namespace hsa;

struct hsa_kv8 {
  hsa_kv8_config cfg;
  hsa_kv8_buffers buf;
  float scale;
  int dev, nsm;
  CUtensorMap tm_k, tm_v;
  int last_cuda_error;
  uint64_t wait_ns;  // bound of the attention kernels' waits
};

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

bool config_ok(const hsa_kv8_config* c) {
  if (!c) return false;
  if (c->num_kv_heads < 1 || c->num_heads < c->num_kv_heads || c->num_heads > 1024 || c->num_heads % c->num_kv_heads) return false;
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->page_tokens != HSA_PAGE_TOKENS) return false;
  if (c->max_pages < 1 || c->max_blocks < 1 || c->max_tokens < 1) return false;
  if (c->max_batch < 1 || c->max_batch > 4096) return false;
  // items of an attention launch: (sequence, key head, 8 rows or more)
  if ((static_cast<int64_t>(c->max_tokens) * (c->num_heads / c->num_kv_heads) / 8 + 1) * c->max_batch * c->num_kv_heads >= (1ll << 31)) return false;
  if (static_cast<int64_t>(c->max_pages) * c->num_kv_heads * kBlock >= (1ll << 31)) return false;  // rows of a pool: TMA coordinates
  if (static_cast<int64_t>(c->max_blocks) * kBlock >= (1ll << 31)) return false;                   // lengths are int32
  if (!(c->softmax_scale >= 0.f) || !std::isfinite(c->softmax_scale)) return false;
  return c->flags == 0;
}

int cuda_fail(hsa_kv8* ctx, cudaError_t e) {
  if (ctx) ctx->last_cuda_error = static_cast<int>(e);
  return HSA_ERR_CUDA;
}

bool tensor_ok(const void* p, int64_t ts, int64_t hs, int D) {
  return p && aligned(p, 16) && ts >= D && hs >= D && (ts % 8) == 0 && (hs % 8) == 0;
}

// Rows of a call; false where they do not fit.
bool rows_ok(const hsa_kv8* ctx, int32_t n_tokens, int32_t batch, const int32_t* start, int32_t max_rows, Kv8Rows* out) {
  if (batch < 1 || batch > ctx->cfg.max_batch || n_tokens < 1 || n_tokens > ctx->cfg.max_tokens) return false;
  if (max_rows < 1 || max_rows > n_tokens || !aligned(start, 4)) return false;
  if (!start && (n_tokens % batch || n_tokens / batch > max_rows)) return false;
  *out = Kv8Rows{start, n_tokens, batch, max_rows, n_tokens / batch};
  return true;
}

// The context's device is the current one?
bool on_device(hsa_kv8* ctx) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == ctx->dev;
}

// workspace: status word, tickets, parts
constexpr int kMaxCtas = 160;  // CTAs of an attention launch (one to an SM)
constexpr size_t kStatusBytes = 256, kTicketBytes = 1280;
static_assert(2 * kMaxCtas * 4 <= kTicketBytes, "two tickets to a CTA");

// floats of a part: what the kernel for many rows leaves, where a call can have that many
size_t part_floats(const hsa_kv8_config* c) {
  const int64_t rows = static_cast<int64_t>(c->max_tokens) * (c->num_heads / c->num_kv_heads);
  return rows > kv8_decode_rows(c->head_dim) ? kv8_chunk_slot(c->head_dim) : kv8_decode_slot(c->head_dim);
}

// A pool as rows of head_dim bytes, read a page tile (64 rows) at a time into the swizzle that spans a row.
bool encode_pool(CUtensorMap* tm, void* base, uint64_t rows, int D) {
  void* p = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
    return false;
  const auto enc = reinterpret_cast<CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill)>(p);
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(D), rows}, strides[1] = {static_cast<cuuint64_t>(D)};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(D), kBlock}, ones[2] = {1, 1};
  return enc(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
             D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

extern "C" {

int hsa_kv8_query_sizes(const hsa_kv8_config* cfg, hsa_kv8_sizes* out) {
  if (!config_ok(cfg) || !out) return HSA_ERR_INVALID_ARG;
  const size_t pages = cfg->max_pages, H = cfg->num_kv_heads, D = cfg->head_dim;
  out->k_pool = out->v_pool = pages * H * kBlock * D;
  out->k_scale = out->v_scale = pages * H * 4;
  out->page_table = static_cast<size_t>(cfg->max_batch) * cfg->max_blocks * 4;
  out->ksum = static_cast<size_t>(cfg->max_batch) * H * cfg->max_blocks * D * 4;
  out->workspace = kStatusBytes + kTicketBytes + 2 * kMaxCtas * part_floats(cfg) * 4;
  return HSA_OK;
}

int hsa_kv8_create(hsa_kv8** out, const hsa_kv8_config* cfg, const hsa_kv8_buffers* b) {
  if (!out) return HSA_ERR_INVALID_ARG;
  *out = nullptr;
  if (!config_ok(cfg) || !b) return HSA_ERR_INVALID_ARG;
  if (!b->k_pool || !b->v_pool || !b->k_scale || !b->v_scale || !b->page_table || !b->workspace) return HSA_ERR_INVALID_ARG;
  if (!aligned(b->k_pool, 256) || !aligned(b->v_pool, 256) || !aligned(b->workspace, 256) || !aligned(b->k_scale, 16) ||
      !aligned(b->v_scale, 16) || !aligned(b->page_table, 16) || !aligned(b->ksum, 16))
    return HSA_ERR_INVALID_ARG;
  int dev = 0, cc_major = 0, nsm = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return HSA_ERR_CUDA;
  cudaDeviceGetAttribute(&cc_major, cudaDevAttrComputeCapabilityMajor, dev);
  cudaDeviceGetAttribute(&nsm, cudaDevAttrMultiProcessorCount, dev);
  if (cc_major != 10) return HSA_ERR_UNSUPPORTED;  // sm_100a only, no fallback
  hsa_kv8* ctx = new (std::nothrow) hsa_kv8();
  if (!ctx) return HSA_ERR_INVALID_ARG;
  ctx->cfg = *cfg;
  ctx->buf = *b;
  ctx->scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / std::sqrt(static_cast<float>(cfg->head_dim));
  ctx->dev = dev;
  ctx->nsm = nsm;
  ctx->last_cuda_error = 0;
  ctx->wait_ns = 2'000'000'000;
  cudaError_t e = cudaMemset(b->workspace, 0, kStatusBytes + kTicketBytes);
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = kv8_append_init(cfg->head_dim);
  if (e == cudaSuccess) e = kv8_decode_init(cfg->head_dim);
  if (e == cudaSuccess) e = kv8_chunk_init(cfg->head_dim);
  const uint64_t rows = static_cast<uint64_t>(cfg->max_pages) * cfg->num_kv_heads * kBlock;
  if (e != cudaSuccess || !encode_pool(&ctx->tm_k, b->k_pool, rows, cfg->head_dim) ||
      !encode_pool(&ctx->tm_v, b->v_pool, rows, cfg->head_dim)) {
    delete ctx;
    return HSA_ERR_CUDA;
  }
  *out = ctx;
  return HSA_OK;
}

int hsa_kv8_append(hsa_kv8* ctx, const void* k, const void* v, int32_t n_tokens, int32_t batch, int64_t tok_stride,
                   int64_t head_stride, const int32_t* token_start_dev, int32_t max_new, const int32_t* held_dev,
                   const hsa_rope_args* rope, void* stream) {
  if (!ctx || !on_device(ctx)) return HSA_ERR_INVALID_ARG;
  if (n_tokens == 0) return HSA_OK;
  const hsa_kv8_config& c = ctx->cfg;
  Kv8AppendArgs a{};
  if (!rows_ok(ctx, n_tokens, batch, token_start_dev, max_new, &a.rows)) return HSA_ERR_INVALID_ARG;
  if (!tensor_ok(k, tok_stride, head_stride, c.head_dim) || !tensor_ok(v, tok_stride, head_stride, c.head_dim))
    return HSA_ERR_INVALID_ARG;
  if (!held_dev || !aligned(held_dev, 4)) return HSA_ERR_INVALID_ARG;
  if (rope && !rope_args(rope, c.head_dim, n_tokens, false, &a.rope)) return HSA_ERR_INVALID_ARG;
  a.has_rope = rope != nullptr;
  a.k = static_cast<const __nv_bfloat16*>(k);
  a.v = static_cast<const __nv_bfloat16*>(v);
  a.ts = tok_stride;
  a.hs = head_stride;
  a.held = held_dev;
  a.H = c.num_kv_heads;
  a.max_pages = c.max_pages;
  a.max_blocks = c.max_blocks;
  a.table = ctx->buf.page_table;
  a.k_pool = static_cast<uint8_t*>(ctx->buf.k_pool);
  a.v_pool = static_cast<uint8_t*>(ctx->buf.v_pool);
  a.k_scale = ctx->buf.k_scale;
  a.v_scale = ctx->buf.v_scale;
  a.ksum = ctx->buf.ksum;
  a.status = static_cast<int32_t*>(ctx->buf.workspace);
  const cudaError_t e = launch_kv8_append(a, c.head_dim, ctx->nsm, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? HSA_OK : cuda_fail(ctx, e);
}

int hsa_kv8_attend(hsa_kv8* ctx, const void* q, int32_t n_tokens, int32_t batch, int64_t tok_stride,
                   int64_t head_stride, const int32_t* token_start_dev, int32_t max_q, const int32_t* lengths_dev,
                   int32_t causal, const int32_t* sel_idx_dev, const int32_t* sel_cnt_dev, int32_t max_topk, void* out,
                   int64_t out_tok_stride, int64_t out_head_stride, float* lse_dev, void* stream) {
  if (!ctx || !on_device(ctx)) return HSA_ERR_INVALID_ARG;
  if (n_tokens == 0) return HSA_OK;
  const hsa_kv8_config& c = ctx->cfg;
  Kv8AttendArgs a{};
  if (!rows_ok(ctx, n_tokens, batch, token_start_dev, max_q, &a.rows)) return HSA_ERR_INVALID_ARG;
  if (!tensor_ok(q, tok_stride, head_stride, c.head_dim) || !tensor_ok(out, out_tok_stride, out_head_stride, c.head_dim))
    return HSA_ERR_INVALID_ARG;
  if (!lengths_dev || !aligned(lengths_dev, 4) || !aligned(lse_dev, 4)) return HSA_ERR_INVALID_ARG;
  if (!sel_idx_dev != !sel_cnt_dev) return HSA_ERR_INVALID_ARG;
  if (sel_idx_dev && (max_topk < 1 || !aligned(sel_idx_dev, 4) || !aligned(sel_cnt_dev, 4))) return HSA_ERR_INVALID_ARG;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.out = static_cast<__nv_bfloat16*>(out);
  a.lse = lse_dev;
  a.ts = tok_stride;
  a.hs = head_stride;
  a.ots = out_tok_stride;
  a.ohs = out_head_stride;
  a.lengths = lengths_dev;
  a.Hq = c.num_heads;
  a.Hkv = c.num_kv_heads;
  a.group = c.num_heads / c.num_kv_heads;
  a.max_pages = c.max_pages;
  a.max_blocks = c.max_blocks;
  a.causal = causal != 0;
  a.sel_idx = sel_idx_dev;
  a.sel_cnt = sel_cnt_dev;
  a.max_topk = max_topk;
  a.scale_log2 = ctx->scale * 1.4426950408889634f;
  a.table = ctx->buf.page_table;
  a.k_pool = static_cast<const uint8_t*>(ctx->buf.k_pool);
  a.v_pool = static_cast<const uint8_t*>(ctx->buf.v_pool);
  a.k_scale = ctx->buf.k_scale;
  a.v_scale = ctx->buf.v_scale;
  a.status = static_cast<int32_t*>(ctx->buf.workspace);
  uint8_t* ws = static_cast<uint8_t*>(ctx->buf.workspace);
  Kv8Work w{};
  w.tickets = reinterpret_cast<int32_t*>(ws + kStatusBytes);
  w.parts = reinterpret_cast<float*>(ws + kStatusBytes + kTicketBytes);
  w.look = ctx->wait_ns < kPollNs ? static_cast<uint32_t>(2 * ctx->wait_ns) : 0;  // (at 2 GHz)
  w.first_try = w.look ? 0 : kMaxPolls - static_cast<uint32_t>(ctx->wait_ns / kPollNs);
  const int ctas = ctx->nsm < kMaxCtas ? ctx->nsm : kMaxCtas;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = static_cast<int64_t>(max_q) * a.group <= kv8_decode_rows(c.head_dim)
                            ? launch_kv8_decode(a, w, c.head_dim, ctas, ctx->tm_k, ctx->tm_v, st)
                            : launch_kv8_chunk(a, w, c.head_dim, ctas, ctx->tm_k, ctx->tm_v, st);
  return e == cudaSuccess ? HSA_OK : cuda_fail(ctx, e);
}

int hsa_kv8_device_status(hsa_kv8* ctx, int32_t* status_out) {
  if (!ctx || !status_out || !on_device(ctx)) return HSA_ERR_INVALID_ARG;
  int32_t v = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(&v, ctx->buf.workspace, 4, cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && v != 0) e = cudaMemset(ctx->buf.workspace, 0, kStatusBytes + kTicketBytes);
  if (e == cudaSuccess && v != 0) e = cudaDeviceSynchronize();  // (the fill is not ordered with what other streams are given next)
  if (e != cudaSuccess) return cuda_fail(ctx, e);
  *status_out = v;
  return HSA_OK;
}

int hsa_kv8_set_wait_limit_ns(hsa_kv8* ctx, uint64_t wait_ns) {
  if (!ctx || wait_ns == 0 || wait_ns > 2'500'000'000) return HSA_ERR_INVALID_ARG;
  ctx->wait_ns = wait_ns;
  return HSA_OK;
}

int hsa_kv8_last_cuda_error(hsa_kv8* ctx) { return ctx ? ctx->last_cuda_error : 0; }

int hsa_kv8_destroy(hsa_kv8* ctx) {
  if (!ctx) return HSA_ERR_INVALID_ARG;
  delete ctx;
  return HSA_OK;
}

}  // extern "C"
