// C-ABI entry points of the cache in pages and of the log probabilities (include/redrafter.h).  Checks of arguments and launches.
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include <cmath>
#include <new>

#include "logprobs.cuh"
#include "pages.cuh"
#include "rd_internal.cuh"

using namespace rd;

namespace {
struct alignas(64) MapBox {   // opaque storage of one CUtensorMap
  unsigned char bytes[128];
};
constexpr int MAX_ROWS = 1 << 30;     // rows of a call, and what a window is cut to (a sequence has fewer tokens): positions less a window fit 32 bits
constexpr int MAX_GROUP = 1024;        // query heads of a key and value head
constexpr int TOKEN_MAX_GRID = 160;   // upper bound of the SM count that the parts are sized for
}  // namespace

struct rd_pages {
  MapBox map_parts;   // the pool's rows, min(page_size, 64) to a box (bf16)
  MapBox map_rows;    // the same in boxes of 64 columns
  PageView pv;
  int dtype, device;
  int32_t* scratch;
  char* parts;      // joins of the attention kernel for single tokens
  char* row_parts;  // ... of the one for many rows
  int grid;         // SMs
  int64_t launches;
  char err[256];
};

namespace {

thread_local char g_pages_err[256] = "";      // why the last redrafter_pages_init failed
thread_local char g_logprob_err[256] = "";    // why the last redrafter_token_logprobs failed

int fail_to(char (&err)[256], int code, const char* fmt, va_list ap) {
  vsnprintf(err, sizeof(err), fmt, ap);
  return code;
}
int fail(rd_pages* h, int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  fail_to(h->err, code, fmt, ap);
  va_end(ap);
  return code;
}
int init_fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  fail_to(g_pages_err, code, fmt, ap);
  va_end(ap);
  return code;
}
int logprob_fail(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  fail_to(g_logprob_err, code, fmt, ap);
  va_end(ap);
  return code;
}

bool view_of(const rd_page_cache* c, PageView* pv) {
  if (!c || c->struct_bytes != (int32_t)sizeof(rd_page_cache)) return false;
  if (c->dtype != RD_DTYPE_FP32 && c->dtype != RD_DTYPE_BF16) return false;
  if (c->n_layers <= 0 || c->n_kv_heads <= 0 || c->n_pages <= 0 || c->max_seqs <= 0 || c->max_seq_pages <= 0) return false;
  pv->pool = c->pool; pv->table = c->page_table; pv->lens = c->lens; pv->refs = c->refs; pv->free_bits = c->free_bits; pv->status = nullptr;
  pv->n_layers = c->n_layers; pv->H = c->n_kv_heads; pv->hd = c->head_dim; pv->es = c->dtype == RD_DTYPE_FP32 ? 4 : 2;
  pv->ps = c->page_size; pv->n_pages = c->n_pages; pv->max_seqs = c->max_seqs; pv->max_pages = c->max_seq_pages;
  pv->ps_log2 = 0;
  while ((1 << pv->ps_log2) < pv->ps && pv->ps_log2 < 8) ++pv->ps_log2;
  return true;
}

// head_dim 64 or 128, pages of 16 to 128 tokens; the pool's rows, the table's entries and a sequence's tokens times its heads
// (two at least, so that a position plus a tile fits, too) countable in 31 bits: what the kernels count in 32 bits then fits.
bool view_shape_ok(const PageView& pv) {
  if (pv.hd != 64 && pv.hd != 128) return false;
  if (pv.ps < 16 || pv.ps > 128 || (1 << pv.ps_log2) != pv.ps) return false;
  if ((double)pv.n_layers * 2 * pv.n_pages * pv.H * pv.ps >= 2147483648.0) return false;   // rows of the pool
  if ((double)pv.n_layers * 2 * pv.H * pv.hd >= 2147483648.0) return false;
  if ((double)pv.max_seqs * pv.max_pages >= 2147483648.0) return false;
  if ((double)pv.max_pages * pv.ps * (pv.H > 2 ? pv.H : 2) >= 2147483648.0) return false;
  return true;
}

size_t scratch_bytes(const PageView& pv) { return (pages_scratch_ints(pv) * 4 + 255) / 256 * 256; }
size_t page_workspace(const PageView& pv) { return 256 + scratch_bytes(pv) + pages_token_part_bytes(pv, TOKEN_MAX_GRID) + pages_rows_part_bytes(pv, TOKEN_MAX_GRID); }

// What every call on a handle checks first.
int enter(rd_pages* h, int n) {
  if (!h) return RD_ERR_INVALID_ARG;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev != h->device)
    return fail(h, RD_ERR_STATE, "current device %d is not the device %d this handle was made on", dev, h->device);
  if (n < 0) return fail(h, RD_ERR_INVALID_ARG, "n = %d", n);
  return RD_OK;
}
// ... and those that take a list of sequences of the table.
int enter_list(rd_pages* h, int n) {
  if (int rc = enter(h, n)) return rc;
  if (n > h->pv.max_seqs) return fail(h, RD_ERR_INVALID_ARG, "%d sequences, the table has %d", n, h->pv.max_seqs);
  return RD_OK;
}

int rows_ok(rd_pages* h, int layer, const int32_t* row_off, int n, int n_rows) {
  if (layer < 0 || layer >= h->pv.n_layers) return fail(h, RD_ERR_INVALID_ARG, "layer %d of %d", layer, h->pv.n_layers);
  if (n_rows < 0 || n_rows > MAX_ROWS) return fail(h, RD_ERR_INVALID_ARG, "%d rows", n_rows);
  if (!row_off && n_rows != n) return fail(h, RD_ERR_INVALID_ARG, "%d rows for %d sequences of one row each", n_rows, n);
  return RD_OK;
}

bool aligned16(const void* p, long long stride, int es) { return ((uintptr_t)p & 15) == 0 && (stride * es) % 16 == 0; }

#define PCK(expr)                                                                                            \
  do {                                                                                                       \
    cudaError_t e__ = (expr);                                                                                \
    if (e__ != cudaSuccess) return fail(h, RD_ERR_CUDA, "%s: %s", #expr, cudaGetErrorString(e__));           \
  } while (0)

}  // namespace

namespace rd {

const PageView& pages_view(const rd_pages* h) { return h->pv; }
int pages_device(const rd_pages* h) { return h->device; }

cudaError_t pages_extend_for(rd_pages* h, const int32_t* seqs, const int32_t* n_new, int n, int* launches, cudaStream_t st) {
  int mine = 0;
  const cudaError_t e = launch_pages_extend(h->pv, seqs, n_new, n, h->scratch, &mine, st);
  h->launches += mine;
  *launches += mine;
  return e;
}

// The kernel for the rows at hand: single tokens; many rows on the tensor cores; many rows of the fp32 configuration.
cudaError_t pages_attention_for(rd_pages* h, const PageRows& rows, PageAttention a, int* launches, cudaStream_t st) {
  int mine = 0;
  a.window = a.window < MAX_ROWS ? a.window : MAX_ROWS;
  cudaError_t e;
  if (rows.max_rows > 1 && h->pv.es == 2) {
    e = launch_pages_rows(h->map_rows.bytes, h->pv, rows, a, h->row_parts, h->grid, &mine, st);
  } else {
    e = rows.max_rows == 1 ? launch_pages_token(h->map_parts.bytes, h->pv, rows, a, h->parts, h->grid, st) : launch_pages_attention_fp32(h->pv, rows, a, st);
    mine = 1;
  }
  h->launches += mine;
  if (launches) *launches += mine;
  return e;
}

}  // namespace rd

extern "C" {

size_t redrafter_pages_workspace_bytes(const rd_page_cache* cache) {
  PageView pv;
  if (!view_of(cache, &pv) || !view_shape_ok(pv)) return 0;
  return page_workspace(pv);
}

size_t redrafter_pages_pool_bytes(const rd_page_cache* cache) {
  PageView pv;
  if (!view_of(cache, &pv) || !view_shape_ok(pv)) return 0;
  return (size_t)pv.n_layers * 2 * pv.n_pages * pv.H * pv.ps * pv.hd * pv.es;
}

int redrafter_pages_init(const rd_page_cache* cache, void* workspace, size_t ws_bytes, rd_pages** out) {
  if (!cache || !workspace || !out) return init_fail(RD_ERR_INVALID_ARG, "null argument");
  *out = nullptr;
  PageView pv;
  if (!view_of(cache, &pv)) return init_fail(RD_ERR_INVALID_ARG, "struct_bytes, dtype or a size is out of range");
  if (!pv.pool || !pv.table || !pv.lens || !pv.refs || !pv.free_bits) return init_fail(RD_ERR_INVALID_ARG, "null buffer");
  if (!view_shape_ok(pv)) return init_fail(RD_ERR_SHAPE, "head_dim %d (64 or 128), page_size %d (16, 32, 64 or 128), or 2^31 rows of the pool, entries of the table or tokens times heads of a sequence", pv.hd, pv.ps);
  if (((uintptr_t)pv.pool | (uintptr_t)workspace) & 255) return init_fail(RD_ERR_INVALID_ARG, "pool and workspace have to be 256-byte aligned");
  if (ws_bytes < page_workspace(pv)) return init_fail(RD_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", ws_bytes, page_workspace(pv));
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return init_fail(RD_ERR_CUDA, "no current device");
  rd_pages* h = new (std::nothrow) rd_pages();
  if (!h) return init_fail(RD_ERR_INVALID_ARG, "out of host memory");
  h->pv = pv; h->dtype = cache->dtype; h->device = dev; h->launches = 0; h->err[0] = 0;
  h->pv.status = (int32_t*)workspace;
  h->scratch = (int32_t*)((char*)workspace + 256);
  h->parts = (char*)h->scratch + scratch_bytes(pv);
  h->row_parts = h->parts + pages_token_part_bytes(pv, TOKEN_MAX_GRID);
  cudaError_t e = cudaDeviceGetAttribute(&h->grid, cudaDevAttrMultiProcessorCount, dev);
  if (h->grid > TOKEN_MAX_GRID) h->grid = TOKEN_MAX_GRID;
  if (e == cudaSuccess && pv.es == 2) {
    const uint64_t pool_rows = (uint64_t)pv.n_layers * 2 * pv.n_pages * pv.H * pv.ps;
    const uint32_t box = pv.ps < 64 ? pv.ps : 64;
    int rc = tc_make_map_parts(h->map_parts.bytes, pv.pool, pool_rows, pv.hd, box);
    if (!rc) rc = tc_make_map(h->map_rows.bytes, pv.pool, pool_rows, pv.hd, box);
    if (rc) {
      delete h;
      return init_fail(RD_ERR_CUDA, "cuTensorMapEncodeTiled failed with %d for the pool", rc);
    }
    e = pages_rows_prepare(pv.hd);
  }
  if (e == cudaSuccess && pv.es == 4) e = pages_attention_fp32_prepare(pv.hd);
  if (e == cudaSuccess) e = pages_token_prepare(pv);
  if (e == cudaSuccess) e = cudaMemsetAsync(h->parts, 0, pages_token_part_bytes(pv, TOKEN_MAX_GRID), 0);
  if (e == cudaSuccess) e = cudaMemsetAsync(workspace, 0, 256, 0);
  if (e == cudaSuccess) e = launch_pages_scratch(h->pv, h->scratch, 0);
  if (e == cudaSuccess) e = cudaStreamSynchronize(0);
  if (e != cudaSuccess) {
    delete h;
    return init_fail(RD_ERR_CUDA, "clearing the workspace: %s", cudaGetErrorString(e));
  }
  h->launches = 1;
  *out = h;
  return RD_OK;
}

int redrafter_pages_destroy(rd_pages* h) {
  if (!h) return RD_ERR_INVALID_ARG;
  delete h;
  return RD_OK;
}

const char* redrafter_pages_last_error(const rd_pages* h) { return h ? h->err : g_pages_err; }

int64_t redrafter_pages_launch_count(const rd_pages* h) { return h ? h->launches : 0; }

int redrafter_pages_reset(rd_pages* h, void* stream) {
  if (int rc = enter(h, 0)) return rc;
  PCK(launch_pages_reset(h->pv, h->scratch, (cudaStream_t)stream));
  h->launches++;
  return RD_OK;
}

int redrafter_pages_extend(rd_pages* h, const int32_t* seqs, const int32_t* n_new, int32_t n, void* stream) {
  if (int rc = enter_list(h, n)) return rc;
  if (n == 0) return RD_OK;   // (an empty list may be null)
  if (!n_new) return fail(h, RD_ERR_INVALID_ARG, "n_new is null");
  int launches = 0;
  PCK(launch_pages_extend(h->pv, seqs, n_new, n, h->scratch, &launches, (cudaStream_t)stream));
  h->launches += launches;
  return RD_OK;
}

int redrafter_pages_fork(rd_pages* h, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  if (int rc = enter_list(h, n)) return rc;
  if (n == 0) return RD_OK;
  if (!src || !dst) return fail(h, RD_ERR_INVALID_ARG, "null list");
  PCK(launch_pages_fork(h->pv, src, dst, n, (cudaStream_t)stream));
  h->launches++;
  return RD_OK;
}

int redrafter_pages_compact(rd_pages* h, const int32_t* seqs, const int32_t* n_rows, const int32_t* n_keep, const int32_t* rows,
                            int32_t row_stride, int32_t n, void* stream) {
  if (int rc = enter_list(h, n)) return rc;
  if (n == 0) return RD_OK;
  if (!n_rows || !n_keep) return fail(h, RD_ERR_INVALID_ARG, "null list");
  if (rows && row_stride <= 0) return fail(h, RD_ERR_INVALID_ARG, "row_stride %d", row_stride);
  int launches = 0;
  PCK(launch_pages_compact(h->pv, seqs, n_rows, n_keep, rows, row_stride, n, h->scratch, &launches, (cudaStream_t)stream));
  h->launches += launches;
  return RD_OK;
}

int redrafter_pages_trim(rd_pages* h, const int32_t* seqs, int32_t window, int32_t sinks, int32_t n, void* stream) {
  if (int rc = enter_list(h, n)) return rc;
  if (window < 1 || sinks < 0) return fail(h, RD_ERR_INVALID_ARG, "window %d, sinks %d", window, sinks);
  if (n == 0) return RD_OK;
  PCK(launch_pages_trim(h->pv, seqs, window, sinks, n, (cudaStream_t)stream));
  h->launches++;
  return RD_OK;
}

int redrafter_pages_free(rd_pages* h, const int32_t* seqs, int32_t n, void* stream) {
  if (int rc = enter_list(h, n)) return rc;
  if (n == 0) return RD_OK;
  PCK(launch_pages_free(h->pv, seqs, n, (cudaStream_t)stream));
  h->launches++;
  return RD_OK;
}

int redrafter_pages_write(rd_pages* h, int32_t layer, const int32_t* seqs, const int32_t* row_off, int32_t n, int32_t n_rows, const void* k,
                          int64_t k_stride, const void* v, int64_t v_stride, void* stream) {
  if (int rc = enter_list(h, n)) return rc;
  if (int rc = rows_ok(h, layer, row_off, n, n_rows)) return rc;
  if (n == 0 || n_rows == 0) return RD_OK;
  if (!k || !v) return fail(h, RD_ERR_INVALID_ARG, "k or v is null");
  const long long row = (long long)h->pv.H * h->pv.hd;
  if (k_stride < row || v_stride < row) return fail(h, RD_ERR_SHAPE, "row strides %lld and %lld, a row has %lld elements", (long long)k_stride, (long long)v_stride, row);
  if (!aligned16(k, k_stride, h->pv.es) || !aligned16(v, v_stride, h->pv.es)) return fail(h, RD_ERR_SHAPE, "rows of k and v have to begin on 16-byte boundaries");
  const PageRows rows{seqs, row_off, n, n_rows, n_rows};
  PCK(launch_pages_write(h->pv, layer, rows, k, k_stride, v, v_stride, (cudaStream_t)stream));
  h->launches++;
  return RD_OK;
}

int redrafter_pages_attention(rd_pages* h, int32_t layer, const int32_t* seqs, const int32_t* row_off, int32_t n, int32_t n_rows, int32_t max_rows,
                              int32_t n_heads, const void* q, int64_t q_stride, void* out, int64_t out_stride, float* lse, float scale,
                              int32_t window, int32_t sinks, void* stream) {
  if (int rc = enter(h, n)) return rc;
  if (int rc = rows_ok(h, layer, row_off, n, n_rows)) return rc;
  if (n_heads <= 0 || n_heads % h->pv.H || n_heads / h->pv.H > MAX_GROUP) return fail(h, RD_ERR_SHAPE, "%d query heads on %d key and value heads", n_heads, h->pv.H);
  if (window < 0 || sinks < 0) return fail(h, RD_ERR_INVALID_ARG, "window %d, sinks %d", window, sinks);
  if (!std::isfinite(scale) || scale < 0.f) return fail(h, RD_ERR_INVALID_ARG, "scale %g", (double)scale);
  if (max_rows < 0) return fail(h, RD_ERR_INVALID_ARG, "max_rows %d", max_rows);
  if (((long long)n + n_rows) * n_heads >= (1ll << 31)) return fail(h, RD_ERR_SHAPE, "%d sequences and %d rows of %d heads", n, n_rows, n_heads);   // (the fp32 kernel's grid)
  if (n == 0 || n_rows == 0) return RD_OK;
  if (!q || !out) return fail(h, RD_ERR_INVALID_ARG, "q or out is null");
  const long long row = (long long)n_heads * h->pv.hd;
  if (q_stride < row || out_stride < row) return fail(h, RD_ERR_SHAPE, "row strides %lld and %lld, a row has %lld elements", (long long)q_stride, (long long)out_stride, row);
  if (!aligned16(q, q_stride, h->pv.es) || !aligned16(out, out_stride, h->pv.es)) return fail(h, RD_ERR_SHAPE, "rows of q and out have to begin on 16-byte boundaries");
  const PageRows rows{seqs, row_off, n, n_rows, !row_off ? 1 : max_rows > 0 ? max_rows : n_rows};
  PageAttention a;
  a.q = q; a.out = out; a.lse = lse; a.q_stride = q_stride; a.out_stride = out_stride; a.heads = n_heads; a.layer = layer;
  a.window = window; a.sinks = window ? sinks : 0;
  a.scale = scale > 0.f ? scale : 1.f / sqrtf((float)h->pv.hd);
  PCK(pages_attention_for(h, rows, a, nullptr, (cudaStream_t)stream));
  return RD_OK;
}

int redrafter_pages_poll(rd_pages* h, void* stream) {
  if (int rc = enter(h, 0)) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  int32_t v = 0;
  PCK(cudaMemcpyAsync(&v, h->pv.status, sizeof(v), cudaMemcpyDeviceToHost, st));
  PCK(cudaStreamSynchronize(st));
  if (v == 0) return RD_OK;
  PCK(cudaMemsetAsync(h->pv.status, 0, sizeof(int32_t), st));
  if (v & DEV_ERR_TIMEOUT) return fail(h, RD_ERR_TIMEOUT, "device status 0x%x: a bounded wait gave up", v);
  if (v & DEV_ERR_CAPACITY) return fail(h, RD_ERR_CAPACITY, "device status 0x%x: too few free pages, a call that extends changed nothing", v);
  return fail(h, RD_ERR_INVALID_ARG, "device status 0x%x: a sequence, length, row or page out of range was skipped", v);
}

int redrafter_token_logprobs(const rd_logprobs* args, void* stream) {
  if (!args || args->struct_bytes != (int32_t)sizeof(rd_logprobs)) return logprob_fail(RD_ERR_INVALID_ARG, "null argument or struct_bytes");
  const rd_logprobs& p = *args;
  if (p.dtype != RD_DTYPE_FP32 && p.dtype != RD_DTYPE_BF16) return logprob_fail(RD_ERR_INVALID_ARG, "dtype %d", p.dtype);
  if (p.rows < 0 || p.n_logit_rows < 0 || p.vocab <= 0 || p.vocab > (1 << 30)) return logprob_fail(RD_ERR_INVALID_ARG, "%d rows of %d, vocabulary %d", p.rows, p.n_logit_rows, p.vocab);
  if (p.top < 0 || p.top > LOGPROB_MAX_TOP || p.top > p.vocab) return logprob_fail(RD_ERR_SHAPE, "top %d of %d (at most %d)", p.top, p.vocab, LOGPROB_MAX_TOP);
  if (!(p.temperature > 0.f) || !std::isfinite(p.temperature) || !std::isfinite(1.5f / p.temperature)) return logprob_fail(RD_ERR_INVALID_ARG, "temperature %g", (double)p.temperature);
  if (p.rows == 0) return RD_OK;
  if (!p.logits || (p.logprob && !p.tokens) || (p.top && (!p.top_ids || !p.top_logprobs))) return logprob_fail(RD_ERR_INVALID_ARG, "null buffer");
  if (!p.row_index && p.rows > p.n_logit_rows) return logprob_fail(RD_ERR_INVALID_ARG, "%d rows of %d", p.rows, p.n_logit_rows);
  if (p.row_stride < p.vocab) return logprob_fail(RD_ERR_SHAPE, "row stride %lld below the vocabulary %d", (long long)p.row_stride, p.vocab);
  const size_t es = p.dtype == RD_DTYPE_FP32 ? 4 : 2;
  if ((uintptr_t)p.logits % es) return logprob_fail(RD_ERR_INVALID_ARG, "logits are not aligned to their type");
  LogprobArgs a;
  a.logits = p.logits; a.row_stride = p.row_stride; a.row_index = p.row_index; a.tokens = p.tokens; a.rows = p.rows; a.vocab = p.vocab;
  a.n_logit_rows = p.n_logit_rows; a.top = p.top; a.inv_t = 1.f / p.temperature;
  a.logprob = p.logprob; a.entropy = p.entropy; a.top_ids = p.top_ids; a.top_logprobs = p.top_logprobs;
  const cudaError_t e = launch_logprobs(p.dtype, a, (cudaStream_t)stream);
  if (e != cudaSuccess) return logprob_fail(RD_ERR_CUDA, "log probabilities: %s", cudaGetErrorString(e));
  return RD_OK;
}

const char* redrafter_token_logprobs_error(void) { return g_logprob_err; }

}  // extern "C"
