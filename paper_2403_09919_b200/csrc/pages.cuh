// Internal declarations of the cache in pages (include/redrafter.h, "A key-value cache in pages").
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "redrafter.h"

namespace rd {

// What the kernels need of a cache: sizes and the caller's buffers.
struct PageView {
  void* pool;           // [n_layers][2][n_pages][H][ps][hd]
  int32_t* table;       // [max_seqs][max_pages]
  int32_t* lens;        // [max_seqs]
  int32_t* refs;        // [n_pages]
  uint32_t* free_bits;  // [ceil(n_pages / 32)]
  int32_t* status;      // device status word (DEV_ERR_*)
  int n_layers, H, hd, es;   // es: bytes of an element
  int ps, ps_log2, n_pages, max_seqs, max_pages;
};

// The rows of one call: row r of sequence i of the list lies at position lens - m + (r - row_off[i]), m its number of rows.
struct PageRows {
  const int32_t* seqs;      // [n] rows of the page table, or nullptr: 0 .. n-1
  const int32_t* row_off;   // [n + 1] first row of each, or nullptr: one row per sequence
  int n, n_rows;
  int max_rows;             // the most rows an entry may bring
};

#ifdef __CUDACC__
// First row and number of rows of entry i, kept inside [0, n_rows) whatever row_off holds.
__device__ __forceinline__ void page_rows_of(const PageRows& r, int i, int* first, int* m) {
  if (!r.row_off) { *first = i; *m = 1; return; }
  const int a = min(max(r.row_off[i], 0), r.n_rows), b = min(max(r.row_off[i + 1], 0), r.n_rows);
  *first = a; *m = max(0, b - a);
}
// Sequence of entry i, or -1.
__device__ __forceinline__ int page_seq_of(const PageView& pv, const int32_t* seqs, int i) {
  const int s = seqs ? seqs[i] : i;
  return (unsigned)s < (unsigned)pv.max_seqs ? s : -1;
}
// Length of sequence s, kept inside what its row of the table can hold.
__device__ __forceinline__ int page_len_of(const PageView& pv, int s) {
  const long long most = min((long long)pv.max_pages * pv.ps, 0x7fffffffll);
  return (int)min(max((long long)pv.lens[s], 0ll), most);
}
#endif

// ---- pages.cu
size_t pages_scratch_ints(const PageView& pv);
cudaError_t launch_pages_scratch(const PageView& pv, int32_t* scratch, cudaStream_t st);
cudaError_t launch_pages_reset(const PageView& pv, int32_t* scratch, cudaStream_t st);
cudaError_t launch_pages_extend(const PageView& pv, const int32_t* seqs, const int32_t* n_new, int n, int32_t* scratch, int* launches, cudaStream_t st);
cudaError_t launch_pages_fork(const PageView& pv, const int32_t* src, const int32_t* dst, int n, cudaStream_t st);
cudaError_t launch_pages_compact(const PageView& pv, const int32_t* seqs, const int32_t* n_rows, const int32_t* n_keep, const int32_t* rows,
                                 int row_stride, int n, int32_t* scratch, int* launches, cudaStream_t st);
cudaError_t launch_pages_trim(const PageView& pv, const int32_t* seqs, int window, int sinks, int n, cudaStream_t st);
cudaError_t launch_pages_free(const PageView& pv, const int32_t* seqs, int n, cudaStream_t st);
cudaError_t launch_pages_write(const PageView& pv, int layer, const PageRows& rows, const void* k, long long k_stride, const void* v,
                               long long v_stride, cudaStream_t st);

// ---- attention over pages
struct PageAttention {
  const void* q;         // [n_rows][heads][hd], rows q_stride elements apart
  void* out;             // likewise
  float* lse;            // [n_rows][heads] or nullptr
  long long q_stride, out_stride;
  int heads, layer, window, sinks;   // window 0: every earlier key
  float scale;
};
// one token per sequence
size_t pages_token_part_bytes(const PageView& pv, int grid);
cudaError_t pages_token_prepare(const PageView& pv);
cudaError_t launch_pages_token(const void* map, const PageView& pv, const PageRows& rows, const PageAttention& a, void* parts, int grid, cudaStream_t st);
// many rows per sequence, bf16
cudaError_t pages_rows_prepare(int hd);
size_t pages_rows_part_bytes(const PageView& pv, int grid);
cudaError_t launch_pages_rows(const void* map, const PageView& pv, const PageRows& rows, const PageAttention& a, void* parts, int sms, int* launches,
                              cudaStream_t st);
// many rows per sequence, fp32
cudaError_t pages_attention_fp32_prepare(int hd);
cudaError_t launch_pages_attention_fp32(const PageView& pv, const PageRows& rows, const PageAttention& a, cudaStream_t st);

// ---- pages_api.cu: a handle for the engine's own passes (rd_handle), which prompts and autoregressive steps may run on
const PageView& pages_view(const rd_pages* h);
int pages_device(const rd_pages* h);
cudaError_t pages_extend_for(rd_pages* h, const int32_t* seqs, const int32_t* n_new, int n, int* launches, cudaStream_t st);
cudaError_t pages_attention_for(rd_pages* h, const PageRows& rows, PageAttention a, int* launches, cudaStream_t st);

}  // namespace rd
