// Attention over a cache in pages, the plain kernel: a warp per row and head, any type and head dimension of the library.
// Latency of a warp's chain of keys bounds it; it serves the small fp32 model and head dimension 64, and works out single
// rows for the tensor-core kernel where that one cannot.
#include "pages_attention.cuh"
#include "pdl.cuh"

namespace rd {

namespace {

constexpr int PLAIN_WARPS = 4;

template <typename T, int HD>
__global__ void __launch_bounds__(PLAIN_WARPS * 32) pages_attention_plain_kernel(PageView pv, PageRows rows, PageAttention a) {
  pdl_enter();
  const int row = blockIdx.x, head = blockIdx.y * PLAIN_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  int i, first, m_rows;
  if (!entry_of_row(rows, row, &i, &first, &m_rows) || head >= a.heads) return;
  constexpr int N = HD / 32;
  float q[N], o[N], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int d = 0; d < N; ++d) o[d] = 0.f;
  const int s = page_seq_of(pv, rows.seqs, i);
  if (m_rows > rows.max_rows) {
    if (lane == 0) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
    return;
  }
  const int pos = s < 0 ? -1 : page_len_of(pv, s) - m_rows + (row - first);
  if (s < 0 && lane == 0) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
  if (pos >= 0) {
    load_dims(reinterpret_cast<const T*>(a.q) + (long long)row * a.q_stride + (long long)head * HD + lane * N, q);
    attend_row_warp<T, HD>(pv, a.layer, pv.table + (size_t)s * pv.max_pages, head / (a.heads / pv.H), pos, a.window, a.sinks, a.scale * LOG2E, q, o,
                           &m, &l);
  }
  store_row_warp<T, HD>(a, row, head, o, m, l);
}

}  // namespace

cudaError_t launch_pages_attention_plain(const PageView& pv, int dtype, const PageRows& rows, const PageAttention& a, cudaStream_t st) {
  const dim3 grid(rows.n_rows, (a.heads + PLAIN_WARPS - 1) / PLAIN_WARPS);
  auto go = [&](auto kernel) { launch_pdl(kernel, grid, PLAIN_WARPS * 32, 0, st, pv, rows, a); };
  if (dtype == RD_DTYPE_FP32) pv.hd == 64 ? go(pages_attention_plain_kernel<float, 64>) : go(pages_attention_plain_kernel<float, 128>);
  else pv.hd == 64 ? go(pages_attention_plain_kernel<__nv_bfloat16, 64>) : go(pages_attention_plain_kernel<__nv_bfloat16, 128>);
  return cudaGetLastError();
}

}  // namespace rd
