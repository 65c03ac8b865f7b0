// Attention of many rows per sequence over a cache in pages for the fp32 configuration: a warp per row and head, keys one after
// another in 32 bits (tensor cores have no fp32 products; TF32 would round K to 11 bits).  The latency of a warp's chain of keys
// bounds it; the configuration is for checks of small models.
#include "pages_attention.cuh"
#include "pdl.cuh"

namespace rd {

namespace {

constexpr int PLAIN_WARPS = 4;

template <int HD>
__global__ void __launch_bounds__(PLAIN_WARPS * 32) pages_attention_fp32_kernel(PageView pv, PageRows rows, PageAttention a) {
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
    load_dims(reinterpret_cast<const float*>(a.q) + (long long)row * a.q_stride + (long long)head * HD + lane * N, q);
    attend_row_warp<float, HD>(pv, a.layer, pv.table + (size_t)s * pv.max_pages, head / (a.heads / pv.H), pos, a.window, a.sinks, a.scale * LOG2E, q, o,
                           &m, &l);
  }
  store_row_warp<float, HD>(a, row, head, o, m, l);
}

}  // namespace

cudaError_t launch_pages_attention_fp32(const PageView& pv, const PageRows& rows, const PageAttention& a, cudaStream_t st) {
  const dim3 grid(rows.n_rows, (a.heads + PLAIN_WARPS - 1) / PLAIN_WARPS);
  if (pv.hd == 64) launch_pdl(pages_attention_fp32_kernel<64>, grid, PLAIN_WARPS * 32, 0, st, pv, rows, a);
  else launch_pdl(pages_attention_fp32_kernel<128>, grid, PLAIN_WARPS * 32, 0, st, pv, rows, a);
  return cudaGetLastError();
}

}  // namespace rd
