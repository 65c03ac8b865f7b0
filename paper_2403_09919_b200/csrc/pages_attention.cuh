// What the attention kernels over pages share: which keys a row sees, and one row worked through by one warp.
#pragma once
#include "pages.cuh"
#include "rd_internal.cuh"

namespace rd {

#ifdef __CUDACC__
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// A row at position pos sees the keys [0, sink_end) and [start, pos].
__device__ __forceinline__ void visible_keys(int pos, int window, int sinks, int* sink_end, int* start) {
  *start = window > 0 ? max(0, pos - window + 1) : 0;   // (pos < 2^31, window > 0: no overflow)
  *sink_end = min(sinks, *start);
}

// Consecutive rows of an entry; n_rows: rows times pack (query heads that share a tile); pos0: position of the first row.
struct RowsTile {
  int row0, n_rows, pos0, seq;
};

// A lane's entry of a group of 32: its first row, rows, tiles of ROWS, sequence and length.
template <int ROWS> struct RowsEntries {
  int first = 0, m = 0, tiles = 0, seq = -1, len = 0, group = -1;

  __device__ __forceinline__ void look_up(const PageView& pv, const PageRows& rows, int pack, int i0) {
    if (i0 == group) return;
    group = i0; first = m = tiles = len = 0; seq = -1;
    const int i = i0 + (int)(threadIdx.x & 31);
    if (i >= rows.n) return;
    seq = page_seq_of(pv, rows.seqs, i);
    page_rows_of(rows, i, &first, &m);
    if (seq >= 0) len = page_len_of(pv, seq);
    tiles = m > rows.max_rows ? 0 : (int)(((long long)m * pack + ROWS - 1) / ROWS);
  }
  // Tile `slot` of all entries' (whole warp): false if there is none.
  __device__ __forceinline__ bool find(const PageView& pv, const PageRows& rows, int pack, int slot, RowsTile& it) {
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int i0 = 0; i0 < rows.n; i0 += 32) {
      look_up(pv, rows, pack, i0);
      int incl = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      const int at = before + incl - tiles;
      const uint32_t here = __ballot_sync(0xffffffffu, slot >= at && slot < at + tiles);
      if (here) {
        const int src = __ffs(here) - 1;
        const int skip = (slot - __shfl_sync(0xffffffffu, at, src)) * ROWS, rows_here = __shfl_sync(0xffffffffu, m, src);
        it.row0 = __shfl_sync(0xffffffffu, first, src) + skip;
        it.n_rows = min(ROWS, (rows_here - skip) * pack);   // (pack > 1: one item, skip is 0)
        it.pos0 = __shfl_sync(0xffffffffu, len, src) - rows_here + skip;
        it.seq = __shfl_sync(0xffffffffu, seq, src);
        return true;
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
    return false;
  }
};

// HD / 32 consecutive elements of a row per lane, as floats.
template <typename T, int N> __device__ __forceinline__ void load_dims(const T* p, float (&v)[N]);
template <> __device__ __forceinline__ void load_dims<float, 4>(const float* p, float (&v)[4]) {
  const float4 a = *reinterpret_cast<const float4*>(p);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
template <> __device__ __forceinline__ void load_dims<float, 2>(const float* p, float (&v)[2]) {
  const float2 a = *reinterpret_cast<const float2*>(p);
  v[0] = a.x; v[1] = a.y;
}
template <> __device__ __forceinline__ void load_dims<__nv_bfloat16, 4>(const __nv_bfloat16* p, float (&v)[4]) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xffff0000u);
  v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xffff0000u);
}
template <> __device__ __forceinline__ void load_dims<__nv_bfloat16, 2>(const __nv_bfloat16* p, float (&v)[2]) {
  const uint32_t a = *reinterpret_cast<const uint32_t*>(p);
  v[0] = __uint_as_float(a << 16); v[1] = __uint_as_float(a & 0xffff0000u);
}

// One row of one head by one warp (HD / 32 dimensions a lane): keys one page after another, eight at a time, running maximum
// and sum of the softmax in base 2 and 32 bits.  Keys in pages that the table does not name are left out and reported.
// scale2: scale * log2(e).  Leaves the unscaled output, the maximum (base 2) and the sum.
template <typename T, int HD>
__device__ __forceinline__ void attend_row_warp(const PageView& pv, int layer, const int32_t* table_row, int kv_head, int pos, int window, int sinks,
                                                float scale2, const float (&q)[HD / 32], float (&o)[HD / 32], float* m_out, float* l_out) {
  constexpr int N = HD / 32, BATCH = 8;
  const int lane = threadIdx.x & 31;
  const size_t page_elems = (size_t)pv.H * pv.ps * HD, plane = (size_t)pv.n_pages * page_elems;
  const T* kp = reinterpret_cast<const T*>(pv.pool) + (size_t)layer * 2 * plane + (size_t)kv_head * pv.ps * HD + lane * N;
  float m = -INFINITY, l = 0.f;
#pragma unroll
  for (int d = 0; d < N; ++d) o[d] = 0.f;
  int sink_end, start;
  visible_keys(pos, window, sinks, &sink_end, &start);
  for (int part = 0; part < 2; ++part) {
    const int from = part ? start : 0, to = part ? pos + 1 : sink_end;
    for (int j = from; j < to;) {
      const int page = table_row[j >> pv.ps_log2], slot = j & (pv.ps - 1), here = min(pv.ps - slot, to - j);
      if ((unsigned)page >= (unsigned)pv.n_pages) {
        if (lane == 0) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
        j += here;
        continue;
      }
      const T* k = kp + (size_t)page * page_elems + (size_t)slot * HD;
      for (int b = 0; b < here; b += BATCH) {
        float s[BATCH];
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
          s[x] = 0.f;
          if (b + x < here) {
            float kv[N];
            load_dims(k + (size_t)(b + x) * HD, kv);
#pragma unroll
            for (int d = 0; d < N; ++d) s[x] = fmaf(q[d], kv[d], s[x]);
          }
        }
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
#pragma unroll
          for (int w = 16; w; w >>= 1) s[x] += __shfl_xor_sync(0xffffffffu, s[x], w);
        }
        float mb = m;
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
          s[x] = b + x < here ? s[x] * scale2 : -INFINITY;
          mb = fmaxf(mb, s[x]);
        }
        const float ref = mb == -INFINITY ? 0.f : mb, corr = exp2f(m - ref);
        m = mb;
        l *= corr;
#pragma unroll
        for (int d = 0; d < N; ++d) o[d] *= corr;
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
          if (b + x >= here) break;
          const float p = exp2f(s[x] - ref);
          l += p;
          float vv[N];
          load_dims(k + plane + (size_t)(b + x) * HD, vv);
#pragma unroll
          for (int d = 0; d < N; ++d) o[d] = fmaf(p, vv[d], o[d]);
        }
      }
      j += here;
    }
  }
  *m_out = m; *l_out = l;
}

// o / l into the output and m + log l into lse (natural logarithm).  A row without keys is zeros and -inf.
template <typename T, int HD>
__device__ __forceinline__ void store_row_warp(const PageAttention& a, long long row, int head, const float (&o)[HD / 32], float m, float l) {
  constexpr int N = HD / 32;
  const int lane = threadIdx.x & 31;
  const float inv = l == 0.f ? 0.f : 1.f / l;   // (NaN stays NaN)
  T* out = reinterpret_cast<T*>(a.out) + row * a.out_stride + (long long)head * HD + lane * N;
#pragma unroll
  for (int d = 0; d < N; ++d) out[d] = from_f<T>(o[d] * inv);
  if (a.lse && lane == 0) a.lse[row * a.heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
}
#endif

}  // namespace rd
