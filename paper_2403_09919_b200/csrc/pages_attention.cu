// Attention of many rows per sequence over a cache in pages for the fp32 configuration, on the CUDA cores (tensor cores have no fp32
// products; TF32 would round K to 11 bits).
//
// A tile is 32 rows of a query head against chunks of 64 keys in shared memory; a thread has four rows (its 16 neighbours the same
// ones) and every 16th key for the scores, then the weights of its rows and four dimensions (eight of 128) for the output: 64
// multiply-adds for eight 16-byte loads.  Running maximum and sum of the softmax in base 2 and 32 bits.  The tile's keys are shared
// by a cluster of up to 8 CTAs where there are few tiles, joined over distributed shared memory in their order.  Keys that a row
// does not see take part in nothing: scores are selected, and chunks that only some rows see add V under the rows' masks.
//
// Bounds: instruction issue where there are many tiles (8 sequences of 2000 tokens, 256 rows, 4 heads of 64: 208 us, 20 of the CUDA
// cores' 74 TFLOP/s; issue slots 68 % while a CTA is there, 97 on the busiest SM, multiply-adds 39; 512 CTAs of which 444 fit at a
// time), else the chain of a tile's chunks, some 1.1 us each (256 rows of 8192 tokens 143 us, of 1000 tokens 24.5; a warp a row and head
// took 2134 and 260).
#include <cooperative_groups.h>

#include "pages_attention.cuh"
#include "pdl.cuh"

namespace rd {

namespace {

namespace cg = cooperative_groups;

constexpr int FR_ROWS = 32, FR_KEYS = 64, FR_THREADS = 128, FR_MAX_SHARE = 8;
template <int HD> constexpr size_t fp32_rows_smem() { return (size_t)(FR_ROWS * (HD + 4) + 2 * FR_KEYS * (HD + 4) + FR_ROWS * (FR_KEYS + 4)) * 4; }

// Bits 0 .. n-1 of 64.
__device__ __forceinline__ uint64_t low_bits64(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull; }

__device__ __forceinline__ void fma4(float4& a, float p, const float4& v) {
  a.x = fmaf(p, v.x, a.x); a.y = fmaf(p, v.y, a.y); a.z = fmaf(p, v.z, a.z); a.w = fmaf(p, v.w, a.w);
}

template <int HD>
__global__ void __launch_bounds__(FR_THREADS) pages_attention_fp32_kernel(const PageView pv, const PageRows rows, const PageAttention a) {
  extern __shared__ __align__(16) float smem[];
  constexpr int PITCH = HD + 4, PP = FR_KEYS + 4, PIECES = HD / 4, HALVES = HD / 64;
  float *s_q = smem, *s_k = s_q + FR_ROWS * PITCH, *s_v = s_k + FR_KEYS * PITCH, *s_p = s_v + FR_KEYS * PITCH;
  __shared__ float2 s_ml[FR_ROWS];
  pdl_enter();
  cg::cluster_group cluster = cg::this_cluster();
  const int S = gridDim.y, part = blockIdx.y, t = threadIdx.x, ty = t >> 4, tx = t & 15;
  RowsEntries<FR_ROWS> e;
  int total = 0;
  for (int i0 = 0; i0 < rows.n; i0 += 32) {
    e.look_up(pv, rows, 1, i0);
    total += __reduce_add_sync(0xffffffffu, e.tiles);
    if (blockIdx.x == 0 && part == 0 && t < 32 && (e.m > rows.max_rows || (e.m > 0 && e.seq < 0))) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
  }
  const int slot = blockIdx.x / a.heads, head = blockIdx.x - slot * a.heads, kv_head = head / (a.heads / pv.H);
  RowsTile it{};
  if (slot >= total || !e.find(pv, rows, 1, total - 1 - slot, it)) return;   // (the whole cluster)
  const int end = max(0, it.pos0 + it.n_rows), start = a.window > 0 ? max(0, it.pos0 - a.window + 1) : 0, sink_end = min(a.sinks, start);
  const int first_chunk = start / FR_KEYS, sink_chunks = min((sink_end + FR_KEYS - 1) / FR_KEYS, first_chunk);
  const int chunks = end > 0 ? sink_chunks + (end + FR_KEYS - 1) / FR_KEYS - first_chunk : 0;
  const int c0 = (int)((long long)chunks * part / S), c1 = (int)((long long)chunks * (part + 1) / S);
  const float scale2 = a.scale * LOG2E;
  for (int x = t; x < FR_ROWS * PIECES; x += FR_THREADS) {
    const int r = x / PIECES, d = (x - r * PIECES) * 4;
    float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < it.n_rows) q = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + (long long)(it.row0 + r) * a.q_stride + (long long)head * HD + d);
    *reinterpret_cast<float4*>(s_q + r * PITCH + d) = make_float4(q.x * scale2, q.y * scale2, q.z * scale2, q.w * scale2);
  }
  float m[4], l[4];
  float4 o[4][HALVES];
  int pos[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY; l[i] = 0.f;
    pos[i] = it.pos0 + min(ty * 4 + i, it.n_rows - 1);   // (rows behind the tile's last do as that one does, for nothing)
#pragma unroll
    for (int h = 0; h < HALVES; ++h) o[i][h] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const size_t page_elems = (size_t)pv.H * pv.ps * HD, plane = (size_t)pv.n_pages * page_elems;
  const float* pool = reinterpret_cast<const float*>(pv.pool) + (size_t)a.layer * 2 * plane + (size_t)kv_head * pv.ps * HD;
  const int32_t* table = pv.table + (size_t)max(it.seq, 0) * pv.max_pages;
  for (int c = c0; c < c1; ++c) {
    const int k0 = (c < sink_chunks ? c : first_chunk + c - sink_chunks) * FR_KEYS;
    __syncthreads();   // the chunk before has been read
#pragma unroll 4
    for (int x = t; x < FR_KEYS * PIECES; x += FR_THREADS) {
      const int key = x / PIECES, d = (x - key * PIECES) * 4, j = k0 + key;
      if (j >= end || (j >= sink_end && j < start)) continue;   // (nobody sees it)
      const int page = table[j >> pv.ps_log2];
      const bool there = (unsigned)page < (unsigned)pv.n_pages;
      if (!there) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
      const float* src = pool + (there ? (size_t)page * page_elems + (size_t)(j & (pv.ps - 1)) * HD + d : 0);
      const uint32_t bytes = there ? 16u : 0u, dk = (uint32_t)__cvta_generic_to_shared(s_k + key * PITCH + d), dv = (uint32_t)__cvta_generic_to_shared(s_v + key * PITCH + d);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dk), "l"(src), "r"(bytes) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dv), "l"(src + (there ? plane : 0)), "r"(bytes) : "memory");
    }
    asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    const bool all = k0 + FR_KEYS - 1 <= it.pos0 && (a.window == 0 || k0 > it.pos0 + it.n_rows - 1 - a.window);   // every row sees all of it
    uint64_t seen[4];
    float s[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      seen[i] = all ? ~0ull : low_bits64(pos[i] + 1 - k0) & ((a.window > 0 ? ~low_bits64(pos[i] - a.window + 1 - k0) : ~0ull) | low_bits64(a.sinks - k0));
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
    }
#pragma unroll 4
    for (int d = 0; d < HD; d += 4) {
      float4 q[4], k[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const float4*>(s_q + (ty * 4 + i) * PITCH + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4*>(s_k + (tx + 16 * j) * PITCH + d);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = fmaf(q[i].x, k[j].x, fmaf(q[i].y, k[j].y, fmaf(q[i].z, k[j].z, fmaf(q[i].w, k[j].w, s[i][j]))));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = (seen[i] >> (tx + 16 * j)) & 1ull ? s[i][j] : -INFINITY;
      float mx = fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3]));
#pragma unroll
      for (int w = 8; w; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float m_new = fmaxf(m[i], mx), ref = m_new == -INFINITY ? 0.f : m_new, corr = exp2f(m[i] - ref);
      m[i] = m_new;
      l[i] *= corr;
#pragma unroll
      for (int h = 0; h < HALVES; ++h) { o[i][h].x *= corr; o[i][h].y *= corr; o[i][h].z *= corr; o[i][h].w *= corr; }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2f(s[i][j] - ref);
        l[i] += p;
        s_p[(ty * 4 + i) * PP + tx + 16 * j] = p;
      }
    }
    __syncwarp();   // (a row's weights are its own warp's)
    for (int k = 0; k < FR_KEYS; k += 4) {
      float4 p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const float4*>(s_p + (ty * 4 + i) * PP + k);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          const float4 v = *reinterpret_cast<const float4*>(s_v + (k + y) * PITCH + h * 64 + tx * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (all || ((seen[i] >> (k + y)) & 1ull)) fma4(o[i][h], y == 0 ? p[i].x : y == 1 ? p[i].y : y == 2 ? p[i].z : p[i].w, v);
        }
      }
    }
  }
  // ---- join the cluster's CTAs: each a share of the rows
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int w = 8; w; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
    if (tx == 0) s_ml[ty * 4 + i] = make_float2(m[i], l[i]);
#pragma unroll
    for (int h = 0; h < HALVES; ++h) *reinterpret_cast<float4*>(s_k + (ty * 4 + i) * PITCH + h * 64 + tx * 4) = o[i][h];
  }
  if (S > 1) cluster.sync();
  else __syncthreads();
  const int each = FR_ROWS / S;
  for (int x = t; x < each * PIECES; x += FR_THREADS) {
    const int r = part * each + x / PIECES, d = (x % PIECES) * 4;
    if (r >= it.n_rows) continue;
    float2 ml[FR_MAX_SHARE];
    float M = -INFINITY, L = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int c = 0; c < FR_MAX_SHARE; ++c) {
      if (c >= S) break;
      ml[c] = *(S > 1 ? cluster.map_shared_rank(&s_ml[r], c) : &s_ml[r]);
      M = fmaxf(M, ml[c].x);
    }
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int c = 0; c < FR_MAX_SHARE; ++c) {
      if (c >= S) break;
      const float* from = s_k + r * PITCH + d;
      const float f = exp2f(ml[c].x - ref);
      L = fmaf(f, ml[c].y, L);
      fma4(v, f, *reinterpret_cast<const float4*>(S > 1 ? cluster.map_shared_rank(from, c) : from));
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + (long long)(it.row0 + r) * a.out_stride + (long long)head * HD + d) =
        make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    if (d == 0 && a.lse) a.lse[(long long)(it.row0 + r) * a.heads + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * LN2;
  }
  if (S > 1) cluster.sync();   // the others' shared memory has been read
}

}  // namespace

cudaError_t pages_attention_fp32_prepare(int hd) {
  return hd == 64 ? cudaFuncSetAttribute(pages_attention_fp32_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)fp32_rows_smem<64>())
                  : cudaFuncSetAttribute(pages_attention_fp32_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)fp32_rows_smem<128>());
}

cudaError_t launch_pages_attention_fp32(const PageView& pv, const PageRows& rows, const PageAttention& a, cudaStream_t st) {
  const long long tiles = (rows.n_rows + (long long)(FR_ROWS - 1) * rows.n) / FR_ROWS * a.heads;   // at most
  // up to four CTAs an SM (three fit at a time) hide a chunk's loads (8 sequences of 2000 tokens, 256 rows: 208 us, with at most two 269; a window of 200 keys,
  // which more of them would cut too short: 41.6, with eight 48.9)
  int S = 1;
  while (S < FR_MAX_SHARE && tiles * S * 2 <= 4 * 148) S *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)tiles, S);
  cfg.blockDim = FR_THREADS;
  cfg.dynamicSmemBytes = pv.hd == 64 ? fp32_rows_smem<64>() : fp32_rows_smem<128>();
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1; attr[1].val.clusterDim.y = S; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = pv.hd == 64 ? cudaLaunchKernelEx(&cfg, pages_attention_fp32_kernel<64>, pv, rows, a) : cudaLaunchKernelEx(&cfg, pages_attention_fp32_kernel<128>, pv, rows, a);
  return e ? e : cudaGetLastError();
}

}  // namespace rd
