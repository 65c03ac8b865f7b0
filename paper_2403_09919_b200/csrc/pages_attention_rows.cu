// Attention of many rows per sequence over a cache in pages (bf16) on the 5th-generation tensor cores: prompts and pieces of
// prompts, causal, with a sliding window and first tokens that stay visible.
//
// One CTA = a query head and up to 256 consecutive rows of a sequence in two tiles of 128, A and B.  Keys come in chunks of
// 128, put together from boxes of min(page_size, 64) keys: the boxes that hold sinks, then those from the first row's window
// on, so a handful of sinks does not cost a chunk of its own.
//   S = Q K^T    tcgen05.mma, Q and K K-major in shared memory, S in tensor memory (128 columns a tile)
//   softmax      one thread a row (= lane of tensor memory), the row's 128 scores in registers: no exchange between threads.
//                Base 2; the reference of a row follows its maximum only when that has grown by more than 2^8, so that the
//                running output is rescaled a few times a row at most (weights up to 2^8 cost nothing in bf16 or fp32);
//                weights rounded to bf16 over the first 64 columns of S
//   O += P V     tcgen05.mma with P read from tensor memory and V as it lies in its pages (MN-major)
// The two tiles take turns: while one's scores go through the softmax, the tensor cores work on the other's products.  The
// tensor pipe works off its instructions in order, so that a tile's scores are complete only when its previous P V is too:
// the softmax warps may then rescale O themselves, and the next S may overwrite P without a wait.
// Tensor memory: columns 0 and 128 S (and P) of A and B, 256 and 384 their O.
// Roles: warp 0 TMA, warp 1 MMA (the whole warp runs the loop, an elected lane issues), warps 2 and 3 look through V,
// warps 4-7 softmax A, 8-11 softmax B.  Registers: 384 x 168 = 64,512 at launch; 4 warps go down to 96 and 8 up to 200
// (128 x 96 + 256 x 200 = 63,488).  Every wait is bounded; on expiry the CTA reports and leaves.
//
// Anything may lie in keys that a row does not see.  Scores are masked by selection.  V's rows that no row of the CTA sees are
// overwritten by zeros, and chunks that only some rows see are looked through: where such a chunk holds NaN or infinities,
// 0 x V would reach the others, and the CTA's rows are worked out one by one instead.
//
// Bounds: 2 x 1024 cycles of exponentials a chunk and pair of tiles (16 a cycle and SM) against 2048 of products.
#include <cuda.h>

#include "pages_attention.cuh"
#include "pdl.cuh"
#include "tcgen05.cuh"

namespace rd {

namespace {

constexpr int RW_TILE = 128;         // rows of a tile
constexpr int RW_KEYS = 128;         // keys of a chunk
constexpr int RW_STAGES = 2;
constexpr int RW_THREADS = 384;
constexpr uint32_t RW_BLOCK = 128 * 128;   // bytes of 128 rows of 64 columns
constexpr float RW_SLACK = 8.f;

struct RowsParams {
  PageView pv;
  PageRows rows;
  PageAttention a;
};

__device__ __forceinline__ uint64_t desc_mnmajor_v(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(RW_BLOCK >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tmem_st32_u32(uint32_t taddr, const uint32_t (&r)[32]) {
  tmem_st32(taddr, reinterpret_cast<const float*>(r));
}
// Bits 0 .. n-1.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// What the rows of a CTA see, as a list of boxes.
struct BoxList {
  int box, sink_boxes, first_box, n_boxes;
  int sinks, start, end;   // keys that some row sees: [0, sinks) and [start, end)
  __device__ __forceinline__ int base(int b) const {   // first key of box b; behind the list: out of sight of everything
    return b >= n_boxes ? 0x40000000 : (b < sink_boxes ? b : first_box + b - sink_boxes) * box;
  }
};

template <int HD> constexpr size_t rows_smem() { return 1024 + (size_t)(2 + 2 * RW_STAGES) * (HD / 64) * RW_BLOCK + 256 + 64; }

template <int HD>
__global__ void __launch_bounds__(RW_THREADS, 1)
    pages_rows_kernel(const __grid_constant__ CUtensorMap map, const RowsParams p) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int HALVES = HD / 64;
  constexpr uint32_t TILE = HALVES * RW_BLOCK;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t sQ = base, sK = sQ + 2 * TILE, sV = sK + RW_STAGES * TILE, bar0 = sV + RW_STAGES * TILE;
  enum { Q_FULL = 0, K_FULL = 1, K_EMPTY = 3, V_FULL = 5, V_OK = 7, V_EMPTY = 9, S_FULL = 11, P_FULL = 13, O_FULL = 15, N_BARS = 17 };
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint8_t* misc = gen + (bar0 - base) + 8 * N_BARS;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
  volatile int* s_unclean = reinterpret_cast<volatile int*>(misc + 8);   // V holds NaN or infinities that not every row sees
  volatile int* s_entry = reinterpret_cast<volatile int*>(misc + 12);    // [2] entry and its pair of tiles; entry -1: nothing to do
  int* s_scan = reinterpret_cast<int*>(misc + 24);                       // [RW_THREADS / 32]

  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
    mbar_init(bar(Q_FULL), 8);
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(K_FULL + s), 1); mbar_init(bar(K_EMPTY + s), 1);
      mbar_init(bar(V_FULL + s), 1); mbar_init(bar(V_OK + s), 2); mbar_init(bar(V_EMPTY + s), 1);
      mbar_init(bar(S_FULL + s), 1); mbar_init(bar(P_FULL + s), 4); mbar_init(bar(O_FULL + s), 1);
    }
    *abort_flag = 0; *s_unclean = 0; *s_entry = -1;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_enter();
  const PageView& pv = p.pv;
  // ---- which entry and rows: pairs of tiles are counted over the entries; the last ones are handed out first, since later
  // rows of a sequence have more keys
  {
    const int per = (p.rows.n + RW_THREADS - 1) / RW_THREADS, e0 = min((int)threadIdx.x * per, p.rows.n), e1 = min(e0 + per, p.rows.n);
    auto pairs_of = [&](int i) {
      int first, m;
      page_rows_of(p.rows, i, &first, &m);
      return m > p.rows.max_rows ? 0 : (m + 2 * RW_TILE - 1) / (2 * RW_TILE);
    };
    int mine = 0;
    for (int i = e0; i < e1; ++i) mine += pairs_of(i);
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    int before = incl - mine, total = 0;
    for (int w = 0; w < RW_THREADS / 32; ++w) {
      if (w < warp) before += s_scan[w];
      total += s_scan[w];
    }
    const int slot = total - 1 - (int)(blockIdx.x / p.a.heads);   // < 0: the grid provides more than there are
    if (slot >= before && slot < before + mine) {
      int i = e0, at = before;
      for (;; ++i) {
        const int n = pairs_of(i);
        if (slot < at + n) break;
        at += n;
      }
      s_entry[0] = i; s_entry[1] = slot - at;
    }
    if (blockIdx.x == 0)   // entries that cannot be answered
      for (int i = e0; i < e1; ++i) {
        int first, m;
        page_rows_of(p.rows, i, &first, &m);
        if (m > p.rows.max_rows || (m > 0 && page_seq_of(pv, p.rows.seqs, i) < 0)) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
      }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int entry = s_entry[0], head = (int)(blockIdx.x % p.a.heads);
  int row0 = 0, n_rows = 0, pos0 = 0, seq = -1, len = 0;   // first row of the CTA, its rows, the first row's position
  if (entry >= 0) {
    int first, m;
    page_rows_of(p.rows, entry, &first, &m);
    seq = page_seq_of(pv, p.rows.seqs, entry);
    len = seq >= 0 ? page_len_of(pv, seq) : 0;
    const int skip = s_entry[1] * 2 * RW_TILE;
    row0 = first + skip;
    n_rows = min(2 * RW_TILE, m - skip);
    pos0 = len - m + skip;
  }
  const int window = p.a.window, kv_head = head / (p.a.heads / pv.H);
  const int n_tiles = n_rows > RW_TILE ? 2 : n_rows > 0 ? 1 : 0;
  BoxList bl;
  bl.box = min(pv.ps, 64);
  const int pos_last = pos0 + n_rows - 1;
  bl.end = n_rows > 0 ? max(0, pos_last + 1) : 0;
  bl.start = window > 0 ? max(0, pos0 - window + 1) : 0;
  bl.sinks = min(p.a.sinks, bl.start);
  bl.first_box = bl.start / bl.box;
  bl.sink_boxes = min((bl.sinks + bl.box - 1) / bl.box, bl.first_box);
  bl.n_boxes = bl.end > 0 ? bl.sink_boxes + (bl.end + bl.box - 1) / bl.box - bl.first_box : 0;
  const int per_chunk = RW_KEYS / bl.box;
  const int n_chunks = (bl.n_boxes + per_chunk - 1) / per_chunk;
  // chunks that a tile works on: A stops behind its own last row's key, B begins (without sinks) where its first row's window does
  const int end_a = n_tiles == 2 ? max(0, min(pos0 + RW_TILE, bl.end)) : bl.end;
  const int boxes_a = end_a > 0 ? bl.sink_boxes + (end_a + bl.box - 1) / bl.box - bl.first_box : 0;
  const int start_b = window > 0 ? max(0, pos0 + RW_TILE - window + 1) : 0;
  int from[2], to[2];
  from[0] = 0;
  to[0] = n_tiles > 0 ? min(n_chunks, (boxes_a + per_chunk - 1) / per_chunk) : 0;
  from[1] = p.a.sinks == 0 ? max(0, start_b / bl.box - bl.first_box) / per_chunk : 0;
  to[1] = n_tiles == 2 ? n_chunks : 0;
  if (n_tiles < 2) from[1] = 0;
  auto active = [&](int tile, int c) { return c >= from[tile] && c < to[tile]; };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
    if (warp == 0) {
      // ===================== TMA: lane = (box, half) of the chunk =====================
      const long long pool_rows = (long long)pv.n_layers * 2 * pv.n_pages * pv.H * pv.ps, plane_rows = (long long)pv.n_pages * pv.H * pv.ps;
      const int box = lane / HALVES, half = lane - box * HALVES;
      const bool mine = box < per_chunk;
      auto row_of = [&](int c, int which) -> int {   // row of the pool at which this lane's box begins
        const int key = bl.base(c * per_chunk + box);
        if (!mine || key >= bl.end) return (int)pool_rows;   // (behind the pool's last row the copy fills in zeros)
        const int page = pv.table[(size_t)seq * pv.max_pages + (key >> pv.ps_log2)];
        if ((unsigned)page >= (unsigned)pv.n_pages) {
          // a page that has been trimmed may share a box's place with the window's edge only if nothing of it is seen
          if (key + bl.box > bl.start || key < bl.sinks) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
          return (int)pool_rows;
        }
        return (int)((((long long)p.a.layer * 2 * pv.n_pages + page) * pv.H + kv_head) * pv.ps + (key & (pv.ps - 1)) + which * plane_rows);
      };
      const uint32_t place = (uint32_t)(half * RW_BLOCK + box * bl.box * 128);
      bool ok = true;
      auto load = [&](uint32_t dst, uint32_t b, int row) {
        if (lane == 0) mbar_expect_tx(b, TILE);
        __syncwarp();
        if (mine) tma_load_2d(dst + place, &map, b, half * 64, row);
      };
      auto wait_warp = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag, pv.status)) != 0; };
      for (int c = 0; c < 2 && c < n_chunks; ++c) load(sK + c * TILE, bar(K_FULL + c), row_of(c, 0));
      for (int c = 0; c < n_chunks; ++c) {
        const int s = c & 1;
        const uint32_t ph = (c >> 1) & 1;
        const int vrow = row_of(c, 1), krow = c + 2 < n_chunks ? row_of(c + 2, 0) : 0;
        if (c >= 2 && !(ok = wait_warp(bar(V_EMPTY + s), ph ^ 1u))) break;
        load(sV + s * TILE, bar(V_FULL + s), vrow);
        if (c + 2 < n_chunks) {
          if (!(ok = wait_warp(bar(K_EMPTY + s), ph))) break;
          load(sK + s * TILE, bar(K_FULL + s), krow);
        }
      }
      if (!ok || *abort_flag) {   // copies already issued land before the CTA's shared memory is given back
        const unsigned long long t0 = now_ns();
        while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
      }
    } else if (warp == 1) {
      // ===================== MMA =====================
      if (n_chunks > 0) {
        uint32_t leader;
        asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\tselp.u32 %0, 1, 0, P;\n\t}" : "=r"(leader));
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(RW_TILE >> 4) << 24);
        const uint32_t idesc_qk = idesc | ((uint32_t)(RW_KEYS >> 3) << 17), idesc_pv = idesc | (1u << 16) | ((uint32_t)(HD >> 3) << 17);
        auto wait_warp = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag, pv.status)) != 0; };
        auto issue_qk = [&](int tile, int c) {
          const uint64_t qd = desc_kmajor(sQ + (uint32_t)tile * TILE), kd = desc_kmajor(sK + (uint32_t)(c & 1) * TILE);
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
              const uint64_t off = (uint64_t)(((uint32_t)(kk >> 2) * RW_BLOCK + (uint32_t)(kk & 3) * 32u) >> 4);
              umma_bf16(tmem + (uint32_t)tile * 128u, qd + off, kd + off, idesc_qk, kk > 0 ? 1u : 0u);
            }
            umma_commit(bar(S_FULL + tile));
          }
          __syncwarp();
        };
        bool ok = wait_warp(bar(Q_FULL), 0);
        if (ok) ok = wait_warp(bar(K_FULL), 0);
        if (ok) {
          tc_fence_after();
          for (int tile = 0; tile < 2; ++tile)
            if (active(tile, 0)) issue_qk(tile, 0);
          if (leader) umma_commit(bar(K_EMPTY));
          __syncwarp();
        }
        for (int c = 0; c < n_chunks && ok; ++c) {
          const int s = c & 1;
          const uint32_t ph = (c >> 1) & 1;
          if (!(ok = wait_warp(bar(V_OK + s), ph))) break;
          if (c + 1 < n_chunks && !(ok = wait_warp(bar(K_FULL + (s ^ 1)), ((c + 1) >> 1) & 1))) break;
          for (int tile = 0; tile < 2; ++tile) {
            if (active(tile, c)) {
              if (!(ok = wait_warp(bar(P_FULL + tile), (uint32_t)((c - from[tile]) & 1)))) break;
              tc_fence_after();
              const uint64_t vd = desc_mnmajor_v(sV + (uint32_t)s * TILE);
              if (leader) {
#pragma unroll
                for (int kk = 0; kk < RW_KEYS / 16; ++kk)
                  umma_bf16_ts(tmem + 256u + (uint32_t)tile * 128u, tmem + (uint32_t)tile * 128u + (uint32_t)kk * 8u, vd + (uint64_t)(kk * 128), idesc_pv,
                               (c > from[tile] || kk > 0) ? 1u : 0u);
                if (c + 1 == to[tile]) umma_commit(bar(O_FULL + tile));
              }
              __syncwarp();
            }
            if (c + 1 < n_chunks && active(tile, c + 1)) issue_qk(tile, c + 1);
          }
          if (!ok) break;
          if (leader) {
            umma_commit(bar(V_EMPTY + s));
            if (c + 1 < n_chunks) umma_commit(bar(K_EMPTY + (s ^ 1)));
          }
          __syncwarp();
        }
      }
    } else {
      // ===================== V: zeros where no row looks, a look at what only some rows see =====================
      const int t = threadIdx.x - 64;
      for (int c = 0; c < n_chunks; ++c) {
        const int s = c & 1;
        if (!__all_sync(0xffffffffu, mbar_wait(bar(V_FULL + s), (c >> 1) & 1, abort_flag, pv.status))) break;
        bool all = true;   // every row of the CTA sees all of the chunk
        for (int b = 0; b < per_chunk; ++b) {
          const int k0 = bl.base(c * per_chunk + b);
          all = all && k0 + bl.box - 1 <= pos0 && (window == 0 || k0 > pos_last - window || k0 + bl.box <= bl.sinks);
        }
        if (!all) {
          bool unclean = false;
          for (int e = t; e < HALVES * 128 * 8; e += 64) {   // 16-byte pieces: (half, key, piece)
            const int key = (e >> 3) & 127;
            const int k = bl.base(c * per_chunk + key / bl.box) + (key & (bl.box - 1));
            uint4* at = reinterpret_cast<uint4*>(gen + (sV - base) + s * TILE + (size_t)e * 16);
            if (k >= bl.end || (k >= bl.sinks && k < bl.start)) {
              *at = make_uint4(0u, 0u, 0u, 0u);
            } else {
              const uint4 v = *at;
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int j = 0; j < 4; ++j) unclean = unclean || (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
            }
          }
          if (unclean) *s_unclean = 1;
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(V_OK + s));
      }
    }
  } else {
    // ===================== softmax and output: one thread a row =====================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    const int tile = (warp - 4) >> 2, w4 = warp & 3;   // (a warp may touch the lane quarter warp mod 4 of tensor memory)
    const int t = w4 * 32 + lane, r_cta = tile * RW_TILE + t;
    const int t_rows = min(RW_TILE, n_rows - tile * RW_TILE);   // rows of the tile, <= 0: none
    const bool valid = t < t_rows;
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    if (n_chunks > 0) {
      // the tile's Q, K-major and swizzled: 16-byte piece c of row r lies at piece c ^ (r & 7) of its 128 bytes
      constexpr int PIECES = HD / 8, ROWS_PASS = 32 / PIECES;
      const int piece = lane % PIECES;
      const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.a.q) + (long long)(row0 + tile * RW_TILE) * p.a.q_stride + (long long)head * HD + piece * 8;
      uint8_t* dst = gen + tile * TILE + (piece >> 3) * RW_BLOCK;
#pragma unroll 8
      for (int i = 0; i < 32 / ROWS_PASS; ++i) {
        const int r = w4 * 32 + i * ROWS_PASS + lane / PIECES;
        const uint4 v = r < t_rows ? *reinterpret_cast<const uint4*>(q + (long long)r * p.a.q_stride) : make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(dst + r * 128 + (((piece & 7) ^ (r & 7)) << 4)) = v;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(Q_FULL));
    }
    auto wait_all = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag, pv.status)) != 0; };
    const float scale2 = p.a.scale * LOG2E;
    const int pos = valid ? pos0 + r_cta : -1, lo = window > 0 ? pos - window + 1 : 0;   // sees [lo, pos] and the sinks
    const int tile_pos0 = pos0 + tile * RW_TILE, tile_pos1 = tile_pos0 + t_rows - 1;
    const uint32_t s_addr = tmem + lanes + (uint32_t)tile * 128u, o_addr = s_addr + 256u;
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int c = from[tile]; c < to[tile]; ++c) {
      const int it = c - from[tile];
      if (!(ok = wait_all(bar(S_FULL + tile), (uint32_t)(it & 1)))) break;
      tc_fence_after();
      float sc[RW_KEYS];
#pragma unroll
      for (int g = 0; g < RW_KEYS / 32; ++g) tmem_ld32_nowait(s_addr + g * 32, sc + g * 32);
      bool all = true;   // every row of the tile sees all of the chunk
      for (int b = 0; b < per_chunk; ++b) {
        const int k0 = bl.base(c * per_chunk + b);
        all = all && k0 + bl.box - 1 <= tile_pos0 && (window == 0 || k0 > tile_pos1 - window || k0 + bl.box <= bl.sinks);
      }
      tmem_ld_wait();
      if (!all) {
#pragma unroll
        for (int g = 0; g < RW_KEYS / 16; ++g) {   // sixteen keys lie in one box
          const int k0 = bl.base(c * per_chunk + g * 16 / bl.box) + ((g * 16) & (bl.box - 1));
          const uint32_t seen = low_bits(pos + 1 - k0) & (~low_bits(lo - k0) | low_bits(p.a.sinks - k0));
#pragma unroll
          for (int j = 0; j < 16; ++j) sc[g * 16 + j] = ((seen >> j) & 1u) ? sc[g * 16 + j] : -INFINITY;
        }
      }
      float mx4[4] = {sc[0], sc[1], sc[2], sc[3]};
#pragma unroll
      for (int j = 4; j < RW_KEYS; ++j) mx4[j & 3] = fmaxf(mx4[j & 3], sc[j]);
      const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * scale2;
      const bool moves = mx > m + RW_SLACK || (m == -INFINITY && mx > m);
      if (__any_sync(0xffffffffu, moves)) {
        const float corr = !moves ? 1.f : fast_exp2(m - mx);
        if (moves) m = mx;
        l *= corr;
        if (it > 0) {   // the tile's earlier products are complete (its scores were issued behind them)
#pragma unroll
          for (int g = 0; g < HD / 32; ++g) {
            float ov[32];
            tmem_ld32_nowait(o_addr + g * 32, ov);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) ov[j] *= corr;
            tmem_st32(o_addr + g * 32, ov);
          }
        }
      }
      const float ref = m == -INFINITY ? 0.f : m;
      float sum4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t pk[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float a = fast_exp2(fmaf(sc[g * 64 + 2 * j], scale2, -ref)), b = fast_exp2(fmaf(sc[g * 64 + 2 * j + 1], scale2, -ref));
          sum4[(2 * j) & 3] += a; sum4[(2 * j + 1) & 3] += b;
          pk[j] = pack_bf16(a, b);
        }
        tmem_st32_u32(s_addr + g * 32, pk);
      }
      l += (sum4[0] + sum4[1]) + (sum4[2] + sum4[3]);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(P_FULL + tile));
    }
    // ---- output
    const bool any = to[tile] > from[tile];
    if (ok && any) ok = wait_all(bar(O_FULL + tile), 0);
    if (ok && t_rows > 0) {
      if (*s_unclean) {
        for (int r = w4 * 32; r < min(t_rows, w4 * 32 + 32); ++r) {   // (rare) the warp's rows, one after another
          const long long row = row0 + tile * RW_TILE + r;
          float q[HD / 32], o[HD / 32], rm = -INFINITY, rl = 0.f;
#pragma unroll
          for (int d = 0; d < HD / 32; ++d) o[d] = 0.f;
          load_dims(reinterpret_cast<const __nv_bfloat16*>(p.a.q) + row * p.a.q_stride + (long long)head * HD + lane * (HD / 32), q);
          if (tile_pos0 + r >= 0)
            attend_row_warp<__nv_bfloat16, HD>(pv, p.a.layer, pv.table + (size_t)seq * pv.max_pages, kv_head, tile_pos0 + r, window, p.a.sinks, scale2, q, o,
                                               &rm, &rl);
          store_row_warp<__nv_bfloat16, HD>(p.a, row, head, o, rm, rl);
        }
      } else {
        tc_fence_after();
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const long long row = row0 + r_cta;
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.a.out) + row * p.a.out_stride + (long long)head * HD;
#pragma unroll 1
        for (int g = 0; g < HD / 32; ++g) {
          float ov[32];
          if (any) {
            tmem_ld32_nowait(o_addr + g * 32, ov);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) ov[j] = 0.f;
          }
          if (valid) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              *reinterpret_cast<uint4*>(out + g * 32 + j * 8) =
                  make_uint4(pack_bf16(ov[j * 8] * inv, ov[j * 8 + 1] * inv), pack_bf16(ov[j * 8 + 2] * inv, ov[j * 8 + 3] * inv),
                             pack_bf16(ov[j * 8 + 4] * inv, ov[j * 8 + 5] * inv), pack_bf16(ov[j * 8 + 6] * inv, ov[j * 8 + 7] * inv));
          }
        }
        if (valid && p.a.lse) p.a.lse[row * p.a.heads + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
      }
    }
  }
  // ---- everyone meets, then the allocating warp frees the tensor memory
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

}  // namespace

cudaError_t pages_rows_prepare(int hd) {
  return hd == 64 ? cudaFuncSetAttribute(pages_rows_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)rows_smem<64>())
                  : cudaFuncSetAttribute(pages_rows_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)rows_smem<128>());
}

// map: the pool as [rows][head_dim], boxes of min(page_size, 64) rows and 64 columns.
cudaError_t launch_pages_rows(const void* map, const PageView& pv, const PageRows& rows, const PageAttention& a, cudaStream_t st) {
  RowsParams p;
  p.pv = pv; p.rows = rows; p.a = a;
  const long long slots = rows.n_rows / (2 * RW_TILE) + (long long)rows.n;   // pairs of tiles, at most
  if (slots * a.heads > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  const unsigned grid = (unsigned)(slots * a.heads);
  if (pv.hd == 64) launch_pdl(pages_rows_kernel<64>, grid, RW_THREADS, rows_smem<64>(), st, *(const CUtensorMap*)map, p);
  else launch_pdl(pages_rows_kernel<128>, grid, RW_THREADS, rows_smem<128>(), st, *(const CUtensorMap*)map, p);
  return cudaGetLastError();
}

}  // namespace rd
