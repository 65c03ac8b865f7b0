// Attention of many rows per sequence over a cache in pages (bf16) on the 5th-generation tensor cores: prompts and pieces of
// prompts, causal, with a sliding window and first tokens that stay visible.
//
// One item = a query head and up to 256 consecutive rows of a sequence in two tiles of 128, A and B.  Keys come in chunks of
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
// The CTAs stay (one per SM) and take one item after another, so that the next one's Q, K and V are on their way while the last
// products and the output of one are finished.
// Few items (up to half the SMs) leave SMs idle and take long over long contexts: their keys are then shared by up to 8 CTAs, at
// least 4 chunks each, which leave unscaled outputs, maxima and sums (fp32) in the workspace, joined by rows_join_kernel.  Bf16, one
// sequence, 32 query heads on 8, one CTA an item | shared: 256 rows of 8192 tokens 120 | 46.5 us, 500 rows 121 | 76; up to 16 CTAs
// are slower again (64 rows of 8192 tokens 30.8 us with 8, 37.8 with 16: the join).
// Few rows on grouped heads (rows x group up to 256) fill a tile with all the query heads of a key and value head: K and V are read
// and multiplied once for all of them.  A head an item | packed: 16 sequences of 2000 tokens, 6 rows each 122 | 36 us; 64 of 500
// tokens, 4 rows each 140 | 51; 17 rows of 8192 tokens 39.4 | 26.9; 60 rows of 300 tokens 15.1 | 18.5 (the one that loses: two
// tiles after one another where idle SMs could take one each; the contexts' lengths stand on the device, and from about 1000 tokens
// on it wins).
// Launches that need neither take the forms without them (4096 rows: 2 us less than one kernel for all).
// Roles: warp 0 finds the items and loads K and V by TMA, warp 1 MMA (the whole warp runs the loop, an elected lane issues), warps
// 2 and 3 look through V, warps 4-7 softmax A, 8-11 softmax B.  Registers: 384 x 168 = 64,512 at launch; 4 warps go down to 120 and 8 up to 192
// (128 x 120 + 256 x 192 = 64,512).  Every wait is bounded; on expiry the CTA reports and leaves.
//
// Anything may lie in keys that a row does not see.  Scores are masked by selection.  V's rows that no row of the CTA sees are
// overwritten by zeros, and chunks that only some rows see are looked through: where such a chunk holds NaN or infinities,
// 0 x V would reach the others, and the CTA's rows are worked out one by one instead.
//
// Bounds: a chunk and pair of tiles takes some 3300 cycles where all of it is seen, against 2048 of products and 2 x 1024 of
// exponentials (16 a cycle and SM); chunks that need masks take 1300 more, an item's set-up and output 5000.  What bounds it is each
// tile's chain of scores, softmax and products, of which the other tile hides a part.  4096 rows of 32 heads, window 1024: 128 us
// with the write of K and V (466 TFLOP/s of what the rows see; 512 items in four waves of 148).  Tried and slower: a warp issuing
// for each tile (132 us), an eighth to a quarter of the exponentials as polynomials (130 to 134).
#include <cuda.h>

#include <type_traits>

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
// A row's largest score may exceed its reference by this much (log2).  Its weight is then rounded to bf16 like the others, where the
// maximum as the reference would make it exactly one: 2.15e-3 of the output's norm against 64 bits (4096 rows, window 1024) and 2.27e-3
// (pieces of prompts, window 512), with the maximum 2.09e-3 and 2.16e-3 at 136.8 us for 128.1 and 44.6 for 42.0; the output's own rounding
// alone is 1.62e-3 and 1.66e-3.  One bf16 part a weight, as attention_t5.cu has it for prompts on the contiguous cache.
constexpr float RW_SLACK = 8.f;
constexpr int RW_SLOTS = 4;                // published items
constexpr int RW_MAX_SPLIT = 8, RW_MIN_CHUNKS = 4;   // CTAs that share an item's keys; chunks that each of them takes at least
constexpr int RW_ROWS = 2 * RW_TILE;

struct RowsParams {
  PageView pv;
  PageRows rows;
  PageAttention a;
  int grid;        // CTAs of the launch
  int pack;        // query heads that share a tile: 1, or all of a key and value head's (then an entry's rows are one item)
  float* parts;    // [CTAs][rows_part_floats]: what they leave of an item that several work on
};
// A part: the unscaled output [HD / 4][RW_ROWS] of four dimensions each (a warp's store covers 512 bytes), then maximum (base 2) and
// sum of every row.  A sum of NaN asks for the row to be worked out by itself.
template <int HD> __host__ __device__ constexpr int rows_part_floats() { return RW_ROWS * (HD + 2); }

__device__ __forceinline__ uint64_t desc_mnmajor_v(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(RW_BLOCK >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void tmem_st32_u32(uint32_t taddr, const uint32_t (&r)[32]) {
  tmem_st32(taddr, reinterpret_cast<const float*>(r));
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&u)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(taddr));
}
// Bits 0 .. n-1.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// What a CTA works on next, worked out by the producer warp and published two items ahead.
struct RowsItem : RowsTile {
  int head;   // of the heads / pack; -1: there is nothing left
  // The keys as a list of boxes: 0 .. sink_boxes - 1 hold sinks, those from `first` on are box b + skew of the sequence, and the
  // places between them are left empty.
  int n_chunks, sink_boxes, skew, first;
  int start, end, sinks;      // keys that some row sees: [0, sinks) and [start, end)
  int to_a, from_b, to_b;     // chunks that a tile works on; A from the first
  int c0, c1, part;           // SPLIT: chunks of this CTA; its part, -1: all of them
  int all_from, all_to_a, all_to_b, all_from_b;   // chunks that every row of a tile (A: all_from .. all_to_a) sees whole
  int unclean;                // V holds NaN or infinities that only some of the rows see

  template <bool SPLIT> __device__ __forceinline__ int begin() const { return SPLIT ? c0 : 0; }
  template <bool SPLIT> __device__ __forceinline__ int end_chunk() const { return SPLIT ? c1 : n_chunks; }
  template <bool SPLIT> __device__ __forceinline__ int from(int tile) const { return tile ? from_b : begin<SPLIT>(); }
  __device__ __forceinline__ int to(int tile) const { return tile ? to_b : to_a; }
  template <bool SPLIT> __device__ __forceinline__ bool active(int tile, int c) const { return c >= from<SPLIT>(tile) && c < to(tile); }
  template <bool SPLIT> __device__ __forceinline__ bool has(int tile) const { return to(tile) > from<SPLIT>(tile); }
  // first key of box b; a place that is left empty: out of sight of everything
  __device__ __forceinline__ int base(int b, int box_log2) const {
    return b < sink_boxes ? b << box_log2 : b < first ? 0x7fffff00 : (b + skew) << box_log2;
  }
};

// Row x of an item is token x / pack of its rows, query head x mod pack of those that share the tile.
__device__ __forceinline__ void plan_rows(RowsItem& r, int window, int sinks, int box_log2, int pack) {
  const int box = 1 << box_log2, pc_log2 = 7 - box_log2, per_chunk = 1 << pc_log2;
  const bool two = r.n_rows > RW_TILE;
  const int last = (r.n_rows - 1) / pack, last_a = min(last, (RW_TILE - 1) / pack), first_b = RW_TILE / pack;   // tokens of the item
  r.end = max(0, r.pos0 + last + 1);
  r.start = window > 0 ? max(0, r.pos0 - window + 1) : 0;
  r.sinks = min(sinks, r.start);
  const int first_box = r.start >> box_log2, end_box = (r.end + box - 1) >> box_log2;
  r.sink_boxes = min((r.sinks + box - 1) >> box_log2, first_box);
  r.n_chunks = r.end > 0 ? (r.sink_boxes + end_box - first_box + per_chunk - 1) >> pc_log2 : 0;
  // The list ends with a chunk: what is left empty lies before the window's boxes, so that the diagonal of rows that end on a
  // multiple of 128 crosses one chunk a tile.
  r.skew = end_box - (r.n_chunks << pc_log2);
  r.first = first_box - r.skew;
  // A stops behind its own last row's key, B begins (without sinks) where its first row's window does
  const int end_a = max(0, r.pos0 + last_a + 1), start_b = window > 0 ? max(0, r.pos0 + first_b - window + 1) : 0;
  r.to_a = !two ? r.n_chunks : end_a > 0 ? min(r.n_chunks, (((end_a + box - 1) >> box_log2) - r.skew + per_chunk - 1) >> pc_log2) : 0;
  r.from_b = two && sinks == 0 && r.n_chunks > 0 ? max(0, (start_b >> box_log2) - r.skew) >> pc_log2 : 0;
  r.to_b = two ? r.n_chunks : 0;
  r.c0 = 0; r.c1 = r.n_chunks; r.part = -1;
  // Chunk c of the window's part holds the keys k0 .. k0 + 127, k0 = (c * per_chunk + skew) * box.  Rows at positions p .. q see
  // all of it if k0 + 127 <= p and k0 > q - window.
  auto all_to = [&](int p) { return p < RW_KEYS - 1 ? 0 : (((p - (RW_KEYS - 1)) >> box_log2) - r.skew + per_chunk) >> pc_log2; };
  auto all_from = [&](int q) {
    const int c0 = (r.first + per_chunk - 1) >> pc_log2;   // the first chunk without sinks and empty places
    return window > 0 && q >= window ? max(c0, (((q - window + box) >> box_log2) - r.skew + per_chunk - 1) >> pc_log2) : c0;
  };
  r.all_from = all_from(r.pos0 + last_a);
  r.all_to_a = all_to(r.pos0);
  r.all_from_b = all_from(r.pos0 + last);
  r.all_to_b = all_to(r.pos0 + first_b);
}

// Most CTAs that may share an item's keys: beyond 1 every CTA of the launch has one item at most.
__device__ __forceinline__ int split_of(long long items, int grid) { return items > 0 ? (int)max(1ll, min((long long)RW_MAX_SPLIT, grid / items)) : 1; }
// ... and those that do.
__device__ __forceinline__ int parts_of(const RowsItem& r, int split) { return min(split, max(1, r.n_chunks / RW_MIN_CHUNKS)); }
// What CTA w of the launch takes of an item that `split` CTAs may share: false for nothing.
__device__ __forceinline__ bool cut_keys(RowsItem& r, int split, int w) {
  const int n = parts_of(r, split), s = w % split;
  if (s >= n) return false;
  if (n > 1) {
    r.part = w;
    r.c0 = r.n_chunks * s / n; r.c1 = r.n_chunks * (s + 1) / n;
    r.to_a = min(r.to_a, r.c1);
    r.from_b = max(r.from_b, r.c0); r.to_b = min(r.to_b, r.c1);
  }
  return true;
}

__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {   // zeros where there is nothing
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16u : 0u) : "memory");
}

constexpr int RW_STAGE_OUT = 32 * 128;     // bytes of a softmax warp's output on its way: 32 rows of 64 columns
template <int HD> constexpr size_t rows_smem() { return 1024 + (size_t)(2 + 2 * RW_STAGES) * (HD / 64) * RW_BLOCK + 8 * RW_STAGE_OUT + 1024; }

// PACK: p.pack > 1.
template <int HD, bool SPLIT, bool PACK>
__global__ void __launch_bounds__(RW_THREADS, 1)
    pages_rows_kernel(const __grid_constant__ CUtensorMap map, const RowsParams p) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int HALVES = HD / 64;
  constexpr uint32_t TILE = HALVES * RW_BLOCK;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t sQ = base, sK = sQ + 2 * TILE, sV = sK + RW_STAGES * TILE, sO = sV + RW_STAGES * TILE, bar0 = sO + 8 * RW_STAGE_OUT;
  enum { K_FULL = 0, K_EMPTY = 2, V_FULL = 4, V_OK = 6, V_EMPTY = 8, Q_FULL = 10, S_FULL = 12, P_HALF = 14, P_FULL = 16, O_FULL = 18, O_EMPTY = 20,
         ITEM_FULL = 22, ITEM_EMPTY = 26, N_BARS = 30 };
  auto bar = [&](int i) { return bar0 + 8u * i; };
  uint8_t* misc = gen + (bar0 - base) + 8 * N_BARS;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 4);
  RowsItem* s_item = reinterpret_cast<RowsItem*>(misc + 16);   // [RW_SLOTS]; guarded by ITEM_FULL and ITEM_EMPTY
  const PageView& pv = p.pv;

  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(K_FULL + s), 1); mbar_init(bar(K_EMPTY + s), 1);
      mbar_init(bar(V_FULL + s), 1); mbar_init(bar(V_OK + s), 2); mbar_init(bar(V_EMPTY + s), 1);
      mbar_init(bar(Q_FULL + s), 4); mbar_init(bar(S_FULL + s), 1); mbar_init(bar(P_HALF + s), 4); mbar_init(bar(P_FULL + s), 4);
      mbar_init(bar(O_FULL + s), 1); mbar_init(bar(O_EMPTY + s), 4);
    }
    for (int s = 0; s < RW_SLOTS; ++s) { mbar_init(bar(ITEM_FULL + s), 1); mbar_init(bar(ITEM_EMPTY + s), 1 + 2 + 8); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_launch_dependents();   // (in this order: rows_join_kernel looks at the lists and lengths before its own wait)

  const int pack = PACK ? p.pack : 1, heads = p.a.heads / pack;   // an item is one of `heads`
  const int window = p.a.window, sinks = p.a.sinks, group = heads / pv.H, box_log2 = min(pv.ps_log2, 6), per_chunk = RW_KEYS >> box_log2;
  auto wait_warp = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(b, parity, abort_flag, pv.status)) != 0; };
  // item k of this CTA is in its slot, for the warps that are told: false when the wait gave up
  auto next_item = [&](int k) { return wait_warp(bar(ITEM_FULL + (k & 3)), (uint32_t)((k >> 2) & 1)); };
  auto release_item = [&](int k) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(ITEM_EMPTY + (k & 3)));
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 120;");
    if (warp == 0) {
      // ===================== producer: what comes next, and K and V by TMA (lane = (box, half) of the chunk) =====================
      const int n = p.rows.n;
      RowsEntries<RW_ROWS> e;
      int total = 0;   // pairs of tiles of all entries
      for (int i0 = 0; i0 < n; i0 += 32) {
        e.look_up(pv, p.rows, pack, i0);
        total += __reduce_add_sync(0xffffffffu, e.tiles);
        if (blockIdx.x == 0 && (e.m > p.rows.max_rows || (e.m > 0 && e.seq < 0))) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);   // cannot be answered
      }
      const int split = SPLIT ? split_of((long long)total * heads, p.grid) : 1;
      const long long pool_rows = (long long)pv.n_layers * 2 * pv.n_pages * pv.H * pv.ps, plane_rows = (long long)pv.n_pages * pv.H * pv.ps;
      const int box = lane / HALVES, half = lane - box * HALVES;
      const uint32_t place = (uint32_t)(half * RW_BLOCK + ((box << box_log2) * 128));
      bool ok = true;
      uint32_t g = 0;   // chunks of K and V so far
      // works out item k of this CTA and publishes it; the pairs are handed out last first: later rows of a sequence have more keys
      auto publish = [&](int k) {
        const long long index = SPLIT && split > 1 ? (k == 0 ? blockIdx.x / split : (long long)total * heads) : blockIdx.x + (long long)k * gridDim.x;
        const int slot = index < (long long)total * heads ? total - 1 - (int)(index / heads) : -1;
        RowsItem it{};
        it.head = -1;
        if (slot >= 0 && e.find(pv, p.rows, pack, slot, it)) {
          plan_rows(it, window, sinks, box_log2, pack);
          if (!SPLIT || cut_keys(it, split, blockIdx.x)) it.head = (int)(index % heads);
        }
        if (k >= RW_SLOTS && !(ok = wait_warp(bar(ITEM_EMPTY + (k & 3)), (uint32_t)(((k >> 2) & 1) ^ 1)))) return;
        if (lane == 0) {
          s_item[k & 3] = it;
          mbar_arrive(bar(ITEM_FULL + (k & 3)));
        }
        __syncwarp();
      };
      publish(0);
      for (int k = 0; ok; ++k) {
        if (s_item[k & 3].head < 0) break;
        publish(k + 1);
        if (!ok) break;
        const RowsItem it = s_item[k & 3];
        const int kv_head = it.head / group;
        const bool mine = box < per_chunk;
        auto row_of = [&](int c, int which) -> int {   // row of the pool at which this lane's box begins
          const int key = it.base(c * per_chunk + box, box_log2);
          if (!mine || key >= it.end) return (int)pool_rows;   // (behind the pool's last row the copy fills in zeros)
          const int page = pv.table[(size_t)it.seq * pv.max_pages + (key >> pv.ps_log2)];
          if ((unsigned)page >= (unsigned)pv.n_pages) {   // trimmed, or bad: reported where a row sees something of it
            if (key + (1 << box_log2) > it.start || key < it.sinks) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
            return (int)pool_rows;
          }
          return (int)((((long long)p.a.layer * 2 * pv.n_pages + page) * pv.H + kv_head) * pv.ps + (key & (pv.ps - 1)) + which * plane_rows);
        };
        auto load = [&](uint32_t dst, uint32_t b, int row) {
          if (lane == 0) mbar_expect_tx(b, TILE);
          __syncwarp();
          if (mine) tma_load_2d(dst + place, &map, b, half * 64, row);
        };
        auto load_k = [&](int c, int row) {
          const uint32_t x = g + c, s = x & 1;
          if (x >= 2 && !(ok = wait_warp(bar(K_EMPTY + s), ((x >> 1) & 1) ^ 1u))) return;
          load(sK + s * TILE, bar(K_FULL + s), row);
        };
        g -= it.template begin<SPLIT>();   // (chunk c of the item is chunk g + c of the CTA)
        if (it.template end_chunk<SPLIT>() > it.template begin<SPLIT>()) load_k(it.template begin<SPLIT>(), row_of(it.template begin<SPLIT>(), 0));
        for (int c = it.template begin<SPLIT>(); c < it.template end_chunk<SPLIT>() && ok; ++c) {   // K a chunk ahead of V: its slot comes free earlier
          const uint32_t x = g + c, s = x & 1;
          const int vrow = row_of(c, 1), krow = c + 1 < it.template end_chunk<SPLIT>() ? row_of(c + 1, 0) : 0;
          if (c + 1 < it.template end_chunk<SPLIT>()) load_k(c + 1, krow);
          if (!ok) break;
          if (x >= 2 && !(ok = wait_warp(bar(V_EMPTY + s), ((x >> 1) & 1) ^ 1u))) break;
          load(sV + s * TILE, bar(V_FULL + s), vrow);
        }
        g += it.template end_chunk<SPLIT>();
      }
      if (!ok || *abort_flag) {   // copies already issued land before the CTA's shared memory is given back
        const unsigned long long t0 = now_ns();
        while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
      }
    } else if (warp == 1) {
      // ===================== MMA =====================
      uint32_t leader;
      asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\tselp.u32 %0, 1, 0, P;\n\t}" : "=r"(leader));
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(RW_TILE >> 4) << 24);
      const uint32_t idesc_qk = idesc | ((uint32_t)(RW_KEYS >> 3) << 17), idesc_pv = idesc | (1u << 16) | ((uint32_t)(HD >> 3) << 17);
      uint32_t g = 0, np_a = 0, np_b = 0, ni_a = 0, ni_b = 0;   // chunks; chunks and items that a tile has worked on
      bool ok = true;
      for (int k = 0; ok; ++k) {
        if (!next_item(k) || s_item[k & 3].head < 0) break;
        const RowsItem it = s_item[k & 3];
        auto issue_qk = [&](int tile, int c) {
          if (c == it.template from<SPLIT>(tile)) {   // the tile's first of this item
            if (!wait_warp(bar(Q_FULL + tile), (tile ? ni_b : ni_a) & 1)) return false;
            tc_fence_after();
          }
          const uint64_t qd = desc_kmajor(sQ + (uint32_t)tile * TILE), kd = desc_kmajor(sK + ((g + c) & 1) * TILE);
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
              const uint64_t off = (uint64_t)(((uint32_t)(kk >> 2) * RW_BLOCK + (uint32_t)(kk & 3) * 32u) >> 4);
              umma_bf16(tmem + (uint32_t)tile * 128u, qd + off, kd + off, idesc_qk, kk > 0 ? 1u : 0u);
            }
            umma_commit(bar(S_FULL + tile));
          }
          __syncwarp();
          return true;
        };
        g -= it.template begin<SPLIT>();
        if (it.template end_chunk<SPLIT>() > it.template begin<SPLIT>()) {
          const uint32_t x = g + it.template begin<SPLIT>();
          if (!(ok = wait_warp(bar(K_FULL + (x & 1)), (x >> 1) & 1))) break;
          tc_fence_after();
          for (int tile = 0; tile < 2 && ok; ++tile)
            if (it.template active<SPLIT>(tile, it.template begin<SPLIT>())) ok = issue_qk(tile, it.template begin<SPLIT>());
          if (!ok) break;
          if (leader) umma_commit(bar(K_EMPTY + (x & 1)));
          __syncwarp();
        }
        for (int c = it.template begin<SPLIT>(); c < it.template end_chunk<SPLIT>() && ok; ++c) {
          const uint32_t x = g + c, s = x & 1;
          if (!(ok = wait_warp(bar(V_OK + s), (x >> 1) & 1))) break;   // V, and the next chunk's K
#pragma unroll
          for (int tile = 0; tile < 2; ++tile) {
            if (it.template active<SPLIT>(tile, c)) {
              const uint64_t vd = desc_mnmajor_v(sV + s * TILE);
              const uint32_t ni = tile ? ni_b : ni_a;
              if (c == it.template from<SPLIT>(tile) && ni > 0 && !(ok = wait_warp(bar(O_EMPTY + tile), (ni - 1) & 1))) break;   // the output before has been read
              for (int hf = 0; hf < 2; ++hf) {   // the weights come in two halves
                if (!(ok = wait_warp(bar((hf ? P_FULL : P_HALF) + tile), (tile ? np_b : np_a) & 1))) break;
                tc_fence_after();
                if (leader) {
#pragma unroll
                  for (int kk = 0; kk < RW_KEYS / 32; ++kk)
                    umma_bf16_ts(tmem + 256u + (uint32_t)tile * 128u, tmem + (uint32_t)tile * 128u + (uint32_t)(hf * 4 + kk) * 8u,
                                 vd + (uint64_t)((hf * 4 + kk) * 128), idesc_pv, (c > it.template from<SPLIT>(tile) || hf > 0 || kk > 0) ? 1u : 0u);
                  if (hf && c + 1 == it.to(tile)) umma_commit(bar(O_FULL + tile));
                }
                __syncwarp();
              }
              if (!ok) break;
              ++(tile ? np_b : np_a);
              if (c + 1 == it.to(tile)) ++(tile ? ni_b : ni_a);
            }
            if (c + 1 < it.template end_chunk<SPLIT>() && it.template active<SPLIT>(tile, c + 1) && !(ok = issue_qk(tile, c + 1))) break;
          }
          if (!ok) break;
          if (leader) {
            umma_commit(bar(V_EMPTY + s));
            if (c + 1 < it.template end_chunk<SPLIT>()) umma_commit(bar(K_EMPTY + (s ^ 1)));
          }
          __syncwarp();
        }
        g += it.template end_chunk<SPLIT>();
        release_item(k);
      }
    } else {
      // ===================== V: zeros where no row looks, a look at what only some rows see =====================
      const int t = threadIdx.x - 64, t_key = t >> 3;   // 8 threads a key and half, 8 keys at a time
      uint32_t g = 0;
      bool ok = true;
      for (int k = 0; ok; ++k) {
        if (!next_item(k) || s_item[k & 3].head < 0) break;
        const RowsItem it = s_item[k & 3];
        g -= it.template begin<SPLIT>();
        for (int c = it.template begin<SPLIT>(); c < it.template end_chunk<SPLIT>(); ++c) {
          const uint32_t x = g + c, s = x & 1;
          const bool all = c >= it.all_from_b && c < it.all_to_a;   // every row of the CTA sees all of the chunk
          if (!(ok = wait_warp(bar(V_FULL + s), (x >> 1) & 1))) break;
          if (!all) {
            uint32_t bad = 0;   // bits 15 and 31: an exponent of all ones among what was looked at
            uint8_t* at0 = gen + (sV - base) + s * TILE + t * 16;
            auto place = [&](int gr, int e) { return reinterpret_cast<uint4*>(at0 + (e >> 1) * RW_BLOCK + gr * 2048 + (e & 1) * 1024); };
#pragma unroll 2
            for (int gr = 0; gr < 8; ++gr) {   // sixteen keys, which lie in one box
              const int b0 = it.base(c * per_chunk + ((gr * 16) >> box_log2), box_log2), k0 = b0 + ((gr * 16) & ((1 << box_log2) - 1));
              if (b0 >= it.end) continue;    // (a box that has not been loaded: zeros)
              uint4 v[2 * HALVES];
#pragma unroll
              for (int e = 0; e < 2 * HALVES; ++e) v[e] = *place(gr, e);
              auto look = [&](const uint4& x) {
                bad |= ((x.x & 0x7fff7fffu) + 0x00800080u) | ((x.y & 0x7fff7fffu) + 0x00800080u) | ((x.z & 0x7fff7fffu) + 0x00800080u) |
                       ((x.w & 0x7fff7fffu) + 0x00800080u);
              };
              if (k0 + 16 <= it.end && (k0 + 16 <= it.sinks || k0 >= it.start)) {
#pragma unroll
                for (int e = 0; e < 2 * HALVES; ++e) look(v[e]);
              } else {
#pragma unroll
                for (int e = 0; e < 2 * HALVES; ++e) {
                  const int key = k0 + t_key + (e & 1) * 8;
                  if (key >= it.end || (key >= it.sinks && key < it.start)) *place(gr, e) = make_uint4(0u, 0u, 0u, 0u);
                  else look(v[e]);
                }
              }
            }
            const bool unclean = (bad & 0x80008000u) != 0;
            if (unclean) *reinterpret_cast<volatile int*>(&s_item[k & 3].unclean) = 1;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          // (the next chunk's K is waited for here: the MMA warp has no time to spare)
          if (c + 1 < it.template end_chunk<SPLIT>() && !(ok = wait_warp(bar(K_FULL + (s ^ 1)), ((x + 1) >> 1) & 1))) break;
          __syncwarp();   // (all lanes' zeros and looks before the one arrival)
          if (lane == 0) mbar_arrive(bar(V_OK + s));
        }
        g += it.template end_chunk<SPLIT>();
        release_item(k);
      }
    }
  } else {
    // ===================== softmax and output: one thread a row =====================
    asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
    const int tile = (warp - 4) >> 2, w4 = warp & 3;   // (a warp may touch the lane quarter warp mod 4 of tensor memory)
    const int t = w4 * 32 + lane;
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16;
    const uint32_t s_addr = tmem + lanes + (uint32_t)tile * 128u, o_addr = s_addr + 256u;
    const float scale2 = p.a.scale * LOG2E;
    const uint64_t scale22 = pair(scale2, scale2);
    // place x of an item: its row of the call (after row0) and query head (after head * pack)
    auto row_of = [&](int x) { return PACK ? x / pack : x; };
    auto sub_of = [&](int x) { return PACK ? x % pack : 0; };
    // the tile's Q, K-major and swizzled: 16-byte piece c of row r lies at piece c ^ (r & 7) of its 128 bytes.  A tile's Q may be
    // overwritten once the scores of its last chunk have been seen.
    auto load_q = [&](const RowsItem& x) {
      constexpr int PIECES = HD / 8, ROWS_PASS = 32 / PIECES;
      const int piece = lane % PIECES, rows = x.n_rows - tile * RW_TILE, r0 = w4 * 32 + lane / PIECES;
      const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.a.q) + (long long)(x.row0 + (PACK ? 0 : tile * RW_TILE)) * p.a.q_stride + (long long)x.head * pack * HD + piece * 8;
      const uint32_t dst = sQ + tile * TILE + (piece >> 3) * RW_BLOCK;
#pragma unroll 4
      for (int i = 0; i < 32 / ROWS_PASS; ++i) {
        const int r = r0 + i * ROWS_PASS;
        const int at = PACK ? tile * RW_TILE + (r < rows ? r : 0) : r < rows ? r : 0;
        cp_async16(dst + r * 128 + (((piece & 7) ^ (r & 7)) << 4), q + (long long)row_of(at) * p.a.q_stride + sub_of(at) * HD, r < rows);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto q_loaded = [&]() {
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(Q_FULL + tile));
    };
    uint32_t n_s = 0, n_item = 0;   // chunks and items that the tile has worked on
    bool ok = next_item(0), more = ok && s_item[0].head >= 0;
    if (more && s_item[0].template has<SPLIT>(tile)) { load_q(s_item[0]); q_loaded(); }
    for (int k = 0; ok && more; ++k) {
      const RowsItem& it = s_item[k & 3];
      const int head = it.head, from = it.template from<SPLIT>(tile), to = it.to(tile), first = it.first, skew = it.skew;
      const int t_rows = min(RW_TILE, it.n_rows - tile * RW_TILE);   // rows of the tile, <= 0: none
      const bool valid = t < t_rows, has = to > from;
      const int place0 = PACK ? tile * RW_TILE : 0, row0 = it.row0 + (PACK ? 0 : tile * RW_TILE), pos0 = it.pos0 + (PACK ? 0 : tile * RW_TILE);
      const int all_from = tile ? it.all_from_b : it.all_from, all_to = tile ? it.all_to_b : it.all_to_a;
      const int pos = valid ? pos0 + row_of(place0 + t) : -1, lo = window > 0 ? pos - window + 1 : 0;   // sees [lo, pos] and the sinks
      float m = -INFINITY, l = 0.f;
      bool next_q = false;
      auto look_ahead = [&]() {   // what comes next, and its Q on the way
        if (!next_item(k + 1)) return false;
        const RowsItem& next = s_item[(k + 1) & 3];
        more = next.head >= 0;
        next_q = more && next.template has<SPLIT>(tile);
        if (next_q) load_q(next);
        return true;
      };
      for (int c = from; c < to; ++c, ++n_s) {
        const bool all = c >= all_from && c < all_to;   // every row of the tile sees all of the chunk
        if (!(ok = wait_warp(bar(S_FULL + tile), n_s & 1))) break;
        tc_fence_after();
        if (c + 1 == to && !(ok = look_ahead())) break;   // the tile's last scores: its Q is free
        float sc[RW_KEYS];
#pragma unroll
        for (int g = 0; g < RW_KEYS / 32; ++g) tmem_ld32_nowait(s_addr + g * 32, sc + g * 32);
        tmem_ld_wait();
        if (!all) {
          uint32_t seen[RW_KEYS / 32];
          const int b0 = c << (7 - box_log2);
          if (b0 >= first) {   // the window's part: one run of keys
            const int k0 = (b0 + skew) << box_log2, x0 = lo - k0, x1 = pos + 1 - k0, x2 = sinks - k0;
#pragma unroll
            for (int g = 0; g < RW_KEYS / 32; ++g) seen[g] = low_bits(x1 - 32 * g) & (~low_bits(x0 - 32 * g) | low_bits(x2 - 32 * g));
          } else {
#pragma unroll
            for (int g = 0; g < RW_KEYS / 32; ++g) seen[g] = 0;
#pragma unroll 1
            for (int e = 0; e < RW_KEYS / 16; ++e) {   // sixteen keys lie in one box
              const int at = e * 16, k0 = it.base(b0 + (at >> box_log2), box_log2) + (at & ((1 << box_log2) - 1));
              const uint32_t w = (low_bits(pos + 1 - k0) & (~low_bits(lo - k0) | low_bits(sinks - k0)) & 0xffffu) << (16 * (e & 1));
#pragma unroll
              for (int g = 0; g < RW_KEYS / 32; ++g) seen[g] |= g == e >> 1 ? w : 0u;
            }
          }
#pragma unroll
          for (int g = 0; g < RW_KEYS / 32; ++g) {
            if (__all_sync(0xffffffffu, seen[g] == 0xffffffffu)) continue;
#pragma unroll
            for (int j = 0; j < 32; ++j) sc[g * 32 + j] = ((seen[g] >> j) & 1u) ? sc[g * 32 + j] : -INFINITY;
          }
        }
        float mx4[4] = {sc[0], sc[1], sc[2], sc[3]};
#pragma unroll
        for (int j = 4; j + 8 <= RW_KEYS; j += 8) {
#pragma unroll
          for (int i = 0; i < 4; ++i) mx4[i] = max3(mx4[i], sc[j + i], sc[j + 4 + i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) mx4[i] = fmaxf(mx4[i], sc[RW_KEYS - 4 + i]);
        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * scale2;
        const bool moves = mx > m + RW_SLACK || (m == -INFINITY && mx > m);
        if (__any_sync(0xffffffffu, moves)) {
          const float corr = !moves ? 1.f : fast_exp2(m - mx);
          if (moves) m = mx;
          l *= corr;
          if (c > from) {   // the tile's earlier products are complete (its scores were issued behind them)
#pragma unroll 1
            for (int g = 0; g < HD / 16; ++g) {   // (sixteen at a time: the row's scores take the registers)
              uint32_t ov[16];
              tmem_ld16(o_addr + g * 16, ov);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) ov[j] = __float_as_uint(__uint_as_float(ov[j]) * corr);
              tmem_st16_u32(o_addr + g * 16, ov);
            }
          }
        }
        const float ref = m == -INFINITY ? 0.f : m;
        const uint64_t neg = pair(-ref, -ref);
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          uint32_t pk[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            float a, b;
            unpair(fma2(pair(sc[g * 64 + 2 * j], sc[g * 64 + 2 * j + 1]), scale22, neg), a, b);
            a = fast_exp2(a); b = fast_exp2(b);
            sum[j & 1] = add2(sum[j & 1], pair(a, b));
            pk[j] = pack_bf16(a, b);
          }
          tmem_st32_u32(s_addr + g * 32, pk);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar((g ? P_FULL : P_HALF) + tile));
        }
        float s0, s1;
        unpair(add2(sum[0], sum[1]), s0, s1);
        l += s0 + s1;
      }
      if (!ok) break;
      if (!has && !(ok = look_ahead())) break;
      if (next_q) q_loaded();   // the next scores are worked on while this output is finished
      if (has && !(ok = wait_warp(bar(O_FULL + tile), n_item & 1))) break;
      const bool unclean = *reinterpret_cast<volatile int*>(&s_item[k & 3].unclean) != 0;
      const int part = SPLIT ? it.part : -1;
      if (t_rows > 0 && part >= 0) {   // for rows_join_kernel
        float* mine = p.parts + (size_t)part * rows_part_floats<HD>();
        if (has && !unclean) {
          tc_fence_after();
#pragma unroll 1
          for (int g = 0; g < HD / 16; ++g) {
            uint32_t ov[16];
            tmem_ld16(o_addr + g * 16, ov);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 4; ++j)
              reinterpret_cast<uint4*>(mine)[(g * 4 + j) * RW_ROWS + tile * RW_TILE + t] = make_uint4(ov[4 * j], ov[4 * j + 1], ov[4 * j + 2], ov[4 * j + 3]);
          }
        }
        reinterpret_cast<float2*>(mine + RW_ROWS * HD)[tile * RW_TILE + t] = make_float2(m, unclean ? __uint_as_float(0x7fffffffu) : l);
      }
      if (t_rows > 0 && part < 0 && !unclean) {
        tc_fence_after();
        const float inv = l == 0.f ? 0.f : 1.f / l;
        // through shared memory, so that a store covers 128 bytes of each of four rows (16 bytes of 32 rows cost 9000 cycles a tile)
        uint8_t* mine = gen + (sO - base) + (warp - 4) * RW_STAGE_OUT;
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.a.out) + (long long)(row0 + (PACK ? 0 : w4 * 32)) * p.a.out_stride + (long long)head * pack * HD + (lane & 7) * 8;
#pragma unroll 1
        for (int g = 0; g < HD / 64; ++g) {   // (short loops: this code runs once an item, and what it costs is its fetch)
#pragma unroll 1
          for (int h = 0; h < 4; ++h) {
            uint32_t ov[16];
            if (has) {
              tmem_ld16(o_addr + g * 64 + h * 16, ov);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int j = 0; j < 16; ++j) ov[j] = 0u;
            }
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = pack_bf16(__uint_as_float(ov[2 * j]) * inv, __uint_as_float(ov[2 * j + 1]) * inv);
#pragma unroll
            for (int j = 0; j < 2; ++j)
              *reinterpret_cast<uint4*>(mine + lane * 128 + (((h * 2 + j) ^ (lane & 7)) << 4)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
          }
          __syncwarp();
#pragma unroll 4
          for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + (lane >> 3);
            const int at = PACK ? place0 + w4 * 32 + r : r;
            if (w4 * 32 + r < t_rows)
              *reinterpret_cast<uint4*>(out + (long long)row_of(at) * p.a.out_stride + sub_of(at) * HD + g * 64) = *reinterpret_cast<const uint4*>(mine + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
          }
          __syncwarp();
        }
        if (valid && p.a.lse) p.a.lse[(long long)(row0 + row_of(place0 + t)) * p.a.heads + head * pack + sub_of(place0 + t)] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
      }
      if (has) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(O_EMPTY + tile));
        ++n_item;
      }
      if (t_rows > 0 && part < 0 && unclean) {
        for (int x = w4 * 32; x < min(t_rows, w4 * 32 + 32); ++x) {   // (rare) the warp's rows, one after another
          const long long row = row0 + row_of(place0 + x);
          const int mine = head * pack + sub_of(place0 + x);
          float q[HD / 32], o[HD / 32], rm = -INFINITY, rl = 0.f;
#pragma unroll
          for (int d = 0; d < HD / 32; ++d) o[d] = 0.f;
          load_dims(reinterpret_cast<const __nv_bfloat16*>(p.a.q) + row * p.a.q_stride + (long long)mine * HD + lane * (HD / 32), q);
          if (pos0 + row_of(place0 + x) >= 0)
            attend_row_warp<__nv_bfloat16, HD>(pv, p.a.layer, pv.table + (size_t)it.seq * pv.max_pages, head / group, pos0 + row_of(place0 + x), window, sinks, scale2, q,
                                               o, &rm, &rl);
          store_row_warp<__nv_bfloat16, HD>(p.a, row, mine, o, rm, rl);
        }
      }
      release_item(k);
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

// The parts of items whose keys several CTAs shared: grid (item, 32 of its rows), a thread a row and four of its dimensions at a time.
constexpr int JOIN_THREADS = 256;

template <int HD>
__global__ void __launch_bounds__(JOIN_THREADS) rows_join_kernel(const RowsParams p) {
  constexpr int WARPS = JOIN_THREADS / 32, PER = HD / 4 / WARPS, PITCH = HD + 8;
  __shared__ __align__(16) __nv_bfloat16 s_out[32 * PITCH];
  __shared__ uint32_t s_alone;
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PageView& pv = p.pv;
  const int window = p.a.window, sinks = p.a.sinks, pack = p.pack, heads = p.a.heads / pack;
  RowsEntries<RW_ROWS> e;
  int total = 0;
  for (int i0 = 0; i0 < p.rows.n; i0 += 32) {
    e.look_up(pv, p.rows, pack, i0);
    total += __reduce_add_sync(0xffffffffu, e.tiles);
  }
  RowsItem it{};
  if ((long long)blockIdx.x < (long long)total * heads && e.find(pv, p.rows, pack, total - 1 - (int)(blockIdx.x / heads), it))
    plan_rows(it, window, sinks, min(pv.ps_log2, 6), pack);   // (else no rows)
  pdl_wait();
  const int split = split_of((long long)total * heads, p.grid), n = parts_of(it, split), head0 = (int)(blockIdx.x % heads) * pack, x0 = blockIdx.y * 32, here = min(32, it.n_rows - x0);
  if (n == 1 || here <= 0) return;   // (written by the one CTA that worked on it)
  const int x = x0 + lane;
  const float* part0 = p.parts + (size_t)blockIdx.x * split * rows_part_floats<HD>();
  float m[RW_MAX_SPLIT], M = -INFINITY, L = 0.f;
#pragma unroll
  for (int s = 0; s < RW_MAX_SPLIT; ++s) {
    const float2 st = s < n && lane < here ? reinterpret_cast<const float2*>(part0 + (size_t)s * rows_part_floats<HD>() + RW_ROWS * HD)[x] : make_float2(-INFINITY, 0.f);
    m[s] = st.y == 0.f ? -INFINITY : st.x;   // (no key of the part: nothing has been left)
    M = fmaxf(M, m[s]);
  }
  const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
  for (int s = 0; s < RW_MAX_SPLIT; ++s) {
    const float l = s < n && lane < here ? reinterpret_cast<const float2*>(part0 + (size_t)s * rows_part_floats<HD>() + RW_ROWS * HD)[x].y : 0.f;
    const float f = l == 0.f ? 0.f : fast_exp2(m[s] - ref);
    L = fmaf(f, l, L);
    m[s] = f;
  }
  const uint32_t alone = __ballot_sync(0xffffffffu, L != L);   // rows that see NaN or infinities, or whose part met some
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int g = warp * PER + k;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int s = 0; s < RW_MAX_SPLIT; ++s) {
      if (s < n && m[s] != 0.f && lane < here) {
        const float4 o = reinterpret_cast<const float4*>(part0 + (size_t)s * rows_part_floats<HD>())[g * RW_ROWS + x];
        v.x = fmaf(m[s], o.x, v.x); v.y = fmaf(m[s], o.y, v.y); v.z = fmaf(m[s], o.z, v.z); v.w = fmaf(m[s], o.w, v.w);
      }
    }
    *reinterpret_cast<uint2*>(&s_out[lane * PITCH + g * 4]) = make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
  }
  if (threadIdx.x == 0) s_alone = alone;
  __syncthreads();
  constexpr int PIECES = HD / 8;
  for (int i = threadIdx.x; i < here * PIECES; i += JOIN_THREADS) {
    const int r = i / PIECES, c = i - r * PIECES;
    if ((s_alone >> r) & 1u) continue;
    *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.a.out) + (long long)(it.row0 + (x0 + r) / pack) * p.a.out_stride + (long long)(head0 + (x0 + r) % pack) * HD + c * 8) =
        *reinterpret_cast<const uint4*>(&s_out[r * PITCH + c * 8]);
  }
  if (warp == 0 && lane < here && p.a.lse && !((alone >> lane) & 1u))
    p.a.lse[(long long)(it.row0 + x / pack) * p.a.heads + head0 + x % pack] = L == 0.f ? -INFINITY : (M + log2f(L)) * LN2;
  for (int r = warp; r < here; r += WARPS) {
    if (!((alone >> r) & 1u)) continue;
    const int token = (x0 + r) / pack, head = head0 + (x0 + r) % pack;
    const long long row = it.row0 + token;
    float q[HD / 32], o[HD / 32], rm = -INFINITY, rl = 0.f;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) o[d] = 0.f;
    load_dims(reinterpret_cast<const __nv_bfloat16*>(p.a.q) + row * p.a.q_stride + (long long)head * HD + lane * (HD / 32), q);
    if (it.pos0 + token >= 0)
      attend_row_warp<__nv_bfloat16, HD>(pv, p.a.layer, pv.table + (size_t)it.seq * pv.max_pages, head / (p.a.heads / pv.H), it.pos0 + token, window, sinks,
                                         p.a.scale * LOG2E, q, o, &rm, &rl);
    store_row_warp<__nv_bfloat16, HD>(p.a, row, head, o, rm, rl);
  }
}

}  // namespace

size_t pages_rows_part_bytes(const PageView& pv, int grid) {
  return pv.es == 2 ? (size_t)grid * (pv.hd == 64 ? rows_part_floats<64>() : rows_part_floats<128>()) * 4 : 0;
}

// Calls f(kernel, shared memory) for each form of the kernel.
template <typename F> static cudaError_t for_rows_kernels(int hd, F f) {
  cudaError_t e = cudaSuccess;
  auto forms = [&](auto hd_c) {
    constexpr int HD = decltype(hd_c)::value;
    e = f(false, false, pages_rows_kernel<HD, false, false>, rows_smem<HD>());
    if (e == cudaSuccess) e = f(true, false, pages_rows_kernel<HD, true, false>, rows_smem<HD>());
    if (e == cudaSuccess) e = f(false, true, pages_rows_kernel<HD, false, true>, rows_smem<HD>());
    if (e == cudaSuccess) e = f(true, true, pages_rows_kernel<HD, true, true>, rows_smem<HD>());
  };
  hd == 64 ? forms(std::integral_constant<int, 64>{}) : forms(std::integral_constant<int, 128>{});
  return e;
}

cudaError_t pages_rows_prepare(int hd) {
  return for_rows_kernels(hd, [](bool, bool, auto kernel, size_t smem) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
}

// map: the pool as [rows][head_dim], boxes of min(page_size, 64) rows and 64 columns.  parts: pages_rows_part_bytes.  sms: CTAs at most.
cudaError_t launch_pages_rows(const void* map, const PageView& pv, const PageRows& rows, const PageAttention& a, void* parts, int sms, int* launches,
                              cudaStream_t st) {
  RowsParams p;
  p.pv = pv; p.rows = rows; p.a = a; p.parts = (float*)parts;
  const long long rows_most = rows.max_rows < rows.n_rows ? rows.max_rows : rows.n_rows;   // rows of an entry that is answered
  const int group = a.heads / pv.H;
  p.pack = group > 1 && rows_most * group <= RW_ROWS ? group : 1;
  const int heads = a.heads / p.pack;
  // items at most, and about (their number stands on the device; with fewer, the form that does not share answers as well)
  const long long most = p.pack > 1 ? (long long)rows.n * heads : (rows.n_rows + (long long)(RW_ROWS - 1) * rows.n) / RW_ROWS * heads;
  const long long filled = ((long long)rows.n_rows * p.pack + RW_ROWS - 1) / RW_ROWS, about = (filled > rows.n ? filled : rows.n) * heads;
  const bool split = about * 2 <= sms, pack = p.pack > 1;
  // (no more CTAs than can share: rows_join_kernel's begin beside them on SMs that are left, 1.5 us)
  const long long ctas = split && most * 2 <= sms ? most * (sms / most < RW_MAX_SPLIT ? sms / most : RW_MAX_SPLIT) : split ? sms : most;
  p.grid = (int)(ctas < sms ? ctas : sms);
  const cudaError_t e = for_rows_kernels(pv.hd, [&](bool split_form, bool pack_form, auto kernel, size_t smem) {
    if (pack_form != pack || split_form != split) return cudaSuccess;
    launch_pdl(kernel, p.grid, RW_THREADS, smem, st, *(const CUtensorMap*)map, p);
    ++*launches;
    return cudaGetLastError();
  });
  if (e || !split) return e;
  const dim3 join((unsigned)(most < p.grid / 2 ? most : p.grid / 2), (unsigned)(rows_most * p.pack < RW_ROWS ? (rows_most * p.pack + 31) / 32 : RW_ROWS / 32));
  if (join.x == 0) return e;
  if (pv.hd == 64) launch_pdl(rows_join_kernel<64>, join, JOIN_THREADS, 0, st, p);
  else launch_pdl(rows_join_kernel<128>, join, JOIN_THREADS, 0, st, p);
  ++*launches;
  return cudaGetLastError();
}

}  // namespace rd
