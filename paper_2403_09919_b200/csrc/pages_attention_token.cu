// Attention of one new token per sequence over a cache in pages: the keys are split evenly over the SMs and the parts
// joined in the same launch.
//
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(scale log2(e) q . k_j - m),  m the running maximum
//
// The cache's stream bounds it (every visible K and V is read once, for all query heads of its key and value head), so the
// design is about keeping that stream full whatever the lengths are:
//   - The work is a line of units: chunks of 64 keys, for each sequence and key and value head (and, beyond 16 query heads on
//     one of those, each 16 of them: an "item").  CTA c of G takes the units [T c / G, T (c + 1) / G), wherever sequences
//     begin and end; the line is worked out on the device from the lengths, so nothing has to be planned on the host.
//   - A producer warp copies chunks by TMA, a page's rows at a time, into a ring of six stages of 32 KB that runs ahead over
//     the ends of items: while a part is joined and written, the stream goes on.
//   - Four warps take 16 keys of every chunk each, on their own: scores by mma (16 query rows; a single token has few rows,
//     so the tensor cores are nowhere near their rate), running maximum and sum per row, V by ldmatrix.trans.  Weights go in two
//     bf16 parts, as in attention_kl.cu, which serves single tokens on the contiguous cache; the second takes the tile's rows 8 to 15
//     where up to 8 query heads leave them free, and products of its own beyond.
//     What the warps hold is joined in shared memory at the end of an item.
//   - An item that crosses CTAs leaves its parts (unscaled output, maximum, sum, fp32) in the workspace; the last CTA to
//     arrive joins them in the order of the CTAs, so that the result does not depend on who is last.
// Measured with the write of the tokens' K and V before it (a launch of its own, 4 us of these): 16 sequences, 296 MB of K and V,
// 62.2 us (4.8 TB/s); 1.29 GB 207 us (6.2 TB/s, 0.95 of a copy); a window of 254 MB 53.5 us; one sequence of 900 tokens (14.8 MB)
// 10.1 us, a chain of latencies: the write's, three looks into the tables, a page's copy, the products, the join.
// Keys outside the row's sight are masked by selection and their V is replaced by zeros bit by bit: they may hold anything.
#include <cuda.h>

#include <type_traits>

#include "pages_attention.cuh"
#include "pdl.cuh"
#include "tcgen05.cuh"

namespace rd {

namespace {

constexpr int TK_KEYS = 64;          // keys of a chunk
constexpr int TK_WARPS = 4;          // consumer warps, 16 keys each
constexpr int TK_THREADS = TK_WARPS * 32 + 32;
constexpr int TK_STAGES = 6;
// Units that a CTA takes at least where an item is cut, and chunks of an item that is not: the more rows a part has, the longer the
// join of many (900 tokens of 32 heads: 8.5 us with 3, 9.2 with 4, 10.0 with 6; 16 query heads on one, 16384 tokens: 28.3 with 6, 22.6
// with 10, 40000: 55.8 and 39.2, but 16 sequences of 2000: 14.8 and 18.2; fp32, whose chunks take longer, 1000 tokens of 4 heads: 7.8 with
// 1, 10.7 with 3).
constexpr int TK_MIN_UNITS = 3, TK_MIN_UNITS_WIDE = 10, TK_WHOLE = 10;
constexpr int TK_JOIN = 8, TK_REST = 2;   // parts that a thread of the join has under way; parts left that it takes one by one

struct TokenParams {
  PageView pv;
  PageRows rows;
  PageAttention a;
  int group, tiles;     // query heads per key and value head; tiles of 16 of them
  float* parts;         // [grid][2][16][HD + 4]: unscaled output, maximum, sum
  int32_t* arrived;     // [grid], zero between launches
};

// The chunks of one entry: the ones that hold sinks, then those from the window's first key on.
struct Span {
  int len, start, sink_end, sink_chunks, first_chunk, chunks;
};

__device__ __forceinline__ Span span_of(const TokenParams& p, int i, int* seq, int* row) {
  Span s;
  int first, m;
  page_rows_of(p.rows, i, &first, &m);
  *row = first;
  *seq = page_seq_of(p.pv, p.rows.seqs, i);
  s.len = *seq >= 0 ? page_len_of(p.pv, *seq) : 0;
  visible_keys(s.len - 1, p.a.window, p.a.sinks, &s.sink_end, &s.start);
  s.first_chunk = s.start / TK_KEYS;
  s.sink_chunks = min((s.sink_end + TK_KEYS - 1) / TK_KEYS, s.first_chunk);
  s.chunks = s.sink_chunks + (s.len + TK_KEYS - 1) / TK_KEYS - s.first_chunk;
  s.chunks = m == 1 ? max(s.chunks, 1) : 0;   // (an empty sequence still writes its zeros)
  return s;
}

// A place on the line of units.
struct Cursor {
  int i, item, chunk;        // entry, item of it (key and value head, tile of query heads), chunk of the item
  int seq, row;
  Span s;
  long long item_begin;      // unit at which the item begins
};

__device__ __forceinline__ void next_unit(const TokenParams& p, int items, Cursor& c) {
  if (++c.chunk < c.s.chunks) return;
  c.chunk = 0;
  c.item_begin += c.s.chunks;
  if (++c.item < items) return;
  c.item = 0;
  do {
    if (++c.i >= p.rows.n) { c.s.chunks = 0; return; }
    c.s = span_of(p, c.i, &c.seq, &c.row);
  } while (c.s.chunks == 0);
}

__device__ __forceinline__ int first_key(const Span& s, int chunk) {
  return (chunk < s.sink_chunks ? chunk : s.first_chunk + chunk - s.sink_chunks) * TK_KEYS;
}

// This CTA's part of the line of units (whole CTA).
struct Share {
  Cursor first;
  long long T;       // units of the line
  int G, n_units;    // CTAs that take part; units of this one
};
struct ShareScratch {
  long long before;            // chunks before the CTA's first entry
  long long scan[TK_WARPS + 1];
  int filled[TK_WARPS + 1];
  int entry, last;             // that entry; whether this CTA joins an item's parts
};

// An entry that cannot be answered.
__device__ __forceinline__ void report_entry(const TokenParams& p, int i) {
  int first, m;
  page_rows_of(p.rows, i, &first, &m);
  if (m > 1 || (m == 1 && page_seq_of(p.pv, p.rows.seqs, i) < 0)) atomicOr(p.pv.status, DEV_ERR_INDEX_RANGE);
}

// a * b / c of counts that mostly fit 32 bits (a 64-bit division costs a few hundred cycles, as much as a look into the cache).
__device__ __forceinline__ long long mul_div(long long a, int b, long long c) {
  if (a < (1 << 24) && c < (1 << 24) && b < 256) return (uint32_t)a * (uint32_t)b / (uint32_t)c;
  return a * b / c;
}

// CTAs that take part: T units in `all` items of C = T / all chunks on average.  Where items are as long as each other the cuts then
// fall on their ends, so that a CTA leaves one part and joins once (one sequence of 900 tokens, 32 heads: 9.3 us in 3 CTAs an item,
// 13.5 over all 148; 300 tokens: 6.1 an item a CTA, 7.8 over all).
__device__ __forceinline__ int ctas_for(long long T, long long all, int grid, int min_units, int whole) {
  if (T <= 0) return 0;
  if (all <= grid) {
    const int items = (int)all, C = (int)min(T / items, 1ll << 20);
    return items * (C <= whole ? 1 : max(1, min(grid / items, C / min_units)));
  }
  // whole items where that costs the longest CTA four units at most (16 sequences of 200 tokens, 32 heads: 15.2 us, cut 17.8)
  const long long per = (all + grid - 1) / grid;
  return all % per == 0 && per * T <= (T / grid + 4) * all ? (int)(all / per) : grid;
}

__device__ __forceinline__ Share share_of(const TokenParams& p, int items, int min_units, int whole, ShareScratch& sc) {
  Share sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (p.rows.n <= 32) {   // a lane per entry, every warp for itself (one user's 900 tokens: 0.8 us less than over the CTA's memory)
    Span s{};
    int seq = -1, row = 0;
    if (lane < p.rows.n) s = span_of(p, lane, &seq, &row);
    int incl = s.chunks;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    sh.T = (long long)__shfl_sync(0xffffffffu, incl, 31) * items;
    sh.G = ctas_for(sh.T, (long long)__popc(__ballot_sync(0xffffffffu, s.chunks > 0)) * items, gridDim.x, min_units, whole);
    sh.n_units = 0;
    const int c = blockIdx.x;
    if (c == 0 && warp == 0 && lane < p.rows.n) report_entry(p, lane);
    if (c >= sh.G) return sh;
    const long long u0 = mul_div(sh.T, c, sh.G);
    sh.n_units = (int)(mul_div(sh.T, c + 1, sh.G) - u0);
    const long long target = mul_div(u0, 1, items);
    const int at = __ffs(__ballot_sync(0xffffffffu, target >= incl - s.chunks && target < incl)) - 1;
    Cursor& f = sh.first;
    f.i = at;
    f.s.len = __shfl_sync(0xffffffffu, s.len, at); f.s.start = __shfl_sync(0xffffffffu, s.start, at);
    f.s.sink_end = __shfl_sync(0xffffffffu, s.sink_end, at); f.s.sink_chunks = __shfl_sync(0xffffffffu, s.sink_chunks, at);
    f.s.first_chunk = __shfl_sync(0xffffffffu, s.first_chunk, at); f.s.chunks = __shfl_sync(0xffffffffu, s.chunks, at);
    f.seq = __shfl_sync(0xffffffffu, seq, at); f.row = __shfl_sync(0xffffffffu, row, at);
    const int r = (int)(u0 - (long long)__shfl_sync(0xffffffffu, incl - s.chunks, at) * items);   // (units of one entry)
    f.item = r / f.s.chunks;
    f.chunk = r - f.item * f.s.chunks;
    f.item_begin = u0 - f.chunk;
    return sh;
  }
  const int per = (p.rows.n + TK_THREADS - 1) / TK_THREADS, e0 = min((int)threadIdx.x * per, p.rows.n), e1 = min(e0 + per, p.rows.n);
  long long mine = 0;
  int filled = 0;
  for (int i = e0; i < e1; ++i) {
    int seq, row;
    const int n = span_of(p, i, &seq, &row).chunks;
    mine += n;
    filled += n > 0;
  }
  filled = __reduce_add_sync(0xffffffffu, filled);
  long long before = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += v;
  }
  if (lane == 31) { sc.scan[warp] = before; sc.filled[warp] = filled; }
  __syncthreads();
  long long chunks = 0;
  before -= mine;
  filled = 0;
  for (int w = 0; w <= TK_WARPS; ++w) {
    if (w < warp) before += sc.scan[w];
    chunks += sc.scan[w];
    filled += sc.filled[w];
  }
  sh.T = chunks * items;
  sh.G = ctas_for(sh.T, (long long)filled * items, gridDim.x, min_units, whole);
  sh.n_units = 0;
  const int c = blockIdx.x;
  if (c == 0)
    for (int i = e0; i < e1; ++i) report_entry(p, i);
  if (c >= sh.G) return sh;
  const long long u0 = mul_div(sh.T, c, sh.G);
  sh.n_units = (int)(mul_div(sh.T, c + 1, sh.G) - u0);
  const long long target = mul_div(u0, 1, items);   // chunk count at which the CTA's first entry lies
  if (target >= before && target < before + mine) {
    int i = e0, seq, row;
    long long at = before;
    for (;; ++i) {
      const int n = span_of(p, i, &seq, &row).chunks;
      if (target < at + n) break;
      at += n;
    }
    sc.entry = i;
    sc.before = at;
  }
  __syncthreads();
  sh.first.i = sc.entry;
  sh.first.s = span_of(p, sh.first.i, &sh.first.seq, &sh.first.row);
  const int r = (int)(u0 - sc.before * items);   // (units of one entry)
  sh.first.item = r / sh.first.s.chunks;
  sh.first.chunk = r - sh.first.item * sh.first.s.chunks;
  sh.first.item_begin = u0 - sh.first.chunk;
  return sh;
}

// An item's CTAs, from its first unit and its chunks.
__device__ __forceinline__ int cta_of_unit(long long unit, long long T, int G) {
  if (unit < (1 << 23) && T < (1 << 24) && G < 256) return (int)(((uint32_t)(unit + 1) * (uint32_t)G - 1) / (uint32_t)T);
  return (int)(((unit + 1) * G - 1) / T);
}

__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(TK_WARPS * 32) : "memory"); }

// The warps' outputs (s_out [TK_WARPS][R][HD + 4]), maxima and sums (s_stat) joined into the output, or into this CTA's part of an
// item that it shares: by all consumers, 4 dimensions a thread.
template <typename T, int HD, int R>
__device__ __forceinline__ void join_warps(const TokenParams& p, const float* s_stat, const float* s_out, bool whole, int first_cta, int row_out, long long head0,
                                           int q_rows) {
  constexpr int PITCH = HD + 4;
  const int c = blockIdx.x;
  float* part = p.parts + ((size_t)c * 2 + (c == first_cta ? 1 : 0)) * 16 * PITCH;   // an item that begins here and goes on: slot 1
  for (int e = threadIdx.x; e < q_rows * (HD / 4); e += TK_WARPS * 32) {
    const int row = e / (HD / 4), d = (e - row * (HD / 4)) * 4;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < TK_WARPS; ++w) M = fmaxf(M, s_stat[w * 16 + row]);
    const float ref = M == -INFINITY ? 0.f : M;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < TK_WARPS; ++w) {
      const float f = fast_exp2(s_stat[w * 16 + row] - ref);
      const float4 x = *reinterpret_cast<const float4*>(s_out + (w * R + row) * PITCH + d);
      L = fmaf(f, s_stat[TK_WARPS * 16 + w * 16 + row], L);
      v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
    }
    if (whole) {
      const float inv = L == 0.f ? 0.f : 1.f / L;
      T* out = reinterpret_cast<T*>(p.a.out) + (long long)row_out * p.a.out_stride + (head0 + row) * HD + d;
      out[0] = from_f<T>(v.x * inv); out[1] = from_f<T>(v.y * inv); out[2] = from_f<T>(v.z * inv); out[3] = from_f<T>(v.w * inv);
      if (d == 0 && p.a.lse) p.a.lse[(long long)row_out * p.a.heads + head0 + row] = L == 0.f ? -INFINITY : (M + log2f(L)) * LN2;
    } else {
      *reinterpret_cast<float4*>(part + row * PITCH + d) = v;
      if (d == 0) *reinterpret_cast<float2*>(part + row * PITCH + HD) = make_float2(M, L);
    }
  }
}

// The parts of an item joined in the order of its CTAs, by the consumers of the last one to arrive: TK_JOIN parts' loads under way at a
// time, the last batch filled up with the last part, and up to TK_REST that are left one by one.  What fills a batch up is selected away and
// not branched over: the compiler moves the loads behind the branches, one after another (16384 tokens of 16 query heads on one: 32.4 us,
// this 22.7; 8000 of 32 on 8, 18 parts: 13.9, 11.7).  Sixteen at a time: 40000 tokens of 16 on one 31.8 us for 39.9, but one user's 900
// tokens (three parts) 10.45 for 10.1; four: 56 and 9.9.
template <typename T, int HD>
__device__ __forceinline__ void join_parts(const TokenParams& p, int first_cta, int last_cta, int row_out, long long head0, int q_rows) {
  constexpr int PITCH = HD + 4;
  const size_t step = (size_t)2 * 16 * PITCH;
  const int others = last_cta - first_cta;
  auto batches = [&](auto take) {   // take(first, constant of the batch's size)
    int k0 = 0;
    for (; others - k0 > TK_REST; k0 += TK_JOIN) take(k0, std::integral_constant<int, TK_JOIN>{});
#pragma unroll 1
    for (; k0 < others; ++k0) take(k0, std::integral_constant<int, 1>{});
  };
  for (int e = threadIdx.x; e < q_rows * (HD / 4); e += TK_WARPS * 32) {
    const int row = e / (HD / 4), d = (e - row * (HD / 4)) * 4;
    const float* at0 = p.parts + ((size_t)first_cta * 2 + 1) * 16 * PITCH + row * PITCH;   // the first CTA's slot 1, the others' slot 0
    const float* at = p.parts + (size_t)(first_cta + 1) * step + row * PITCH;
    float M = __ldcg(at0 + HD);
    batches([&](int k0, auto size) {
      constexpr int N = decltype(size)::value;
      float x[N];
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = __ldcg(at + min(k0 + k, others - 1) * step + HD);
#pragma unroll
      for (int k = 0; k < N; ++k) M = fmaxf(M, x[k]);
    });
    const float ref = M == -INFINITY ? 0.f : M;
    float f = fast_exp2(__ldcg(at0 + HD) - ref);
    float L = f * __ldcg(at0 + HD + 1);
    float4 v = __ldcg(reinterpret_cast<const float4*>(at0 + d));
    v.x *= f; v.y *= f; v.z *= f; v.w *= f;
    batches([&](int k0, auto size) {
      constexpr int N = decltype(size)::value;
      float2 st[N];
      float4 x[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float* part = at + min(k0 + k, others - 1) * step;
        st[k] = __ldcg(reinterpret_cast<const float2*>(part + HD));
        x[k] = __ldcg(reinterpret_cast<const float4*>(part + d));
      }
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const bool there = k0 + k < others;
        f = there ? fast_exp2(st[k].x - ref) : 0.f;
        L = fmaf(f, there ? st[k].y : 0.f, L);
        v.x = fmaf(f, there ? x[k].x : 0.f, v.x); v.y = fmaf(f, there ? x[k].y : 0.f, v.y);
        v.z = fmaf(f, there ? x[k].z : 0.f, v.z); v.w = fmaf(f, there ? x[k].w : 0.f, v.w);
      }
    });
    const float inv = L == 0.f ? 0.f : 1.f / L;
    T* out = reinterpret_cast<T*>(p.a.out) + (long long)row_out * p.a.out_stride + (head0 + row) * HD + d;
    out[0] = from_f<T>(v.x * inv); out[1] = from_f<T>(v.y * inv); out[2] = from_f<T>(v.z * inv); out[3] = from_f<T>(v.w * inv);
    if (d == 0 && p.a.lse) p.a.lse[(long long)row_out * p.a.heads + head0 + row] = L == 0.f ? -INFINITY : (M + log2f(L)) * LN2;
  }
  if (threadIdx.x == 0) p.arrived[first_cta] = 0;
}

// One box of a chunk of the cursor's item: the page (-1: not in the pool, reported), its first token there.
struct PageBox {
  bool wanted;
  int page, slot;
};
__device__ __forceinline__ PageBox page_box(const TokenParams& p, const Cursor& c, int chunk, int box, bool in) {
  const PageView& pv = p.pv;
  const int rows = min(pv.ps, TK_KEYS), k0 = first_key(c.s, chunk) + box * rows;
  PageBox b{in && k0 < c.s.len && c.seq >= 0 && !(k0 >= c.s.sink_end && k0 + rows <= c.s.start), -1, k0 & (pv.ps - 1)};   // (not what lies between the sinks and the window)
  if (b.wanted) {
    b.page = pv.table[(size_t)c.seq * pv.max_pages + (k0 >> pv.ps_log2)];
    if ((unsigned)b.page >= (unsigned)pv.n_pages) { b.page = -1; atomicOr(pv.status, DEV_ERR_INDEX_RANGE); }
  }
  return b;
}

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two weights in two bf16 parts each: the leading bits, cut off, and what is left, rounded (off by 2^-16 of the weight at most; one
// part alone 2^-8).  The last bit is set first, so that what is left is never zero: 0 times an infinite V would not be infinite.
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t* high, uint32_t* low) {
  const uint32_t a = __float_as_uint(x) | 1u, b = __float_as_uint(y) | 1u;
  *high = __byte_perm(a, b, 0x7632);
  *low = pack_bf16(__uint_as_float(a) - __uint_as_float(a & 0xffff0000u), __uint_as_float(b) - __uint_as_float(b & 0xffff0000u));
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
               "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
               : "memory");
}

template <int HD> __host__ __device__ constexpr int token_stage_bytes() { return 2 * TK_KEYS * HD * 2; }
template <int HD> __host__ __device__ constexpr int token_pitch() { return HD + 4; }   // floats of a row of parts; also keeps the joins free of bank conflicts
template <int HD> constexpr size_t token_smem() {
  return 1024 + (size_t)TK_STAGES * token_stage_bytes<HD>() + (size_t)TK_WARPS * 16 * 2 * 4 + (size_t)TK_WARPS * 16 * token_pitch<HD>() * 4 + 256;
}

// WIDE: more than 8 query heads in an item (rows 8 to 15 of the tile are in use).
template <int HD, bool WIDE>
__global__ void __launch_bounds__(TK_THREADS, 1) pages_token_kernel(const __grid_constant__ CUtensorMap map, const TokenParams p) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int STAGE = token_stage_bytes<HD>(), PITCH = token_pitch<HD>(), KSTEPS = HD / 16;
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  float* s_stat = reinterpret_cast<float*>(gen + TK_STAGES * STAGE);   // [2][TK_WARPS][16] maxima, sums
  float* s_out = s_stat + 2 * TK_WARPS * 16;                           // [TK_WARPS][16][PITCH] the warps' outputs
  uint8_t* misc = reinterpret_cast<uint8_t*>(s_out + TK_WARPS * 16 * PITCH);
  const uint32_t bars = smem_u32(misc);   // full, then empty
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 16 * TK_STAGES);
  ShareScratch& share = *reinterpret_cast<ShareScratch*>(misc + 16 * TK_STAGES + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PageView& pv = p.pv;
  if (threadIdx.x == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
    for (int s = 0; s < TK_STAGES; ++s) { mbar_init(bars + 8u * s, 1); mbar_init(bars + 8u * (TK_STAGES + s), TK_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_enter();

  const int items = pv.H * p.tiles, c = blockIdx.x;
  const Share sh = share_of(p, items, WIDE ? TK_MIN_UNITS_WIDE : TK_MIN_UNITS, TK_WHOLE, share);
  if (sh.n_units == 0) return;
  Cursor cur = sh.first;
  const int n_units = sh.n_units, G = sh.G;
  const long long T = sh.T;

  const int box_rows = min(pv.ps, TK_KEYS), boxes = TK_KEYS / box_rows;
  if (warp == TK_WARPS) {
    // ===================== producer =====================
    const long long pool_rows = (long long)pv.n_layers * 2 * pv.n_pages * pv.H * pv.ps, plane_rows = (long long)pv.n_pages * pv.H * pv.ps;
    const int units = 32 / boxes, u = lane / boxes, box = lane - u * boxes;   // lane = (unit of a group, box): a group's pages in one look
    bool ok = true;
    for (int n = 0; n < n_units && ok;) {
      const int h = cur.item / p.tiles, many = min(min(units, cur.s.chunks - cur.chunk), n_units - n);
      const PageBox b = page_box(p, cur, cur.chunk + u, box, u < many);
      for (int x = 0; x < many; ++x, ++n) {
        const int st = n % TK_STAGES;
        if (n >= TK_STAGES && !(ok = __all_sync(0xffffffffu, mbar_wait(bars + 8u * (TK_STAGES + st), ((n / TK_STAGES) & 1) ^ 1u, abort_flag, pv.status)))) break;
        const bool mine = u == x && b.wanted;
        const uint32_t count = __popc(__ballot_sync(0xffffffffu, mine));
        if (lane == 0) mbar_expect_tx(bars + 8u * st, count * (uint32_t)(2 * box_rows * HD * 2));
        __syncwarp();
        if (mine) {
          // (behind the pool's last row the copy fills in zeros)
          const long long row = b.page >= 0 ? (((long long)p.a.layer * 2 * pv.n_pages + b.page) * pv.H + h) * pv.ps + b.slot : pool_rows;
          const uint32_t dst = base + (uint32_t)(st * STAGE + box * box_rows * HD * 2);
          tma_load_3d(dst, &map, bars + 8u * st, 0, (int)row, 0);
          tma_load_3d(dst + STAGE / 2, &map, bars + 8u * st, 0, (int)(b.page >= 0 ? row + plane_rows : pool_rows), 0);
        }
      }
      if (ok && n < n_units) { cur.chunk += many - 1; next_unit(p, items, cur); }
    }
    if (!ok) {   // copies already issued land before the CTA's shared memory is given back
      const unsigned long long t0 = now_ns();
      while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
    return;
  }

  // ===================== consumers =====================
  const int g = lane >> 2, t4 = lane & 3;
  const float scale2 = p.a.scale * LOG2E;
  uint32_t q[KSTEPS][4];
  float o[HD / 8][4];
  float m[2], l[2];
  // this warp's 16 keys of a chunk lie in one page
  const int wkey = warp * 16, wbox = wkey / box_rows, wrow = wkey - wbox * box_rows;
  const uint32_t wbase = base + (uint32_t)(wbox * box_rows * HD * 2 + wrow * 128), half_step = (uint32_t)box_rows * 128u;
  // ldmatrix addresses: lane l gives row (l & 7) of matrix l >> 3
  const int mat = lane >> 3, mrow = lane & 7;
  const int krow = (mat >> 1) * 8 + mrow, kcol = mat & 1;   // K: keys 0-7 | 0-7 | 8-15 | 8-15, dimensions 0-7 | 8-15 | ...
  const int vrow = (mat & 1) * 8 + mrow, vcol = mat >> 1;   // V: keys 0-7 | 8-15 | 0-7 | 8-15, dimensions 0-7 | 0-7 | 8-15 | 8-15
  bool ok = true;
  for (int n = 0; n < n_units;) {
    const Cursor item = cur;
    const int h = item.item / p.tiles, tile = item.item - h * p.tiles;
    const int q_rows = min(16, p.group - tile * 16);
    const int todo = min(item.s.chunks - item.chunk, n_units - n);
    const long long head0 = (long long)h * p.group + tile * 16;
    // the query rows as A fragments (zeros behind the last one)
    {
      const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(p.a.q) + (long long)item.row * p.a.q_stride + head0 * HD + 2 * t4;
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k) {
        q[k][0] = g < q_rows ? *reinterpret_cast<const uint32_t*>(src + g * HD + 16 * k) : 0u;
        q[k][2] = g < q_rows ? *reinterpret_cast<const uint32_t*>(src + g * HD + 16 * k + 8) : 0u;
        q[k][1] = WIDE && g + 8 < q_rows ? *reinterpret_cast<const uint32_t*>(src + (g + 8) * HD + 16 * k) : 0u;
        q[k][3] = WIDE && g + 8 < q_rows ? *reinterpret_cast<const uint32_t*>(src + (g + 8) * HD + 16 * k + 8) : 0u;
      }
    }
#pragma unroll
    for (int d = 0; d < HD / 8; ++d) { o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f; }
    m[0] = m[1] = -INFINITY; l[0] = l[1] = 0.f;
    for (int x = 0; x < todo; ++x, ++n) {
      const int st = n % TK_STAGES;
      const int k0 = first_key(item.s, item.chunk + x) + wkey;
      ok = __all_sync(0xffffffffu, mbar_wait(bars + 8u * st, (n / TK_STAGES) & 1, abort_flag, pv.status));
      if (!ok) { n += todo - x; break; }   // (the warps still meet below, and the parts' counters come back to zero)
      const uint32_t sk = wbase + (uint32_t)(st * STAGE), sv = sk + STAGE / 2;
      // which of the 16 keys the row sees
      uint32_t seen = 0xffffu;
      if (k0 + 16 > item.s.len || (k0 < item.s.start && k0 + 16 > item.s.sink_end)) {
        seen = 0;
#pragma unroll
        for (int b = 0; b < 16; ++b) seen |= (k0 + b < item.s.len && (k0 + b >= item.s.start || k0 + b < item.s.sink_end)) ? 1u << b : 0u;
      }
      if (seen) {
        float c0[4] = {0.f, 0.f, 0.f, 0.f}, c1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KSTEPS; ++k) {
          uint32_t b[4];
          const int col = 2 * k + kcol;   // 16-byte column of the row
          ldsm4(sk + (uint32_t)(col >> 3) * half_step + krow * 128 + (((col & 7) ^ (krow & 7)) << 4), b);
          mma_bf16(c0, q[k], b[0], b[1]);
          mma_bf16(c1, q[k], b[2], b[3]);
        }
        // keys 2 t4, 2 t4 + 1 in c0 and 8 further in c1; rows g in [0], [1] and g + 8 in [2], [3]
        if (seen != 0xffffu) {
          const uint32_t w = seen >> (2 * t4);
          if (!(w & 1u)) c0[0] = c0[2] = -INFINITY;
          if (!(w & 2u)) c0[1] = c0[3] = -INFINITY;
          if (!(w & 256u)) c1[0] = c1[2] = -INFINITY;
          if (!(w & 512u)) c1[1] = c1[3] = -INFINITY;
        }
        uint32_t pa[4], pb[4];   // the weights in two parts
#pragma unroll
        for (int r = 0; r < (WIDE ? 2 : 1); ++r) {
          float mx = fmaxf(fmaxf(c0[2 * r], c0[2 * r + 1]), fmaxf(c1[2 * r], c1[2 * r + 1]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          const float m_new = fmaxf(m[r], mx * scale2);
          const float ref = m_new == -INFINITY ? 0.f : m_new;
          if (__any_sync(0xffffffffu, m_new != m[r])) {
            const float corr = fast_exp2(m[r] - ref);
            l[r] *= corr;
#pragma unroll
            for (int d = 0; d < HD / 8; ++d) {
              o[d][2 * r] *= corr; o[d][2 * r + 1] *= corr;
              if (!WIDE) { o[d][2] *= corr; o[d][3] *= corr; }
            }
            m[r] = m_new;
          }
          const float p0 = fast_exp2(fmaf(c0[2 * r], scale2, -ref)), p1 = fast_exp2(fmaf(c0[2 * r + 1], scale2, -ref));
          const float p2 = fast_exp2(fmaf(c1[2 * r], scale2, -ref)), p3 = fast_exp2(fmaf(c1[2 * r + 1], scale2, -ref));
          l[r] += (p0 + p1) + (p2 + p3);
          split_bf16(p0, p1, &pa[r], &pb[r]); split_bf16(p2, p3, &pa[r + 2], &pb[r + 2]);
        }
        if (!WIDE) { pa[1] = pb[0]; pa[3] = pb[2]; }   // (rows 8 to 15 of the tile are free)
        const uint32_t z0 = ((seen >> (2 * t4)) & 1u ? 0xffffu : 0u) | ((seen >> (2 * t4 + 1)) & 1u ? 0xffff0000u : 0u);
        const uint32_t z1 = ((seen >> (2 * t4 + 8)) & 1u ? 0xffffu : 0u) | ((seen >> (2 * t4 + 9)) & 1u ? 0xffff0000u : 0u);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) {
          uint32_t b[4];
          const int col = 2 * d + vcol;
          ldsm4_trans(sv + (uint32_t)(col >> 3) * half_step + vrow * 128 + (((col & 7) ^ (vrow & 7)) << 4), b);
          if (seen != 0xffffu) { b[0] &= z0; b[1] &= z1; b[2] &= z0; b[3] &= z1; }
          mma_bf16(o[2 * d], pa, b[0], b[1]);
          mma_bf16(o[2 * d + 1], pa, b[2], b[3]);
          if (WIDE) {
            mma_bf16(o[2 * d], pb, b[0], b[1]);
            mma_bf16(o[2 * d + 1], pb, b[2], b[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bars + 8u * (TK_STAGES + st));
    }
    // ---- join the warps through shared memory
    consumers_sync();   // the join before has been read
#pragma unroll
    for (int r = 0; r < (WIDE ? 2 : 1); ++r) {
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
      l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
      if (t4 == 0) {
        s_stat[warp * 16 + g + 8 * r] = m[r];
        s_stat[TK_WARPS * 16 + warp * 16 + g + 8 * r] = l[r];
      }
      if (g + 8 * r < q_rows) {
        float* dst = s_out + (warp * 16 + g + 8 * r) * PITCH + 2 * t4;
#pragma unroll
        for (int d = 0; d < HD / 8; ++d) *reinterpret_cast<float2*>(dst + 8 * d) = WIDE ? make_float2(o[d][2 * r], o[d][2 * r + 1]) : make_float2(o[d][0] + o[d][2], o[d][1] + o[d][3]);
      }
    }
    consumers_sync();
    const bool whole = todo == item.s.chunks;
    const int first_cta = whole ? c : cta_of_unit(item.item_begin, T, G);
    join_warps<__nv_bfloat16, HD, 16>(p, s_stat, s_out, whole, first_cta, item.row, head0, q_rows);
    if (!whole) {
      // ---- the last of the item's CTAs joins their parts
      const int last_cta = cta_of_unit(item.item_begin + item.s.chunks - 1, T, G);
      consumers_sync();
      if (threadIdx.x == 0) share.last = chain_arrive_count(p.arrived + first_cta) == last_cta - first_cta;
      consumers_sync();
      if (share.last) join_parts<__nv_bfloat16, HD>(p, first_cta, last_cta, item.row, head0, q_rows);
    }
    if (n < n_units) {
      cur.chunk += todo - 1;
      next_unit(p, items, cur);
    }
  }
}

// ---------------------------------------------------------------- fp32
// The same line of units for the fp32 configuration, on the CUDA cores.  A page's rows of a head are one run of bytes, copied as it
// is; a warp takes 16 keys of a chunk, two lanes a key for the scores (each half of the dimensions, beginning at a place of its own
// so that eight lanes read eight different banks' worth), then all lanes the dimensions of the output.
template <int HD, int R> __host__ __device__ constexpr int token_stages_f32() { return HD * R == 2048 ? 2 : 3; }   // (16 query heads of dimension 128: their parts take the room)
template <int HD> __host__ __device__ constexpr int token_stage_f32() { return 2 * TK_KEYS * HD * 4; }
template <int HD, int R> constexpr size_t token_smem_f32() {
  return 128 + (size_t)token_stages_f32<HD, R>() * token_stage_f32<HD>() + (size_t)R * HD * 4 + (size_t)TK_WARPS * 16 * 2 * 4 + (size_t)TK_WARPS * R * token_pitch<HD>() * 4 + 256;
}

// R: most query heads of an item.
template <int HD, int R>
__global__ void __launch_bounds__(TK_THREADS, 1) pages_token_f32_kernel(const TokenParams p) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int TF_STAGES = token_stages_f32<HD, R>(), STAGE = token_stage_f32<HD>(), PITCH = token_pitch<HD>(), N = HD / 32, QUADS = HD / 8;   // QUADS: 16-byte pieces of half a row
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 127u) & ~127u;
  uint8_t* gen = smem_raw + (base - raw);
  float* s_q = reinterpret_cast<float*>(gen + TF_STAGES * STAGE);      // [R][HD]
  float* s_stat = s_q + R * HD;                                        // [2][TK_WARPS][16]
  float* s_out = s_stat + 2 * TK_WARPS * 16;                           // [TK_WARPS][R][PITCH]
  uint8_t* misc = reinterpret_cast<uint8_t*>(s_out + TK_WARPS * R * PITCH);
  const uint32_t bars = smem_u32(misc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(misc + 16 * TF_STAGES);
  ShareScratch& share = *reinterpret_cast<ShareScratch*>(misc + 16 * TF_STAGES + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PageView& pv = p.pv;
  if (threadIdx.x == 0) {
    for (int s = 0; s < TF_STAGES; ++s) { mbar_init(bars + 8u * s, 1); mbar_init(bars + 8u * (TF_STAGES + s), TK_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_enter();
  const int items = pv.H * p.tiles, c = blockIdx.x;
  const Share sh = share_of(p, items, 1, 1, share);
  if (sh.n_units == 0) return;
  Cursor cur = sh.first;
  const int n_units = sh.n_units, G = sh.G;
  const long long T = sh.T;
  const int box_rows = min(pv.ps, TK_KEYS), boxes = TK_KEYS / box_rows;
  if (warp == TK_WARPS) {
    bool ok = true;
    const size_t plane = (size_t)pv.n_pages * pv.H * pv.ps * HD;
    const int units = 32 / boxes, u = lane / boxes, box = lane - u * boxes;
    const uint32_t bytes = (uint32_t)(box_rows * HD * 4);
    for (int n = 0; n < n_units && ok;) {
      const int h = cur.item / p.tiles, many = min(min(units, cur.s.chunks - cur.chunk), n_units - n);
      const PageBox b = page_box(p, cur, cur.chunk + u, box, u < many);
      for (int x = 0; x < many; ++x, ++n) {
        const int st = n % TF_STAGES;
        if (n >= TF_STAGES && !(ok = __all_sync(0xffffffffu, mbar_wait(bars + 8u * (TF_STAGES + st), ((n / TF_STAGES) & 1) ^ 1u, abort_flag, pv.status)))) break;
        const bool mine = u == x && b.wanted && b.page >= 0;
        const uint32_t count = __popc(__ballot_sync(0xffffffffu, mine));
        if (u == x && b.wanted && b.page < 0) {   // (reported; zeros, as the copy of the other type fills in, not what the slot held before)
          for (uint32_t e = 0; e < bytes; e += 16)
            for (int kv = 0; kv < 2; ++kv) *reinterpret_cast<float4*>(gen + st * STAGE + kv * (STAGE / 2) + (size_t)box * bytes + e) = make_float4(0.f, 0.f, 0.f, 0.f);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        if (lane == 0) mbar_expect_tx(bars + 8u * st, count * 2 * bytes);
        __syncwarp();
        if (mine) {
          const float* src = reinterpret_cast<const float*>(pv.pool) + (size_t)p.a.layer * 2 * plane + (((size_t)b.page * pv.H + h) * pv.ps + b.slot) * HD;
          const uint32_t dst = base + (uint32_t)(st * STAGE) + (uint32_t)box * bytes;
          bulk_load(dst, src, bytes, bars + 8u * st);
          bulk_load(dst + STAGE / 2, src + plane, bytes, bars + 8u * st);
        }
      }
      if (ok && n < n_units) { cur.chunk += many - 1; next_unit(p, items, cur); }
    }
    if (!ok) {
      const unsigned long long t0 = now_ns();
      while (now_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
    return;
  }
  const float scale2 = p.a.scale * LOG2E;
  const int key = lane >> 1, half = lane & 1, rot = lane & 7, wkey = warp * 16;
  bool ok = true;
  for (int n = 0; n < n_units;) {
    const Cursor item = cur;
    const int h = item.item / p.tiles, tile = item.item - h * p.tiles;
    const int q_rows = min(16, p.group - tile * 16);
    const int todo = min(item.s.chunks - item.chunk, n_units - n);
    const long long head0 = (long long)h * p.group + tile * 16;
    consumers_sync();   // the item before is done with its query rows
    for (int e = threadIdx.x; e < q_rows * HD; e += TK_WARPS * 32)
      s_q[e] = reinterpret_cast<const float*>(p.a.q)[(long long)item.row * p.a.q_stride + head0 * HD + e] * scale2;
    consumers_sync();
    float o[R][N], m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
      for (int d = 0; d < N; ++d) o[r][d] = 0.f;
    }
    for (int x = 0; x < todo; ++x, ++n) {
      const int st = n % TF_STAGES, k0 = first_key(item.s, item.chunk + x) + wkey, j = k0 + key;
      ok = __all_sync(0xffffffffu, mbar_wait(bars + 8u * st, (n / TF_STAGES) & 1, abort_flag, pv.status));
      if (!ok) { n += todo - x; break; }   // (the warps still meet below, and the parts' counters come back to zero)
      const bool seen = j < item.s.len && (j >= item.s.start || j < item.s.sink_end);
      const uint32_t any = __ballot_sync(0xffffffffu, seen);
      if (any) {
        const float4* kr = reinterpret_cast<const float4*>(gen + st * STAGE + (size_t)(wkey + key) * HD * 4 + half * HD * 2);
        float s[R];
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = 0.f;
#pragma unroll 4
        for (int i = 0; i < QUADS; ++i) {
          const int at = (i + rot) % QUADS;
          const float4 kv = kr[at];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (r >= q_rows) break;
            const float4 qv = *reinterpret_cast<const float4*>(s_q + r * HD + half * (HD / 2) + at * 4);
            s[r] = fmaf(kv.x, qv.x, fmaf(kv.y, qv.y, fmaf(kv.z, qv.z, fmaf(kv.w, qv.w, s[r]))));
          }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
          if (r >= q_rows) break;
          s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
          s[r] = seen ? s[r] : -INFINITY;
          float mx = s[r];
#pragma unroll
          for (int w = 2; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
          const float m_new = fmaxf(m[r], mx), ref = m_new == -INFINITY ? 0.f : m_new, corr = exp2f(m[r] - ref);
          m[r] = m_new;
          s[r] = exp2f(s[r] - ref);
          l[r] = l[r] * corr + (half ? 0.f : s[r]);
#pragma unroll
          for (int d = 0; d < N; ++d) o[r][d] *= corr;
        }
        const float* vr = reinterpret_cast<const float*>(gen + st * STAGE + STAGE / 2) + (size_t)wkey * HD + lane * N;
#pragma unroll 4
        for (int y = 0; y < 16; ++y) {
          if (!((any >> (2 * y)) & 1u)) continue;   // (what is not seen may be anything)
          float v[N];
          load_dims(vr + y * HD, v);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (r >= q_rows) break;
            const float w = __shfl_sync(0xffffffffu, s[r], 2 * y);
#pragma unroll
            for (int d = 0; d < N; ++d) o[r][d] = fmaf(w, v[d], o[r][d]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bars + 8u * (TF_STAGES + st));
    }
    // ---- join the warps
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= q_rows) break;
#pragma unroll
      for (int w = 1; w < 32; w <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], w);
      if (lane == 0) {
        s_stat[warp * 16 + r] = m[r];
        s_stat[TK_WARPS * 16 + warp * 16 + r] = l[r];
      }
#pragma unroll
      for (int d = 0; d < N; ++d) s_out[(warp * R + r) * PITCH + lane * N + d] = o[r][d];
    }
    consumers_sync();
    const bool whole = todo == item.s.chunks;
    const int first_cta = whole ? c : cta_of_unit(item.item_begin, T, G);
    join_warps<float, HD, R>(p, s_stat, s_out, whole, first_cta, item.row, head0, q_rows);
    if (!whole) {
      const int last_cta = cta_of_unit(item.item_begin + item.s.chunks - 1, T, G);
      consumers_sync();
      if (threadIdx.x == 0) share.last = chain_arrive_count(p.arrived + first_cta) == last_cta - first_cta;
      consumers_sync();
      if (share.last) join_parts<float, HD>(p, first_cta, last_cta, item.row, head0, q_rows);
    }
    if (n < n_units) {
      cur.chunk += todo - 1;
      next_unit(p, items, cur);
    }
  }
}

}  // namespace

size_t pages_token_part_bytes(const PageView& pv, int grid) {
  return ((size_t)grid * 2 * 16 * (pv.hd + 4) * 4 + 255) / 256 * 256 + ((size_t)grid * 4 + 255) / 256 * 256;
}

// Calls f(kernel, shared memory) for the kernel of these sizes, or for all of the type and head dimension (group < 0).
template <typename F> static cudaError_t for_token_kernels(int es, int hd, int group, F f) {
  cudaError_t e = cudaSuccess;
  auto pick = [&](bool mine, auto kernel, size_t smem) { if (e == cudaSuccess && (group < 0 || mine)) e = f(kernel, smem); };
  auto bf16 = [&](auto hd_c) {
    constexpr int HD = decltype(hd_c)::value;
    pick(group <= 8, pages_token_kernel<HD, false>, token_smem<HD>());
    pick(group > 8, pages_token_kernel<HD, true>, token_smem<HD>());
  };
  auto fp32 = [&](auto hd_c) {
    constexpr int HD = decltype(hd_c)::value;
    pick(group == 1, pages_token_f32_kernel<HD, 1>, token_smem_f32<HD, 1>());
    pick(group > 1 && group <= 4, pages_token_f32_kernel<HD, 4>, token_smem_f32<HD, 4>());
    pick(group > 4, pages_token_f32_kernel<HD, 16>, token_smem_f32<HD, 16>());
  };
  using C64 = std::integral_constant<int, 64>;
  using C128 = std::integral_constant<int, 128>;
  if (es == 2) hd == 64 ? bf16(C64{}) : bf16(C128{});
  else hd == 64 ? fp32(C64{}) : fp32(C128{});
  return e;
}

cudaError_t pages_token_prepare(const PageView& pv) {
  return for_token_kernels(pv.es, pv.hd, -1, [](auto k, size_t smem) { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
}

// map: the pool's rows in boxes of min(page_size, 64) (bf16).  parts: pages_token_part_bytes, its counters zero.  grid: the SMs.
cudaError_t launch_pages_token(const void* map, const PageView& pv, const PageRows& rows, const PageAttention& a, void* parts, int grid, cudaStream_t st) {
  TokenParams p;
  p.pv = pv; p.rows = rows; p.a = a;
  p.group = a.heads / pv.H; p.tiles = (p.group + 15) / 16;
  p.parts = (float*)parts;
  p.arrived = (int32_t*)((char*)parts + ((size_t)grid * 2 * 16 * (pv.hd + 4) * 4 + 255) / 256 * 256);
  return for_token_kernels(pv.es, pv.hd, p.group, [&](auto k, size_t smem) {
    if constexpr (std::is_invocable_v<decltype(k), CUtensorMap, TokenParams>) launch_pdl(k, grid, TK_THREADS, smem, st, *(const CUtensorMap*)map, p);
    else launch_pdl(k, grid, TK_THREADS, smem, st, p);
    return cudaGetLastError();
  });
}

}  // namespace rd
