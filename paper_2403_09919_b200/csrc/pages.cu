// Management of a key-value cache in pages: allocation with copy on write, sharing between sequences, the accept step's
// compaction (Section 3.4) on pages, and release.  Whole numbers and moved rows; everything is decided on the device, so a
// serving loop never waits for the host and the calls can be captured.
//
// The state is a page table, lengths, a reference count per page and a bit per page that says it is free.  There is no free
// list: which page a sequence gets is the lowest free one in the order of the call's sequences, found by a scan of the bits,
// and releases only count down and set bits.  The result therefore does not depend on the order in which atomics land.
//
// Bounds: the tables are a few kilobytes (latency of a launch or two: four branches of a small fp32 cache, given up and made again,
// 9.0 us in four launches); copies of shared pages and moved rows are bandwidth, every byte read and written once with 16-byte accesses (201 MB for
// 32 branches over 8 layers 44 us, of which 13 are the launches and look-ups before).
#include "pages.cuh"
#include "pdl.cuh"
#include "rd_internal.cuh"

namespace rd {

namespace {

constexpr int EXTEND_THREADS = 1024;

// Workspace of the management calls (int32 words).
struct PageScratch {
  int32_t* job_count;   // [4] number of copy jobs of the extend in flight
  int32_t* mark;        // [max_seqs]  lowest entry of the list that names the sequence; INT_MAX between calls
  int32_t* need;        // [max_seqs]  pages an entry needs | its offset in the order of the list
  int32_t* offset;      // [max_seqs]
  int32_t* jobs;        // [max_seqs][3] source page, target page, rows of a copy
  int32_t* ok;          // [max_seqs]  compaction: the entry passed its checks
  int32_t* sharers;     // [n_pages]   entries of the call that write into the page; 0 between calls
  int32_t* last_sharer; // [n_pages]   highest of them + 1; 0 between calls
  int32_t* found;       // [n_pages]   free pages in ascending order
};

__host__ __device__ inline PageScratch page_scratch(const PageView& pv, int32_t* base) {
  PageScratch s;
  const size_t S = pv.max_seqs, P = pv.n_pages;
  s.job_count = base; base += 4;
  s.mark = base; base += S;
  s.need = base; base += S;
  s.offset = base; base += S;
  s.jobs = base; base += 3 * S;
  s.ok = base; base += S;
  s.sharers = base; base += P;
  s.last_sharer = base; base += P;
  s.found = base;
  return s;
}

__device__ __forceinline__ int held_pages(const PageView& pv, int len) { return (int)(((long long)len + pv.ps - 1) >> pv.ps_log2); }

// Exclusive scan of a pair over the CTA's EXTEND_THREADS threads; totals in *ta, *tb.
__device__ __forceinline__ void scan_pair(int& a, int& b, int* ta, int* tb, int (*warp_tot)[2]) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int a0 = a, b0 = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int va = __shfl_up_sync(0xffffffffu, a, o), vb = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) { a += va; b += vb; }
  }
  __syncthreads();   // the totals of an earlier scan have been read
  if (lane == 31) { warp_tot[w][0] = a; warp_tot[w][1] = b; }
  __syncthreads();
  int sa = 0, sb = 0, ra = 0, rb = 0;
#pragma unroll
  for (int i = 0; i < EXTEND_THREADS / 32; ++i) {
    if (i < w) { sa += warp_tot[i][0]; sb += warp_tot[i][1]; }
    ra += warp_tot[i][0]; rb += warp_tot[i][1];
  }
  a += sa - a0; b += sb - b0;
  *ta = ra; *tb = rb;
}

// Whether an earlier entry of the list names the same sequence (whole CTA).
__device__ __forceinline__ bool named_before(const int32_t* list, int i, int s) {
  bool dup = false;
  if (list)
    for (int j = threadIdx.x; j < i; j += blockDim.x) dup = dup || list[j] == s;
  return __syncthreads_or(dup);
}

// A page loses one of its names; the last one frees it.
__device__ __forceinline__ void drop_page(const PageView& pv, int p) {
  if ((unsigned)p >= (unsigned)pv.n_pages) { atomicOr(pv.status, DEV_ERR_INDEX_RANGE); return; }
  const int before = atomicSub(&pv.refs[p], 1);
  if (before == 1) atomicOr(&pv.free_bits[p >> 5], 1u << (p & 31));
  else if (before <= 0) { atomicAdd(&pv.refs[p], 1); atomicOr(pv.status, DEV_ERR_INDEX_RANGE); }
}

// ---------------------------------------------------------------- reset
__global__ void pages_reset_kernel(PageView pv, int32_t* scratch) {
  pdl_enter();
  const PageScratch sc = page_scratch(pv, scratch);
  const long long t0 = (long long)blockIdx.x * blockDim.x + threadIdx.x, stride = (long long)gridDim.x * blockDim.x;
  for (long long i = t0; i < (long long)pv.max_seqs * pv.max_pages; i += stride) pv.table[i] = -1;
  for (long long i = t0; i < pv.max_seqs; i += stride) { pv.lens[i] = 0; sc.mark[i] = 0x7fffffff; }
  for (long long i = t0; i < pv.n_pages; i += stride) { pv.refs[i] = 0; sc.sharers[i] = 0; sc.last_sharer[i] = 0; }
  for (long long i = t0; i < (pv.n_pages + 31) / 32; i += stride) {
    const int left = pv.n_pages - (int)i * 32;
    pv.free_bits[i] = left >= 32 ? 0xffffffffu : (1u << left) - 1u;
  }
}

// Only the scratch: a handle on tables that are already in use.
__global__ void pages_scratch_kernel(PageView pv, int32_t* scratch) {
  pdl_enter();
  const PageScratch sc = page_scratch(pv, scratch);
  const long long t0 = (long long)blockIdx.x * blockDim.x + threadIdx.x, stride = (long long)gridDim.x * blockDim.x;
  for (long long i = t0; i < pv.max_seqs; i += stride) sc.mark[i] = 0x7fffffff;
  for (long long i = t0; i < pv.n_pages; i += stride) { sc.sharers[i] = 0; sc.last_sharer[i] = 0; }
}

// ---------------------------------------------------------------- extend
// One CTA: the lists are short and every step needs the one before for all entries.  All entries or none: a call that finds
// too few free pages changes nothing.
//
// Copy on write: an entry whose last page is partly filled writes into that page.  As if the entries came one after another,
// each that finds the page shared takes a copy and gives its name up, so the last of `refs` sharers keeps the page: entry i
// copies unless the call's writers are all the page's names and i is the last of them.  Counting (atomicAdd) and finding the
// last (atomicMax) do not depend on the order in which they land.
__global__ void __launch_bounds__(EXTEND_THREADS) pages_extend_kernel(PageView pv, const int32_t* __restrict__ seqs,
                                                                      const int32_t* __restrict__ n_new, int n, int32_t* scratch) {
  pdl_enter();
  __shared__ int warp_tot[EXTEND_THREADS / 32][2];
  const PageScratch sc = page_scratch(pv, scratch);
  const int t = threadIdx.x;
  // a sequence named twice: its first entry counts
  if (seqs) {
    for (int i = t; i < n; i += EXTEND_THREADS) {
      const int s = page_seq_of(pv, seqs, i);
      if (s >= 0) atomicMin(&sc.mark[s], i);
    }
    __syncthreads();
  }
  // what each entry writes into; need = -1 marks an entry that is refused
  auto entry = [&](int i, int* s, int* len, int* add) {
    *s = page_seq_of(pv, seqs, i);
    if (*s < 0 || (seqs && sc.mark[*s] != i)) return false;
    *len = pv.lens[*s]; *add = n_new[i];
    return *len >= 0 && *add >= 0 && (long long)*len + *add <= min((long long)pv.max_pages << pv.ps_log2, 0x7fffffffll);
  };
  auto last_page = [&](int s, int len) { return pv.table[(size_t)s * pv.max_pages + (len >> pv.ps_log2)]; };
  for (int i = t; i < n; i += EXTEND_THREADS) {
    int s, len, add, need = 0;
    bool ok = entry(i, &s, &len, &add);
    if (ok && add > 0 && (len & (pv.ps - 1))) {
      const int p = last_page(s, len);
      if ((unsigned)p < (unsigned)pv.n_pages) {
        atomicAdd(&sc.sharers[p], 1);
        atomicMax(&sc.last_sharer[p], i + 1);
      } else ok = false;
    }
    if (ok) need = held_pages(pv, len + add) - held_pages(pv, len);
    else atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
    sc.need[i] = ok ? need : -1;
  }
  __syncthreads();
  // offsets of the entries' pages and copies, in the order of the list
  int base_pages = 0, base_jobs = 0;
  for (int i0 = 0; i0 < n; i0 += EXTEND_THREADS) {
    const int i = i0 + t;
    int pages = 0, copies = 0;
    if (i < n && sc.need[i] >= 0) {
      int s, len, add;
      entry(i, &s, &len, &add);
      if (add > 0 && (len & (pv.ps - 1))) {
        const int p = last_page(s, len);
        copies = !(sc.sharers[p] >= pv.refs[p] && sc.last_sharer[p] == i + 1);
      }
      pages = sc.need[i] + copies;
    }
    const int mine = pages, my_copies = copies;
    int tp, tj;
    scan_pair(pages, copies, &tp, &tj, warp_tot);
    if (i < n && sc.need[i] >= 0) {
      sc.offset[i] = base_pages + pages;
      sc.need[i] = mine * 2 + my_copies;
      if (my_copies) sc.jobs[3 * (size_t)i] = base_jobs + copies;   // (its place among the jobs; filled in below)
    }
    base_pages += tp; base_jobs += tj;
  }
  __syncthreads();
  const int total = base_pages;
  // the lowest free pages
  const int words = (pv.n_pages + 31) >> 5;
  int found = 0;
  for (int w0 = 0; w0 < words && found < total; w0 += EXTEND_THREADS) {
    const int w = w0 + t;
    uint32_t bits = 0;
    if (w < words) {
      bits = pv.free_bits[w];
      const int left = pv.n_pages - w * 32;
      if (left < 32) bits &= (1u << left) - 1u;
    }
    int rank = __popc(bits), none = 0, tf, tn;
    scan_pair(rank, none, &tf, &tn, warp_tot);
    rank += found;
    while (bits && rank < total) {
      sc.found[rank++] = w * 32 + __ffs(bits) - 1;
      bits &= bits - 1;
    }
    found += tf;
  }
  __syncthreads();
  const bool enough = found >= total;
  if (enough) {
    for (int k = t; k < total; k += EXTEND_THREADS) {
      const int p = sc.found[k];
      atomicAnd(&pv.free_bits[p >> 5], ~(1u << (p & 31)));
      pv.refs[p] = 1;
    }
  } else if (t == 0) {
    atomicOr(pv.status, DEV_ERR_CAPACITY);
  }
  // a page's counters back to zero before its entries' lengths change
  for (int i = t; i < n; i += EXTEND_THREADS) {
    int s, len, add;
    if (sc.need[i] < 0) continue;
    entry(i, &s, &len, &add);
    if (add > 0 && (len & (pv.ps - 1))) {
      const int p = last_page(s, len);
      sc.sharers[p] = 0; sc.last_sharer[p] = 0;
    }
  }
  __syncthreads();
  // the pages into the tables: a warp per entry
  if (enough) {
    const int lane = t & 31;
    for (int i = t >> 5; i < n; i += EXTEND_THREADS / 32) {
      if (sc.need[i] < 0) continue;
      const int s = page_seq_of(pv, seqs, i), len = pv.lens[s], add = n_new[i];
      const int pages = sc.need[i] >> 1, copy = sc.need[i] & 1, off = sc.offset[i], held = held_pages(pv, len);
      int32_t* row = pv.table + (size_t)s * pv.max_pages;
      __syncwarp();
      if (copy && lane == 0) {
        const int old = row[held - 1], p = sc.found[off];
        atomicSub(&pv.refs[old], 1);
        row[held - 1] = p;
        const int j = sc.jobs[3 * (size_t)i];
        sc.offset[i] = old;   // (kept until the jobs are written: their places may be other entries' own)
        sc.need[i] = 2 * p + 1;
        sc.ok[i] = j;
      } else if (lane == 0) {
        sc.need[i] = 0;
      }
      for (int k = copy + lane; k < pages; k += 32) row[held + k - copy] = sc.found[off + k];
      __syncwarp();
      if (lane == 0 && !copy) pv.lens[s] = len + add;
    }
  }
  __syncthreads();
  for (int i = t; i < n; i += EXTEND_THREADS) {
    const int s = page_seq_of(pv, seqs, i);
    if (enough && sc.need[i] > 0) {
      const int j = sc.ok[i], len = pv.lens[s];
      sc.jobs[3 * (size_t)j] = sc.offset[i]; sc.jobs[3 * (size_t)j + 1] = sc.need[i] >> 1; sc.jobs[3 * (size_t)j + 2] = len & (pv.ps - 1);
      pv.lens[s] = len + n_new[i];
    }
    if (seqs && s >= 0) sc.mark[s] = 0x7fffffff;
  }
  if (t == 0) sc.job_count[0] = enough ? base_jobs : 0;
}

// The same for up to EXTEND_FEW entries, an entry a thread, with what is passed on in registers and shared memory: the chain of
// dependent looks into global memory (sequence, length, last page, its count) is what such a call costs (four branches given up, made
// and extended: 13.4 us with the kernel above, 8.9 with this one).
constexpr int EXTEND_FEW = 256, EXTEND_FOUND = 2048;   // entries; pages whose numbers fit shared memory

__global__ void __launch_bounds__(EXTEND_FEW) pages_extend_few_kernel(PageView pv, const int32_t* __restrict__ seqs, const int32_t* __restrict__ n_new,
                                                                      int n, int32_t* scratch) {
  __shared__ int s_seq[EXTEND_FEW], s_found[EXTEND_FOUND];
  __shared__ int2 s_scan[2][EXTEND_FEW / 32];
  pdl_enter();
  const PageScratch sc = page_scratch(pv, scratch);
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, words = (pv.n_pages + 31) >> 5;
  auto free_word = [&](int w) {
    if (w >= words) return 0u;
    const int left = pv.n_pages - w * 32;
    return pv.free_bits[w] & (left < 32 ? (1u << left) - 1u : 0xffffffffu);
  };
  uint32_t bits = free_word(t);   // (on its way while the entries are looked up)
  auto scan = [&](int2 v, int which, int2* total) {   // exclusive scan over the CTA
    const int2 own = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int a = __shfl_up_sync(0xffffffffu, v.x, o), b = __shfl_up_sync(0xffffffffu, v.y, o);
      if (lane >= o) { v.x += a; v.y += b; }
    }
    if (lane == 31) s_scan[which][warp] = v;
    __syncthreads();
    *total = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < EXTEND_FEW / 32; ++w) {
      const int2 x = s_scan[which][w];
      if (w < warp) { v.x += x.x; v.y += x.y; }
      total->x += x.x; total->y += x.y;
    }
    return make_int2(v.x - own.x, v.y - own.y);
  };
  const int s = t < n ? page_seq_of(pv, seqs, t) : -1, add = t < n ? n_new[t] : 0;
  if (seqs) {
    s_seq[t] = s;
    __syncthreads();
  }
  int len = 0, pages = 0, copies = 0, last = -1;
  bool ok = s >= 0 && add >= 0, partly = false;
  if (ok) {
    len = pv.lens[s];
    ok = len >= 0 && (long long)len + add <= min((long long)pv.max_pages << pv.ps_log2, 0x7fffffffll);
    if (seqs)
      for (int j = 0; j < t; ++j) ok = ok && s_seq[j] != s;   // a sequence named twice: its first entry counts
    partly = ok && add > 0 && (len & (pv.ps - 1));
  }
  int32_t* row = pv.table + (size_t)max(s, 0) * pv.max_pages;
  int names = 1;
  if (partly) {
    last = row[len >> pv.ps_log2];
    ok = partly = (unsigned)last < (unsigned)pv.n_pages;
    if (partly) names = pv.refs[last];
  }
  // (a page with one name has one writer: only shared ones are counted)
  const bool shared = partly && names > 1;
  if (shared) {
    atomicAdd(&sc.sharers[last], 1);
    atomicMax(&sc.last_sharer[last], t + 1);
  }
  if (__syncthreads_or(shared)) {
    if (shared) copies = !(sc.sharers[last] >= names && sc.last_sharer[last] == t + 1);
    __syncthreads();
    if (shared) { sc.sharers[last] = 0; sc.last_sharer[last] = 0; }
  }
  const int held = held_pages(pv, len);
  if (ok) pages = held_pages(pv, len + add) - held + copies;
  else if (t < n) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
  int2 all;
  const int2 off = scan(make_int2(pages, copies), 0, &all);
  const int total = all.x;
  // the lowest free pages
  int* found = total <= EXTEND_FOUND ? s_found : sc.found;
  int have = 0;
  for (int w0 = 0; w0 < words && have < total; w0 += EXTEND_FEW) {
    if (w0 > 0) {
      __syncthreads();   // (the sums of the tile before have been read)
      bits = free_word(w0 + t);
    }
    int2 sum;
    int rank = have + scan(make_int2(__popc(bits), 0), 1, &sum).x;
    while (bits && rank < total) {
      found[rank++] = (w0 + t) * 32 + __ffs(bits) - 1;
      bits &= bits - 1;
    }
    have += sum.x;
  }
  const bool enough = have >= total;
  __syncthreads();
  if (t == 0) {
    sc.job_count[0] = enough ? all.y : 0;
    if (!enough) atomicOr(pv.status, DEV_ERR_CAPACITY);
  }
  if (!enough) return;
  for (int k = t; k < total; k += EXTEND_FEW) {
    const int p = found[k];
    atomicAnd(&pv.free_bits[p >> 5], ~(1u << (p & 31)));
    pv.refs[p] = 1;
  }
  if (ok && add > 0) {
    if (copies) {
      const int p = found[off.x];
      atomicSub(&pv.refs[last], 1);
      row[held - 1] = p;
      sc.jobs[3 * (size_t)off.y] = last; sc.jobs[3 * (size_t)off.y + 1] = p; sc.jobs[3 * (size_t)off.y + 2] = len & (pv.ps - 1);
    }
    for (int k = copies; k < pages; ++k) row[held + k - copies] = found[off.x + k];
    pv.lens[s] = len + add;
  }
}

// The filled rows of shared pages into their writers' copies: one run of rows per (job, layer, K or V, head), 16 bytes a
// thread and four loads in flight.
constexpr int COPY_THREADS = 256;

__global__ void __launch_bounds__(COPY_THREADS) pages_copy_kernel(PageView pv, const int32_t* scratch) {
  pdl_enter();
  const PageScratch sc = page_scratch(pv, const_cast<int32_t*>(scratch));
  const int planes = pv.n_layers * 2;
  const long long units = (long long)sc.job_count[0] * planes * pv.H;
  const int row16 = pv.hd * pv.es / 16;   // 16-byte pieces of a row
  const size_t block16 = (size_t)pv.ps * row16;
  uint4* pool = reinterpret_cast<uint4*>(pv.pool);
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int h = (int)(u % pv.H);
    const long long r = u / pv.H;
    const int plane = (int)(r % planes), job = (int)(r / planes);
    const int from = sc.jobs[3 * (size_t)job], to = sc.jobs[3 * (size_t)job + 1], n16 = sc.jobs[3 * (size_t)job + 2] * row16;
    const uint4* src = pool + (((size_t)plane * pv.n_pages + from) * pv.H + h) * block16;
    uint4* dst = pool + (((size_t)plane * pv.n_pages + to) * pv.H + h) * block16;
    for (int e0 = 0; e0 < n16; e0 += 4 * COPY_THREADS) {
      uint4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = e0 + k * COPY_THREADS + threadIdx.x;
        if (e < n16) v[k] = __ldcs(src + e);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int e = e0 + k * COPY_THREADS + threadIdx.x;
        if (e < n16) __stcs(dst + e, v[k]);
      }
    }
  }
}

// ---------------------------------------------------------------- fork
// A CTA per entry.  Refused: a target that holds tokens, is named twice, or is also a source of the call (what a source holds
// is what it held before the call).
__global__ void __launch_bounds__(128) pages_fork_kernel(PageView pv, const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int n) {
  pdl_enter();
  const int i = blockIdx.x;
  const int a = page_seq_of(pv, src, i), b = page_seq_of(pv, dst, i);
  bool bad = a < 0 || b < 0;
  if (!bad) {
    for (int j = threadIdx.x; j < n; j += blockDim.x) bad = bad || src[j] == b || (j < i && dst[j] == b);
    bad = bad || pv.lens[b] != 0 || pv.lens[a] < 0 || pv.lens[a] > (long long)pv.max_pages * pv.ps;
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
    return;
  }
  const int len = pv.lens[a], held = held_pages(pv, len);
  const int32_t* from = pv.table + (size_t)a * pv.max_pages;
  int32_t* to = pv.table + (size_t)b * pv.max_pages;
  for (int c = threadIdx.x; c < held; c += blockDim.x) {
    const int p = from[c];
    to[c] = p;
    if ((unsigned)p < (unsigned)pv.n_pages) atomicAdd(&pv.refs[p], 1);
    else if (p != -1) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
  }
  if (threadIdx.x == 0) pv.lens[b] = len;
}

// ---------------------------------------------------------------- compact
// The checks of one entry (whole CTA): 0 <= keep <= rows <= length, the kept rows ascend inside the sequence's last `rows`
// ones, and no page that a row moves into is shared.
__device__ __forceinline__ bool compact_ok(const PageView& pv, const int32_t* seqs, const int32_t* n_rows, const int32_t* n_keep,
                                           const int32_t* rows, int row_stride, int i, int* s_out, int* base_out, int* keep_out) {
  const int s = page_seq_of(pv, seqs, i);
  bool bad = s < 0;
  int len = 0, m = 0, keep = 0;
  if (!bad) {
    len = pv.lens[s]; m = n_rows[i]; keep = n_keep[i];
    bad = len < 0 || (long long)len > (long long)pv.max_pages * pv.ps || m < 0 || m > len || keep < 0 || keep > m || (rows && keep > row_stride);
  }
  const bool dup = named_before(seqs, i, s);
  if (!bad && !dup && rows)
    for (int j = threadIdx.x; j < keep; j += blockDim.x) {
      const int r = rows[(size_t)i * row_stride + j], before = j ? rows[(size_t)i * row_stride + j - 1] : -1;
      if (r <= before || r >= m) { bad = true; continue; }
      if (r != j) {
        const int p = pv.table[(size_t)s * pv.max_pages + ((len - m + j) >> pv.ps_log2)];
        const int q = pv.table[(size_t)s * pv.max_pages + ((len - m + r) >> pv.ps_log2)];
        bad = bad || (unsigned)p >= (unsigned)pv.n_pages || (unsigned)q >= (unsigned)pv.n_pages || pv.refs[p] != 1;
      }
    }
  *s_out = s; *base_out = len - m; *keep_out = keep;
  return !__syncthreads_or(bad || dup);
}

// Kept rows to the front: grid (entry, share of the layers' planes and heads).  A thread owns 16 bytes of the rows of one
// (layer, K or V, head) and walks the kept rows in batches: their sources ascend and no target lies behind its source, so the
// loads of a batch never read what an earlier store wrote over.
constexpr int MOVE_THREADS = 256, MOVE_BATCH = 8;

__global__ void __launch_bounds__(MOVE_THREADS) pages_move_kernel(PageView pv, const int32_t* __restrict__ seqs, const int32_t* __restrict__ n_rows,
                                                                  const int32_t* __restrict__ n_keep, const int32_t* __restrict__ rows,
                                                                  int row_stride, int32_t* scratch) {
  pdl_enter();
  const PageScratch sc = page_scratch(pv, scratch);
  const int i = blockIdx.x;
  int s, base, keep;
  const bool ok = compact_ok(pv, seqs, n_rows, n_keep, rows, row_stride, i, &s, &base, &keep);
  if (blockIdx.y == 0 && threadIdx.x == 0) sc.ok[i] = ok;
  if (!ok) return;
  const int row16 = pv.hd * pv.es / 16, per = MOVE_THREADS / row16;
  const int col = threadIdx.x % row16, lane = threadIdx.x / row16;
  const int units = pv.n_layers * 2 * pv.H;
  const size_t block16 = (size_t)pv.ps * row16;
  uint4* pool = reinterpret_cast<uint4*>(pv.pool);
  const int32_t* table = pv.table + (size_t)s * pv.max_pages;
  for (int u = blockIdx.y * per + lane; u < units && lane < per; u += gridDim.y * per) {
    const int plane = u / pv.H, h = u - plane * pv.H;
    auto at = [&](int slot) {
      return pool + (((size_t)plane * pv.n_pages + table[slot >> pv.ps_log2]) * pv.H + h) * block16 + (size_t)(slot & (pv.ps - 1)) * row16 + col;
    };
    for (int j0 = 0; j0 < keep; j0 += MOVE_BATCH) {
      uint4 v[MOVE_BATCH];
      uint32_t moved = 0;
#pragma unroll
      for (int k = 0; k < MOVE_BATCH; ++k) {
        const int j = j0 + k;
        if (j < keep) {
          const int r = rows[(size_t)i * row_stride + j];
          if (r != j) { v[k] = *at(base + r); moved |= 1u << k; }
        }
      }
#pragma unroll
      for (int k = 0; k < MOVE_BATCH; ++k)
        if ((moved >> k) & 1u) *at(base + j0 + k) = v[k];
    }
  }
}

// Pages of columns [from, to) of a sequence's row of the table given back (whole CTA).
__device__ __forceinline__ void release_columns(const PageView& pv, int s, int from, int to) {
  int32_t* row = pv.table + (size_t)s * pv.max_pages;
  for (int c = from + threadIdx.x; c < to; c += blockDim.x) {
    const int p = row[c];
    if (p != -1) drop_page(pv, p);
    row[c] = -1;
  }
}

// The new lengths, and what lies behind them given back.  moved: the rows have been checked by pages_move_kernel.
__global__ void __launch_bounds__(128) pages_shrink_kernel(PageView pv, const int32_t* __restrict__ seqs, const int32_t* __restrict__ n_rows,
                                                           const int32_t* __restrict__ n_keep, int moved, const int32_t* scratch) {
  pdl_enter();
  const PageScratch sc = page_scratch(pv, const_cast<int32_t*>(scratch));
  const int i = blockIdx.x;
  int s, base, keep;
  bool ok;
  if (moved) {
    ok = sc.ok[i] != 0;
    if (ok) { s = page_seq_of(pv, seqs, i); keep = n_keep[i]; base = pv.lens[s] - n_rows[i]; }
  } else {
    ok = compact_ok(pv, seqs, n_rows, n_keep, nullptr, 0, i, &s, &base, &keep);
  }
  if (!ok) {
    if (threadIdx.x == 0) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
    return;
  }
  const int len = pv.lens[s];
  __syncthreads();
  release_columns(pv, s, held_pages(pv, base + keep), held_pages(pv, len));
  if (threadIdx.x == 0) pv.lens[s] = base + keep;
}

// ---------------------------------------------------------------- trim, free
__global__ void __launch_bounds__(128) pages_trim_kernel(PageView pv, const int32_t* __restrict__ seqs, int window, int sinks) {
  pdl_enter();
  const int s = page_seq_of(pv, seqs, blockIdx.x);
  if (named_before(seqs, blockIdx.x, s)) return;
  if (s < 0 || pv.lens[s] < 0 || pv.lens[s] > (long long)pv.max_pages * pv.ps) {
    if (threadIdx.x == 0) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
    return;
  }
  const long long hidden = (long long)pv.lens[s] - window;   // positions below this one, from the sinks on, are out of sight
  release_columns(pv, s, (int)(((long long)sinks + pv.ps - 1) >> pv.ps_log2), hidden > 0 ? (int)(hidden >> pv.ps_log2) : 0);
}

__global__ void __launch_bounds__(128) pages_free_kernel(PageView pv, const int32_t* __restrict__ seqs) {
  pdl_enter();
  const int s = page_seq_of(pv, seqs, blockIdx.x);
  if (named_before(seqs, blockIdx.x, s)) return;   // (a sequence that has been freed is empty)
  if (s < 0 || pv.lens[s] < 0 || pv.lens[s] > (long long)pv.max_pages * pv.ps) {
    if (threadIdx.x == 0) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
    return;
  }
  const int len = pv.lens[s];
  __syncthreads();
  release_columns(pv, s, 0, held_pages(pv, len));
  if (threadIdx.x == 0) pv.lens[s] = 0;
}

// ---------------------------------------------------------------- write
// K and V of new rows into their pages, 16 bytes a thread: grid (row, share of a row's pieces).
constexpr int WRITE_THREADS = 128;

__global__ void __launch_bounds__(WRITE_THREADS) pages_write_kernel(PageView pv, int layer, PageRows rows, const uint4* __restrict__ k, long long k_stride16,
                                                                    const uint4* __restrict__ v, long long v_stride16) {
  pdl_enter();
  const int row = blockIdx.x, row16 = pv.hd * pv.es / 16, n16 = pv.H * row16, e = blockIdx.y * WRITE_THREADS + threadIdx.x;
  uint4 a, b;   // requested before the row's place is looked up
  if (e < n16) { a = __ldcs(k + row * k_stride16 + e); b = __ldcs(v + row * v_stride16 + e); }
  int i = row, first, m;
  if (rows.row_off) {   // the entry whose rows hold this one: the last whose first row is not behind it
    int lo = 0, hi = rows.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (rows.row_off[mid] <= row) lo = mid; else hi = mid;
    }
    i = lo;
  }
  page_rows_of(rows, i, &first, &m);
  if (row < first || row >= first + m) return;   // behind the last sequence's rows
  const int s = page_seq_of(pv, rows.seqs, i);
  const bool dup = named_before(rows.seqs, i, s);
  bool bad = s < 0 || dup;
  int page = -1, slot = 0;
  if (!bad) {
    const int pos = page_len_of(pv, s) - m + (row - first);
    bad = pos < 0;
    if (!bad) {
      page = pv.table[(size_t)s * pv.max_pages + (pos >> pv.ps_log2)];
      slot = pos & (pv.ps - 1);
      bad = (unsigned)page >= (unsigned)pv.n_pages || pv.refs[page] != 1;
    }
  }
  if (bad) {
    if (threadIdx.x == 0 && blockIdx.y == 0) atomicOr(pv.status, DEV_ERR_INDEX_RANGE);
    return;
  }
  if (e >= n16) return;
  const int h = e / row16, c = e - h * row16;
  const size_t plane16 = (size_t)pv.n_pages * pv.H * pv.ps * row16;
  uint4* dst = reinterpret_cast<uint4*>(pv.pool) + (size_t)layer * 2 * plane16 + (((size_t)page * pv.H + h) * pv.ps + slot) * row16 + c;
  dst[0] = a;
  dst[plane16] = b;
}

}  // namespace

size_t pages_scratch_ints(const PageView& pv) { return 4 + (size_t)pv.max_seqs * 7 + (size_t)pv.n_pages * 3; }

static int reset_blocks(const PageView& pv) {
  const long long most = (long long)pv.max_seqs * pv.max_pages > pv.n_pages ? (long long)pv.max_seqs * pv.max_pages : pv.n_pages;
  const long long b = (most + 255) / 256;
  return b > 1024 ? 1024 : (int)b;
}

cudaError_t launch_pages_scratch(const PageView& pv, int32_t* scratch, cudaStream_t st) {
  launch_pdl(pages_scratch_kernel, reset_blocks(pv), 256, 0, st, pv, scratch);
  return cudaGetLastError();
}

cudaError_t launch_pages_reset(const PageView& pv, int32_t* scratch, cudaStream_t st) {
  launch_pdl(pages_reset_kernel, reset_blocks(pv), 256, 0, st, pv, scratch);
  return cudaGetLastError();
}

cudaError_t launch_pages_extend(const PageView& pv, const int32_t* seqs, const int32_t* n_new, int n, int32_t* scratch, int* launches, cudaStream_t st) {
  if (n <= EXTEND_FEW) launch_pdl(pages_extend_few_kernel, 1, EXTEND_FEW, 0, st, pv, seqs, n_new, n, scratch);
  else launch_pdl(pages_extend_kernel, 1, EXTEND_THREADS, 0, st, pv, seqs, n_new, n, scratch);
  if (cudaError_t e = cudaGetLastError()) return e;
  ++*launches;
  const long long units = (long long)n * pv.n_layers * 2 * pv.H;
  launch_pdl(pages_copy_kernel, units < 148 * 8 ? (int)units : 148 * 8, COPY_THREADS, 0, st, pv, scratch);
  ++*launches;
  return cudaGetLastError();
}

cudaError_t launch_pages_fork(const PageView& pv, const int32_t* src, const int32_t* dst, int n, cudaStream_t st) {
  launch_pdl(pages_fork_kernel, n, 128, 0, st, pv, src, dst, n);
  return cudaGetLastError();
}

cudaError_t launch_pages_compact(const PageView& pv, const int32_t* seqs, const int32_t* n_rows, const int32_t* n_keep, const int32_t* rows,
                                 int row_stride, int n, int32_t* scratch, int* launches, cudaStream_t st) {
  if (rows) {
    const int per = MOVE_THREADS / (pv.hd * pv.es / 16), units = pv.n_layers * 2 * pv.H;
    const int shares = (units + per - 1) / per;
    launch_pdl(pages_move_kernel, dim3(n, shares < 64 ? shares : 64), MOVE_THREADS, 0, st, pv, seqs, n_rows, n_keep, rows, row_stride, scratch);
    if (cudaError_t e = cudaGetLastError()) return e;
    ++*launches;
  }
  launch_pdl(pages_shrink_kernel, n, 128, 0, st, pv, seqs, n_rows, n_keep, rows ? 1 : 0, scratch);
  ++*launches;
  return cudaGetLastError();
}

cudaError_t launch_pages_trim(const PageView& pv, const int32_t* seqs, int window, int sinks, int n, cudaStream_t st) {
  launch_pdl(pages_trim_kernel, n, 128, 0, st, pv, seqs, window, sinks);
  return cudaGetLastError();
}

cudaError_t launch_pages_free(const PageView& pv, const int32_t* seqs, int n, cudaStream_t st) {
  launch_pdl(pages_free_kernel, n, 128, 0, st, pv, seqs);
  return cudaGetLastError();
}

cudaError_t launch_pages_write(const PageView& pv, int layer, const PageRows& rows, const void* k, long long k_stride, const void* v,
                               long long v_stride, cudaStream_t st) {
  const int n16 = pv.H * pv.hd * pv.es / 16;
  launch_pdl(pages_write_kernel, dim3(rows.n_rows, (n16 + WRITE_THREADS - 1) / WRITE_THREADS), WRITE_THREADS, 0, st, pv, layer, rows,
             (const uint4*)k, k_stride * pv.es / 16, (const uint4*)v, v_stride * pv.es / 16);
  return cudaGetLastError();
}

}  // namespace rd
