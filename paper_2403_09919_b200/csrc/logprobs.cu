// Log probabilities of given tokens with the distribution's entropy and its most likely tokens, one pass over the logits.
//
//   y_v = x_v / T,  lse = log sum_v exp(y_v),  logprob = y_t - lse,  entropy = lse - sum_v p_v y_v,  p_v = exp(y_v - lse)
//
// A row is one cluster of 1 to 8 CTAs whose threads take its 16-byte pieces in turn.  Each thread keeps, in 32 bits, the
// running maximum r of x and, with d = (x - r) log2(e) / T, s = sum 2^d and u = sum 2^d d, from which logprob = (x_t - r) / T -
// log s and entropy = log s - ln 2 u / s; they are joined over the lanes, warps and CTAs in a fixed order.  (The difference
// x - r is formed first: it is exact where it matters, so that no log probability comes out above 0.)
//
// The most likely tokens (larger logit first, lower index first among equals) need no second pass over the row: the k-th
// largest of the maxima of 64 or 128 groups of threads is a bound that at least k elements reach and, in expectation, few more
// (k + k^2 / 128 or so); only threads whose own maximum reaches it read their pieces again (from the L2) and list what
// reaches the bound, and the list is ranked by counting.  Where fewer than k groups hold anything above -inf, what is above it
// and the first 1024 elements are listed.  Rows with NaN or +inf, and lists that overflow, take one maximum after another.
//
// A thread takes batches of four pieces, with one maximum, one comparison and at most one change of reference a batch, and packed fp32 (a
// comparison and two selections for each element's place alone had made the scan several times as long).  1296 rows of 32000 in fp32,
// top 20: 38.3 us, 0.66 of a copy's rate.  No unit is at its limit there (issue slots 47 %, exponentials' pipe 28 %, DRAM 49 % of ncu's
// peak): a row's tail -- bound, list, ranks, a barrier each -- loads nothing, and the SM's two other CTAs hide only a part of it.  6 rows
// 6.0 us, the chain of a first load and that tail.
#include <cooperative_groups.h>

#include "logprobs.cuh"
#include "pdl.cuh"
#include "rd_internal.cuh"

namespace rd {

namespace {

namespace cg = cooperative_groups;

constexpr int LP_THREADS = 512, LP_WARPS = LP_THREADS / 32, LP_GROUPS = 128, LP_LIST = 2048;   // LP_GROUPS: most groups of threads
typedef unsigned long long u64;

// Order of the tokens as one number: larger logit first (NaN above all, as sorting puts it), lower index first.  No key is ~0, which
// stands above them all: +inf is 0xff800000 in the upper half, NaN 0xfffffffe.
__device__ __forceinline__ u64 rank_key(float x, uint32_t index) {
  uint32_t u = __float_as_uint(x + 0.f);   // (-0 is 0)
  u = x != x ? 0xfffffffeu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return ((u64)u << 32) | (0xffffffffu - index);
}
__device__ __forceinline__ float key_logit(u64 key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u == 0xfffffffeu ? 0x7fffffffu : (u & 0x80000000u) ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ uint32_t key_index(u64 key) { return 0xffffffffu - (uint32_t)key; }

template <typename T> struct Pieces;   // 16 bytes as floats
template <> struct Pieces<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ uint4 nothing() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }   // -inf
  static __device__ __forceinline__ void unpack(const uint4& v, float* x) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
  }
};
template <> struct Pieces<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ uint4 nothing() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
  static __device__ __forceinline__ void unpack(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
};

// r: largest x so far, s and u relative to it.
struct Sums { float r, s, u; };


__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ Sums rebase(const Sums& a, float r, float c2) {
  if (a.r == r || a.r == -INFINITY) return Sums{r, a.s, a.u};   // (nothing but -inf so far: s and u are zero, or NaN)
  const float d = (a.r - r) * c2, c = ex2(d);
  return Sums{r, a.s * c, c == 0.f ? 0.f * a.s : c * fmaf(a.s, d, a.u)};
}
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float c2) {
  const float r = fmaxf(a.r, b.r);
  const Sums x = rebase(a, r, c2), y = rebase(b, r, c2);
  return Sums{r, x.s + y.s, x.u + y.u};
}

// Over groups of N lanes: one change of reference each, then plain sums.
template <int N> __device__ __forceinline__ Sums join_lanes(Sums a, float c2) {
  float r = a.r;
#pragma unroll
  for (int w = 1; w < N; w <<= 1) r = fmaxf(r, __shfl_xor_sync(0xffffffffu, r, w));
  a = rebase(a, r, c2);
#pragma unroll
  for (int w = 1; w < N; w <<= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, w);
    a.u += __shfl_xor_sync(0xffffffffu, a.u, w);
  }
  return a;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
typedef float2 f2;
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("{\n\t.reg .b64 w, x, y, z;\n\tmov.b64 w, {%2, %3};\n\tmov.b64 x, {%4, %5};\n\tmov.b64 y, {%6, %7};\n\tfma.rn.f32x2 z, w, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}

// Adds N values; returns their maximum (NaN left out).
template <int N> __device__ __forceinline__ float add_values(Sums& a, const float (&x)[N], float c2) {
  float m = x[0];
  if constexpr (N > 1) {
    float m2 = x[1];
#pragma unroll
    for (int i = 2; i + 4 <= N; i += 4) { m = max3(m, x[i], x[i + 1]); m2 = max3(m2, x[i + 2], x[i + 3]); }
    m = max3(m, m2, x[N - 2]);
    m = fmaxf(m, x[N - 1]);
  }
  if (m > a.r) a = rebase(a, m, c2);
  const float ref = a.r == -INFINITY ? 0.f : a.r;
  if constexpr (N == 1) {
    const float d = (x[0] - ref) * c2, e = ex2(d);
    a.s += e;
    a.u = fmaf(e, fmaxf(d, -1024.f), a.u);   // (2^-1024 is zero, and 0 * -inf would not be)
  } else {
    const f2 nr = make_float2(-ref, -ref), cc = make_float2(c2, c2);
    f2 s2 = make_float2(a.s, 0.f), u2 = make_float2(a.u, 0.f);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const f2 d = mul2(add2(make_float2(x[i], x[i + 1]), nr), cc);
      const f2 e = make_float2(ex2(d.x), ex2(d.y));
      s2 = add2(s2, e);
      u2 = fma2(e, make_float2(fmaxf(d.x, -1024.f), fmaxf(d.y, -1024.f)), u2);
    }
    a.s = s2.x + s2.y; a.u = u2.x + u2.y;
  }
  return m;
}

// Most tokens that groups of PER threads find: the top-th largest of the groups' maxima is the bound.
constexpr int most_top(int per) { return LP_THREADS / per; }
constexpr int LP_FEW_TOP = 32, LP_FEW = 8, LP_MANY = 4;   // threads of a group for up to LP_FEW_TOP tokens, and for more
static_assert(most_top(LP_FEW) >= LP_FEW_TOP && most_top(LP_MANY) >= LOGPROB_MAX_TOP && LOGPROB_MAX_TOP <= LP_GROUPS && 8 * LOGPROB_MAX_TOP <= LP_LIST,
              "groups enough for the bound, room for the lists of a row's eight CTAs");

// PER: threads of a group.
template <typename T, int PER>
__global__ void __launch_bounds__(LP_THREADS, sizeof(T) == 2 ? 3 : 0) logprob_kernel(LogprobArgs a) {
  pdl_enter();
  using P = Pieces<T>;
  constexpr int N = P::N, UNROLL = 4;
  __shared__ u64 s_best[LP_GROUPS];
  __shared__ __align__(16) float s_group[LP_GROUPS];
  __shared__ u64 s_list[LP_LIST];
  __shared__ u64 s_top[LOGPROB_MAX_TOP];
  __shared__ Sums s_sums[LP_WARPS];
  __shared__ Sums s_total;
  __shared__ float s_bound;
  __shared__ int s_count, s_n_who;
  __shared__ short s_who[LP_THREADS];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), part = (int)cluster.block_rank();
  const int row = blockIdx.x / S, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int at = a.row_index ? a.row_index[row] : row;
  const float nan = __uint_as_float(0x7fffffffu);
  if (at < 0 || at >= a.n_logit_rows) {   // (the whole cluster)
    if (part == 0) {
      if (t == 0 && a.logprob) a.logprob[row] = nan;
      if (t == 0 && a.entropy) a.entropy[row] = nan;
      for (int k = t; k < a.top; k += LP_THREADS) {
        a.top_ids[(size_t)row * a.top + k] = -1;
        a.top_logprobs[(size_t)row * a.top + k] = nan;
      }
    }
    return;
  }
  const T* x = reinterpret_cast<const T*>(a.logits) + (long long)at * a.row_stride;
  const float c2 = a.inv_t * 1.4426950408889634f;
  float x_token = nan;
  if (part == 0 && t == 0) {
    s_count = s_n_who = 0;
    if (a.tokens && a.logprob) {
      const int tok = a.tokens[row];
      if ((unsigned)tok < (unsigned)a.vocab) x_token = to_f<T>(x[tok]);
    }
  } else if (t == 0) {
    s_count = s_n_who = 0;
  }
  // the row's elements: single ones up to a 16-byte boundary (head), pieces, single ones behind the last piece
  const int head = min((int)(((16 - ((uintptr_t)x & 15)) & 15) / sizeof(T)), a.vocab);
  const int pieces = (a.vocab - head) / N, tail0 = head + pieces * N;
  const uint4* body = reinterpret_cast<const uint4*>(x + head);
  const int single = part == 0 ? (t < head ? t : t - head < a.vocab - tail0 ? tail0 + t - head : -1) : -1;   // this thread's single element
  const int step = S * LP_THREADS, p0 = part * LP_THREADS + t;
  Sums sum{-INFINITY, 0.f, 0.f};
  float best = -INFINITY;   // this thread's largest
  for (int p = p0; p < pieces; p += UNROLL * step) {
    uint4 raw[UNROLL];
    if (p + (UNROLL - 1) * step < pieces) {
#pragma unroll
      for (int k = 0; k < UNROLL; ++k) raw[k] = body[p + k * step];
    } else {   // the last batch is filled up with -inf
#pragma unroll
      for (int k = 0; k < UNROLL; ++k) raw[k] = p + k * step < pieces ? body[p + k * step] : P::nothing();
    }
    constexpr int TAKE = N * UNROLL <= 16 ? UNROLL : 2;   // pieces at a time
#pragma unroll
    for (int k = 0; k < UNROLL; k += TAKE) {
      float v[TAKE * N];
#pragma unroll
      for (int i = 0; i < TAKE; ++i) P::unpack(raw[k + i], v + i * N);
      best = fmaxf(best, add_values(sum, v, c2));
    }
  }
  if (single >= 0) {
    const float v[1] = {to_f<T>(x[single])};
    best = fmaxf(best, add_values(sum, v, c2));
  }
  // ---- the CTA's sums and the maxima of its groups of threads
  sum = join_lanes<32>(sum, c2);
  if (lane == 0) s_sums[warp] = sum;
  if (a.top) {
    float g = best;
#pragma unroll
    for (int w = 1; w < PER; w <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, w));
    if (t % PER == 0) s_group[t / PER] = g;
  }
  __syncthreads();
  if (warp == 0) {
    Sums q = lane < LP_WARPS ? s_sums[lane] : Sums{-INFINITY, 0.f, 0.f};
    q = join_lanes<LP_WARPS>(q, c2);
    if (lane == 0) s_total = q;
  }
  if (a.top) {
    // the bound: the group maximum that is the top-th largest (equal ones write the same); a group's threads share the others
    constexpr int GROUPS = LP_THREADS / PER;
    static_assert(GROUPS <= LP_GROUPS && GROUPS % (4 * PER) == 0 && 32 % PER == 0, "a thread's share of the maxima is read 16 bytes at a time");
    const float g = s_group[t / PER];
    int above = 0, not_below = 0;
#pragma unroll
    for (int j = 0; j < GROUPS / PER; j += 4) {
      const float4 o = *reinterpret_cast<const float4*>(&s_group[(t % PER) * (GROUPS / PER) + j]);
      above += (o.x > g) + (o.y > g) + (o.z > g) + (o.w > g);
      not_below += (o.x >= g) + (o.y >= g) + (o.z >= g) + (o.w >= g);
    }
    int both = above + (not_below << 16);
#pragma unroll
    for (int w = 1; w < PER; w <<= 1) both += __shfl_xor_sync(0xffffffffu, both, w);
    if ((both & 0xffff) < a.top && (both >> 16) >= a.top) s_bound = g;
  }
  __syncthreads();
  if (a.top) {
    const float total = s_total.s;
    bool rounds = total != total;
    if (!rounds) {
      const float bound = s_bound;
      auto offer = [&](float v, int index) {
        if (bound == -INFINITY ? v > bound || index < 1024 : v >= bound) {
          const int place = atomicAdd(&s_count, 1);
          if (place < LP_LIST) s_list[place] = rank_key(v, (uint32_t)index);
        }
      };
      if (best >= bound) s_who[atomicAdd(&s_n_who, 1)] = (short)t;
      __syncthreads();
      const int n_who = s_n_who;
      for (int w = warp; w < n_who; w += LP_WARPS) {   // a warp looks through what one of those threads has read
        const int who = s_who[w];
        for (int p = part * LP_THREADS + who + lane * step; p < pieces; p += 32 * step) {
          float v[N];
          P::unpack(body[p], v);
#pragma unroll
          for (int j = 0; j < N; ++j) offer(v[j], head + p * N + j);
        }
      }
      if (single >= 0) offer(to_f<T>(x[single]), single);
      __syncthreads();
      rounds = s_count > LP_LIST;
    }
    if (rounds) {   // one maximum after another, each below the one before
      u64 before = ~0ull;   // (above every key)
      for (int r = 0; r < a.top; ++r) {
        u64 m = 0;
        auto look = [&](float v, int index) {
          const u64 key = rank_key(v, (uint32_t)index);
          if (key < before && key > m) m = key;
        };
        for (int p = p0; p < pieces; p += step) {
          float v[N];
          P::unpack(body[p], v);
          for (int j = 0; j < N; ++j) look(v[j], head + p * N + j);
        }
        if (single >= 0) look(to_f<T>(x[single]), single);
#pragma unroll
        for (int w = 1; w < 32; w <<= 1) {
          const u64 o = __shfl_xor_sync(0xffffffffu, m, w);
          m = o > m ? o : m;
        }
        __syncthreads();
        if (lane == 0) s_best[warp] = m;
        __syncthreads();
        m = 0;
        for (int w = 0; w < LP_WARPS; ++w) m = s_best[w] > m ? s_best[w] : m;
        if (t == 0) s_top[r] = m;
        before = m;
        if (m == 0) before = 1;   // nothing left: zeros follow
      }
      __syncthreads();
    } else {
      const int n = s_count;
      for (int k = t; k < a.top; k += LP_THREADS) if (k >= n) s_top[k] = 0;   // fewer elements than asked for in this CTA's share
      for (int e = t; e < n; e += LP_THREADS) {
        const u64 key = s_list[e];
        int above = 0;
        for (int j = 0; j < n; ++j) above += s_list[j] > key;
        if (above < a.top) s_top[above] = key;
      }
      __syncthreads();
    }
  }
  // ---- over the cluster's CTAs
  if (S > 1) {
    cluster.sync();
    if (part == 0) {
      if (t == 0) {
        Sums q = s_total;
        for (int c = 1; c < S; ++c) q = join(q, *cluster.map_shared_rank(&s_total, c), c2);
        s_sums[0] = q;
      }
      if (a.top) {
        const int n = S * a.top;   // <= LP_LIST
        for (int e = t; e < n; e += LP_THREADS) s_list[e] = *cluster.map_shared_rank(&s_top[e % a.top], e / a.top);
        __syncthreads();
        for (int e = t; e < n; e += LP_THREADS) {
          const u64 key = s_list[e];
          if (!key) continue;
          int above = 0;
          for (int j = 0; j < n; ++j) above += s_list[j] > key;
          if (above < a.top) s_best[above] = key;   // (top <= LP_GROUPS)
        }
      }
      __syncthreads();
    }
    cluster.sync();   // the others' shared memory has been read
    if (part != 0) return;
  }
  const Sums q = S > 1 ? s_sums[0] : s_total;
  const u64* top = S > 1 ? s_best : s_top;
  const float ln2 = 0.6931471805599453f, ref = q.r == -INFINITY ? 0.f : q.r;
  const float log_s = logf(q.s);
  if (t == 0 && a.logprob) a.logprob[row] = (x_token - ref) * a.inv_t - log_s;
  if (t == 0 && a.entropy) a.entropy[row] = log_s - q.u / q.s * ln2;
  for (int k = t; k < a.top; k += LP_THREADS) {
    const u64 key = top[k];
    a.top_ids[(size_t)row * a.top + k] = (int32_t)key_index(key);
    a.top_logprobs[(size_t)row * a.top + k] = (key_logit(key) - ref) * a.inv_t - log_s;
  }
}

}  // namespace

cudaError_t launch_logprobs(int dtype, const LogprobArgs& a, cudaStream_t st) {
  // CTAs per row: more than one where rows are long and few.  Fp32, us with 1, 2, 4, 8: 6 x 32000 6.0, 6.4, 6.2, 7.4; 6 x 64000 8.3,
  // 7.6, 6.9, 7.4; 6 x 128000 12.9, 10.0, 8.2, 8.1; 74 x 64000 8.6, 8.0, 9.9, 16.8; 148 x 32000 6.4, 9.3, 14.4, 29.7.
  int S = 1;
  while (S < 8 && (long long)a.rows * S * 2 <= 148 && a.vocab / (2 * S) >= 16384) S *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.rows * S);
  cfg.blockDim = LP_THREADS;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = S; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  // up to 32 tokens are found with 64 groups (1296 x 32000, top 20: 39.8 us against 46.4 with 128; top 64: 94 against 56)
  auto go = [&](auto kernel) { return cudaLaunchKernelEx(&cfg, kernel, a); };
  const cudaError_t e = dtype == RD_DTYPE_FP32 ? (a.top <= LP_FEW_TOP ? go(logprob_kernel<float, LP_FEW>) : go(logprob_kernel<float, LP_MANY>))
                                               : (a.top <= LP_FEW_TOP ? go(logprob_kernel<__nv_bfloat16, LP_FEW>) : go(logprob_kernel<__nv_bfloat16, LP_MANY>));
  return e ? e : cudaGetLastError();
}

}  // namespace rd
