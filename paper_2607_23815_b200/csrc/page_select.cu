// attn_select_pages: which pages of its context a query attends over, by the pages' summaries (kv_page_bounds).
//
// score(page) = max over the group's query heads of sum_d (q_d >= 0 ? q_d hi_d : q_d lo_d): no key of the page can have a larger product with any of
// those heads.  Chosen are the n_first first and n_last last pages and those others that score highest, ties to the lowest index.
//
// The order is that of the scores as defined, not of a rounded sum.  Scores are first summed in 32 bits, with an error of at most `err` (below);
// if the last page chosen and the best one left are further apart than two errors, no rounding has decided anything.  If not (a few rows in a hundred
// of normal data, and wherever scores are equal, infinite or not numbers), the pages within two errors of the border are scored again in 64 bits, in
// which the products of bf16 values are exact, and the choice is made among them.
//
// What bounds it: HBM (4 D bytes a page and KV head, read once) where there are many rows, latency where there are few, so a row's pages are then
// shared out over a cluster whose CTAs push their scores into the shared memory of the first, which chooses.
#include <math.h>

#include "common.cuh"
#include "page_mma.cuh"
#include "sm100_ptx.cuh"

namespace kvattn {
using namespace ptx;

struct SelectArgs {
  PoolView pool;
  const __nv_bfloat16* q;       // [batch][Hq][D]
  const __nv_bfloat16* bounds;  // [num_pages][Hkv][2][D]
  const int* block_tables;
  const int* ctx_lens;
  int* pages;                   // [batch][Hkv][n_select]
  int* counts;                  // [batch][Hkv]
  int max_pages, bound_pages;   // bound_pages: the keys there is shared memory for
  int n_q_heads, n_select, n_first, n_last, splits;
};

constexpr int kSelWarps = 8;
constexpr int kSelThreads = kSelWarps * 32;
constexpr int kSelMaxSplits = 8;
constexpr int kSelMaxPages = 24576;  // 192 KB of keys
constexpr int kBins = 256;
typedef unsigned long long u64;

// Keys in the order of the values, whatever is not a number above all of them; -0 and 0 are the same.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (isnan(x)) return 0xffffffffu;
  const uint32_t b = x == 0.f ? 0u : __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
__device__ __forceinline__ u64 key_of(double x) {
  if (isnan(x)) return ~0ull;
  const u64 b = x == 0.0 ? 0ull : (u64)__double_as_longlong(x);
  return b >> 63 ? ~b : b | (1ull << 63);
}

struct SelectShared {
  u64 lo, hi;                  // range of the keys still in question
  u64 warp_lo[kSelWarps], warp_hi[kSelWarps];
  unsigned hist[kBins];
  int need, bin;
  int warp_ge[kSelWarps], warp_eq[kSelWarps];
  uint32_t bmax[kSelMaxSplits];  // largest magnitude among the bounds each CTA has read (bf16 bits)
  uint32_t warp_bmax[kSelWarps];
  float qsum;
};

// The `need` largest of keys[0 .. m) are those >= ge and the first `eq` of those that equal ge - 1.
struct Choice {
  u64 ge;
  int eq;
};

__device__ __forceinline__ u64 warp_min(u64 v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = min(v, (u64)__shfl_xor_sync(0xffffffffu, v, off));
  return v;
}
__device__ __forceinline__ u64 warp_max(u64 v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = max(v, (u64)__shfl_xor_sync(0xffffffffu, v, off));
  return v;
}

// Smallest of the threads' lo and largest of their hi, for all of them.
__device__ __forceinline__ void block_range(SelectShared& sh, u64& lo, u64& hi) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  lo = warp_min(lo);
  hi = warp_max(hi);
  __syncthreads();  // (the arrays may still be read for the range before)
  if (lane == 0) {
    sh.warp_lo[warp] = lo;
    sh.warp_hi[warp] = hi;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kSelWarps; ++w) {
    lo = min(lo, sh.warp_lo[w]);
    hi = max(hi, sh.warp_hi[w]);
  }
}

// By the bits of the keys, eight at a time, counted from the highest in which the keys in question differ; 1 <= need <= m.
__device__ __forceinline__ Choice choose(SelectShared& sh, const u64* keys, int m, int need) {
  const int tid = threadIdx.x, lane = tid & 31;
  u64 lo = ~0ull, hi = 0;
  for (int i = tid; i < m; i += kSelThreads) {
    lo = min(lo, keys[i]);
    hi = max(hi, keys[i]);
  }
  block_range(sh, lo, hi);
  while (lo < hi) {
    const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - 8);
    for (int b = tid; b < kBins; b += kSelThreads) sh.hist[b] = 0;
    __syncthreads();
    for (int i = tid; i < m; i += kSelThreads) {
      const u64 k = keys[i];
      if (k >= lo && k <= hi) atomicAdd(&sh.hist[(unsigned)((k - lo) >> shift)], 1u);
    }
    __syncthreads();
    if (tid < 32) {  // the bin that the last one needed lies in: lane 31 has the highest eight bins
      unsigned mine[kBins / 32], sum = 0;
#pragma unroll
      for (int i = 0; i < kBins / 32; ++i) {
        mine[i] = sh.hist[lane * (kBins / 32) + i];
        sum += mine[i];
      }
      unsigned above = sum;  // then: in this lane's bins and those above
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const unsigned x = __shfl_down_sync(0xffffffffu, above, off);
        if (lane + off < 32) above += x;
      }
      above -= sum;
      if (above < (unsigned)need && above + sum >= (unsigned)need) {
#pragma unroll
        for (int i = kBins / 32 - 1; i >= 0; --i) {
          if (above + mine[i] >= (unsigned)need) {
            sh.bin = lane * (kBins / 32) + i;
            sh.need = need - above;
            break;
          }
          above += mine[i];
        }
      }
    }
    __syncthreads();
    const u64 start = lo + ((u64)sh.bin << shift);
    need = sh.need;
    if (sh.hist[sh.bin] == (unsigned)need) return Choice{start, 0};
    if (hi - start >= 1ull << shift) hi = start + ((1ull << shift) - 1);
    lo = start;
    __syncthreads();  // (bin, need and the counts are read before they are written again)
  }
  return Choice{lo + 1, need};  // all that is left is equal (lo = ~0: ge wraps to 0, see taken())
}

// Is a key among the chosen for sure / one of the equals of which only some are?  (Keys of ~0 make ge wrap around to 0.)
__device__ __forceinline__ bool surely(const Choice& c, u64 k) { return c.ge == 0 && c.eq > 0 ? false : k >= c.ge; }
__device__ __forceinline__ bool equals(const Choice& c, u64 k) { return c.eq > 0 && k == c.ge - 1; }

// Sum over kLanes neighbouring lanes of each of v[0 .. N): the lanes share out the sums; returns the largest of the N.
template <int N, int kLanes>
__device__ __forceinline__ float largest_sum(float (&v)[N]) {
  const int lane = threadIdx.x & 31;
  int n = N;
#pragma unroll
  for (int off = kLanes / 2; off > 0; off >>= 1) {
    if (n > 1) {
      n >>= 1;
      const bool up = lane & off;
#pragma unroll
      for (int i = 0; i < N / 2; ++i)
        if (i < n) {
          const float give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
          v[i] = keep + __shfl_xor_sync(0xffffffffu, give, off);
        }
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], off);
    }
  }
  float best = v[0];
#pragma unroll
  for (int off = kLanes / 2, k = N; k > 1; off >>= 1, k >>= 1) {
    const float other = __shfl_xor_sync(0xffffffffu, best, off);
    best = isnan(best) || best > other ? best : other;
  }
  return best;
}

template <int kDims>
__device__ __forceinline__ void load_dims(uint32_t (&w)[kDims / 2], const __nv_bfloat16* p) {
  if constexpr (kDims == 8)
    asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
  else
    asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
}
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The score by its definition, in 64 bits, for the whole warp.
template <int D, int G>
__device__ __forceinline__ u64 exact_key(const __nv_bfloat16* q, const __nv_bfloat16* bounds) {
  constexpr int kDims = D / 32;
  const int lane = threadIdx.x & 31;
  double best = -INFINITY;
#pragma unroll 1
  for (int g = 0; g < G; ++g) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kDims; ++i) {
      const int d = lane * kDims + i;
      const double x = (double)__bfloat162float(q[g * D + d]);
      sum += x * (double)__bfloat162float(x >= 0.0 ? bounds[D + d] : bounds[d]);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    best = isnan(best) || best > sum ? best : sum;
  }
  return key_of(best);
}

template <int D, int G>
__global__ void __launch_bounds__(kSelThreads) select_pages_kernel(const SelectArgs a) {
  constexpr int kDims = G == 8 ? 4 : 8;      // of a lane (its q takes 2 G kDims registers)
  constexpr int kLanes = D / kDims;          // of a page
  constexpr int kAtOnce = 32 / kLanes;       // pages of a warp's load
  constexpr int kDeep = 4;                   // loads in flight
  extern __shared__ u64 keys[];
  __shared__ SelectShared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, sub = lane / kLanes, dim0 = lane % kLanes * kDims;
  const int splits = a.splits, row = blockIdx.x / splits, rank = blockIdx.x - row * splits;
  const int Hkv = a.pool.n_kv_heads, seq = row / Hkv, kvh = row - seq * Hkv;
  if (splits > 1) cluster_arrive();
  ptx::dependency_wait();

  const int L = ptx::ld_plain(a.ctx_lens + seq);
  const bool fits = L <= a.max_pages * (int64_t)kPageSize && L <= a.bound_pages * (int64_t)kPageSize;
  if (!fits && rank == 0 && tid == 0) report(a.pool.status, KV_ERR_BOUNDS);  // left unwritten
  const int nb = fits && L > 0 ? (int)(((int64_t)L + kPageSize - 1) / kPageSize) : 0;
  int* list = a.pages + (int64_t)row * a.n_select;
  if (nb <= a.n_select) {  // every page is chosen
    if (splits > 1) cluster_wait();
    if (fits && rank == 0) {
      for (int i = tid; i < a.n_select; i += kSelThreads) list[i] = i < nb ? i : -1;
      if (tid == 0) a.counts[row] = nb;
    }
    return;
  }

  // ---- scores of the pages n_first .. nb - n_last - 1; key i is that of page n_first + i
  const int m = nb - a.n_first - a.n_last, need = a.n_select - a.n_first - a.n_last;
  const __nv_bfloat16* q = a.q + ((int64_t)seq * a.n_q_heads + kvh * G) * D;
  const int* table = a.block_tables + (int64_t)seq * a.max_pages + a.n_first;
  const int64_t page_stride = (int64_t)Hkv * 2 * D;
  const __nv_bfloat16* base = a.bounds + (int64_t)kvh * 2 * D;
  if (need > 0) {
    const int runs = kSelWarps * splits, run = rank * kSelWarps + warp;
    const int begin = (int)((int64_t)m * run / runs), end = (int)((int64_t)m * (run + 1) / runs);
    auto table_entry = [&](int i) {
      int pg = 0;
      if (i < end) {
        pg = ptx::ld_plain(table + i);
        if ((unsigned)pg >= (unsigned)a.pool.num_pages) {
          report(a.pool.status, KV_ERR_BOUNDS);
          pg = 0;  // stay inside; the result of this row is flagged, not trusted
        }
      }
      return pg;
    };
    int cur = table_entry(begin + lane), nxt = table_entry(begin + 32 + lane), at = begin;
    float qp[G][kDims], qn[G][kDims], qsum = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      uint32_t w[kDims / 2];
      load_dims<kDims>(w, q + g * D + dim0);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kDims; ++i) {
        const float x = i & 1 ? high_half(w[i / 2]) : low_half(w[i / 2]);
        qp[g][i] = x >= 0.f ? x : 0.f;
        qn[g][i] = x >= 0.f ? 0.f : x;  // (not a number: here, and so in every score)
        sum += fabsf(x);
      }
#pragma unroll
      for (int off = kLanes / 2; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      qsum = isnan(qsum) || qsum > sum ? qsum : sum;
    }
    if (tid == 0) sh.qsum = qsum;
    if (splits > 1) cluster_wait();  // the first CTA runs: its shared memory may be written
    const uint32_t keys0 = splits > 1 ? cluster_addr(ptx::smem_u32(keys), 0) : 0;
    uint32_t big = 0;  // largest magnitude among the bounds, two at a time
    for (int i0 = begin; i0 < end; i0 += kAtOnce * kDeep) {
      if (i0 - at >= 32) {
        cur = nxt;
        at += 32;
        nxt = table_entry(at + 32 + lane);
      }
      uint32_t lo[kDeep][kDims / 2], hi[kDeep][kDims / 2];
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        const int pg = __shfl_sync(0xffffffffu, cur, i0 - at + u * kAtOnce + sub);
        const __nv_bfloat16* src = base + pg * page_stride + dim0;
        if (i0 + u * kAtOnce + sub < end) {
          load_dims<kDims>(lo[u], src);
          load_dims<kDims>(hi[u], src + D);
        } else {
#pragma unroll
          for (int w = 0; w < kDims / 2; ++w) lo[u][w] = hi[u][w] = 0;
        }
      }
#pragma unroll
      for (int u = 0; u < kDeep; ++u) {
        float sum[G];
#pragma unroll
        for (int g = 0; g < G; ++g) sum[g] = 0.f;
#pragma unroll
        for (int w = 0; w < kDims / 2; ++w) {
          big = __vmaxu2(big, __vmaxu2(lo[u][w] & 0x7fff7fffu, hi[u][w] & 0x7fff7fffu));
          const float l0 = low_half(lo[u][w]), l1 = high_half(lo[u][w]), h0 = low_half(hi[u][w]), h1 = high_half(hi[u][w]);
#pragma unroll
          for (int g = 0; g < G; ++g) {
            sum[g] = fmaf(qp[g][2 * w], h0, sum[g]);
            sum[g] = fmaf(qn[g][2 * w], l0, sum[g]);
            sum[g] = fmaf(qp[g][2 * w + 1], h1, sum[g]);
            sum[g] = fmaf(qn[g][2 * w + 1], l1, sum[g]);
          }
        }
        const float best = largest_sum<G, kLanes>(sum);
        const int i = i0 + u * kAtOnce + sub;
        if (lane % kLanes == 0 && i < end) {
          const u64 key = (u64)key_of(best) << 32;
          if (splits > 1)
            asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(keys0 + i * 8), "l"(key) : "memory");
          else
            keys[i] = key;
        }
      }
    }
    big = max(big & 0xffffu, big >> 16);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, off));
    if (lane == 0) sh.warp_bmax[warp] = big;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
      for (int w = 0; w < kSelWarps; ++w) big = max(big, sh.warp_bmax[w]);
      if (splits > 1)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(ptx::smem_u32(&sh.bmax[rank]), 0)), "r"(big) : "memory");
      else
        sh.bmax[0] = big;
    }
    if (splits > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
  } else if (splits > 1) {
    cluster_wait();
  }
  ptx::launch_dependents();
  if (rank != 0) return;

  // ---- the choice, by the first CTA
  Choice ch{~0ull, 0};
  if (need > 0) {
    ch = choose(sh, keys, m, need);
    uint32_t big = 0;
    for (int s = 0; s < splits; ++s) big = max(big, sh.bmax[s]);
    // A sum of a lane takes 2 kDims roundings, the sum over the lanes five at most, and so each partial sum of at most (sum |q|) max |bound| is
    // rounded no more than 21 times, each by 2^-24 of itself: below 2^-19 of it in all.  Twice that for the sum of |q| itself; what is too small
    // for 32 bits adds less than 2^-140.
    const float err = sh.qsum * low_half(big) * 0x1p-18f + 0x1p-140f;
    u64 lo = ~0ull, hi = 0;  // the smallest key chosen, the largest one left
    int seen_eq = 0;
    for (int i = tid; i < m; i += kSelThreads) {
      const u64 k = keys[i];
      if (surely(ch, k)) lo = min(lo, k);
      else hi = max(hi, k);
      seen_eq |= equals(ch, k);
    }
    if (__syncthreads_or(seen_eq)) lo = min(lo, ch.ge - 1);  // (equals chosen and, maybe, equals left)
    block_range(sh, lo, hi);
    const float kept = value_of((uint32_t)(lo >> 32)), left = value_of((uint32_t)(hi >> 32));
    if (m > need && !(kept - left > 2.f * err)) {
      for (int i0 = warp; i0 < m; i0 += kSelWarps) {
        const float v = value_of((uint32_t)(keys[i0] >> 32));
        u64 k = v > kept + 2.f * err ? ~0ull : 0ull;
        if (k == 0 && !(v < kept - 2.f * err)) {
          int pg = ptx::ld_plain(table + i0);
          if ((unsigned)pg >= (unsigned)a.pool.num_pages) pg = 0;  // (reported above)
          k = exact_key<D, G>(q, base + pg * page_stride);
        }
        __syncwarp();
        if (lane == 0) keys[i0] = k;
      }
      __syncthreads();
      ch = choose(sh, keys, m, need);
    }
  }

  // ---- the list, ascending: a warp takes a run of the keys
  const int begin = (int)((int64_t)m * warp / kSelWarps), end = (int)((int64_t)m * (warp + 1) / kSelWarps);
  int ge = 0, eq = 0;
  if (need > 0) {
    for (int i0 = begin; i0 < end; i0 += 32) {
      const bool in = i0 + lane < end;
      const u64 k = in ? keys[i0 + lane] : 0;
      ge += __popc(__ballot_sync(0xffffffffu, in && surely(ch, k)));
      eq += __popc(__ballot_sync(0xffffffffu, in && equals(ch, k)));
    }
  }
  if (lane == 0) {
    sh.warp_ge[warp] = ge;
    sh.warp_eq[warp] = eq;
  }
  __syncthreads();
  int out = a.n_first, eq_left = ch.eq;
  for (int w = 0; w < warp; ++w) {
    out += sh.warp_ge[w] + min(eq_left, sh.warp_eq[w]);
    eq_left -= min(eq_left, sh.warp_eq[w]);
  }
  if (need > 0) {
    for (int i0 = begin; i0 < end; i0 += 32) {
      const bool in = i0 + lane < end;
      const u64 k = in ? keys[i0 + lane] : 0;
      const unsigned eqs = __ballot_sync(0xffffffffu, in && equals(ch, k));
      const bool take = in && (surely(ch, k) || (equals(ch, k) && __popc(eqs & ((1u << lane) - 1)) < eq_left));
      const unsigned takes = __ballot_sync(0xffffffffu, take);
      if (take) list[out + __popc(takes & ((1u << lane) - 1))] = a.n_first + i0 + lane;
      out += __popc(takes);
      eq_left -= min(eq_left, __popc(eqs));
    }
  }
  for (int i = tid; i < a.n_first; i += kSelThreads) list[i] = i;
  for (int i = tid; i < a.n_last; i += kSelThreads) list[a.n_select - a.n_last + i] = nb - a.n_last + i;
  if (tid == 0) a.counts[row] = a.n_select;
}

template <int D, int G>
static kv_status_t launch_select_variant(const kv_pool_t* p, const SelectArgs& a, int rows, cudaStream_t st) {
  static std::atomic<bool> ready[kMaxDevices];
  const auto prepare = [] {
    return cudaFuncSetAttribute(select_pages_kernel<D, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSelMaxPages * 8) == cudaSuccess &&
           cudaFuncSetAttribute(select_pages_kernel<D, G>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
  };
  if (!once_per_device(ready, p->device, prepare)) {
    cudaGetLastError();
    return KV_ERR_CUDA;
  }
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3((unsigned)(rows * a.splits));
  cfg.blockDim = dim3(kSelThreads);
  cfg.dynamicSmemBytes = (size_t)a.bound_pages * 8;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)a.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.splits > 1 ? 2 : 1;
  KV_CUDA_OK(cudaLaunchKernelEx(&cfg, select_pages_kernel<D, G>, a));
  count_launch();
  return KV_OK;
}

template <int D>
static kv_status_t launch_select(const kv_pool_t* p, const SelectArgs& a, int rows, int group, cudaStream_t st) {
  switch (group) {
    case 1: return launch_select_variant<D, 1>(p, a, rows, st);
    case 2: return launch_select_variant<D, 2>(p, a, rows, st);
    case 4: return launch_select_variant<D, 4>(p, a, rows, st);
    default: return launch_select_variant<D, 8>(p, a, rows, st);
  }
}

}  // namespace kvattn

using namespace kvattn;

extern "C" kv_status_t attn_select_pages(kv_pool_t* p, const void* q, int n_q_heads, const void* bounds, const int* block_tables, int max_pages,
                                         const int* ctx_lens, int batch, int max_ctx_len, int n_select, int n_first, int n_last, int* pages,
                                         int* counts, void* stream) {
  if (p == nullptr || batch < 0 || max_pages < 0 || max_ctx_len < 0 || n_select < 1 || n_first < 0 || n_last < 0) return KV_ERR_INVALID;
  if ((int64_t)n_first + n_last > n_select) return KV_ERR_INVALID;
  if (n_q_heads <= 0 || n_q_heads % p->n_kv_heads != 0) return KV_ERR_UNSUPPORTED;
  const int group = n_q_heads / p->n_kv_heads;
  if (!(group == 1 || group == 2 || group == 4 || group == 8)) return KV_ERR_UNSUPPORTED;
  if (batch == 0) return KV_OK;
  if (q == nullptr || bounds == nullptr || block_tables == nullptr || ctx_lens == nullptr || pages == nullptr || counts == nullptr) return KV_ERR_INVALID;
  if ((((uintptr_t)q) | ((uintptr_t)bounds)) & 15) return KV_ERR_INVALID;
  if (max_ctx_len > (int64_t)max_pages * kPageSize) return KV_ERR_INVALID;
  if (!on_pool_device(p)) return KV_ERR_INVALID;
  const int64_t rows = (int64_t)batch * p->n_kv_heads, bound = ((int64_t)max_ctx_len + kPageSize - 1) / kPageSize;
  if (bound > kSelMaxPages || rows * kSelMaxSplits > 0x7fffffffLL) return KV_ERR_UNSUPPORTED;
  SelectArgs a{p->view(), (const __nv_bfloat16*)q, (const __nv_bfloat16*)bounds, block_tables, ctx_lens, pages, counts, max_pages, (int)bound,
               n_q_heads, n_select, n_first, n_last, 1};
  // As many CTAs to a row as the device has room for beside the other rows, while a warp still has sixteen pages.
  const int sms = sm_count_of(p->device);
  while (a.splits < kSelMaxSplits && rows * a.splits * 2 <= 2 * sms && bound >= (int64_t)a.splits * 2 * kSelWarps * 16) a.splits *= 2;
  return p->head_dim == 128 ? launch_select<128>(p, a, (int)rows, group, (cudaStream_t)stream)
                            : launch_select<64>(p, a, (int)rows, group, (cudaStream_t)stream);
}
