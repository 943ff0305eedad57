// attn_select_pages: which pages of its context a query attends over, by the pages' summaries (kv_page_bounds).
//
// score(page) = max over the group's query heads of sum_d (q_d >= 0 ? q_d hi_d : q_d lo_d): no key of the page can have a larger product with any of
// those heads.  Chosen are the n_first first and n_last last pages and those others that score highest, ties to the lowest index.
//
// The order is that of the scores as defined, not of a rounded sum.  Scores are first summed by the tensor cores, with an error of at most `err` (below);
// if the last page chosen and the best one left are further apart than two errors, no rounding has decided anything.  If not (a few rows in a hundred
// of normal data, and wherever scores are equal, infinite or not numbers), the pages within two errors of the border are scored again in 64 bits, in
// which the products of bf16 values are exact, and the choice is made among them.
//
// What bounds it: HBM (4 D bytes a page and KV head, read once) where there are many rows, latency where there are few, so a row's pages are then
// shared out over a cluster whose CTAs push their scores into the shared memory of the first, which chooses.  A score is a product of (q+, q-), the
// positive and the negative part of q, with (hi, lo): sixteen pages by eight heads in an mma.sync.m16n8k16 whose A fragments are the 16-byte chunks as
// they lie.  (The lanes' own multiplications, G for every element, and their sums by shuffles took 103 us where this takes 25; the tensor
// pipe is busy a tenth of the time.)  32 documents of 8192-16384 tokens, 64/8 heads of 128: 25.4 us, 3.9 TB/s; 15 us of it are the bytes, the rest is what a
// row has in front of them (length, page ids, the first pages: three trips to memory) and behind them (the choice, 2 to 3 us), at which no other row's
// pages are read: the rows are on the device all at once.  256 sequences of 1024-4096: 42 us, 4.1 TB/s.  One of 15000: 5.7 us.  What has been left:
// rows of the next round fetched in front of the choice, which only batches of more than four rows to an SM would gain by.
#include <math.h>

#include <type_traits>

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
  int group, n_select, n_first, n_last, splits;
};

constexpr int kSelMaxSplits = 8;
constexpr int kSelMaxWarps = 16;
constexpr int kSelMaxPages = 24576;  // 198 KB of keys and marks
constexpr int kBins = 256;
constexpr int kNear = 32;
constexpr int kFew = 128;  // pages whose order is found by comparing each with each
typedef unsigned long long u64;

// Keys in the order of the values, whatever is not a number above all of them; -0 and 0 are the same.  A page has room for 64 bits in shared memory:
// the sum of 32 bits takes the upper half, the exact score all of it.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = x == 0.f ? 0u : __float_as_uint(x);
  return isnan(x) ? 0xffffffffu : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
constexpr u64 kBelow = 0, kAbove = ~0ull;  // keys of no value
__device__ __forceinline__ u64 key_of(double x) {
  if (isnan(x)) return kAbove - 1;
  const u64 b = x == 0.0 ? 0ull : (u64)__double_as_longlong(x);
  return b >> 63 ? ~b : b | (1ull << 63);
}
template <typename Key>
__device__ __forceinline__ Key key_at(const u64* keys, int i) {
  if constexpr (sizeof(Key) == 4) return reinterpret_cast<const uint32_t*>(keys)[2 * i + 1];
  else return keys[i];
}

struct SelectShared {
  uint4 q[3][4][32];  // [negative elements, positive ones, all without their signs][16-byte chunk 4 j + c of head r, by j][lane (r, c)]
  float qsum[kSelMaxWarps];
  unsigned hist[3][kBins];
  // of each run of pages: the smallest and the largest key, the largest sum of magnitudes of a score's terms (bits)
  uint32_t run_lo[kSelMaxSplits * kSelMaxWarps], run_hi[kSelMaxSplits * kSelMaxWarps], run_reach[kSelMaxSplits * kSelMaxWarps];
  uint32_t warp_kept[kSelMaxWarps], warp_left[kSelMaxWarps];
  u64 warp_lo[kSelMaxWarps], warp_hi[kSelMaxWarps];
  int warp_above[kSelMaxWarps];
  // the first of the pages near the border
  int near_count, near_page[kNear];
  u64 near_key[kNear];
};

// The chosen of the keys are those >= ge and the first `eq` of those that equal ge - 1.
struct Choice {
  u64 ge;
  int eq;
};
__device__ __forceinline__ bool surely(const Choice& c, u64 k) { return k >= c.ge; }
__device__ __forceinline__ bool equals(const Choice& c, u64 k) { return c.eq > 0 && k == c.ge - 1; }

// The `need` largest of the keys in [lo, hi], by their bits, eight at a time, counted from the highest in which lo and hi differ; there are `need` of
// them at least, 1 <= need.  One barrier a turn: every warp looks through the counts by itself, and there are three sets of them, so that the one that
// is cleared for the next turn has been read by all.  turn: of the block's turns so far; set turn % 3 is clear.
template <typename Key>
__device__ __forceinline__ Choice choose(SelectShared& sh, const u64* keys, int m, int need, Key lo, Key hi, int& turn) {
  const int tid = threadIdx.x, lane = tid & 31;
  while (lo < hi) {
    const Key span = hi - lo;
    const int bits = sizeof(Key) == 4 ? 32 - __clz((int)span) : 64 - __clzll((long long)span), shift = bits > 8 ? bits - 8 : 0;
    unsigned* hist = sh.hist[turn % 3];
    unsigned* next = sh.hist[(turn + 1) % 3];
    ++turn;
    for (int b = tid; b < kBins; b += blockDim.x) next[b] = 0;
    for (int i = tid; i < m; i += blockDim.x) {
      const Key k = key_at<Key>(keys, i);
      if (k >= lo && k <= hi) atomicAdd(&hist[(unsigned)((k - lo) >> shift)], 1u);
    }
    __syncthreads();
    // the bin that the last one needed lies in: lane 31 has the highest eight bins
    const uint4 h0 = *reinterpret_cast<const uint4*>(hist + 8 * lane), h1 = *reinterpret_cast<const uint4*>(hist + 8 * lane + 4);
    const unsigned h[8] = {h0.x, h0.y, h0.z, h0.w, h1.x, h1.y, h1.z, h1.w};
    const unsigned sum = h[0] + h[1] + h[2] + h[3] + h[4] + h[5] + h[6] + h[7];
    unsigned above = sum;  // then: in the bins above this lane's
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const unsigned x = __shfl_down_sync(0xffffffffu, above, off);
      if (lane + off < 32) above += x;
    }
    above -= sum;
    unsigned bin = 0, count = 0, rest = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
      if (above < (unsigned)need && above + h[i] >= (unsigned)need) {
        bin = 8 * lane + i;
        count = h[i];
        rest = need - above;
      }
      above += h[i];
    }
    const int at = __ffs(__ballot_sync(0xffffffffu, count != 0)) - 1;
    bin = __shfl_sync(0xffffffffu, bin, at);
    count = __shfl_sync(0xffffffffu, count, at);
    need = __shfl_sync(0xffffffffu, rest, at);
    const Key start = lo + ((Key)bin << shift);
    if (count == (unsigned)need) return Choice{start, 0};
    if ((Key)(hi - start) >> shift != 0) hi = start + (((Key)1 << shift) - 1);
    lo = start;
  }
  return Choice{(u64)lo + 1, need};  // all that is left is equal
}

// The larger of the magnitudes of two pairs of bf16 (not a number, if one of them is not).
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmax2_nan(__habs2(*reinterpret_cast<const __nv_bfloat162*>(&a)), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// The score by its definition, in 64 bits, for the whole warp.
template <int D>
__device__ __forceinline__ u64 exact_key(const __nv_bfloat16* q, const __nv_bfloat16* bounds, int group) {
  constexpr int kDims = D / 32, kWords = kDims / 2;  // of a lane
  const int lane = threadIdx.x & 31;
  auto load = [&](const __nv_bfloat16* p, uint32_t (&w)[kWords]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = (uint32_t)ptx::ld_plain(reinterpret_cast<const int*>(p + lane * kDims) + i);
  };
  auto value = [](const uint32_t (&w)[kWords], int i) { return (double)__uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); };
  uint32_t lo[kWords], hi[kWords], x[8][kWords];
  load(bounds, lo);
  load(bounds + D, hi);
#pragma unroll
  for (int g = 0; g < 8; ++g)
    if (g < group) load(q + g * D, x[g]);
  double sum[8];
#pragma unroll
  for (int g = 0; g < 8; ++g) {
    sum[g] = 0.0;
    if (g < group) {
#pragma unroll
      for (int i = 0; i < kDims; ++i) {
        const double v = value(x[g], i);
        sum[g] += v * (v >= 0.0 ? value(hi, i) : value(lo, i));
      }
    }
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
#pragma unroll
    for (int g = 0; g < 8; ++g) sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], off);
  double best = sum[0];
#pragma unroll
  for (int g = 1; g < 8; ++g)
    if (g < group) best = isnan(best) || best > sum[g] ? best : sum[g];
  return key_of(best);
}

// kBlocks: blocks on an SM.  Of more than sixteen warps none has registers for a whole tile on its way.
template <int D, int kWarps, int kBlocks>
__global__ void __launch_bounds__(kWarps * 32, kBlocks) select_pages_kernel(const SelectArgs a) {
  constexpr int NJ = D / 32;  // 16-byte chunks of lo (and of hi) of a page that a lane takes
  constexpr int kThreads = kWarps * 32;
  constexpr bool kRanks = kBlocks == 7;  // (a kernel for rows of few pages)
  extern __shared__ u64 keys[];
  __shared__ __align__(16) SelectShared sh;
  __shared__ __align__(16) uint32_t few_keys[kRanks ? kFew : 4];  // 0 behind the last
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, c = lane & 3;
  const int splits = a.splits, row = blockIdx.x / splits, rank = blockIdx.x - row * splits;
  const int Hkv = a.pool.n_kv_heads, G = a.group, seq = row / Hkv, kvh = row - seq * Hkv;
  const int runs = kWarps * splits, run = rank * kWarps + warp;
  for (int b = tid; b < kBins; b += kThreads) sh.hist[0][b] = 0;
  if constexpr (kRanks)
    for (int i = tid; i < kFew; i += kThreads) few_keys[i] = 0;
  if (tid == 0) sh.near_count = 0;
  if (splits > 1) cluster_arrive();
  ptx::dependency_wait();

  // The length, the first pages and the query at once; what the length rules out is not used.  A warp takes every `runs`-th sixteen pages, the next two
  // sixteens' ids are on their way meanwhile.
  const int L = ptx::ld_plain(a.ctx_lens + seq);
  const int* table = a.block_tables + (int64_t)seq * a.max_pages + a.n_first;
  auto table_entry = [&](int tile, int limit) {  // lanes 0 - 15: of this sixteen, 16 - 31: of the warp's next
    const int i = (tile + (lane >> 4) * runs) * 16 + (lane & 15);
    return i < limit ? ptx::ld_plain(table + i) : 0;
  };
  const int in_table = min(a.max_pages, a.bound_pages) - a.n_first;
  int ids = table_entry(run, in_table), ids_behind = table_entry(run + 2 * runs, in_table);
  const __nv_bfloat16* q = a.q + ((int64_t)seq * Hkv + kvh) * G * D;
  static_assert(kWarps >= NJ, "a warp for every chunk of the query");
  if (warp < NJ) {  // head r's chunks 4 warp + c: the positive elements (for hi) and the others (for lo)
    const uint4 x = r < G ? ptx::ld_plain(reinterpret_cast<const uint4*>(q + r * D) + 4 * warp + c) : make_uint4(0, 0, 0, 0);
    uint4 pos, neg;
    constexpr uint32_t kAbs = 0x7fff7fffu;  // two elements without their signs
    const uint4 any = make_uint4(x.x & kAbs, x.y & kAbs, x.z & kAbs, x.w & kAbs);
    float sum = 0.f;
    bool odd = false;  // an element below the normal numbers, which the tensor cores may take for 0
    auto split = [&](uint32_t w, uint32_t& pos, uint32_t& neg) {
      const uint32_t mask = (w & 0x8000u ? 0xffffu : 0u) | (w & 0x80000000u ? 0xffff0000u : 0u);
      pos = w & ~mask;
      neg = w & mask;
      sum += fabsf(__uint_as_float(w << 16)) + fabsf(__uint_as_float(w & 0xffff0000u));
      odd |= ((w & 0x7f80u) == 0 && (w & 0x7fu) != 0) || ((w & 0x7f800000u) == 0 && (w & 0x7f0000u) != 0);
    };
    split(x.x, pos.x, neg.x);
    split(x.y, pos.y, neg.y);
    split(x.z, pos.z, neg.z);
    split(x.w, pos.w, neg.w);
    sh.q[0][warp][lane] = neg;
    sh.q[1][warp][lane] = pos;
    sh.q[2][warp][lane] = any;
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    sum = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(sum)));  // (not a number: above all)
    if (__any_sync(0xffffffffu, odd)) sum = INFINITY;
    if (lane == 0) sh.qsum[warp] = sum;
  }

  const bool fits = L <= a.max_pages * (int64_t)kPageSize && L <= a.bound_pages * (int64_t)kPageSize;
  if (!fits && rank == 0 && tid == 0) report(a.pool.status, KV_ERR_BOUNDS);  // left unwritten
  const int nb = fits && L > 0 ? (int)(((int64_t)L + kPageSize - 1) / kPageSize) : 0;
  int* list = a.pages + (int64_t)row * a.n_select;
  const int m = nb - a.n_first - a.n_last, need = a.n_select - a.n_first - a.n_last;  // key i is that of page n_first + i
  const int64_t page_stride = (int64_t)Hkv * 2 * D;
  const __nv_bfloat16* base = a.bounds + (int64_t)kvh * 2 * D;
  const bool all = nb <= a.n_select, scored = !all && need > 0, few = kRanks && m <= kFew;

  // ---- scores
  if (scored) {
    if (splits > 1) cluster_wait();  // the first CTA runs: its shared memory may be written
    // where the keys are in this CTA and in the first
    const uint32_t keys_here = few ? ptx::smem_u32(few_keys) : ptx::smem_u32(keys) + 4, keys_at = splits > 1 ? cluster_addr(keys_here, 0) : keys_here;
    const uint32_t key_step = few ? 4 : 8;
    uint32_t reach = 0, least = 0xffffffffu, most = 0;  // reach: the largest sum of the magnitudes of a score's terms (bits)
    const int tiles = (m + 15) / 16;
    // A tile's two pages of this lane.  A part of a tile that has been multiplied is followed by a part of the same or of the next tile, so that loads are
    // under way all the time.
    const uint4* all_bounds = reinterpret_cast<const uint4*>(a.bounds);
    constexpr int kAhead = kWarps * kBlocks > 16 ? 1 : NJ;  // parts of a tile (of this, then of the next) that are on their way
    struct Place { uint32_t src[2]; bool in[2]; };  // (in 16 bytes: 32 bits reach further than any pool's bounds)
    auto find = [&](int n, int tile) {  // the n-th tile of the warp, each once and in order
      if ((n & 1) == 0 && n > 0) {
        ids = ids_behind;
        ids_behind = table_entry(tile + 2 * runs, m);
      }
      Place at;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        int pg = __shfl_sync(0xffffffffu, ids, 16 * (n & 1) + 8 * s + r);
        at.in[s] = 16 * tile + 8 * s + r < m;
        if (at.in[s] && (unsigned)pg >= (unsigned)a.pool.num_pages) {
          report(a.pool.status, KV_ERR_BOUNDS);
          pg = 0;  // stay inside; the result of this row is flagged, not trusted
        }
        at.src[s] = ((uint32_t)pg * Hkv + kvh) * (D / 4) + c;
      }
      return at;
    };
    uint4 lo[kAhead][2], hi[kAhead][2];
    auto load = [&](const Place& at, int j) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        lo[j % kAhead][s] = at.in[s] ? ldg_stream(all_bounds + at.src[s] + 4 * j) : make_uint4(0, 0, 0, 0);
        hi[j % kAhead][s] = at.in[s] ? ldg_stream(all_bounds + at.src[s] + D / 8 + 4 * j) : make_uint4(0, 0, 0, 0);
      }
    };
    Place now{};
    if (run < tiles) {
      now = find(0, run);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) load(now, j);
    }
    __syncthreads();  // (the query is in shared memory)
    for (int tile = run, n = 0; tile < tiles; tile += runs, ++n) {
      const bool more = tile + runs < tiles;
      Place then = now;
      if (more) then = find(n + 1, tile + runs);
      // Sixteen terms to an accumulator of their own, these then added in a tree; the magnitudes of the terms, or more, in a chain beside them.
      float sum[NJ][4], mag[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const uint4 neg = sh.q[0][j][lane], pos = sh.q[1][j][lane], any = sh.q[2][j][lane];
        float part[4][4];
        mma_bf16_16816_first(part[0], lo[j % kAhead][0].x, lo[j % kAhead][1].x, lo[j % kAhead][0].y, lo[j % kAhead][1].y, neg.x, neg.y);
        mma_bf16_16816_first(part[1], lo[j % kAhead][0].z, lo[j % kAhead][1].z, lo[j % kAhead][0].w, lo[j % kAhead][1].w, neg.z, neg.w);
        mma_bf16_16816_first(part[2], hi[j % kAhead][0].x, hi[j % kAhead][1].x, hi[j % kAhead][0].y, hi[j % kAhead][1].y, pos.x, pos.y);
        mma_bf16_16816_first(part[3], hi[j % kAhead][0].z, hi[j % kAhead][1].z, hi[j % kAhead][0].w, hi[j % kAhead][1].w, pos.z, pos.w);
        mma_bf16_16816(mag, larger(lo[j % kAhead][0].x, hi[j % kAhead][0].x), larger(lo[j % kAhead][1].x, hi[j % kAhead][1].x), larger(lo[j % kAhead][0].y, hi[j % kAhead][0].y), larger(lo[j % kAhead][1].y, hi[j % kAhead][1].y),
                       any.x, any.y);
        mma_bf16_16816(mag, larger(lo[j % kAhead][0].z, hi[j % kAhead][0].z), larger(lo[j % kAhead][1].z, hi[j % kAhead][1].z), larger(lo[j % kAhead][0].w, hi[j % kAhead][0].w), larger(lo[j % kAhead][1].w, hi[j % kAhead][1].w),
                       any.z, any.w);
        if (j + kAhead < NJ) load(now, j + kAhead);
        else if (more) load(then, j + kAhead - NJ);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[j][e] = (part[0][e] + part[1][e]) + (part[2][e] + part[3][e]);
      }
#pragma unroll
      for (int step = 1; step < NJ; step *= 2)
#pragma unroll
        for (int j = 0; j + step < NJ; j += 2 * step)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[j][e] += sum[j + step][e];
      now = then;
      // elements 0, 1: page r, heads 2c and 2c + 1; 2, 3: page r + 8
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        float best = fmaxf(2 * c < G ? sum[0][2 * s] : -INFINITY, 2 * c + 1 < G ? sum[0][2 * s + 1] : -INFINITY);
        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 1));
        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 2));
        const int i = 16 * tile + 8 * s + r;
        if (i < m) {
          const uint32_t key = key_of(best);
          least = min(least, key);
          most = max(most, key);
          if (c == s) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(keys_at + i * key_step), "r"(key) : "memory");
        }
        reach = max(reach, max(__float_as_uint(mag[2 * s]) & 0x7fffffffu, __float_as_uint(mag[2 * s + 1]) & 0x7fffffffu));  // (not a number: above all)
      }
    }
    reach = __reduce_max_sync(0xffffffffu, reach);
    least = __reduce_min_sync(0xffffffffu, least);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) {
      const uint32_t lo0 = ptx::smem_u32(&sh.run_lo[run]), hi0 = ptx::smem_u32(&sh.run_hi[run]), reach0 = ptx::smem_u32(&sh.run_reach[run]);
      const uint32_t shift = keys_at - keys_here;  // to the first CTA
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(lo0 + shift), "r"(least) : "memory");
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(hi0 + shift), "r"(most) : "memory");
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(reach0 + shift), "r"(reach) : "memory");
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
  if (rank != 0 || !fits) return;
  if (all) {
    for (int i = tid; i < a.n_select; i += kThreads) list[i] = i < nb ? i : -1;
    if (tid == 0) a.counts[row] = nb;
    return;
  }
  for (int i = tid; i < a.n_first; i += kThreads) list[i] = i;
  for (int i = tid; i < a.n_last; i += kThreads) list[a.n_select - a.n_last + i] = nb - a.n_last + i;
  if (tid == 0) a.counts[row] = a.n_select;
  if (!scored) return;

  // ---- the choice, by the first CTA
  // marks: of each 32 keys, those surely chosen and those that are equal to the last one chosen
  const int groups = (m + 31) / 32;
  uint2* marks = reinterpret_cast<uint2*>(keys + a.bound_pages);
  auto approximate = [&](int i) { return few ? few_keys[i] : key_at<uint32_t>(keys, i); };
  Choice ch{0, 0};
  uint32_t kept, left;  // the smallest key chosen, the largest one left
  int turn = 0;
  if (few) {
    // Every key's rank: how many are larger, or equal and in front of it.  1000 rows of 42 pages 8.5 -> 7.6 us, 800 of 32-44, heads of 128, 9.9 -> 8.3; with
    // 188 pages it is slower than counting by bits.
    for (int g = warp; g < groups; g += kWarps) {
      const int i = 32 * g + lane;
      const uint32_t k = few_keys[i];
      int rank = 0;
      auto count = [&](int from, int to, auto limit) {
#pragma unroll 8
        for (int q = from / 4; q < to / 4; ++q) {
          const uint4 x = reinterpret_cast<const uint4*>(few_keys)[q];
          rank += (x.x > limit(4 * q)) + (x.y > limit(4 * q + 1)) + (x.z > limit(4 * q + 2)) + (x.w > limit(4 * q + 3));
        }
      };
      count(0, 32 * g, [&](int) { return k - 1; });
      count(32 * g, 32 * g + 32, [&](int j) { return j < i ? k - 1 : k; });
      count(32 * g + 32, 32 * groups, [&](int) { return k; });
      const bool in = i < m && rank < need;
      const unsigned ins = __ballot_sync(0xffffffffu, in);
      if (lane == 0) marks[g] = make_uint2(ins, 0);
      if (i < m && rank == need - 1) sh.warp_kept[0] = k;
      if (i < m && rank == need) sh.warp_left[0] = k;
    }
    __syncthreads();
    kept = sh.warp_kept[0];
    left = sh.warp_left[0];
  } else {
    uint32_t least = 0xffffffffu, most = 0;
    for (int i = lane; i < runs; i += 32) {
      least = min(least, sh.run_lo[i]);
      most = max(most, sh.run_hi[i]);
    }
    least = __reduce_min_sync(0xffffffffu, least);
    most = __reduce_max_sync(0xffffffffu, most);
    ch = choose<uint32_t>(sh, keys, m, need, least, most, turn);
    kept = 0xffffffffu;
    left = 0;
    for (int g = warp; g < groups; g += kWarps) {
      const int i = 32 * g + lane;
      const uint32_t k = i < m ? key_at<uint32_t>(keys, i) : 0;
      const bool in = i < m && surely(ch, k), eq = i < m && equals(ch, k);
      const unsigned ins = __ballot_sync(0xffffffffu, in), eqs = __ballot_sync(0xffffffffu, eq);
      if (in || eq) kept = min(kept, k);
      if (i < m && !in) left = max(left, k);  // (of equals, some are chosen and some are left)
      if (lane == 0) marks[g] = make_uint2(ins, eqs);
    }
    kept = __reduce_min_sync(0xffffffffu, kept);
    left = __reduce_max_sync(0xffffffffu, left);
    if (lane == 0) {
      sh.warp_kept[warp] = kept;
      sh.warp_left[warp] = left;
    }
    __syncthreads();
    kept = __reduce_min_sync(0xffffffffu, lane < kWarps ? sh.warp_kept[lane] : 0xffffffffu);
    left = __reduce_max_sync(0xffffffffu, lane < kWarps ? sh.warp_left[lane] : 0);
  }
  uint32_t reach = 0;
  for (int i = lane; i < runs; i += 32) reach = max(reach, sh.run_reach[i]);
  reach = __reduce_max_sync(0xffffffffu, reach);
  // Of what the terms' magnitudes add up to, an accumulator loses 2^-23 with each of its sixteen terms at most, the tree 2^-24 with each of its four
  // steps: below 2^-18.8 in all; their sum as computed, by an accumulator of 128 terms, is short by 2^-16 of itself at most.  Elements of the bounds below
  // the normal numbers may count as 0 (2^-126 |q_d| each), as may sums.
  float qsum = 0.f;  // at least the sum of |q_d| of any head
#pragma unroll
  for (int j = 0; j < NJ; ++j) qsum += sh.qsum[j];
  const float err = __uint_as_float(reach) * 0x1p-18f + qsum * 0x1p-125f + 0x1p-120f;
  const float low = value_of(kept), next = value_of(left);
  if (!(low - next > 2.f * err)) {
    // Those above the band around the border are chosen, those in it scored again: a few, to each warp its share, of which every lane then sees whether
    // its own is among the best; or, where there are more, all of them where they are.
    int above = 0, rest = need;
    for (int g = warp; g < groups; g += kWarps) {
      const int i = 32 * g + lane;
      const float v = i < m ? value_of(approximate(i)) : 0.f;
      const bool over = i < m && v > low + 2.f * err, near = i < m && !over && !(v < low - 2.f * err);
      const unsigned overs = __ballot_sync(0xffffffffu, over);
      above += __popc(overs);
      if (lane == 0) marks[g] = make_uint2(overs, 0);
      if (near) {
        const int at = atomicAdd(&sh.near_count, 1);
        if (at < kNear) sh.near_page[at] = i;
      }
    }
    if (lane == 0) sh.warp_above[warp] = above;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) rest -= sh.warp_above[w];
    auto exact = [&](int i) {
      int pg = ptx::ld_plain(table + i);
      if ((unsigned)pg >= (unsigned)a.pool.num_pages) pg = 0;  // (reported above)
      return exact_key<D>(q, base + pg * page_stride, G);
    };
    const int near_count = sh.near_count;
    if (near_count <= kNear) {
      for (int e = warp; e < near_count; e += kWarps) {
        const u64 k = exact(sh.near_page[e]);
        if (lane == 0) sh.near_key[e] = k;
      }
      __syncthreads();
      if (warp == 0 && lane < near_count) {
        const int i = sh.near_page[lane];
        const u64 k = sh.near_key[lane];
        int better = 0;
        for (int e = 0; e < near_count; ++e) better += sh.near_key[e] > k || (sh.near_key[e] == k && sh.near_page[e] < i);
        if (better < rest) atomicOr(&marks[i / 32].x, 1u << (i % 32));
      }
      ch.eq = 0;
    } else {
      u64 lo = kAbove, hi = kBelow;
      for (int g = warp; g < groups; g += kWarps) {
        const int i = 32 * g + lane;
        const float v = i < m ? value_of(approximate(i)) : 0.f;
        const bool over = i < m && v > low + 2.f * err, near = i < m && !over && !(v < low - 2.f * err);
        u64 mine = over ? kAbove : kBelow;
        for (unsigned open = __ballot_sync(0xffffffffu, near); open != 0; open &= open - 1) {
          const int at = __ffs(open) - 1;
          const u64 k = exact(32 * g + at);
          if (lane == at) mine = k;
          lo = min(lo, k);
          hi = max(hi, k);
        }
        if (i < m) keys[i] = mine;
      }
      if (lane == 0) {
        sh.warp_lo[warp] = lo;
        sh.warp_hi[warp] = hi;
      }
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        lo = min(lo, sh.warp_lo[w]);
        hi = max(hi, sh.warp_hi[w]);
      }
      ch = choose<u64>(sh, keys, m, rest, lo, hi, turn);
      for (int g = warp; g < groups; g += kWarps) {
        const int i = 32 * g + lane;
        const u64 k = i < m ? keys[i] : 0;
        const unsigned ins = __ballot_sync(0xffffffffu, i < m && surely(ch, k)), eqs = __ballot_sync(0xffffffffu, i < m && equals(ch, k));
        if (lane == 0) marks[g] = make_uint2(ins, eqs);
      }
    }
    __syncthreads();
  }

  // The kernel behind this one is let in when the choice is made.  Decode's blocks, let in when the scores were there, took what room these left on the
  // SMs and their clusters found no places beside each other: steps of 9, 30 and 64 sequences (tables, rotary append, bounds, choice, decode; 1000-2000 tokens)
  // 25.5 / 31.4 / 44.9 us, this way 21.3 / 31.2 / 44.5, on two streams 12.9 / 24.2 / 37.8 and 12.8 / 21.8 / 34.7; of one 16.7 and 16.9.
  ptx::launch_dependents();
  // ---- the list, ascending: every warp counts all the marks, 32 groups at a time, and writes the groups that are its own
  int out = a.n_first, eq_before = 0;
  for (int g0 = 0; g0 < groups; g0 += 32) {
    const uint2 mark = g0 + lane < groups ? marks[g0 + lane] : make_uint2(0, 0);
    int n_in = __popc(mark.x), n_eq = __popc(mark.y);
    const int own_in = n_in, own_eq = n_eq;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, n_in, off), y = __shfl_up_sync(0xffffffffu, n_eq, off);
      if (lane >= off) {
        n_in += x;
        n_eq += y;
      }
    }
    const int all_in = __shfl_sync(0xffffffffu, n_in, 31), all_eq = __shfl_sync(0xffffffffu, n_eq, 31);
    const int eqs_at = eq_before + n_eq - own_eq;                                       // equals in front of the group
    const int at = out + n_in - own_in + min(ch.eq, eqs_at) - min(ch.eq, eq_before);    // its first place in the list
    for (int g = (warp - g0 % kWarps + kWarps) % kWarps; g < 32 && g0 + g < groups; g += kWarps) {
      const unsigned ins = __shfl_sync(0xffffffffu, mark.x, g), eqs = __shfl_sync(0xffffffffu, mark.y, g);
      const int first = __shfl_sync(0xffffffffu, at, g), room = ch.eq - __shfl_sync(0xffffffffu, eqs_at, g);
      const unsigned below = (1u << lane) - 1;
      const bool take = (ins >> lane & 1) || ((eqs >> lane & 1) && __popc(eqs & below) < room);
      const unsigned takes = __ballot_sync(0xffffffffu, take);
      if (take) list[first + __popc(takes & below)] = a.n_first + 32 * (g0 + g) + lane;
    }
    out += all_in + min(ch.eq, eq_before + all_eq) - min(ch.eq, eq_before);
    eq_before += all_eq;
  }
}

// Shared memory for the keys of so many pages and for the marks.
static int select_smem(int pages) { return pages * 8 + (pages + 31) / 32 * 8; }

template <int D, int kWarps, int kBlocks>
static kv_status_t launch_select(const kv_pool_t* p, const SelectArgs& a, int rows, cudaStream_t st) {
  static std::atomic<bool> ready[kMaxDevices];
  if (!allow_smem((const void*)select_pages_kernel<D, kWarps, kBlocks>, select_smem(kSelMaxPages), ready, p->device)) return KV_ERR_CUDA;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3((unsigned)(rows * a.splits));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = (size_t)select_smem(a.bound_pages);
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)a.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.splits > 1 ? 2 : 1;
  KV_CUDA_OK(cudaLaunchKernelEx(&cfg, select_pages_kernel<D, kWarps, kBlocks>, a));
  count_launch();
  return KV_OK;
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
  if ((int64_t)p->num_pages * p->n_kv_heads * (p->head_dim / 4) > 0xffffffffLL) return KV_ERR_UNSUPPORTED;  // (64 GB of bounds)
  SelectArgs a{p->view(), (const __nv_bfloat16*)q, (const __nv_bfloat16*)bounds, block_tables, ctx_lens, pages, counts, max_pages, (int)bound,
               group, n_select, n_first, n_last, 1};
  // CTAs of eight warps, two of them to an SM, or of four, four to an SM, and as many to a row as the device holds and find sixteen pages for most of
  // their warps: whatever leaves the SM with most to read the least (an SM reads 64 GB/s at best).  Us with eight warps and 1 / 2 / 4 / 8 CTAs, four warps and
  // 1 / 2 / 4 (heads of 128, 8 to a group): 8 rows of 722 pages 12.0 / 9.1 / 7.9 / 6.7, 16.1 / 11.1 / 8.3; 64 rows of 512-1024 19.8 / 16.8 / 14.6 / 17.8,
  // 27.0 / 19.9 / 16.2; 240 of 63-94 7.7 / 12.6 / - / -, 8.0 / 8.1 / 11.7; 256 of 512-1024 28.4 / 33.1 / - / -, 35.5 / 29.4 / 30.8; 2048 of 64-256 56.0
  // and 41.7 with one.  Few rows that are longer still: sixteen warps, 8 rows of 6250 pages, heads of 64, 15.6 / 13.1 with eight / sixteen.
  // An eighth of the device stays free beside clusters: those that do not find their CTAs' places at once, because of the kernel in front or of how they
  // fall on the SMs, are a second round (96 rows of 188-375 pages 10.9 us with three CTAs each, 9.3 with two; 192 of 63-125 8.8 and 7.3).
  // The rules go by the bound, and a block has shared memory for the keys of as many pages: a bound of 2 or 4 times the longest sequence costs at most 4 %,
  // one of 16 times up to a third, where blocks stop fitting beside each other (32 documents of 8192-16384, 64/8 heads, 26.5 / 27.1 / 27.2 / 33.2 us
  // with 1 / 2 / 4 / 16 times, 256 sequences of 1024-4096 42.2 / 41.9 / 42.4 / 47.4, 1000 rows of 42 pages 8.5 / 8.2 / 8.2 / 11.5).
  const int sms = sm_count_of(p->device);
  const int64_t tiles = (bound + 15) / 16, resident = 16 * (int64_t)sms;  // (warps)
  int warps = 4;
  double least = 1e30;
  for (int w : {8, 4})
    for (int s = 1; s <= kSelMaxSplits && (s == 1 || (8 * rows * s * w <= 7 * resident && 2 * tiles > (int64_t)s * w)); ++s) {
      const double most = (double)((rows * s + sms - 1) / sms) / s;
      if ((w == 8 && rows * w > resident) || most > (w == 8 ? least : 0.9 * least)) continue;
      least = most;
      warps = w;
      a.splits = s;
    }
  if (a.splits == kSelMaxSplits && rows * 16 * a.splits <= resident && tiles > 4 * a.splits * warps) warps = 16;
  // Many rows of few pages take longer to begin and to choose than to read: seven blocks to an SM then, without whole tiles on their way.  Us with four /
  // seven (before the ranks): heads of 128, 800 rows of 32-44 pages 10.2 / 9.9, 2048 of 19-38 19.3 / 15.4; of 64, 1000 of 42 10.8 / 8.5, 1600 of 63-188
  // 21.3 / 19.6; longer rows, 1280 of 125-375, 38.7 / 46.5; fewer rows, heads of 64, 480 of 125-375, 11.7 / 13.5.
  const bool brief = warps == 4 && rows > 4 * sms && tiles <= 12;
  const auto go = [&](auto w, auto b) {
    return p->head_dim == 128 ? launch_select<128, decltype(w)::value, decltype(b)::value>(p, a, (int)rows, (cudaStream_t)stream)
                              : launch_select<64, decltype(w)::value, decltype(b)::value>(p, a, (int)rows, (cudaStream_t)stream);
  };
  using std::integral_constant;
  return warps == 16  ? go(integral_constant<int, 16>(), integral_constant<int, 1>())
         : warps == 8 ? go(integral_constant<int, 8>(), integral_constant<int, 2>())
         : brief      ? go(integral_constant<int, 4>(), integral_constant<int, 7>())
                      : go(integral_constant<int, 4>(), integral_constant<int, 4>());
}
