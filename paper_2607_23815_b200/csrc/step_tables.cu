// kv_step_tables: block tables, positions and slots of a step's new tokens, from the sequences' lengths.
//
// Sequence i holds c_i tokens and stores n_i more.  It has ceil(c_i / 16) pages, so ceil((c_i + n_i) / 16) - ceil(c_i / 16) are
// taken for it from a list, in the order of the sequences: two exclusive sums over the batch (rows, pages) and a search say
// which sequence a row belongs to, its place p there and the p / 16-th page.  A row with p % 16 == 0 opens a page and writes the
// table's entry for it; no other row does.
//
// What bounds it: latency (lengths, then a page id, then stores: 251 rows are 7 KB).  So one launch: every block sums over the whole batch by itself,
// 256 sequences at a time, and then takes its share of those sequences' rows, so that no block waits for another.
#include "common.cuh"
#include "sm100_ptx.cuh"

namespace kvattn {

struct TablesArgs {
  const int* ctx_lens;
  const int* new_lens;
  const int* new_pages;
  const int* cursor;  // or nullptr: 0
  int* block_tables;
  int* cu_new;
  int* positions;     // or nullptr
  int* slots;
  int* next_lens;     // or nullptr
  int* next_cursor;   // or nullptr
  int* status;
  int batch, n_new_pages, max_pages, total_new, num_pages;
  int fill;           // 1: tables, sums, positions, slots
  int advance;        // 1: next_lens, next_cursor
};

constexpr int kTableThreads = 256;  // (251 decode rows 2.9 us with 512, 2.7 with 256, 4.1 with 128; 100000 rows 3.5, 3.4, 4.0)
constexpr unsigned kSumLimit = (1u << 30) + 1;  // sums stay here once they reach it; rows and pages are fewer

__device__ __forceinline__ unsigned add_limited(unsigned a, unsigned b) { return min(a + b, kSumLimit); }

// Sum of v over the threads in front of this one (limited; the order of the additions does not matter to it), *all: over all of them.
__device__ __forceinline__ unsigned block_sum(unsigned v, unsigned* warp_sums, unsigned* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const unsigned x = __shfl_up_sync(0xffffffffu, v, off);
    if (lane >= off) v = add_limited(v, x);
  }
  __syncthreads();  // (warp_sums may still be read for the sum before)
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  unsigned w = lane < kTableThreads / 32 ? warp_sums[lane] : 0;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const unsigned x = __shfl_up_sync(0xffffffffu, w, off);
    if (lane >= off) w = add_limited(w, x);
  }
  const unsigned warps_before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31), lanes_before = __shfl_up_sync(0xffffffffu, v, 1);
  *all = __shfl_sync(0xffffffffu, w, 31);
  return add_limited(warp == 0 ? 0 : warps_before, lane == 0 ? 0 : lanes_before);
}

__global__ void __launch_bounds__(kTableThreads) step_tables_kernel(const TablesArgs a) {
  __shared__ unsigned first_row[kTableThreads];  // of each sequence of the chunk
  __shared__ int ctx[kTableThreads];             // its tokens so far, -1: it gets nothing
  __shared__ unsigned first_page[kTableThreads]; // its first new page, counted from the cursor
  __shared__ unsigned warp_sums[32];
  __shared__ unsigned taken;
  const int tid = threadIdx.x;
  ptx::dependency_wait();
  const int cursor = a.cursor != nullptr ? ptx::ld_plain(a.cursor) : 0;
  const bool cursor_ok = cursor >= 0 && cursor <= a.n_new_pages;
  const unsigned avail = cursor_ok ? a.n_new_pages - cursor : 0;
  const int64_t room = min((int64_t)a.max_pages * kPageSize, (int64_t)0x7fffffff);  // tokens of a sequence: a row of its table, and a length has 31 bits
  const bool speaks = blockIdx.x == 0;  // one block writes what belongs to the sequences, and reports
  bool bad = !cursor_ok;
  if (tid == 0) taken = 0;

  unsigned rows = 0, pages = 0;  // of the sequences in front of the chunk
  for (int base = 0; base < a.batch; base += kTableThreads) {
    const int seq = base + tid;
    const bool in = seq < a.batch;
    const int c = in ? ptx::ld_plain(a.ctx_lens + seq) : 0, n = in ? ptx::ld_plain(a.new_lens + seq) : 0;
    const unsigned n_rows = n > 0 ? min((unsigned)n, kSumLimit) : 0;
    unsigned all_rows, all_pages;
    const unsigned row = add_limited(rows, block_sum(n_rows, warp_sums, &all_rows)), row_end = add_limited(row, n_rows);
    bool ok = c >= 0 && n >= 0 && (int64_t)c + n <= room && row_end <= (unsigned)a.total_new;
    const unsigned need = ok ? pages_of(c + n) - pages_of(c) : 0;
    const unsigned page = add_limited(pages, block_sum(need, warp_sums, &all_pages)), page_end = add_limited(page, need);
    if (need > 0 && page_end > avail) ok = false;  // the list has run out: this sequence and the later ones that need a page get none
    first_row[tid] = in ? row : kSumLimit;
    ctx[tid] = ok ? c : -1;
    first_page[tid] = page;
    if (in) {
      if (!ok) bad = true;
      if (ok && need > 0) atomicMax(&taken, page_end);
      if (speaks && a.fill) a.cu_new[seq] = (int)min(row, (unsigned)a.total_new);
      if (speaks && a.advance && a.next_lens != nullptr) a.next_lens[seq] = ok ? c + n : c;
    }
    __syncthreads();
    const unsigned rows_before = rows;
    rows = add_limited(rows, all_rows);
    pages = add_limited(pages, all_pages);
    if (a.fill) {
      const unsigned end = min(rows, (unsigned)a.total_new);
      const int members = min(kTableThreads, a.batch - base);
      for (unsigned t = rows_before + blockIdx.x * kTableThreads + tid; t < end; t += gridDim.x * kTableThreads) {
        int lo = 0, span = members;  // the last sequence that starts at or before row t
        while (span > 1) {
          const int half = span >> 1;
          if (first_row[lo + half] <= t) { lo += half; span -= half; } else { span = half; }
        }
        int pos = 0, slot = -1;
        if (ctx[lo] >= 0) {
          pos = ctx[lo] + (int)(t - first_row[lo]);
          const int b = pos / kPageSize, owned = pages_of(ctx[lo]);
          int* entry = a.block_tables + (int64_t)(base + lo) * a.max_pages + b;
          const bool fresh = b >= owned;
          const int page = ptx::ld_plain(fresh ? a.new_pages + cursor + first_page[lo] + (b - owned) : entry);
          if ((unsigned)page >= (unsigned)a.num_pages) {
            report(a.status, KV_ERR_BOUNDS);
          } else {
            if (fresh && pos % kPageSize == 0) *entry = page;
            slot = page * kPageSize + pos % kPageSize;
          }
        }
        if (a.positions != nullptr) a.positions[t] = pos;
        a.slots[t] = slot;
      }
    }
  }
  if (a.fill) {
    if (speaks && tid == 0) a.cu_new[a.batch] = (int)min(rows, (unsigned)a.total_new);
    // rows behind the last sequence
    for (unsigned t = min(rows, (unsigned)a.total_new) + blockIdx.x * kTableThreads + tid; t < (unsigned)a.total_new; t += gridDim.x * kTableThreads) {
      if (a.positions != nullptr) a.positions[t] = 0;
      a.slots[t] = -1;
    }
  }
  if (speaks && bad) report(a.status, KV_ERR_BOUNDS);
  __syncthreads();
  if (speaks && a.advance && tid == 0 && a.next_cursor != nullptr) *a.next_cursor = cursor + (int)taken;
}

}  // namespace kvattn

using namespace kvattn;

// Do [a, a + n) and [b, b + n) overlap without being the same?
static bool overlap(const int* a, const int* b, int n) { return a != nullptr && b != nullptr && a != b && a < b + n && b < a + n; }

extern "C" kv_status_t kv_step_tables(kv_pool_t* p, const int* ctx_lens, const int* new_lens, int batch, const int* new_pages,
                                      int n_new_pages, int* block_tables, int max_pages, int total_new, int* cu_new, int* positions,
                                      int* slots, int* next_lens, const int* cursor, int* next_cursor, void* stream) {
  if (p == nullptr || batch < 0 || n_new_pages < 0 || max_pages < 0 || total_new < 0 || cu_new == nullptr) return KV_ERR_INVALID;
  if (batch > 0 && (ctx_lens == nullptr || new_lens == nullptr || (max_pages > 0 && block_tables == nullptr))) return KV_ERR_INVALID;
  if ((n_new_pages > 0 && new_pages == nullptr) || (total_new > 0 && slots == nullptr)) return KV_ERR_INVALID;
  if (overlap(ctx_lens, next_lens, batch)) return KV_ERR_INVALID;
  if (total_new > (1 << 30) || n_new_pages > (1 << 30) || p->num_pages > (1 << 27)) return KV_ERR_UNSUPPORTED;  // (a slot is 31 bits)
  if (!on_pool_device(p)) return KV_ERR_INVALID;
  TablesArgs a{ctx_lens, new_lens, new_pages, cursor, block_tables, cu_new, positions, slots, next_lens, next_cursor, p->d_status,
               batch, n_new_pages, max_pages, total_new, p->num_pages, 1, 1};
  const int64_t want = ((int64_t)total_new + kTableThreads - 1) / kTableThreads, most = 2 * (int64_t)sm_count_of(p->device);
  const unsigned blocks = (unsigned)(want < 1 ? 1 : want < most ? want : most);
  // Lengths or a cursor that are advanced in place may only be written when no block will read them any more: by a launch of one
  // block behind the others, or by the one block there is, whose threads have read what they write.
  const bool in_place = (next_lens != nullptr && next_lens == ctx_lens) || (next_cursor != nullptr && next_cursor == cursor);
  const bool apart = in_place && blocks > 1;
  if (apart) a.advance = 0;
  KV_CUDA_OK(launch_early(step_tables_kernel, blocks, kTableThreads, 0, (cudaStream_t)stream, a));
  count_launch();
  if (apart) {
    a.fill = 0;
    a.advance = 1;
    KV_CUDA_OK(launch_early(step_tables_kernel, 1, kTableThreads, 0, (cudaStream_t)stream, a));
    count_launch();
  }
  return KV_OK;
}
