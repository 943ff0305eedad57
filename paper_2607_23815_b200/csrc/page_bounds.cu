// kv_page_bounds: for every page that rows have been stored in, and every KV head, the smallest and the largest key element of each dim.
//
// bounds[page][head] = (lo[D], hi[D]), lo_d = min over the page's tokens of k_d, hi_d = max.  A row is the last of its page when the next row
// goes to another; its slot then says how many tokens the page holds, and the whole page is read again: nothing is kept from call to call, and
// the result does not depend on how the tokens came.
//
// What bounds it: HBM (16 D bf16 in, 2 D out): 13 documents of 8192-16384 tokens, 8 heads of 128, 58.4 us, 6.2 TB/s; 256 decode rows 2.4 us, a launch and
// two trips to memory.  A warp takes a page's block of one head as it lies, whole lines: a lane's 16-byte chunks are
// those of equal dims (rows r and r + 4 of both groups), so that four lanes at the end, not 16, hold parts of one dim.
#include <cuda_bf16.h>

#include "common.cuh"
#include "page_mma.cuh"
#include "sm100_ptx.cuh"

namespace kvattn {

__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmin2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

constexpr int kBoundsWarps = 8;

// tile: rows a warp looks at (a power of two up to 32), for one head.
template <int D>
__global__ void __launch_bounds__(kBoundsWarps * 32) page_bounds_kernel(PoolView pool, const int* slots, int total, int tile, uint4* bounds) {
  constexpr int kHalves = D / 64;
  const int lane = threadIdx.x & 31, c = lane & 7, r0 = lane >> 3;
  const bool upper = lane & 16, odd = lane & 8;
  const int tiles = (total + tile - 1) / tile;
  const int64_t units = (int64_t)tiles * pool.n_kv_heads;
  const size_t blk = block_bytes(D);
  ptx::dependency_wait();
  for (int64_t u = (int64_t)blockIdx.x * kBoundsWarps + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * kBoundsWarps) {
    const int first = (int)(u / pool.n_kv_heads) * tile, head = (int)(u % pool.n_kv_heads), t = first + lane;
    const int slot = lane < tile && t < total ? ptx::ld_plain(slots + t) : -1;
    const int follow = lane < tile && t + 1 < total ? ptx::ld_plain(slots + t + 1) : -1;
    bool closes = slot >= 0 && (unsigned)follow / kPageSize != (unsigned)slot / kPageSize;
    if (closes && slot / kPageSize >= pool.num_pages) {
      report(pool.status, KV_ERR_BOUNDS);
      closes = false;
    }
    for (unsigned left = __ballot_sync(0xffffffffu, closes); left != 0; left &= left - 1) {
      const int s = __shfl_sync(0xffffffffu, slot, __ffs(left) - 1), page = s / kPageSize, n = s % kPageSize + 1;
      const char* k = reinterpret_cast<const char*>(pool.k) + ((size_t)page * pool.n_kv_heads + head) * blk;
      uint4 x[2][2][kHalves];
#pragma unroll
      for (int grp = 0; grp < 2; ++grp)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            if (8 * grp + r0 + 4 * i < n) x[grp][i][h] = ldg_stream(k + chunk_offset_bytes(8 * grp + r0 + 4 * i, 8 * h + c, D));
      uint32_t lo[kHalves][4], hi[kHalves][4];
#pragma unroll
      for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          lo[h][w] = 0x7f807f80u;  // slots behind the last token hold arbitrary bits: they are left out, not multiplied away
          hi[h][w] = 0xff80ff80u;
        }
#pragma unroll
      for (int grp = 0; grp < 2; ++grp)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (8 * grp + r0 + 4 * i < n) {
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
              const uint32_t v[4] = {x[grp][i][h].x, x[grp][i][h].y, x[grp][i][h].z, x[grp][i][h].w};
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                lo[h][w] = min2(lo[h][w], v[w]);
                hi[h][w] = max2(hi[h][w], v[w]);
              }
            }
          }
      // the lanes of four rows: the lower sixteen go on with lo, the upper with hi, then each eight with one half of the dims
      uint32_t b[kHalves][4], mine[4];
#pragma unroll
      for (int h = 0; h < kHalves; ++h)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t other = __shfl_xor_sync(0xffffffffu, upper ? lo[h][w] : hi[h][w], 16);
          b[h][w] = upper ? max2(hi[h][w], other) : min2(lo[h][w], other);
        }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, odd ? b[0][w] : b[kHalves - 1][w], 8), keep = odd ? b[kHalves - 1][w] : b[0][w];
        mine[w] = upper ? max2(keep, other) : min2(keep, other);
      }
      if (kHalves == 2 || !odd)
        bounds[(((size_t)page * pool.n_kv_heads + head) * 2 + (upper ? 1 : 0)) * (D / 8) + (odd ? 8 : 0) + c] = make_uint4(mine[0], mine[1], mine[2], mine[3]);
    }
  }
}

template <int D>
static cudaError_t launch_bounds(const kv_pool_t* p, const int* slots, int total, void* bounds, cudaStream_t st) {
  // As many rows to a warp as leave every SM 32 warps: a page closes at one row in sixteen of a prefill and at every row of a decode step.
  const int sms = sm_count_of(p->device);
  int tile = 1;
  while (tile < 32 && (int64_t)total * p->n_kv_heads >= (int64_t)2 * tile * sms * 32) tile *= 2;
  const int64_t units = (int64_t)((total + tile - 1) / tile) * p->n_kv_heads, want = (units + kBoundsWarps - 1) / kBoundsWarps, most = (int64_t)sms * 16;
  static std::atomic<bool> allowed[kMaxDevices];
  const int smem = few_blocks_smem(want, sms);
  return launch_early(page_bounds_kernel<D>, (unsigned)(want < most ? want : most), kBoundsWarps * 32,
                      smem > 0 && allow_smem((const void*)page_bounds_kernel<D>, spread_smem(1), allowed, p->device) ? smem : 0, st, p->view(), slots, total,
                      tile, (uint4*)bounds);
}

}  // namespace kvattn

using namespace kvattn;

extern "C" {

size_t kv_page_bounds_bytes(const kv_pool_t* p) {
  return p == nullptr ? 0 : (size_t)p->num_pages * p->n_kv_heads * 2 * p->head_dim * sizeof(__nv_bfloat16);
}

kv_status_t kv_page_bounds(kv_pool_t* p, const int* slots, int total_new, void* bounds, void* stream) {
  if (p == nullptr || total_new < 0) return KV_ERR_INVALID;
  if (p->num_pages > (1 << 27) || total_new > (1 << 30)) return KV_ERR_UNSUPPORTED;
  if (total_new == 0) return KV_OK;
  if (slots == nullptr || bounds == nullptr || (((uintptr_t)bounds) & 15) != 0) return KV_ERR_INVALID;
  if (!on_pool_device(p)) return KV_ERR_INVALID;
  KV_CUDA_OK(p->head_dim == 128 ? launch_bounds<128>(p, slots, total_new, bounds, (cudaStream_t)stream)
                                : launch_bounds<64>(p, slots, total_new, bounds, (cudaStream_t)stream));
  count_launch();
  return KV_OK;
}

}  // extern "C"
