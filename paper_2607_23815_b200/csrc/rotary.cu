// kv_append_rotary: projected rows are rotated by their positions and stored, queries in a tensor, keys and values in their pages.
//
// Pair j of a head's first rot_dim dims turns by theta_j = position[axis_j] * inv_freq_j: (x1, x2) -> (x1 cos - x2 sin, x2 cos + x1 sin).
// theta is a product in 64 bits, brought to a fraction of a turn before it goes to 32: at position 10^6 a 32-bit angle is off by 0.03.
// Rows are widened to 32 bits, rotated and rounded once.  Values are copied.
//
// What bounds it: HBM on steps of many tokens (every row is read once and written once), latency on small ones.  A warp takes eight (D = 64:
// sixteen) rows of a token, whatever mixture of queries, keys and values they are, and each lane the two 16-byte chunks whose dims pair
// up, so that a pair never leaves its lane; the lanes that hold the same dims of different rows share out the sines and cosines.
// 10123 tokens, 32/8 heads of 128, parts of one projection: 40.5 us, 6.1 TB/s of the 248 MB (copy rate 6.55); 9 x 300-2000, heads of 64, three axes:
// 25.7 us, 5.6 TB/s; one token 2.5 us.
// Four blocks of eight warps to an SM (64 registers), which walk the units in one grid's strides: three blocks 41.4 us, more blocks than are resident
// 42.9, all rows of a token to a warp (one set of sines for six units) 44.8, runs of neighbouring units to a warp 49.8, twice the rows in flight per
// warp with three blocks 42.1.
#include "common.cuh"
#include "page_mma.cuh"
#include "sm100_ptx.cuh"

namespace kvattn {

struct RotaryArgs {
  PoolView pool;
  const __nv_bfloat16 *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, out_stride;  // elements from token to token
  __nv_bfloat16* q_out;
  const int* slots;       // or nullptr: every row is one to rotate (no keys and values then)
  const int* positions;   // [n_axes][total]
  const float* inv_freq;  // [rot_dim / 2]
  const int* freq_axis;   // or nullptr: axis 0
  int n_q, n_kv;          // heads of q, of k and of v (0: there are none)
  int n_axes, rot_dim, neighbours, total, slices;
};

constexpr int kRotaryWarps = 8;
constexpr int kRotaryPasses = 2;
constexpr int kRotaryBlocks = 4;  // on an SM

template <int D>
__global__ void __launch_bounds__(kRotaryWarps * 32, kRotaryBlocks) append_rotary_kernel(const RotaryArgs a) {
  constexpr int kLanes = D / 16;          // of a row: a pair of chunks each
  constexpr int kRows = 32 / kLanes;      // of a pass
  constexpr int kShare = 8 / kRows;       // frequencies of which a lane takes the sine and cosine
  const int lane = threadIdx.x & 31, p = lane % kLanes, g = lane / kLanes;
  const bool turns = p < a.rot_dim / 16;
  // the lane's chunks, and the frequency of its first pair
  const int c0 = !turns || a.neighbours ? 2 * p : p, c1 = !turns || a.neighbours ? 2 * p + 1 : p + a.rot_dim / 16;
  const int rows = a.n_q + 2 * a.n_kv;
  const size_t blk = block_bytes(D);
  ptx::dependency_wait();

  double freq[kShare];
  int axis[kShare];
#pragma unroll
  for (int i = 0; i < kShare; ++i) {
    const int f = 8 * p + g * kShare + i;
    freq[i] = 0.0;
    axis[i] = 0;
    if (turns) {
      freq[i] = (double)__int_as_float(ptx::ld_plain(reinterpret_cast<const int*>(a.inv_freq) + f)) * 0.15915494309189535;  // turns per position
      if (a.freq_axis != nullptr) axis[i] = ptx::ld_plain(a.freq_axis + f);
      if ((unsigned)axis[i] >= (unsigned)a.n_axes) {
        report(a.pool.status, KV_ERR_BOUNDS);
        axis[i] = 0;
      }
    }
  }

  const unsigned units = (unsigned)a.total * a.slices;
  bool let_in = false;
  for (unsigned u = blockIdx.x * kRotaryWarps + (threadIdx.x >> 5); u < units; u += gridDim.x * kRotaryWarps) {
    const int t = (int)(u / (unsigned)a.slices), slice = (int)(u - (unsigned)t * a.slices), row0 = slice * (kRows * kRotaryPasses) + g;
    // the rows first: everything else is found while they are on their way
    uint4 x[kRotaryPasses][2];
#pragma unroll
    for (int i = 0; i < kRotaryPasses; ++i) {
      const int r = row0 + i * kRows;
      if (r < rows) {
        const __nv_bfloat16* src = r < a.n_q            ? a.q + t * a.q_stride + r * D
                                   : r < a.n_q + a.n_kv ? a.k + t * a.k_stride + (r - a.n_q) * D
                                                        : a.v + t * a.v_stride + (r - a.n_q - a.n_kv) * D;
        x[i][0] = ptx::ld_plain(reinterpret_cast<const uint4*>(src) + c0);
        x[i][1] = ptx::ld_plain(reinterpret_cast<const uint4*>(src) + c1);
      }
    }
    int slot = 0, follow = -1;
    if (a.slots != nullptr) {
      slot = ptx::ld_plain(a.slots + t);
      if (t + 1 < a.total) follow = ptx::ld_plain(a.slots + t + 1);
    }
    float cs[kShare], sn[kShare];
#pragma unroll
    for (int i = 0; i < kShare; ++i) {
      double turn = (double)ptx::ld_plain(a.positions + (int64_t)axis[i] * a.total + t) * freq[i];
      turn -= rint(turn);
      sincospif((float)(2.0 * turn), &sn[i], &cs[i]);
    }
    float cosv[8], sinv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int from = (i / kShare) * kLanes + p;
      cosv[i] = __shfl_sync(0xffffffffu, cs[i % kShare], from);
      sinv[i] = __shfl_sync(0xffffffffu, sn[i % kShare], from);
    }
    if (!let_in) {
      ptx::launch_dependents();
      let_in = true;
    }
    // The last row of its page clears the slots behind it, as kv_append's does.  One that another row of the page follows does not, even if slots are
    // left out between them: another warp may be storing that row.
    const bool clears = (unsigned)follow / kPageSize != (unsigned)slot / kPageSize;
    if (slot < 0) continue;  // a padding row: nothing of it is written
    const int page = slot / kPageSize, at = slot % kPageSize;
    if (page >= a.pool.num_pages) {
      report(a.pool.status, KV_ERR_BOUNDS);
      continue;
    }
#pragma unroll
    for (int i = 0; i < kRotaryPasses; ++i) {
      const int r = row0 + i * kRows;
      if (r >= rows) continue;
      if (turns && r < a.n_q + a.n_kv) {
        uint32_t* w0 = reinterpret_cast<uint32_t*>(&x[i][0]);
        uint32_t* w1 = reinterpret_cast<uint32_t*>(&x[i][1]);
        auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
        auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
        if (a.neighbours) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float a0 = lo(w0[j]), b0 = hi(w0[j]), a1 = lo(w1[j]), b1 = hi(w1[j]);
            w0[j] = pack_bf16x2(a0 * cosv[j] - b0 * sinv[j], b0 * cosv[j] + a0 * sinv[j]);
            w1[j] = pack_bf16x2(a1 * cosv[4 + j] - b1 * sinv[4 + j], b1 * cosv[4 + j] + a1 * sinv[4 + j]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float a0 = lo(w0[j]), a1 = hi(w0[j]), b0 = lo(w1[j]), b1 = hi(w1[j]);
            const float ca = cosv[2 * j], cb = cosv[2 * j + 1], sa = sinv[2 * j], sb = sinv[2 * j + 1];
            w0[j] = pack_bf16x2(a0 * ca - b0 * sa, a1 * cb - b1 * sb);
            w1[j] = pack_bf16x2(b0 * ca + a0 * sa, b1 * cb + a1 * sb);
          }
        }
      }
      if (r < a.n_q) {
        uint4* dst = reinterpret_cast<uint4*>(a.q_out + t * a.out_stride + r * D);
        dst[c0] = x[i][0];
        dst[c1] = x[i][1];
      } else {
        const bool is_v = r >= a.n_q + a.n_kv;
        const int head = r - a.n_q - (is_v ? a.n_kv : 0);
        char* base = reinterpret_cast<char*>(is_v ? a.pool.v : a.pool.k) + ((size_t)page * a.n_kv + head) * blk;
        *reinterpret_cast<uint4*>(base + chunk_offset_bytes(at, c0, D)) = x[i][0];
        *reinterpret_cast<uint4*>(base + chunk_offset_bytes(at, c1, D)) = x[i][1];
      }
    }
    // The slots behind are shared out over the token's units: they can be fifteen times what the token itself takes, and in the units that hold its
    // keys and values alone they were the longest part of a decode step (40 tokens 4.2 us, this way 3.5; 256 5.8 and 5.2).
    if (clears) {
      constexpr int kChunks = D / 8;  // of a row
      for (int s = at + 1 + slice; s < kPageSize; s += a.slices) {
        const size_t off = ((size_t)page * a.n_kv + lane / kChunks) * blk + chunk_offset_bytes(s, lane % kChunks, D);
        char *kp = reinterpret_cast<char*>(a.pool.k) + off, *vp = reinterpret_cast<char*>(a.pool.v) + off;
#pragma unroll 4
        for (int head = lane / kChunks; head < a.n_kv; head += 32 / kChunks, kp += 32 / kChunks * blk, vp += 32 / kChunks * blk) {
          *reinterpret_cast<uint4*>(kp) = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(vp) = make_uint4(0, 0, 0, 0);
        }
      }
    }
  }
}

static int rotary_slices(int head_dim, int rows) {
  const int step = 32 / (head_dim / 16) * kRotaryPasses;
  return (rows + step - 1) / step;
}

template <int D>
static cudaError_t launch_rotary(const kv_pool_t* p, const RotaryArgs& a, cudaStream_t st) {
  static std::atomic<bool> allowed[kMaxDevices];
  const int sms = sm_count_of(p->device);
  const int64_t want = ((int64_t)a.total * a.slices + kRotaryWarps - 1) / kRotaryWarps, most = (int64_t)sms * kRotaryBlocks;
  const int smem = few_blocks_smem(want, sms);
  return launch_early(append_rotary_kernel<D>, (unsigned)(want < most ? want : most), kRotaryWarps * 32,
                      smem > 0 && allow_smem((const void*)append_rotary_kernel<D>, spread_smem(1), allowed, p->device) ? smem : 0, st, a);
}

}  // namespace kvattn

using namespace kvattn;

extern "C" kv_status_t kv_append_rotary(kv_pool_t* p, const void* q, int64_t q_stride, const void* k_new, int64_t k_stride,
                                        const void* v_new, int64_t v_stride, int n_q_heads, const int* slots, const int* positions,
                                        int n_axes, const float* inv_freq, const int* freq_axis, int rot_dim, int neighbours,
                                        int total_new, void* q_out, int64_t q_out_stride, void* stream) {
  if (p == nullptr || total_new < 0 || n_axes < 1 || rot_dim < 0 || (q != nullptr && n_q_heads <= 0)) return KV_ERR_INVALID;
  const int D = p->head_dim;
  if (rot_dim < 16 || rot_dim % 16 != 0 || rot_dim > D || n_q_heads > (1 << 15) || p->num_pages > (1 << 27)) return KV_ERR_UNSUPPORTED;
  if (total_new == 0) return KV_OK;
  const bool kv = k_new != nullptr || v_new != nullptr;
  if (q == nullptr && !kv) return KV_OK;
  if ((q != nullptr && q_out == nullptr) || (kv && (k_new == nullptr || v_new == nullptr || slots == nullptr))) return KV_ERR_INVALID;
  if (positions == nullptr || inv_freq == nullptr || (n_axes > 1 && freq_axis == nullptr)) return KV_ERR_INVALID;
  const int n_q = q != nullptr ? n_q_heads : 0, n_kv = kv ? p->n_kv_heads : 0;
  // rows are read and written in 16-byte pieces and do not reach into the next token's
  const struct { const void* at; int64_t stride; int heads; } rows[] = {{q, q_stride, n_q}, {k_new, k_stride, n_kv}, {v_new, v_stride, n_kv},
                                                                        {q_out, q_out_stride, n_q}};
  for (const auto& r : rows)
    if (r.heads > 0 && ((((uintptr_t)r.at) & 15) != 0 || (total_new > 1 && (r.stride % 8 != 0 || r.stride < (int64_t)r.heads * D))))
      return KV_ERR_INVALID;
  const int slices = rotary_slices(D, n_q + 2 * n_kv);
  if ((int64_t)total_new * slices > 0x7fffffffLL) return KV_ERR_UNSUPPORTED;
  if (!on_pool_device(p)) return KV_ERR_INVALID;
  const RotaryArgs a{p->view(), (const __nv_bfloat16*)q, (const __nv_bfloat16*)k_new, (const __nv_bfloat16*)v_new, q_stride, k_stride, v_stride,
               q_out_stride, (__nv_bfloat16*)q_out, slots, positions, inv_freq, freq_axis, n_q, n_kv, n_axes, rot_dim, neighbours != 0, total_new, slices};
  KV_CUDA_OK(D == 128 ? launch_rotary<128>(p, a, (cudaStream_t)stream) : launch_rotary<64>(p, a, (cudaStream_t)stream));
  count_launch();
  return KV_OK;
}
