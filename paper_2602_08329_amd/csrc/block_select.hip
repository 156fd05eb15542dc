// Selection of whole blocks by their key bounds.  With q+ = max(q, 0) and
// q- = min(q, 0),
//   sum_d max(q kmin, q kmax) = q+ . kmax + q- . kmin,
// an upper bound of q . k over the block's keys.
//
// block_score: a wave per block, its lanes over the dimensions: the largest
//   bound over the group's heads as an order-preserving key; 0, below every
//   number's key, for NaN and for blocks whose page lies outside the pool.
// block_pick: one workgroup per (batch, kv head): the key of the last chosen
//   block by a radix search over the keys, then the chosen blocks and the set
//   in ascending order (which settles ties).
#include "prhs_internal.h"

namespace prhs {
namespace {

constexpr int kScoreThreads = 256;
constexpr int kScoreBlocks = 64;    // blocks of a score workgroup
constexpr int kPickThreads = 1024;

struct BlockArgs : BlockSelectLaunch {
  uint32_t* keys;   // [units][nbmax], candidate i of a unit at [i]
  int nbmax;
};

struct MiddleBlocks {
  int n0, sink_end, win_start;
  int first, count;   // candidates: blocks [first, first + count)
};

__device__ __forceinline__ MiddleBlocks middle_blocks(const BlockArgs& a, int b) {
  MiddleBlocks m;
  m.n0 = kv_seq_len(a.kv, b);
  m.sink_end = min(a.sink, m.n0);
  m.win_start = max(m.sink_end, m.n0 - a.window);
  m.first = m.sink_end >> a.block_shift;
  m.count = m.win_start > m.sink_end ? ((m.win_start - 1) >> a.block_shift) + 1 - m.first : 0;
  return m;
}

// Chosen blocks of a row with `cand` candidates at length n0.
__device__ __forceinline__ int chosen_blocks(const BlockArgs& a, int n0, int cand) {
  const long long k = a.k_den > 0 ? ((long long)a.k_num * n0) / a.k_den : (long long)a.k;
  const long long kb = (k + (1 << a.block_shift) - 1) >> a.block_shift;
  return (int)min(kb, (long long)cand);
}

// Index of block j of (b, g) among all blocks, or -1.
__device__ __forceinline__ int block_id(const BlockArgs& a, int b, int g, int j) {
  if (!a.kv.paged) return (b * a.kv.hkv + g) * (a.kv.capacity >> a.block_shift) + j;
  const int phys = a.kv.table[(int64_t)b * a.kv.max_pages + j];
  return phys < 0 || phys >= a.kv.num_pages ? -1 : phys * a.kv.hkv + g;
}

template <typename T, int D>
__global__ __launch_bounds__(kScoreThreads) void block_score(BlockArgs a, int chunks) {
  __shared__ float s_q[16 * D];
  const int u = blockIdx.x / chunks, b = u / a.kv.hkv, g = u - b * a.kv.hkv;
  const int G = a.kv.hq / a.kv.hkv;
  const MiddleBlocks m = middle_blocks(a, b);
  const int i0 = (blockIdx.x - u * chunks) * kScoreBlocks, i1 = min(m.count, i0 + kScoreBlocks);
  if (i0 >= m.count) return;
  const T* q = (const T*)a.q + ((size_t)b * a.kv.hq + (size_t)g * G) * D;
  for (int e = threadIdx.x; e < G * D; e += kScoreThreads) s_q[e] = (float)q[e];
  __syncthreads();
  const int lane = threadIdx.x & 63;
  for (int i = i0 + (threadIdx.x >> 6); i < i1; i += kScoreThreads / 64) {
    const int id = block_id(a, b, g, m.first + i);
    uint32_t key = 0u;
    if (id >= 0) {
      const T* lo = (const T*)a.k_min + (int64_t)id * D;
      const T* hi = (const T*)a.k_max + (int64_t)id * D;
      float best = -INFINITY;
      bool nan = false;
      for (int h = 0; h < G; ++h) {
        float s = 0.f;
        for (int d = lane; d < D; d += 64) {
          const float x = s_q[h * D + d];
          s += fmaxf(x, 0.f) * (float)hi[d] + fminf(x, 0.f) * (float)lo[d];
        }
        for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
        nan = nan || !(s == s);
        best = fmaxf(best, s);
      }
      if (!nan) key = score_key(best);
    }
    if (lane == 0) a.keys[(size_t)u * a.nbmax + i] = key;
  }
}

__global__ __launch_bounds__(kPickThreads) void block_pick(BlockArgs a) {
  __shared__ uint32_t s_hist[256];
  __shared__ uint64_t s_scan[kPickThreads / 64 + 1];
  __shared__ uint32_t s_digit, s_left;
  const int u = blockIdx.x, b = u / a.kv.hkv;
  const MiddleBlocks m = middle_blocks(a, b);
  const int kb = chosen_blocks(a, m.n0, m.count);
  const uint32_t* keys = a.keys + (size_t)u * a.nbmax;
  const int tid = threadIdx.x, bs = 1 << a.block_shift;
  // threshold key T: `left` blocks of key T are chosen, and every one above it
  uint32_t T = 0u, left = (uint32_t)kb;
  if (kb > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) s_hist[tid] = 0u;
      __syncthreads();
      const uint32_t mask = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
      for (int i = tid; i < m.count; i += kPickThreads)
        if ((keys[i] & mask) == T) atomicAdd(&s_hist[(keys[i] >> shift) & 255u], 1u);
      __syncthreads();
      if (tid == 0) {
        uint32_t above = 0u;
        int d = 255;
        for (; d > 0 && above + s_hist[d] < left; --d) above += s_hist[d];
        s_digit = (uint32_t)d;
        s_left = left - above;
      }
      __syncthreads();
      T |= s_digit << shift;
      left = s_left;
    }
  }
  int32_t* blk = a.blk_idx + (size_t)u * a.blk_cap;
  int32_t* set = a.set_idx + (size_t)u * a.set_cap;
  uint32_t above = 0u, ties = 0u;   // of the blocks before this chunk
  int first = -1, last = -1;        // first and last chosen block
  for (int base = 0; kb > 0 && base < m.count; base += kPickThreads) {
    const int i = base + tid;
    const uint32_t key = i < m.count ? keys[i] : 0u;
    const bool gt = i < m.count && key > T, eq = i < m.count && key == T;
    uint64_t total;
    const uint64_t before = block_exclusive_scan<kPickThreads, uint64_t>(
        (uint64_t)gt << 32 | (uint64_t)eq, s_scan, &total);
    const uint32_t e = ties + (uint32_t)before;
    if (gt || (eq && e < left)) {
      const uint32_t at = above + (uint32_t)(before >> 32) + min(e, left);
      blk[at] = m.first + i;
    }
    above += (uint32_t)(total >> 32);
    ties += (uint32_t)total;
  }
  __syncthreads();   // the list is read back below
  if (kb > 0) {
    first = blk[0];
    last = blk[kb - 1];
  }
  // the chosen blocks' positions within the middle range [sink_end, win_start)
  const int lo_cut = kb > 0 ? max(0, m.sink_end - first * bs) : 0;
  const int hi_cut = kb > 0 ? max(0, (last + 1) * bs - m.win_start) : 0;
  const int mid = kb * bs - lo_cut - hi_cut;
  for (int i = tid; i < m.sink_end; i += kPickThreads) set[i] = i;
  for (int i = tid; i < mid; i += kPickThreads) {
    const int x = i + lo_cut;
    set[m.sink_end + i] = (blk[x >> a.block_shift] << a.block_shift) + (x & (bs - 1));
  }
  const int nw = m.n0 - m.win_start;
  for (int i = tid; i < nw; i += kPickThreads) set[m.sink_end + mid + i] = m.win_start + i;
  if (tid == 0) {
    a.blk_len[u] = kb;
    a.set_len[u] = m.sink_end + mid + nw;
  }
}

}  // namespace

size_t block_select_workspace_bytes(int units, int max_seq_len, int block_shift) {
  return (size_t)units * ((max_seq_len + (1 << block_shift) - 1) >> block_shift) * sizeof(uint32_t);
}

hipError_t launch_block_select(const BlockSelectLaunch& s, hipStream_t stream) {
  BlockArgs a;
  (BlockSelectLaunch&)a = s;
  a.keys = (uint32_t*)s.ws;
  a.nbmax = (s.kv.max_seq_len + (1 << s.block_shift) - 1) >> s.block_shift;
  const int units = s.kv.batch * s.kv.hkv;
  const int chunks = (a.nbmax + kScoreBlocks - 1) / kScoreBlocks;
  if (chunks > 0) {
    const dim3 grid((unsigned)units * chunks), block(kScoreThreads);
    if (s.dtype == 1) {
      if (s.kv.d == 128) hipLaunchKernelGGL((block_score<__bf16, 128>), grid, block, 0, stream, a, chunks);
      else hipLaunchKernelGGL((block_score<__bf16, 64>), grid, block, 0, stream, a, chunks);
    } else {
      if (s.kv.d == 128) hipLaunchKernelGGL((block_score<float, 128>), grid, block, 0, stream, a, chunks);
      else hipLaunchKernelGGL((block_score<float, 64>), grid, block, 0, stream, a, chunks);
    }
  }
  hipLaunchKernelGGL(block_pick, dim3(units), dim3(kPickThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace prhs
