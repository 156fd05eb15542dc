// What the decode attention kernels share: the launch arguments, the rows a
// unit attends and their row ids, lane-group reductions of a wave, and the
// merge of split partials.
#pragma once

#include "prhs_internal.h"

namespace prhs {
namespace {

constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kRowsPerThread = 8;   // staged list entries per thread
constexpr int kMaxSplits = 4096;
constexpr int kMaxWaves = 8;        // waves of an attention workgroup

struct AttnArgs {
  KvView kv;
  const void* q;
  const int32_t* set_idx;
  const int32_t* set_len;
  const int32_t* tail_start;  // [B] or null: rows also cover [tail_start[b], n_b)
  const int32_t* unit_row;    // [units] or null: pool row of set_idx each unit attends
  const int32_t* unit_tail;   // [units] with unit_row: first position of the unit's tail
  int pool_rows;
  const int32_t* unit_gate;   // [units] or null: the gate's choice per unit
  int units_side;             // 1: only units with unit_gate < 0; 2: only >= 0; else all
  int psaw;                   // nonzero: positions in [psaw_sink, first visible) are skipped
  double psaw_f;              // Eq. psaw factor of the layer (first visible at length n:
  int psaw_sink;              // psaw_first_visible(psaw_f, psaw_sink, n))
  int set_cap;
  float scale_log2;
  int chunk, nsplit;
  float* part_o;    // [B*Hq][nsplit][D]
  float* part_ml;   // [B*Hq][nsplit][2]
  float* out;
  float* lse;
};

// The rows a unit attends, in order: the first `base` come from its index
// set (entries at or beyond t0 are skipped), then the tail positions
// [t0, t0 + L - base).  Dense: rows are the positions [0, n_b).  Without a
// tail t0 = n_b.  L never exceeds set_cap, the bound the split geometry uses.
// The set is row u of set_idx, or with a pool the row unit_row[u] (a row
// outside the pool gives an empty set) and the tail from unit_tail[u].
struct UnitSpan {
  int L, base, t0;
  int mask_lo, mask_hi;  // rows at positions in [mask_lo, mask_hi) are skipped (PSAW)
};

template <bool DENSE>
__device__ __forceinline__ UnitSpan unit_span(const AttnArgs& a, int u, int b, int nb) {
  UnitSpan sp;
  sp.t0 = nb;
  sp.mask_lo = sp.mask_hi = 0;
  if (DENSE) {
    sp.L = sp.base = nb;
    return sp;
  }
  if (a.psaw) {
    sp.mask_lo = a.psaw_sink;
    sp.mask_hi = psaw_first_visible(a.psaw_f, a.psaw_sink, nb);
  }
  int row = u, t0 = nb;
  bool tail = false;
  if (a.unit_row) {
    row = a.unit_row[u];
    t0 = a.unit_tail[u];
    tail = true;
    if (row < 0 || row >= a.pool_rows) {
      sp.L = sp.base = 0;
      return sp;
    }
  } else if (a.tail_start) {
    t0 = a.tail_start[b];
    tail = true;
  }
  int L = a.set_len[row];
  L = L < 0 ? 0 : (L > a.set_cap ? a.set_cap : L);
  sp.base = L;
  if (tail) {
    t0 = t0 < 0 ? 0 : (t0 > nb ? nb : t0);
    sp.t0 = t0;
    L += nb - t0;
    L = L > a.set_cap ? a.set_cap : L;
  }
  sp.L = L;
  return sp;
}

// Units a launch leaves alone (their outputs untouched): with a side filter,
// the ones on the other side of the gate's decision.
__device__ __forceinline__ bool unit_excluded(const AttnArgs& a, int u) {
  if (!a.unit_gate || (a.units_side != 1 && a.units_side != 2)) return false;
  const bool retrieving = a.unit_gate[u] < 0;
  return a.units_side == 1 ? !retrieving : retrieving;
}

// Row id (element offset / d) of position pos of (b, kv head g), or -1 when
// the position lies outside [0, nb) or outside the cache.
template <bool PAGED>
__device__ __forceinline__ int32_t phys_row(const KvView& kv, int b, int g, int pos, int nb) {
  if (pos < 0 || pos >= nb) return -1;
  if (!PAGED) {
    if (pos >= kv.capacity) return -1;
    return (b * kv.hkv + g) * kv.capacity + pos;
  }
  const int page = pos / kv.page_size;
  if (page >= kv.max_pages) return -1;
  const int phys = kv.table[(int64_t)b * kv.max_pages + page];
  if (phys < 0 || phys >= kv.num_pages) return -1;
  return (phys * kv.hkv + g) * kv.page_size + (pos - page * kv.page_size);
}

// Loads the set entries [start, start + chunk) of unit u before the unit's
// length is known, so that these loads share one memory latency with the
// length loads.  Entries at or past the length are loaded and never used; a
// set row holds set_cap entries, so every load stays inside it.
template <bool DENSE>
__device__ __forceinline__ void prefetch_entries(const AttnArgs& a, int u, int start,
                                                 int32_t (&raw)[kRowsPerThread]) {
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) raw[k] = -1;
  if (DENSE) return;
  int row = u;
  bool ok = true;
  if (a.unit_row) {
    row = a.unit_row[u];
    ok = row >= 0 && row < a.pool_rows;
  }
  const int32_t* idx = a.set_idx + (size_t)(ok ? row : 0) * a.set_cap;
  const int lim = min(start + a.chunk, a.set_cap);
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int t = start + (int)threadIdx.x + k * (int)blockDim.x;
    if (ok && t < lim) raw[k] = idx[t];
  }
}

// Positions of the list entries start + threadIdx.x + k * blockDim.x of the
// unit, from the entries prefetch_entries loaded; -1 for none.
template <bool DENSE>
__device__ __forceinline__ void entry_positions(const int32_t (&raw)[kRowsPerThread], int start,
                                                int n, const UnitSpan& sp,
                                                int (&pos)[kRowsPerThread]) {
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int r = threadIdx.x + k * blockDim.x;
    const int t = start + r;
    pos[k] = -1;
    if (r < n) {
      if (DENSE) {
        pos[k] = t;
      } else {
        int p;
        if (t < sp.base) {
          p = raw[k];
          p = p < sp.t0 ? p : -1;
        } else {
          p = sp.t0 + (t - sp.base);
        }
        pos[k] = (p >= sp.mask_lo && p < sp.mask_hi) ? -1 : p;
      }
    }
  }
}

// Resolves list entries [start, start + n) of the unit to row ids in s_row,
// from the entries prefetch_entries loaded; for a paged cache all block-table
// loads of a thread are issued before any is used.  n <= blockDim * 8.
template <bool DENSE, bool PAGED>
__device__ __forceinline__ void stage_rows(const AttnArgs& a, const int32_t (&raw)[kRowsPerThread],
                                           int start, int n, const UnitSpan& sp, int nb, int b,
                                           int g, int32_t* s_row) {
  int pos[kRowsPerThread];
  entry_positions<DENSE>(raw, start, n, sp, pos);
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int r = threadIdx.x + k * blockDim.x;
    if (r < n) s_row[r] = phys_row<PAGED>(a.kv, b, g, pos[k], nb);
  }
  __syncthreads();
}

// Maximum over the lanes col, col + 16, col + 32 and col + 48 (the four
// lane groups of one MFMA column), by the cross-half and cross-row lane
// swaps: each swap of a value with itself leaves a lane holding its own
// value and its partner's, one in each result.
__device__ __forceinline__ float max_over_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Maximum over all 64 lanes, in every lane: rotations by 8, 4, 2 and 1
// inside each row of 16 lanes (DPP row_ror), then across the four rows.
__device__ __forceinline__ float wave_max(float v) {
#define PRHS_ROR_MAX(CTRL)                                                                    \
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), \
                                                          CTRL, 0xF, 0xF, false)))
  PRHS_ROR_MAX(0x128);  // row_ror:8
  PRHS_ROR_MAX(0x124);  // row_ror:4
  PRHS_ROR_MAX(0x122);  // row_ror:2
  PRHS_ROR_MAX(0x121);  // row_ror:1
#undef PRHS_ROR_MAX
  return max_over_groups(v);
}

// Sum over the same four lanes.
__device__ __forceinline__ float sum_over_groups(float v) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Writes out/lse of query head bh from (M, sum, unnormalised numerator).  The
// sum is 0 where no row was attended, and NaN where a logit was.
__device__ __forceinline__ void write_final(const AttnArgs& a, size_t bh, int D, int dim, float M,
                                            float num, float den) {
  a.out[bh * D + dim] = den == 0.f ? 0.f : num / den;
  if (a.lse && dim == 0) a.lse[bh] = den == 0.f ? -INFINITY : (M + log2f(den)) * kLn2;
}

// Combines the split partials of one query head (grid: batch * num_q_heads,
// 256 threads).  Every thread first loads all it may need (the m, l and
// numerators of its first kMergePerThread split slots, for 256 / d split
// groups) together with the unit's lengths, before the number of splits in
// use is known, so the kernel costs one memory latency; slots past that
// number (stale values of earlier calls) are masked, never used in
// arithmetic.  The max, the weights and the sums follow in registers and
// LDS.  Units that fit one split were written by the split kernel and are
// skipped.
constexpr int kMergePerThread = 16;

template <int D, bool DENSE>
__global__ __launch_bounds__(256) void attn_merge(AttnArgs a) {
  constexpr int SG = 256 / D;
  __shared__ float s_red[SG][D];
  __shared__ float s_den[SG];
  __shared__ float s_max[4];
  const int bh = blockIdx.x;
  const int hkv = a.kv.hkv, hq = a.kv.hq, G = hq / hkv;
  const int b = bh / hq, h = bh % hq, u = b * hkv + h / G;
  const float* ml = a.part_ml + (size_t)bh * a.nsplit * 2;
  const float* po = a.part_o + (size_t)bh * a.nsplit * D;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int sg = tid / D, dim = tid - sg * D;
  // the first batch of slots below nsplit (a launch argument: no load
  // waits for another)
  float m0[kMergePerThread], l0[kMergePerThread], o0[kMergePerThread];
#pragma unroll
  for (int k = 0; k < kMergePerThread; ++k) {
    const int s = sg + k * SG;
    const bool in = s < a.nsplit;
    m0[k] = in ? ml[2 * s] : -INFINITY;
    l0[k] = in ? ml[2 * s + 1] : 0.f;
    o0[k] = in ? po[(size_t)s * D + dim] : 0.f;
  }
  if (!DENSE && unit_excluded(a, u)) return;
  const int L = unit_span<DENSE>(a, u, b, kv_seq_len(a.kv, b)).L;
  const int nsp = (L + a.chunk - 1) / a.chunk;
  if (nsp <= 1) return;
  float mx = -INFINITY, num = 0.f, den = 0.f;
  for (int s0 = sg; s0 < nsp; s0 += SG * kMergePerThread) {
    float m[kMergePerThread], l[kMergePerThread], o[kMergePerThread];
#pragma unroll
    for (int k = 0; k < kMergePerThread; ++k) {
      const int s = s0 + k * SG;
      const bool ok = s < nsp;
      if (s0 == sg) {
        m[k] = ok ? m0[k] : -INFINITY;
        l[k] = ok ? l0[k] : 0.f;
        o[k] = ok ? o0[k] : 0.f;
      } else {
        m[k] = ok ? ml[2 * s] : -INFINITY;
        l[k] = ok ? ml[2 * s + 1] : 0.f;
        o[k] = ok ? po[(size_t)s * D + dim] : 0.f;
      }
    }
    // rescale the running sums to the new maximum of this thread; a split whose
    // logits are all NaN has the maximum -inf and the weight 0, which leaves its
    // sums NaN
    float bm = mx;
#pragma unroll
    for (int k = 0; k < kMergePerThread; ++k) bm = fmaxf(bm, m[k]);
    const float ref = bm == -INFINITY ? 0.f : bm;
    const float r = __builtin_amdgcn_exp2f(mx - ref);
    num *= r;
    den *= r;
#pragma unroll
    for (int k = 0; k < kMergePerThread; ++k) {
      const float f = __builtin_amdgcn_exp2f(m[k] - ref);
      num += f * o[k];
      den += f * l[k];
    }
    mx = bm;
  }
  // block-wide maximum
  const float wm = wave_max(mx);
  if (lane == 0) s_max[wave] = wm;
  __syncthreads();
  const float M = fmaxf(fmaxf(s_max[0], s_max[1]), fmaxf(s_max[2], s_max[3]));
  const float f = (mx == -INFINITY || M == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(mx - M);
  s_red[sg][dim] = num * f;
  if (dim == 0) s_den[sg] = den * f;
  __syncthreads();
  if (sg == 0) {
    float tot = 0.f, dt = 0.f;
#pragma unroll
    for (int k = 0; k < SG; ++k) {
      tot += s_red[k][dim];
      dt += s_den[k];
    }
    write_final(a, bh, D, dim, M, tot, dt);
  }
}

struct AttnLayout {
  size_t part_o, part_ml, total;
};

AttnLayout attn_layout(int batch, int hq, int d, int nsplit) {
  const size_t parts = (size_t)batch * hq * nsplit;
  AttnLayout L;
  size_t off = 0;
  L.part_o = off;  off += (parts * d * 4 + 255) & ~(size_t)255;
  L.part_ml = off; off += parts * 2 * 4;
  L.total = off;
  return L;
}

}  // namespace
}  // namespace prhs
