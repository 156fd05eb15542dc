// Decode attention over the 8-bit cache, split-K: for the rows i of a unit's
// list (attention_common.h) with block scales ks, vs
//   x_i = scale ks_i (q . k8_i),   y = sum_i softmax(x)_i vs_i v8_i.
// One workgroup per (unit, split) walks a contiguous chunk of the list with an
// online softmax; a unit of several splits is joined by attn_merge.
//
// e4m3 values are exact in bf16 and fp16, so both products run on MFMA without
// rounding an operand: K as bf16 with q (fp32 queries as three bf16 parts), V as
// fp16 with the weights w_i = p_i vs_i 128 / R, R the largest vs of the chunk.
// p stays below 2^8 (lazy rescaling), so w is at most 2^15, and as an fp16 pair
// hi + lo it keeps 22 bits, or an absolute 2^-25: 2^-32 of the largest weight.
//
// Row ids and scales of the chunk are staged in LDS (a row's scale is that of
// block row_id / block_size).  A wave then walks 32-row tiles, the next tile's
// loads in flight while one is multiplied: K in whole rows (d / 16 lanes of 16
// bytes) through a per-wave LDS tile into operand order, V (rows 16s + 4 grp + e,
// d / 16 bytes per lane) straight into operands by byte permutes.
#include <algorithm>

#include "attention_common.h"
#include "prhs_internal.h"

namespace prhs {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

struct QuantArgs : AttnArgs {
  QuantScales sc;
};

constexpr int kWaves = 4;
constexpr int kMaxChunk = 64 * kWaves * kRowsPerThread;   // rows a workgroup stages
constexpr long long kGroups = 256;                        // workgroups aimed at
constexpr int kNoSplitRows = 512;

// LDS bytes of a wave: its K tile of 32 rows, at the end its G output rows.
__host__ __device__ constexpr int wave_bytes(int D, int G) {
  return ((32 * D > G * (D + 1) * 4 ? 32 * D : G * (D + 1) * 4) + 15) & ~15;
}

// 16-byte chunk c of tile row r in the wave's K tile.
template <int D>
__device__ __forceinline__ int kst_slot(int r, int c) {
  constexpr int CH = D / 16;
  return r * CH + (c ^ (r & (CH - 1)));
}

// Stages row ids and scales of list entries [start, start + n), and entries
// without a row up to the next multiple of 32.  Scales of K carry the softmax
// scale, those of V 128 / R; returns R / 128.
template <bool DENSE, bool PAGED>
__device__ __forceinline__ float stage(const QuantArgs& a, const int32_t (&raw)[kRowsPerThread],
                                       int start, int n, const UnitSpan& sp, int nb, int b, int g,
                                       int32_t* s_row, float* s_ks, float* s_vs, float* s_max) {
  const int n32 = (n + 31) & ~31;
  int pos[kRowsPerThread], row[kRowsPerThread];
  float ks[kRowsPerThread], vs[kRowsPerThread];
  entry_positions<DENSE>(raw, start, n, sp, pos);
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) row[k] = phys_row<PAGED>(a.kv, b, g, pos[k], nb);
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int blk = row[k] < 0 ? 0 : row[k] >> a.sc.block_shift;
    ks[k] = row[k] < 0 ? 0.f : a.sc.k[blk] * a.scale_log2;
    vs[k] = row[k] < 0 ? 0.f : a.sc.v[blk];
    top = fmaxf(top, vs[k]);
  }
  top = wave_max(top);
  if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = top;
  __syncthreads();
  const int nwaves = blockDim.x >> 6;
  for (int w = 0; w < nwaves; ++w) top = fmaxf(top, s_max[w]);
  if (!(top > 0.f)) top = 1.f;
  const float inv = 128.f / top;
#pragma unroll
  for (int k = 0; k < kRowsPerThread; ++k) {
    const int r = threadIdx.x + k * blockDim.x;
    if (r < n32) {
      s_row[r] = row[k];
      s_ks[r] = ks[k];
      s_vs[r] = vs[k] * inv;
    }
  }
  __syncthreads();
  return top * (1.f / 128.f);
}

template <int D>
struct Tile {
  static constexpr int KL = D / 32;   // K loads of 16 bytes per lane
  static constexpr int VW = D / 64;   // words of a V piece
  u32x4_t k[KL];
  uint32_t v[8][VW];
  uint32_t ok;
};

template <int D>
__device__ __forceinline__ void load_tile(Tile<D>& T, const int32_t* s_row, int r0, const uint8_t* kb,
                                          const uint8_t* vb, int lane) {
  constexpr int CH = D / 16, RPI = 64 / CH;
  const int col = lane & 15, grp = lane >> 4;
  int rk[Tile<D>::KL], rv[8];
#pragma unroll
  for (int j = 0; j < Tile<D>::KL; ++j) rk[j] = s_row[r0 + j * RPI + lane / CH];
#pragma unroll
  for (int j = 0; j < 8; ++j) rv[j] = s_row[r0 + 16 * (j >> 2) + grp * 4 + (j & 3)];
#pragma unroll
  for (int j = 0; j < Tile<D>::KL; ++j)
    T.k[j] = stream_load16(kb + (int64_t)max(rk[j], 0) * D + (lane % CH) * 16);
  T.ok = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint8_t* p = vb + (int64_t)max(rv[j], 0) * D + col * (D / 16);
    if constexpr (D == 128) {
      const u32x2_t x = stream_load8(p);
      T.v[j][0] = x[0];
      T.v[j][1] = x[1];
    } else {
      T.v[j][0] = __builtin_nontemporal_load((const uint32_t*)p);
    }
    if (rv[j] >= 0) T.ok |= 1u << j;
  }
}

template <int D>
struct WaveState {
  float m, l;
  f32x4_t o[D / 16];
};

__device__ __forceinline__ bf16x8_t bf16_of_e4m3(uint32_t a, uint32_t b) {
  uint32_t w[4];
  w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false));
  w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true));
  w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false));
  w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true));
  return __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
}

template <bool HI>
__device__ __forceinline__ uint32_t f16_of_e4m3(uint32_t a) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, HI));
}

template <int D, int QP>
__device__ __forceinline__ void consume_tile(Tile<D>& T, WaveState<D>& st,
                                             const bf16x8_t (&qf)[QP][D / 32], const float* s_ks,
                                             const float* s_vs, int r0, u32x4_t* kst, int lane) {
  constexpr int CH = D / 16, RPI = 64 / CH;
  const int col = lane & 15, grp = lane >> 4;
  // K to operand order: lane (col, grp) takes dims grp D/4 .. of rows col and 16 + col
#pragma unroll
  for (int j = 0; j < Tile<D>::KL; ++j) kst[kst_slot<D>(j * RPI + lane / CH, lane % CH)] = T.k[j];
  __builtin_amdgcn_wave_barrier();
  u32x4_t kr[2][CH / 4];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int i = 0; i < CH / 4; ++i) kr[s][i] = kst[kst_slot<D>(16 * s + col, grp * (CH / 4) + i)];
  __builtin_amdgcn_wave_barrier();
  float x[8], w[8];
  float mt = -INFINITY;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
      const u32x4_t c = kr[s][kk >> 1];
      const bf16x8_t kf = bf16_of_e4m3(c[2 * (kk & 1)], c[2 * (kk & 1) + 1]);
#pragma unroll
      for (int part = QP - 1; part >= 0; --part)   // small parts first
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[part][kk], acc, 0, 0, 0);
    }
    const float4 ks = *(const float4*)(s_ks + r0 + 16 * s + 4 * grp);
    const float kse[4] = {ks.x, ks.y, ks.z, ks.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = s * 4 + e;
      x[j] = (T.ok >> j) & 1u ? acc[e] * kse[e] : -INFINITY;
      mt = fmaxf(mt, x[j]);
    }
  }
  // entries without a row read a stand-in row: their V must not count
  if (__builtin_amdgcn_ballot_w64(T.ok != 0xFFu)) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (!((T.ok >> j) & 1u)) {
#pragma unroll
        for (int i = 0; i < Tile<D>::VW; ++i) T.v[j][i] = 0u;
      }
  }
  mt = max_over_groups(mt);
  const float m_new = fmaxf(st.m, mt);
  if (__builtin_amdgcn_ballot_w64(m_new > st.m + 8.f)) {
    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - m_new);
    st.m = m_new;
    st.l *= alpha;
#pragma unroll
    for (int blk = 0; blk < D / 16; ++blk) st.o[blk] *= alpha;
  }
  const float mref = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const float4 vs = *(const float4*)(s_vs + r0 + 16 * s + 4 * grp);
    const float vse[4] = {vs.x, vs.y, vs.z, vs.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = __builtin_amdgcn_exp2f(x[s * 4 + e] - mref);
      st.l += p;
      w[s * 4 + e] = p * vse[e];
    }
  }
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f16x2_t h = __builtin_convertvector(f32x2_t{w[2 * i], w[2 * i + 1]}, f16x2_t);
    hi[i] = __builtin_bit_cast(uint32_t, h);
    lo[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
        f32x2_t{w[2 * i] - (float)h[0], w[2 * i + 1] - (float)h[1]}, f16x2_t));
  }
  const f16x8_t whi = __builtin_bit_cast(f16x8_t, make_uint4(hi[0], hi[1], hi[2], hi[3]));
  const f16x8_t wlo = __builtin_bit_cast(f16x8_t, make_uint4(lo[0], lo[1], lo[2], lo[3]));
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {   // dims 2i, 2i + 1 of the lane's piece
    uint32_t a0[4], a1[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // bytes (row 2j, dim 2i), (row 2j+1, dim 2i), then the same of dim 2i + 1
      const uint32_t y = __builtin_amdgcn_perm(T.v[2 * j + 1][i >> 1], T.v[2 * j][i >> 1],
                                               (i & 1) ? 0x07030602u : 0x05010400u);
      a0[j] = f16_of_e4m3<false>(y);
      a1[j] = f16_of_e4m3<true>(y);
    }
    const f16x8_t v0 = __builtin_bit_cast(f16x8_t, make_uint4(a0[0], a0[1], a0[2], a0[3]));
    const f16x8_t v1 = __builtin_bit_cast(f16x8_t, make_uint4(a1[0], a1[1], a1[2], a1[3]));
    st.o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, whi, st.o[2 * i], 0, 0, 0);
    st.o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, whi, st.o[2 * i + 1], 0, 0, 0);
    st.o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, wlo, st.o[2 * i], 0, 0, 0);
    st.o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, wlo, st.o[2 * i + 1], 0, 0, 0);
  }
}

// The query operand of product kk: dims grp D/4 + 8 kk .. +7 of head col, in QP
// bf16 parts (fp32: the value is the sum of three, 24 bits).
typedef uint32_t u32x4_a2_t __attribute__((ext_vector_type(4), aligned(2)));
template <int D, int QP>
__device__ __forceinline__ void load_query(const void* q, size_t bh, bool on, int grp,
                                           bf16x8_t (&qf)[QP][D / 32]) {
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    const size_t at = bh * D + grp * (D / 4) + 8 * kk;
    if constexpr (QP == 1) {
      const u32x4_t v = *(const u32x4_a2_t*)((const __bf16*)q + at);
      qf[0][kk] = __builtin_bit_cast(bf16x8_t, on ? v : u32x4_t{0u, 0u, 0u, 0u});
    } else {
      const float4 x = load_f32x4((const float*)q + at), y = load_f32x4((const float*)q + at + 4);
      float r[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int part = 0; part < QP; ++part) {
        bf16x8_t h;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[i] = (__bf16)(on ? r[i] : 0.f);
          r[i] -= (float)h[i];
        }
        qf[part][kk] = h;
      }
    }
  }
}

template <int D, bool DENSE, bool PAGED, int QP>
__global__ __launch_bounds__(64 * kWaves) void quant_attn_split(QuantArgs a) {
  // dynamic LDS: per-wave regions, then row ids and scales of the chunk
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
  __shared__ float sm_m[kWaves][16], sm_l[kWaves][16], s_max[kWaves];
  const int split = blockIdx.x % a.nsplit, u = blockIdx.x / a.nsplit;
  const int hkv = a.kv.hkv, hq = a.kv.hq, G = hq / hkv;
  const int wbytes = wave_bytes(D, G);
  const int nwaves = blockDim.x >> 6, staged = blockDim.x * kRowsPerThread;
  int32_t* s_row = (int32_t*)(dyn + (size_t)nwaves * wbytes);
  float* s_ks = (float*)(s_row + staged);
  float* s_vs = s_ks + staged;
  const int b = u / hkv, g = u - b * hkv;
  const int start = split * a.chunk;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, grp = lane >> 4;
  int32_t raw[kRowsPerThread];
  prefetch_entries<DENSE>(a, u, start, raw);
  bf16x8_t qf[QP][D / 32];
  load_query<D, QP>(a.q, (size_t)b * hq + g * G + (col < G ? col : 0), col < G, grp, qf);
  const int nb = kv_seq_len(a.kv, b);
  if (!DENSE && unit_excluded(a, u)) return;
  const UnitSpan sp = unit_span<DENSE>(a, u, b, nb);
  const int L = sp.L;
  if (L == 0 && split == 0) {  // empty set: y = 0, lse = -inf
    for (int e = threadIdx.x; e < G * D; e += blockDim.x)
      write_final(a, (size_t)b * hq + g * G + e / D, D, e % D, -INFINITY, 0.f, 0.f);
    return;
  }
  if (start >= L) return;
  const int n = min(L, start + a.chunk) - start;
  const float unscale = stage<DENSE, PAGED>(a, raw, start, n, sp, nb, b, g, s_row, s_ks, s_vs, s_max);

  const uint8_t* kb = (const uint8_t*)a.kv.k;
  const uint8_t* vb = (const uint8_t*)a.kv.v;
  WaveState<D> st;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) st.o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int ntiles = (n + 31) >> 5;
  const int iters = wave < ntiles ? (ntiles - wave + nwaves - 1) / nwaves : 0;
  if (iters > 0) {
    Tile<D> A, B;
    u32x4_t* kst = (u32x4_t*)(dyn + (size_t)wave * wbytes);
    const int step = 32 * nwaves;
    int r0 = wave * 32;
    load_tile<D>(A, s_row, r0, kb, vb, lane);
    int i = 0;
    for (; i + 2 < iters; i += 2) {
      load_tile<D>(B, s_row, r0 + step, kb, vb, lane);
      consume_tile<D, QP>(A, st, qf, s_ks, s_vs, r0, kst, lane);
      load_tile<D>(A, s_row, r0 + 2 * step, kb, vb, lane);
      consume_tile<D, QP>(B, st, qf, s_ks, s_vs, r0 + step, kst, lane);
      r0 += 2 * step;
    }
    if (i + 1 < iters) {
      load_tile<D>(B, s_row, r0 + step, kb, vb, lane);
      consume_tile<D, QP>(A, st, qf, s_ks, s_vs, r0, kst, lane);
      consume_tile<D, QP>(B, st, qf, s_ks, s_vs, r0 + step, kst, lane);
    } else {
      consume_tile<D, QP>(A, st, qf, s_ks, s_vs, r0, kst, lane);
    }
  }

  st.l = sum_over_groups(st.l);
  if (grp == 0) {
    sm_m[wave][col] = st.m;
    sm_l[wave][col] = st.l;
  }
  if (col < G) {
    float* wo = (float*)(dyn + (size_t)wave * wbytes) + col * (D + 1);
#pragma unroll
    for (int blk = 0; blk < D / 16; ++blk)
#pragma unroll
      for (int i = 0; i < 4; ++i) wo[(grp * 4 + i) * (D / 16) + blk] = st.o[blk][i] * unscale;
  }
  __syncthreads();
  const int nsp = (L + a.chunk - 1) / a.chunk;
  for (int e = threadIdx.x; e < G * D; e += blockDim.x) {
    const int h = e / D, dim = e - h * D;
    float M = -INFINITY;
    for (int w = 0; w < nwaves; ++w) M = fmaxf(M, sm_m[w][h]);
    float num = 0.f, den = 0.f;
    if (M != -INFINITY) {
      for (int w = 0; w < nwaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm_m[w][h] - M);
        num += f * ((const float*)(dyn + (size_t)w * wbytes))[h * (D + 1) + dim];
        den += f * sm_l[w][h];
      }
    }
    const size_t bh = (size_t)b * hq + g * G + h;
    if (nsp == 1) {
      write_final(a, bh, D, dim, M, num, den);
    } else {
      const size_t pidx = bh * a.nsplit + split;
      a.part_o[pidx * D + dim] = num;
      if (dim == 0) {
        a.part_ml[pidx * 2] = M;
        a.part_ml[pidx * 2 + 1] = den;
      }
    }
  }
}

// Rows per workgroup and splits per unit: at most kGroups workgroups, or as many
// as staging needs.
void split_geometry(bool dense, long long units, int rows_cap, int* chunk, int* nsplit) {
  const long long rows = std::max(rows_cap, 1);
  const long long k = std::max(1LL, kGroups / std::max(1LL, units));
  long long c = (rows + k - 1) / k;
  if (!dense && rows <= kNoSplitRows) c = rows;
  c = std::min<long long>((c + 31) / 32 * 32, kMaxChunk);
  *chunk = (int)c;
  *nsplit = (int)((rows + c - 1) / c);
}

template <int D, bool DENSE, bool PAGED, int QP>
hipError_t launch_typed(const QuantArgs& a, hipStream_t stream) {
  const int units = a.kv.batch * a.kv.hkv, G = a.kv.hq / a.kv.hkv;
  const int waves = std::min(kWaves, (a.chunk + 31) / 32);
  const size_t dyn = (size_t)waves * (wave_bytes(D, G) + 64 * kRowsPerThread * 12);
  static_assert(kWaves * (wave_bytes(D, 16) + 64 * kRowsPerThread * 12) <= 65536 - 1024,
                "LDS that needs no attribute");
  hipLaunchKernelGGL((quant_attn_split<D, DENSE, PAGED, QP>), dim3((unsigned)units * a.nsplit),
                     dim3(64 * waves), dyn, stream, a);
  if (a.nsplit > 1)
    hipLaunchKernelGGL((attn_merge<D, DENSE>), dim3(a.kv.batch * a.kv.hq), dim3(256), 0, stream,
                       (const AttnArgs&)a);
  return hipGetLastError();
}

template <int D, bool DENSE>
hipError_t launch_layout(const QuantArgs& a, int dtype, hipStream_t stream) {
  if (a.kv.paged)
    return dtype == 1 ? launch_typed<D, DENSE, true, 1>(a, stream)
                      : launch_typed<D, DENSE, true, 3>(a, stream);
  return dtype == 1 ? launch_typed<D, DENSE, false, 1>(a, stream)
                    : launch_typed<D, DENSE, false, 3>(a, stream);
}

}  // namespace

long long quant_attn_groups(bool dense, int batch, int hkv, int rows_cap) {
  int chunk, nsplit;
  split_geometry(dense, (long long)batch * hkv, rows_cap, &chunk, &nsplit);
  return (long long)batch * hkv * nsplit;
}

size_t quant_attn_call_bytes(bool dense, int batch, int hq, int hkv, int d, int rows_cap) {
  int chunk, nsplit;
  split_geometry(dense, (long long)batch * hkv, rows_cap, &chunk, &nsplit);
  return attn_layout(batch, hq, d, nsplit).total;
}

// A call of fewer sequences may split its units more: a launch has at most
// max(kGroups, units * the splits that staging needs) workgroups, so that many
// partials of hq / hkv heads hold every such call.
size_t quant_attn_workspace_bytes(bool dense, int batch, int hq, int hkv, int d, int rows_cap) {
  const long long units = (long long)batch * hkv, rows = std::max(rows_cap, 1);
  const long long groups = std::max(kGroups, units * ((rows + kMaxChunk - 1) / kMaxChunk));
  const long long per = units > 0 ? (groups + units - 1) / units : 0;
  return std::max(attn_layout(batch, hq, d, (int)per).total,
                  quant_attn_call_bytes(dense, batch, hq, hkv, d, rows_cap));
}

hipError_t launch_quant_attention(const AttnLaunch& s, const QuantScales& scales, bool dense,
                                  hipStream_t stream) {
  QuantArgs a;
  a.sc = scales;
  a.kv = s.kv;
  a.q = s.q;
  a.set_idx = s.set_idx;
  a.set_len = s.set_len;
  a.tail_start = dense ? nullptr : s.tail_start;
  a.unit_row = dense ? nullptr : s.unit_row;
  a.unit_tail = dense ? nullptr : s.unit_tail;
  a.pool_rows = s.pool_rows;
  a.unit_gate = dense ? nullptr : s.unit_gate;
  a.units_side = s.units_side;
  a.psaw = dense ? 0 : s.psaw;
  a.psaw_f = s.psaw_f;
  a.psaw_sink = s.psaw_sink;
  a.set_cap = s.set_cap;
  a.scale_log2 = s.scale * 1.44269504088896340736f;
  split_geometry(dense, (long long)s.kv.batch * s.kv.hkv, dense ? s.kv.max_seq_len : s.set_cap,
                 &a.chunk, &a.nsplit);
  const AttnLayout L = attn_layout(s.kv.batch, s.kv.hq, s.kv.d, a.nsplit);
  a.part_o = (float*)((char*)s.ws + L.part_o);
  a.part_ml = (float*)((char*)s.ws + L.part_ml);
  a.out = s.out;
  a.lse = s.lse;
  if (s.kv.d == 128)
    return dense ? launch_layout<128, true>(a, s.dtype, stream)
                 : launch_layout<128, false>(a, s.dtype, stream);
  return dense ? launch_layout<64, true>(a, s.dtype, stream)
               : launch_layout<64, false>(a, s.dtype, stream);
}

}  // namespace prhs
