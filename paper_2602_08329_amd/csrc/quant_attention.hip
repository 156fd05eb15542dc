// Decode attention over the 8-bit cache, split-K: for the rows i of a unit's
// list (attention_common.h) with block scales ks, vs
//   x_i = scale ks_i (q . k8_i),   y = sum_i softmax(x)_i vs_i v8_i.
// One workgroup per (unit, split) walks a contiguous chunk of the list with an
// online softmax; a unit of several splits is joined by attn_merge.
//
// e4m3 values are exact in bf16, so both products run on MFMA without rounding
// an operand to less than fp32 holds: K with q (fp32 queries as three bf16 parts,
// 24 bits), V with the weights w_i = p_i vs_i r, three bf16 parts as well, r a
// power of two, at most 2^126, that brings the largest vs the wave has met to
// [2^80, 2^81) (a normal one to 1 or more).  p is at most 2^8 (lazy rescaling), so
// sums over 2^22 rows stay below 2^120, and the parts are normal numbers for w down
// to 2^-110, at most that part of the largest weight.  Two fp16 parts have too
// little range: beside a block whose values are 2^20 times the others' they left
// about ten bits of the others' weights.  They cost a product less: one sequence of
// 617 tokens 8.8 us, 9.3 so.
// With at most 8 heads a kv head, two of the parts are two columns of one product
// (the queries stand in the columns twice), else each part is a product.
//
// A wave walks tiles of 32 rows: lane l knows row l of its tile.  List entries
// are read three tiles ahead, their pages two, K, V and scales one, into
// registers in whole rows (d / 16 lanes of 16 bytes).  A tile passes through the
// wave's own LDS, K into operand order, V by transposing reads
// (ds_read_b64_tr_b8: of the 8-byte pieces that a group of 16 lanes addresses,
// lane l receives byte l mod 8 of pieces l / 8, l / 8 + 2, ..).  Every load is
// issued unconditionally, from a stand-in address where there is no row, as one
// behind a branch would make the compiler wait for all of them.
//
// Reading the bytes bounds long streams: 64 sequences of 8k to 16k, 32 over 8
// heads of d 128 (1.59 GB) 242 us, 6.6 TB/s, 8 of 4k with 32 kv heads (269 MB) 42
// us, 6.4 TB/s, where a plain read reaches 7.1.  Few units are bound by the chain of
// loads (list, page, row), the joining of the waves and the second launch: the
// selected set of one 128k sequence (8 units of 2300 rows, 4.8 MB) 10.6 us, in a
// trace 7.8 and 4.0 in attn_merge.
#include <algorithm>
#include <cmath>

#include "attention_common.h"
#include "prhs_internal.h"

namespace prhs {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_a2_t __attribute__((ext_vector_type(4), aligned(2)));

struct QuantArgs : AttnArgs {
  QuantScales sc;
  int by_length;   // workgroups take their units longest sequence first
};

constexpr int kTile = 32;   // rows of a wave's tile

// LDS bytes of a wave: its tile of K, of V and their scales, at the end its G
// output rows.
__host__ __device__ constexpr int wave_bytes(int D, int G) {
  const int tile = 2 * kTile * D + 2 * kTile * 4, out = G * (D + 4) * 4;
  return ((tile > out ? tile : out) + 15) & ~15;
}

// LDS bytes of the query operands, which fp32 queries keep there.
__host__ __device__ constexpr int query_bytes(int D, int QP) {
  return QP > 1 ? QP * (D / 32) * 64 * 16 : 0;
}

// 16-byte chunk c of tile row r: the same chunk of eight rows lies in eight
// different places of a 128-byte line.
template <int D>
__device__ __forceinline__ int tile_slot(int r, int c) {
  return D == 128 ? r * 8 + (c ^ (r & 7)) : r * 4 + (c ^ ((r >> 1) & 3));
}

// A unit's list in tiles: row ids of entry `t` in three steps, each from what the
// one before loaded.
template <bool DENSE, bool PAGED>
struct Rows {
  const int32_t* idx;     // the unit's set
  const int32_t* table;   // its sequence's pages
  UnitSpan sp;
  int nb, base, last_page, hkv, g, num_pages, shift, set_last;

  __device__ __forceinline__ int entry(int t) const { return DENSE ? t : idx[min(t, set_last)]; }
  // position of entry t, -1 for none; end: entries of the list
  __device__ __forceinline__ int pos(int raw, int t, int end) const {
    if (DENSE) return t < end ? t : -1;
    int p = t < sp.base ? (raw < sp.t0 ? raw : -1) : sp.t0 + (t - sp.base);
    if (p >= sp.mask_lo && p < sp.mask_hi) p = -1;
    return t < end && p >= 0 && p < nb ? p : -1;
  }
  __device__ __forceinline__ int page(int p) const {
    return PAGED ? table[min(max(p, 0) >> shift, last_page)] : 0;
  }
  __device__ __forceinline__ int row(int page, int p) const {
    if (p < 0) return -1;
    if (!PAGED) return base + p;
    if (page < 0 || page >= num_pages || (p >> shift) > last_page) return -1;
    return ((page * hkv + g) << shift) + (p & ((1 << shift) - 1));
  }
};

template <int D>
struct Tile {
  static constexpr int KL = D / 32;   // loads of 16 bytes per lane, of K and of V
  u32x4_t k[KL], v[KL];
  float ks, vs;   // of row lane mod 32; 0 without a row
  uint32_t ok;    // rows that are there
};

// Issues the loads of the tile whose row ids the lanes hold.
template <int D>
__device__ __forceinline__ void load_tile(Tile<D>& T, const QuantArgs& a, int row, int lane) {
  constexpr int CH = D / 16, RPI = 64 / CH;
  const uint8_t* kb = (const uint8_t*)a.kv.k;
  const uint8_t* vb = (const uint8_t*)a.kv.v;
  const int r0 = max(row, 0), blk = r0 >> a.sc.block_shift;
  T.ok = (uint32_t)__builtin_amdgcn_ballot_w64(row >= 0);
  T.ks = a.sc.k[blk];
  T.vs = a.sc.v[blk];
#pragma unroll
  for (int j = 0; j < Tile<D>::KL; ++j) {
    const int64_t at = (int64_t)__shfl(r0, j * RPI + lane / CH) * D + (lane % CH) * 16;
    T.k[j] = stream_load16(kb + at);
    T.v[j] = stream_load16(vb + at);
  }
}

// A loaded tile to the wave's LDS, its V scales times r; rows that are not there
// get V = 0 and scales of 0 (their K only reaches logits that are masked).
template <int D>
__device__ __forceinline__ void stage_tile(const Tile<D>& T, float scale_log2, float r, u32x4_t* s_k,
                                           u32x4_t* s_v, float* s_sc, int lane) {
  constexpr int CH = D / 16, RPI = 64 / CH;
#pragma unroll
  for (int j = 0; j < Tile<D>::KL; ++j) {
    const int row = j * RPI + lane / CH, slot = tile_slot<D>(row, lane % CH);
    s_k[slot] = T.k[j];
    s_v[slot] = T.ok == 0xFFFFFFFFu || ((T.ok >> row) & 1u) ? T.v[j] : u32x4_t{0u, 0u, 0u, 0u};
  }
  if (lane < kTile) {
    const bool in = (T.ok >> lane) & 1u;
    s_sc[lane] = in ? T.ks * scale_log2 : 0.f;
    s_sc[kTile + lane] = in ? T.vs * r : 0.f;
  }
}

template <int D>
struct WaveState {
  float m, l;
  int ve;       // exponent bits of the largest V scale met
  float r;      // 2^(80 - that exponent), at most 2^126
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

// The query operands, of product kk dims grp D/4 + 8 kk .. +7 of a lane's head
// (lanes without one take the first head's, to no effect).  bf16: in registers, not
// touched before the first product, as a use waits for all earlier loads.
template <int D, int QP>
struct Query {
  bf16x8_t f[D / 32];

  __device__ __forceinline__ void load(const void* q, size_t at, int) {
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
      const u32x4_t v = *(const u32x4_a2_t*)((const __bf16*)q + at + 8 * kk);
      f[kk] = __builtin_bit_cast(bf16x8_t, v);
    }
  }
  __device__ __forceinline__ void stage(const void*, size_t, int, int, int, u32x4_t*) {}
  __device__ __forceinline__ bf16x8_t part(int, int kk, const u32x4_t*, int) const { return f[kk]; }
};

// fp32: in three bf16 parts (24 bits) in LDS, product kk by wave kk; a barrier
// follows (all products by every wave, without one: 7 units of 16 heads and 11312
// rows 16.0 us, 15.2 so).
template <int D>
struct Query<D, 3> {
  float4 x, y;   // of product wave mod D / 32

  __device__ __forceinline__ void load(const void* q, size_t at, int wave) {
    x = load_f32x4((const float*)q + at + 8 * (wave % (D / 32)));
    y = load_f32x4((const float*)q + at + 8 * (wave % (D / 32)) + 4);
  }
  __device__ __forceinline__ void stage(const void* q, size_t at, int wave, int nwaves, int lane,
                                        u32x4_t* s_q) {
    for (int kk = wave % (D / 32);;) {
      float r[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
      for (int part = 0; part < 3; ++part) {
        bf16x8_t h;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[i] = (__bf16)r[i];
          r[i] -= (float)h[i];
        }
        s_q[(part * (D / 32) + kk) * 64 + lane] = __builtin_bit_cast(u32x4_t, h);
      }
      kk += nwaves;
      if (kk >= D / 32) break;
      x = load_f32x4((const float*)q + at + 8 * kk);
      y = load_f32x4((const float*)q + at + 8 * kk + 4);
    }
  }
  __device__ __forceinline__ bf16x8_t part(int p, int kk, const u32x4_t* s_q, int lane) const {
    return __builtin_bit_cast(bf16x8_t, s_q[(p * (D / 32) + kk) * 64 + lane]);
  }
};

// Lane (col, grp) owns query head col (with !WIDE col mod 8) and in the V product
// the rows 16 s + 4 grp + e of the tile, in the order 4 s + e.
template <int D, int QP, bool WIDE>
__device__ __forceinline__ void consume_tile(uint32_t ok, WaveState<D>& st,
                                             const Query<D, QP>& q, const u32x4_t* s_q,
                                             const u32x4_t* s_k, const u32x4_t* s_v, const float* s_sc,
                                             int lane) {
  constexpr int CH = D / 16;
  const int col = lane & 15, grp = lane >> 4;
  // lane (col, grp) takes dims grp D/4 .. of rows col and 16 + col
  float x[8];
  float mt = -INFINITY;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < CH / 4; ++i) {
      const u32x4_t c = s_k[tile_slot<D>(16 * s + col, grp * (CH / 4) + i)];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int kk = 2 * i + h;
        const bf16x8_t kf = bf16_of_e4m3(c[2 * h], c[2 * h + 1]);
#pragma unroll
        for (int part = QP - 1; part >= 0; --part)   // small parts first
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q.part(part, kk, s_q, lane), acc, 0, 0, 0);
      }
    }
    const float4 ks = *(const float4*)(s_sc + 16 * s + 4 * grp);
    const float kse[4] = {ks.x, ks.y, ks.z, ks.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) x[s * 4 + e] = acc[e] * kse[e];
  }
  if (ok != 0xFFFFFFFFu) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = (ok >> (16 * (j >> 2) + 4 * grp + (j & 3))) & 1u ? x[j] : -INFINITY;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) mt = fmaxf(mt, x[j]);
  // lazy rescaling: the reference st.m moves only when some head of the wave sees
  // its maximum rise by more than 2^8
  if (__builtin_amdgcn_ballot_w64(mt > st.m + 8.f)) {
    const float m_new = fmaxf(st.m, max_over_groups(mt));
    const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m - m_new);
    st.m = m_new;
    st.l *= alpha;
#pragma unroll
    for (int blk = 0; blk < D / 16; ++blk) st.o[blk] *= alpha;
  }
  const float mref = st.m == -INFINITY ? 0.f : st.m;
  float w[8];
  float4 vs[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) vs[s] = *(const float4*)(s_sc + kTile + 16 * s + 4 * grp);
  const float vse[8] = {vs[0].x, vs[0].y, vs[0].z, vs[0].w, vs[1].x, vs[1].y, vs[1].z, vs[1].w};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float p = __builtin_amdgcn_exp2f(x[j] - mref);
    st.l += p;
    w[j] = p * vse[j];
  }
  // The parts of w are its upper eight significant bits, the next eight and the
  // rest, each the upper half of an fp32 word.  Not WIDE: one product with the first
  // in columns 0 .. 7 and the second in 8 .. 15, where lanes take the first off
  // beforehand, and another with the third in columns 8 .. 15.
  constexpr uint32_t kUpper = 0xFFFF0000u;
  constexpr int NP = WIDE ? 3 : 2;
  const uint32_t off = !WIDE && col >= 8 ? kUpper : 0u;
  const uint32_t last = WIDE || col >= 8 ? 0x07060302u : 0x0C0C0C0Cu;   // upper halves, zeros
  bf16x8_t part[NP];
  if (!WIDE)
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] -= __uint_as_float(__float_as_uint(w[j]) & off);
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      u[i] = __builtin_amdgcn_perm(__float_as_uint(w[2 * i + 1]), __float_as_uint(w[2 * i]),
                                   k == NP - 1 ? last : 0x07060302u);
    part[k] = __builtin_bit_cast(bf16x8_t, make_uint4(u[0], u[1], u[2], u[3]));
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] -= __uint_as_float(__float_as_uint(w[j]) & kUpper);
  }
  // lane `col` of a group addresses 8 dims of the group's row col / 2 (in the
  // order of w) and receives dim 16 blk + col of its 8 rows
  const int vr = 16 * (col >> 3) + 4 * grp + ((col >> 1) & 3);
#pragma unroll
  for (int blk = 0; blk < D / 16; ++blk) {
    const uint8_t* at = (const uint8_t*)(s_v + tile_slot<D>(vr, blk)) + 8 * (col & 1);
    const i32x2_t t = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2_t*)at);
    const bf16x8_t v = bf16_of_e4m3((uint32_t)t[0], (uint32_t)t[1]);
#pragma unroll
    for (int k = NP - 1; k >= 0; --k)   // small parts first
      st.o[blk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, part[k], st.o[blk], 0, 0, 0);
  }
}

template <int D, bool DENSE, bool PAGED, int QP, bool WIDE>
__global__ __launch_bounds__(64 * kMaxWaves) void quant_attn_split(QuantArgs a) {
  // dynamic LDS: per-wave regions, then the query operands of fp32 queries
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
  __shared__ float sm_m[kMaxWaves][16], sm_l[kMaxWaves][16];
  __shared__ int s_unit;
  const int split = blockIdx.x % a.nsplit;
  int u = blockIdx.x / a.nsplit;
  if (DENSE && a.by_length) u = unit_of_length_rank(a.kv, a.kv.hkv, u, (int*)dyn, &s_unit);
  const int hkv = a.kv.hkv, hq = a.kv.hq, G = hq / hkv;
  const int wbytes = wave_bytes(D, G);
  const int nwaves = blockDim.x >> 6;
  const int b = u / hkv, g = u - b * hkv;
  const int start = split * a.chunk;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, grp = lane >> 4;
  unsigned char* own = dyn + (size_t)wave * wbytes;
  u32x4_t* s_k = (u32x4_t*)own;
  u32x4_t* s_v = (u32x4_t*)(own + kTile * D);
  float* s_sc = (float*)(own + 2 * kTile * D);
  u32x4_t* s_q = (u32x4_t*)(dyn + (size_t)nwaves * wbytes);

  // list entries, query and lengths load together
  const int step = kTile * nwaves;
  int t = start + wave * kTile + (lane & (kTile - 1));   // this lane's entry
  Rows<DENSE, PAGED> rows;
  if (!DENSE) {
    int row = u;
    if (a.unit_row) {
      row = a.unit_row[u];
      row = row >= 0 && row < a.pool_rows ? row : 0;
    }
    rows.idx = a.set_idx + (size_t)row * a.set_cap;
    rows.set_last = max(a.set_cap, 1) - 1;
  }
  const bool any = DENSE || (a.set_cap > 0 && (!a.unit_row || a.pool_rows > 0));
  int raw0 = any ? rows.entry(t) : -1, raw1 = any ? rows.entry(t + step) : -1,
      raw2 = any ? rows.entry(t + 2 * step) : -1;
  // a dense stream's first tile loads before the lengths are known: its positions
  // are the cache's own, and those behind the length are masked below
  rows.hkv = hkv;
  rows.g = g;
  rows.num_pages = a.kv.num_pages;
  rows.shift = a.sc.block_shift;
  rows.base = (b * hkv + g) * a.kv.capacity;
  // (a table without entries is not read)
  rows.table = PAGED && a.kv.max_pages > 0 ? a.kv.table + (int64_t)b * a.kv.max_pages : a.kv.seq_lens;
  rows.last_page = max(a.kv.max_pages, 1) - 1;
  Query<D, QP> query;
  const int head = WIDE ? col : col & 7;
  const size_t q_at = ((size_t)b * hq + g * G + (head < G ? head : 0)) * D + grp * (D / 4);
  query.load(a.q, q_at, wave);
  Tile<D> T;
  if (DENSE && a.kv.max_seq_len > 0) {
    const int p = min(t, a.kv.max_seq_len - 1);
    load_tile<D>(T, a, rows.row(rows.page(p), p), lane);
  }
  const int nb = kv_seq_len(a.kv, b);
  // the pages of a set's first entries before the lengths are known, as positions
  // of the tail come last
  int g0 = DENSE ? 0 : rows.page(raw0);
  if (!DENSE && unit_excluded(a, u)) return;
  rows.sp = unit_span<DENSE>(a, u, b, nb);
  const int L = rows.sp.L;
  if (L == 0 && split == 0) {  // empty set: y = 0, lse = -inf
    for (int e = threadIdx.x; e < G * D; e += blockDim.x)
      write_final(a, (size_t)b * hq + g * G + e / D, D, e % D, -INFINITY, 0.f, 0.f);
    return;
  }
  if (start >= L) return;
  const int end = min(L, start + a.chunk);
  rows.nb = nb;

  WaveState<D> st;
  st.m = -INFINITY;
  st.l = 0.f;
  st.ve = 0;
  st.r = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) st.o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (QP > 1) {
    query.stage(a.q, q_at, wave, nwaves, lane, s_q);
    lds_barrier();
  }
  const int ntiles = (end - start + kTile - 1) / kTile;
  // (no page of an empty sequence is looked up: its table may be empty too)
  const int iters = nb > 0 && wave < ntiles ? (ntiles - wave + nwaves - 1) / nwaves : 0;
  if (iters > 0) {
    int p1 = rows.pos(raw1, t + step, end);
    if (DENSE) {
      T.ok &= (uint32_t)__builtin_amdgcn_ballot_w64(t < end);
    } else {
      const int p0 = rows.pos(raw0, t, end);
      if (PAGED && __builtin_amdgcn_ballot_w64(p0 >= 0 && p0 != raw0)) g0 = rows.page(p0);
      load_tile<D>(T, a, rows.row(g0, p0), lane);
    }
    int g1 = rows.page(p1);
    for (int i = 0; i < iters; ++i) {
      const uint32_t ok = T.ok;
      const uint32_t vs = (ok >> (lane & (kTile - 1))) & 1u ? __float_as_uint(T.vs) & 0x7FFFFFFFu : 0u;
      if (__builtin_amdgcn_ballot_w64(max((int)(vs >> 23), 1) > st.ve)) {   // a larger V scale than any before
        const int ve = max((int)(wave_umax(vs) >> 23), 1);
        const int re = min(334 - ve, 253);
        // (the ratio of both r may be no fp32 number)
        const int by = st.ve > 0 ? re - (int)(__float_as_uint(st.r) >> 23) : 0;
        st.ve = ve;
        st.r = __uint_as_float((uint32_t)re << 23);
#pragma unroll
        for (int blk = 0; blk < D / 16; ++blk)
#pragma unroll
          for (int i = 0; i < 4; ++i) st.o[blk][i] = __builtin_amdgcn_ldexpf(st.o[blk][i], by);
      }
      __builtin_amdgcn_wave_barrier();
      stage_tile<D>(T, a.scale_log2, st.r, s_k, s_v, s_sc, lane);
      __builtin_amdgcn_wave_barrier();
      load_tile<D>(T, a, rows.row(g1, p1), lane);
      p1 = rows.pos(raw2, t + 2 * step, end);
      g1 = rows.page(p1);
      raw2 = any ? rows.entry(t + 3 * step) : -1;
      t += step;
      consume_tile<D, QP, WIDE>(ok, st, query, s_q, s_k, s_v, s_sc, lane);
    }
  }

  st.l = sum_over_groups(st.l);
  if (grp == 0) {
    sm_m[wave][col] = st.m;
    sm_l[wave][col] = st.l;
  }
  const float unscale = st.r > 0.f ? 1.f / st.r : 0.f;
  __builtin_amdgcn_wave_barrier();
  float* wo = (float*)own + col * (D + 4) + 4 * grp;
#pragma unroll
  for (int blk = 0; blk < D / 16; ++blk) {
    f32x4_t v = st.o[blk] * unscale;
    if (!WIDE)   // parts 8 columns apart
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = add_rotated<0x128>(v[i]);
    if (col < G) *(f32x4_t*)(wo + 16 * blk) = v;
  }
  __syncthreads();
  // four dims a thread and step, the waves' rows read four at a time
  const int nsp = (L + a.chunk - 1) / a.chunk;
  for (int e = threadIdx.x; e < G * (D / 4); e += blockDim.x) {
    const int h = e / (D / 4), dim = 4 * (e - h * (D / 4));
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < kMaxWaves; ++w) M = fmaxf(M, sm_m[min(w, nwaves - 1)][h]);
    f32x4_t num = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
    for (int w0 = 0; w0 < nwaves; w0 += 4)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int w = min(w0 + i, nwaves - 1);
        const float f = w0 + i < nwaves && M != -INFINITY ? __builtin_amdgcn_exp2f(sm_m[w][h] - M) : 0.f;
        num += f * *(const f32x4_t*)(dyn + (size_t)w * wbytes + (h * (D + 4) + dim) * 4);
        den += f * sm_l[w][h];
      }
    const size_t bh = (size_t)b * hq + g * G + h;
    if (nsp == 1) {
      const f32x4_t y = den == 0.f ? f32x4_t{0.f, 0.f, 0.f, 0.f} : num / den;
      *(f32x4_a4_t*)(a.out + bh * D + dim) = y;
      if (a.lse && dim == 0) a.lse[bh] = den == 0.f ? -INFINITY : (M + log2f(den)) * kLn2;
    } else {
      const size_t pidx = bh * a.nsplit + split;
      *(f32x4_a4_t*)(a.part_o + pidx * D + dim) = num;
      if (dim == 0) {
        a.part_ml[pidx * 2] = M;
        a.part_ml[pidx * 2 + 1] = den;
      }
    }
  }
}

// Splits of a unit and rows of a split, a multiple of the tile.  Times in us of
// replayed graphs, d 128 with 4 heads a kv head where nothing else is said.
// Up to 256 units: one workgroup of eight waves a CU (64 units of ragged 16384 rows
// 35.2, two of four waves 44.5), two where that fills the CUs better (96 units of
// ragged 16384 rows in two 54.8, in five 51.3; 72 of 1600 in three 12.7, in seven
// 12.4), but no more splits than is worth their joining, each 0.05 (one unit of
// 32768 rows in 256 20.5, in 64 13.0, of 131072 24.6, in 128 19.6), so that their
// number grows with the root of the rows.  No split of few rows, which saves the
// merge launch (8 units of 600 rows 8.1 whole, 9.0 in four; of 1000 10.4 and 9.2;
// 96 units of 1600 rows 14.0 whole, 13.8 in five; 120 14.2 and 15.3), no split below
// kMinSplit rows, and of more than 128 units only long ones (136 of 12000 rows 76.2
// whole, 70.6 in three, of ragged 16384 92.0 and 78.4; 160 of 4096 29.7 and 32.9).
// More units than CUs: whole, as the workgroups of a CU share it (512 of 16384 rows
// 318, in two 325), but long rows of a few more units than CUs, which wait for the
// CUs that take two (264 of 4096 rows 55.5 whole, 53.8 in four; 320 of 16384 251
// and 207; 384 of 16384 255 and 247).
// The CUs are those of a whole chip, a number and no question to the device, since
// workspaces are sized by it where there is none; on a part of a chip the splits are
// as right, but not the fastest.
constexpr long long kCus = 256;
constexpr int kWholeFew = 850, kWholeMany = 1536, kFewUnits = 64;
constexpr int kMinSplit = 128;
constexpr int kLongRows = 4000;

long long splits_of(long long units, long long rows) {
  if (units > kCus) return units <= 320 && rows >= kLongRows ? 4 : 1;
  if (rows <= (units > kFewUnits ? kWholeMany : kWholeFew)) return 1;
  if (units > kCus / 2 && rows < 2 * kLongRows) return 1;
  long long k = kCus / units;
  if (units > kFewUnits && 2 * kCus / units > 2 * k) k = 2 * kCus / units;
  const long long join = std::max(32LL, (long long)std::sqrt(rows / 16.0));
  return std::max(1LL, std::min({k, join, rows / kMinSplit}));
}

void split_geometry(long long units, int rows_cap, int* chunk, int* nsplit) {
  const long long rows = std::max(rows_cap, 1);
  const long long k = splits_of(std::max(1LL, units), rows);
  const long long c = ((rows + k - 1) / k + kTile - 1) / kTile * kTile;
  *chunk = (int)c;
  *nsplit = (int)((rows + c - 1) / c);
}

// Waves of a workgroup, one for each tile at most: eight where it has a CU to
// itself (256 units of 600 rows 11.0, with four 11.5, with two 14.2) and for long
// streams (64 ragged sequences of up to 16384 rows, 8 kv heads, in length order 238
// us, with four 252, of equal lengths 317 and 315), else four (512 of 600 rows 18.6,
// with eight 19.9).  Short streams of many heads take waves for joining the heads'
// rows too (64 units of 16 heads and 7 rows 5.4 with four waves, 8.4 with one; 512
// of 4 heads and 64 rows 6.0 with their two, 6.4 with four).
int waves_for(long long groups, int chunk, int outputs) {
  const int most = groups <= kCus || chunk > 8192 ? kMaxWaves : 4;
  return std::min(most, std::max(chunk / kTile, std::min(4, outputs / 512)));
}

template <int D, bool DENSE, bool PAGED, int QP, bool WIDE>
hipError_t launch_typed(QuantArgs& a, hipStream_t stream) {
  const int units = a.kv.batch * a.kv.hkv, G = a.kv.hq / a.kv.hkv;
  const int waves = waves_for((long long)units * a.nsplit, a.chunk, G * D);
  // long whole streams on more units than CUs, which take another as they end
  // (64 ragged sequences of 8k to 16k, 8 kv heads: 246 us in index order, 238; of
  // equal lengths 313 and 317)
  a.by_length = DENSE && a.nsplit == 1 && units > kCus && a.chunk > 8192 && a.kv.batch > 1 && a.kv.batch <= 1024;
  const size_t dyn = (size_t)waves * wave_bytes(D, G) + query_bytes(D, QP);
  if (dyn > 49152) {
    const hipError_t e = hipFuncSetAttribute((const void*)quant_attn_split<D, DENSE, PAGED, QP, WIDE>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize,
                                             kMaxWaves * wave_bytes(D, 16) + query_bytes(D, QP));
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((quant_attn_split<D, DENSE, PAGED, QP, WIDE>), dim3((unsigned)units * a.nsplit),
                     dim3(64 * waves), dyn, stream, a);
  if (a.nsplit > 1)
    hipLaunchKernelGGL((attn_merge<D, DENSE>), dim3(a.kv.batch * a.kv.hq), dim3(256), 0, stream,
                       (const AttnArgs&)a);
  return hipGetLastError();
}

template <int D, bool DENSE, bool PAGED>
hipError_t launch_query(QuantArgs& a, int dtype, hipStream_t stream) {
  if (a.kv.hq / a.kv.hkv > 8)
    return dtype == 1 ? launch_typed<D, DENSE, PAGED, 1, true>(a, stream)
                      : launch_typed<D, DENSE, PAGED, 3, true>(a, stream);
  return dtype == 1 ? launch_typed<D, DENSE, PAGED, 1, false>(a, stream)
                    : launch_typed<D, DENSE, PAGED, 3, false>(a, stream);
}

template <int D, bool DENSE>
hipError_t launch_layout(QuantArgs& a, int dtype, hipStream_t stream) {
  return a.kv.paged ? launch_query<D, DENSE, true>(a, dtype, stream)
                    : launch_query<D, DENSE, false>(a, dtype, stream);
}

}  // namespace

long long quant_attn_groups(int batch, int hkv, int rows_cap) {
  int chunk, nsplit;
  split_geometry((long long)batch * hkv, rows_cap, &chunk, &nsplit);
  return (long long)batch * hkv * nsplit;
}

size_t quant_attn_call_bytes(int batch, int hq, int hkv, int d, int rows_cap) {
  int chunk, nsplit;
  split_geometry((long long)batch * hkv, rows_cap, &chunk, &nsplit);
  return attn_layout(batch, hq, d, nsplit).total;
}

// A call of fewer sequences may split its units more: up to 64 units have at most
// 256 splits in all, up to 256 units 512, up to 320 four each, all others one, so
// that many partials of hq / hkv heads hold every smaller call.
size_t quant_attn_workspace_bytes(int batch, int hq, int hkv, int d, int rows_cap) {
  const long long units = (long long)batch * hkv;
  const long long most = units <= kFewUnits ? kCus : units <= kCus ? 2 * kCus : 4 * std::min(units, 320LL);
  const long long groups = std::max(units, most);
  const long long per = units > 0 ? (groups + units - 1) / units : 0;
  return std::max(attn_layout(batch, hq, d, (int)per).total,
                  quant_attn_call_bytes(batch, hq, hkv, d, rows_cap));
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
  split_geometry((long long)s.kv.batch * s.kv.hkv, dense ? s.kv.max_seq_len : s.set_cap, &a.chunk,
                 &a.nsplit);
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
