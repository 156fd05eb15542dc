// Selection of whole blocks by their key bounds.  With q+ = max(q, 0) and
// q- = min(q, 0),
//   sum_d max(q kmin, q kmax) = q+ . kmax + q- . kmin,
// an upper bound of q . k over the keys that the bounds were made of (for an 8-bit
// cache those given to the store, which rounds them to 4 bits): a product of length
// 2d, on MFMA for bf16 and in vector fp32 for fp32 bounds.  What bounds it is
// reading the bounds (4d bytes a block in bf16) once: 512 rows of 4096 blocks at d
// 128 (1.07 GB) 181 us, 5.9 TB/s, where a kernel that only loads them in the same
// order takes 150.  The scoring without its arithmetic takes the same time; the pick
// costs a row of 8192 blocks 7.5 us in a launch of its own.
//
// Scores become order-preserving keys (0, below every number's key, for NaN and
// for blocks whose page lies outside the pool).  The key of the last chosen block
// comes from histograms of narrowing intervals, then one pass in block order
// writes the chosen blocks (which settles ties) and the set.  Two forms:
//   select_blocks   one workgroup per (batch, kv head) scores its blocks into LDS
//                   and picks: one launch;
//   score_blocks    spreads the rows' scores over the chip, keys in the
//   + pick_blocks   workspace, and one workgroup a row picks: two launches.
#include <algorithm>

#include "prhs_internal.h"

namespace prhs {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512;        // scoring workgroups, and select_blocks
constexpr int kWaves = kThreads / 64;
constexpr int kPickThreads = 1024;
constexpr int kBins = 2048;
constexpr int kKeys = 8;             // most keys a thread of the pick holds at a time
constexpr int kRankMax = 64;         // candidates for the last key that one wave ranks
constexpr int kListMax = 4096;       // chosen blocks kept in LDS
constexpr int kLdsKeys = 14336;      // most keys a workgroup holds in LDS (56 KB)

struct BlockArgs : BlockSelectLaunch {
  uint32_t* keys;   // [units][nbmax], candidate i of a unit at [i]
  int nbmax;        // blocks of the longest row, a multiple of kKeys
  int lds_list;     // chosen blocks in LDS
  int chunk;        // score_blocks: candidates of a workgroup
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

// ---- scores -------------------------------------------------------------------

// Slot of 16-byte chunk c of row r in a wave's LDS tile of 16 rows of CH chunks.
template <int CH>
__device__ __forceinline__ int tile_slot(int r, int c) {
  return r * CH + (c ^ (r & (CH - 1)));
}

// Scores of a wave over tiles of kRows candidates: load() issues a tile's loads
// (whole rows, 16 bytes a lane), consume() writes its keys to LDS.
template <typename T, int D, bool PAGED>
struct Scorer;

// bf16: 16 blocks a tile in the columns of v_mfma_f32_16x16x32_bf16, the group's
// heads in its rows.  A tile's rows reach operand order through LDS, as loads in
// operand order would read 64-byte pieces; q+ and q- are read from LDS too, which
// leaves registers for two workgroups a CU.
template <int D, bool PAGED>
struct Scorer<__bf16, D, PAGED> {
  static constexpr int kRows = 16, CH = D / 8, RPI = 64 / CH, KL = D / 32;
  static constexpr int kLdsWave = 16 * D * 2;          // bytes of a wave's tile
  static constexpr int kLdsQuery = 2 * KL * 64 * 16;   // operands of q+, then q-
  int G;
  struct Tile {
    u32x4_t hi[KL], lo[KL];
    int id;   // of block lane mod 16
  };

  __device__ __forceinline__ void init(const BlockArgs& a, int b, int g, unsigned char* lds, int lane) {
    typedef uint32_t u32x4_a2_t __attribute__((ext_vector_type(4), aligned(2)));
    G = a.kv.hq / a.kv.hkv;
    const int wave = threadIdx.x >> 6, head = lane & 15, grp = lane >> 4;
    if (wave < KL) {   // product kk = wave: dims 32 kk + 8 grp .. +7 of head
      const __bf16* q = (const __bf16*)a.q + ((size_t)b * a.kv.hq + (size_t)g * G + (head < G ? head : 0)) * D;
      const u32x4_t v = *(const u32x4_a2_t*)(q + 32 * wave + 8 * grp);
      u32x4_t p, n;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // halves whose sign bit is set are negative
        const uint32_t s = ((v[i] >> 15) & 0x10001u) * 0xFFFFu;
        p[i] = head < G ? v[i] & ~s : 0u;
        n[i] = head < G ? v[i] & s : 0u;
      }
      ((u32x4_t*)lds)[wave * 64 + lane] = p;
      ((u32x4_t*)lds)[(KL + wave) * 64 + lane] = n;
    }
    __syncthreads();
  }

  // id: of block lane mod 16 of the tile, row0: of its first one where the
  // blocks follow each other
  __device__ __forceinline__ void load(Tile& t, const BlockArgs& a, int id, int row0, int last,
                                       int lane) const {
    t.id = id;
#pragma unroll
    for (int j = 0; j < KL; ++j) {
      const int r = j * RPI + lane / CH;
      const int row = PAGED ? max(__shfl(id, r), 0) : min(row0 + r, last);
      const int64_t at = (int64_t)row * D + (lane % CH) * 8;
      t.hi[j] = stream_load16((const __bf16*)a.k_max + at);
      t.lo[j] = stream_load16((const __bf16*)a.k_min + at);
    }
  }

  // LDS operations of one wave complete in order; the wave barriers keep the
  // compiler from moving them across each other.
  __device__ __forceinline__ f32x4_t product(const u32x4_t (&x)[KL], const u32x4_t* q, u32x4_t* tile,
                                             int lane) const {
    const int col = lane & 15, grp = lane >> 4;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < KL; ++j) tile[tile_slot<CH>(j * RPI + lane / CH, lane % CH)] = x[j];
    __builtin_amdgcn_wave_barrier();
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kk = 0; kk < KL; ++kk)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          __builtin_bit_cast(bf16x8_t, q[kk * 64 + lane]),
          __builtin_bit_cast(bf16x8_t, tile[tile_slot<CH>(col, 4 * kk + grp)]), acc, 0, 0, 0);
    return acc;
  }

  __device__ __forceinline__ void consume(const Tile& t, int i0, int end, const unsigned char* q,
                                          u32x4_t* tile, int lane, uint32_t* keys) const {
    const int col = lane & 15, grp = lane >> 4;
    const f32x4_t x = product(t.hi, (const u32x4_t*)q, tile, lane);
    const f32x4_t y = product(t.lo, (const u32x4_t*)q + KL * 64, tile, lane);
    // block col, heads 4 grp + e: the largest key, and the largest of all for NaN
    uint32_t key = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v = x[e] + y[e];
      const uint32_t k = v == v ? score_key(v) : 0xFFFFFFFFu;
      key = max(key, 4 * grp + e < G ? k : 0u);
    }
    const auto h = __builtin_amdgcn_permlane32_swap(key, key, false, false);
    key = max(h[0], h[1]);
    const auto l = __builtin_amdgcn_permlane16_swap(key, key, false, false);
    key = max(l[0], l[1]);
    key = t.id < 0 || key == 0xFFFFFFFFu ? 0u : key;
    if (grp == 0 && i0 + col < end) keys[i0 + col] = key;
  }
};

// fp32: D/4 lanes a block, each with four dims of its bounds and of q+ and q-
// (from LDS), summed over the lanes for each head.
template <int D, bool PAGED>
struct Scorer<float, D, PAGED> {
  static constexpr int CH = D / 4, RPI = 64 / CH, U = 4, kRows = U * RPI;
  static constexpr int kLdsWave = 0;
  static constexpr int kLdsQuery = 2 * 16 * D * 4;
  int G;
  struct Tile {
    float4 hi[U], lo[U];
    int id;   // of row lane mod kRows
  };

  __device__ __forceinline__ void init(const BlockArgs& a, int b, int g, unsigned char* lds, int lane) {
    float* s_q = (float*)lds;
    G = a.kv.hq / a.kv.hkv;
    const float* q = (const float*)a.q + ((size_t)b * a.kv.hq + (size_t)g * G) * D;
    for (int e = threadIdx.x; e < G * D; e += kThreads) {
      const float x = q[e];
      s_q[e] = x > 0.f ? x : (x == x ? 0.f : x);
      s_q[16 * D + e] = x < 0.f ? x : 0.f;
    }
    __syncthreads();
  }

  __device__ __forceinline__ void load(Tile& t, const BlockArgs& a, int id, int row0, int last,
                                       int lane) const {
    t.id = id;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int r = j * RPI + lane / CH;
      const int row = PAGED ? max(__shfl(id, r), 0) : min(row0 + r, last);
      const int64_t at = (int64_t)row * D + (lane % CH) * 4;
      t.hi[j] = stream_load_f32x4((const float*)a.k_max + at);
      t.lo[j] = stream_load_f32x4((const float*)a.k_min + at);
    }
  }

  __device__ __forceinline__ void consume(const Tile& t, int i0, int end, const unsigned char* lds,
                                          u32x4_t*, int lane, uint32_t* keys) const {
    const float* s_q = (const float*)lds;
    float best[U];
    bool nan[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      best[j] = -INFINITY;
      nan[j] = false;
    }
    for (int h = 0; h < G; ++h) {
      const float4 p = *(const float4*)(s_q + h * D + (lane % CH) * 4);
      const float4 n = *(const float4*)(s_q + (16 + h) * D + (lane % CH) * 4);
#pragma unroll
      for (int j = 0; j < U; ++j) {
        float s = p.x * t.hi[j].x;
        s = fmaf(p.y, t.hi[j].y, s);
        s = fmaf(p.z, t.hi[j].z, s);
        s = fmaf(p.w, t.hi[j].w, s);
        s = fmaf(n.x, t.lo[j].x, s);
        s = fmaf(n.y, t.lo[j].y, s);
        s = fmaf(n.z, t.lo[j].z, s);
        s = group_sum<CH>(fmaf(n.w, t.lo[j].w, s));
        nan[j] = nan[j] || !(s == s);
        best[j] = fmaxf(best[j], s);
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int r = j * RPI + lane / CH, i = i0 + r;
      const int id = __shfl(t.id, r);
      if (lane % CH == 0 && i < end) keys[i] = id >= 0 && !nan[j] ? score_key(best[j]) : 0u;
    }
  }
};

// Keys of candidates [begin, end) of unit (b, g), by the workgroup's waves, to
// keys[begin ..] in LDS.  A wave's block-table entries are read two tiles ahead
// and its bounds one; every load is issued unconditionally (past the end the
// last entry, for a lost page block 0), as one behind a branch would make the
// compiler wait for all of them.
template <typename T, int D, bool PAGED>
__device__ __forceinline__ void score_range(const BlockArgs& a, const MiddleBlocks& m, int b, int g,
                                            int begin, int end, unsigned char* lds, uint32_t* keys) {
  typedef Scorer<T, D, PAGED> S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u32x4_t* tile = (u32x4_t*)(lds + S::kLdsQuery + wave * S::kLdsWave);
  S s;
  s.init(a, b, g, lds, lane);
  constexpr int step = S::kRows * kWaves;
  const int32_t* table = a.kv.table + (PAGED ? (int64_t)b * a.kv.max_pages + m.first : 0);
  const int base = (b * a.kv.hkv + g) * (a.kv.capacity >> a.block_shift) + m.first;
  auto entry = [&](int i0) {   // of candidate i0 + lane mod kRows
    return PAGED ? table[min(i0 + lane % S::kRows, end - 1)] : 0;
  };
  auto id_of = [&](int e) {
    if (!PAGED) return 0;
    return e < 0 || e >= a.kv.num_pages ? -1 : e * a.kv.hkv + g;
  };
  int i0 = begin + wave * S::kRows;
  if (i0 >= end) return;
  const int iters = (end - i0 + step - 1) / step;
  typename S::Tile A, B;
  s.load(A, a, id_of(entry(i0)), base + i0, base + end - 1, lane);
  int next = entry(i0 + step);
  int i = 0;
  for (; i + 2 < iters; i += 2) {
    s.load(B, a, id_of(next), base + i0 + step, base + end - 1, lane);
    next = entry(i0 + 2 * step);
    s.consume(A, i0, end, lds, tile, lane, keys);
    s.load(A, a, id_of(next), base + i0 + 2 * step, base + end - 1, lane);
    next = entry(i0 + 3 * step);
    s.consume(B, i0 + step, end, lds, tile, lane, keys);
    i0 += 2 * step;
  }
  if (i + 1 < iters) {
    s.load(B, a, id_of(next), base + i0 + step, base + end - 1, lane);
    s.consume(A, i0, end, lds, tile, lane, keys);
    s.consume(B, i0 + step, end, lds, tile, lane, keys);
  } else {
    s.consume(A, i0, end, lds, tile, lane, keys);
  }
}

// ---- the pick -----------------------------------------------------------------

struct PickLds {
  uint32_t hist[kBins];
  uint32_t scan[kPickThreads / 64 + 1];
  uint32_t red[2 * (kPickThreads / 64)];
  uint32_t cand[kRankMax];
  uint32_t ncand, bin, left, count, key;
};

// A row's n keys over a workgroup of NT threads, R consecutive ones a thread (so
// that a scan over the threads is in block order), in chunks of NT R: one chunk
// stays in registers, more are read again by each pass.
// `keys` holds a multiple of R.
template <int NT, int R>
struct RowKeys {
  typedef uint32_t vec_t __attribute__((ext_vector_type(R), aligned(4)));
  uint32_t x[R];
  const uint32_t* keys;
  int room, n;

  __device__ __forceinline__ void load(int c) {
    const int i = (c * NT + (int)threadIdx.x) * R;
    const vec_t v = *(const vec_t*)(keys + (i < room ? i : 0));
#pragma unroll
    for (int j = 0; j < R; ++j) x[j] = v[j];
  }
  __device__ __forceinline__ void init(const uint32_t* from, int padded) {
    keys = from;
    room = padded;
    load(0);
  }
  __device__ __forceinline__ int chunks() const { return (n + NT * R - 1) / (NT * R); }
  // f(key) for each of this thread's keys
  template <typename F>
  __device__ __forceinline__ void each(F f) {
    const int last = chunks();
    for (int c = 0; c < last; ++c) {
      if (last > 1) load(c);
      const int i = (c * NT + (int)threadIdx.x) * R;
#pragma unroll
      for (int j = 0; j < R; ++j)
        if (i + j < n) f(x[j]);
    }
  }
};

// The k-th largest of a row's keys (1 <= k <= n) and, in *left, how many of the
// chosen k equal it.  Interval [lo, lo + 2^width) of keys, narrowed by histograms
// of its 2048 parts, the first one from the smallest to the largest key; at most
// 64 keys left are ranked by one wave.  A row of 8192 keys takes one histogram as
// a rule, where digits of the keys' own bits take two: scores differ little in
// their exponents.
template <int NT, typename Keys>
__device__ uint32_t kth_key(Keys& keys, uint32_t k, PickLds& s, uint32_t* left) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t inv = 0u, mx = 0u;   // of the smallest key its complement
  keys.each([&](uint32_t x) {
    inv = max(inv, ~x);
    mx = max(mx, x);
  });
  inv = wave_umax(inv);
  mx = wave_umax(mx);
  if (lane == 0) {
    s.red[2 * wave] = inv;
    s.red[2 * wave + 1] = mx;
  }
  for (int i = tid; i < kBins; i += NT) s.hist[i] = 0u;
  if (tid == 0) s.ncand = 0u;
  lds_barrier();
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    inv = max(inv, s.red[2 * w]);
    mx = max(mx, s.red[2 * w + 1]);
  }
  uint32_t lo = ~inv;
  int width = mx > lo ? 32 - __clz((int)(mx - lo)) : 0;
  for (;;) {
    const int shift = max(0, width - 11);
    const uint32_t span = width >= 32 ? 0xFFFFFFFFu : (1u << width) - 1u;   // largest key - lo
    keys.each([&](uint32_t x) {
      if (x >= lo && x - lo <= span) atomicAdd(&s.hist[(x - lo) >> shift], 1u);
    });
    lds_barrier();
    // the bin of the k-th largest, from the top
    constexpr int BPT = kBins / NT;
    uint32_t local = 0u, total;
#pragma unroll
    for (int i = 0; i < BPT; ++i) local += s.hist[kBins - 1 - (tid * BPT + i)];
    uint32_t cum = block_exclusive_scan<NT, uint32_t, false>(local, s.scan, &total);
#pragma unroll
    for (int i = 0; i < BPT; ++i) {
      const int bin = kBins - 1 - (tid * BPT + i);
      const uint32_t c = s.hist[bin];
      if (cum < k && cum + c >= k) {
        s.bin = (uint32_t)bin;
        s.left = k - cum;
        s.count = c;
      }
      cum += c;
    }
    lds_barrier();
    k = s.left;
    lo += s.bin << shift;
    width = shift;
    const uint32_t count = s.count;
    if (shift == 0) {
      *left = k;
      return lo;
    }
    if (count <= (uint32_t)kRankMax) {
      const uint32_t top = (1u << shift) - 1u;
      keys.each([&](uint32_t x) {
        if (x >= lo && x - lo <= top) s.cand[atomicAdd(&s.ncand, 1u)] = x;
      });
      lds_barrier();
      // every wave ranks them itself, so that no barrier follows
      const uint32_t x = (uint32_t)lane < count ? s.cand[lane] : 0u;
      uint32_t above = 0u, same = 0u;
      for (uint32_t c = 0; c < count; ++c) {
        const uint32_t y = (uint32_t)__builtin_amdgcn_readlane((int)x, (int)c);
        above += y > x;
        same += y == x;
      }
      const uint64_t hit = __builtin_amdgcn_ballot_w64((uint32_t)lane < count && above < k && above + same >= k);
      const int at = __ffsll((unsigned long long)hit) - 1;
      *left = k - (uint32_t)__builtin_amdgcn_readlane((int)above, at);
      return (uint32_t)__builtin_amdgcn_readlane((int)x, at);
    }
    for (int i = tid; i < kBins; i += NT) s.hist[i] = 0u;
    lds_barrier();
  }
}

// Writes the chosen blocks of unit u, whose `kb` are some of its candidates, to
// blk_idx and, where they fit, to LDS; first_in, last_in: whether the first and
// the last candidate are among them.
template <int NT, int R>
__device__ __forceinline__ void place_blocks(const BlockArgs& a, const MiddleBlocks& m, int u, int kb,
                                             RowKeys<NT, R>& keys, int32_t* list, PickLds& s,
                                             bool* first_in, bool* last_in) {
  const int tid = threadIdx.x, n = keys.n;
  int32_t* blk = a.blk_idx + (size_t)u * a.blk_cap;
  const uint32_t key0 = keys.keys[0], key1 = keys.keys[n - 1];
  uint32_t left;
  const uint32_t T = kth_key<NT>(keys, (uint32_t)kb, s, &left);
  const int chunks = keys.chunks();
  uint32_t gt_all = 0u, eq_all = 0u;   // keys above and equal to T in earlier chunks
  for (int c = 0; c < chunks; ++c) {
    if (chunks > 1) keys.load(c);
    const int i = (c * NT + tid) * R;
    uint32_t is_gt = 0u, is_eq = 0u;   // bit j: key j of this thread
#pragma unroll
    for (int j = 0; j < R; ++j) {
      is_gt |= (i + j < n && keys.x[j] > T ? 1u : 0u) << j;
      is_eq |= (i + j < n && keys.x[j] == T ? 1u : 0u) << j;
    }
    // of a chunk at most 2^13 keys, so that both counts scan in one word
    const uint32_t mine = (uint32_t)__popc(is_gt) << 16 | (uint32_t)__popc(is_eq);
    uint32_t total;
    const uint32_t before = block_exclusive_scan<NT>(mine, s.scan, &total);
    uint32_t g = gt_all + (before >> 16), e = eq_all + (before & 0xFFFFu);
    for (uint32_t rest = is_gt | is_eq; rest; rest &= rest - 1u) {
      const int j = __ffs((int)rest) - 1;
      const bool above = (is_gt >> j) & 1u;
      if (above || e < left) {   // of equal keys the first `left`
        const uint32_t at = g + min(e, left);
        blk[at] = m.first + i + j;
        if (list) list[at] = m.first + i + j;
      }
      g += above ? 1u : 0u;
      e += above ? 0u : 1u;
    }
    gt_all += total >> 16;
    eq_all += total & 0xFFFFu;
  }
  *first_in = key0 >= T;
  *last_in = key1 > T || (key1 == T && eq_all == left);
}

// Writes unit u's chosen blocks and set from its candidates' keys.
template <int NT, int R>
__device__ __forceinline__ void pick_row(const BlockArgs& a, const MiddleBlocks& m, int u, int kb,
                                         RowKeys<NT, R>& keys, int32_t* s_list, PickLds& s) {
  const int tid = threadIdx.x, n = m.count, bs = 1 << a.block_shift;
  int32_t* blk = a.blk_idx + (size_t)u * a.blk_cap;
  int32_t* set = a.set_idx + (size_t)u * a.set_cap;
  bool first_in = kb > 0, last_in = kb > 0;
  int32_t* list = kb <= a.lds_list ? s_list : nullptr;
  if (kb > 0 && kb < n) {
    keys.n = n;
    place_blocks<NT, R>(a, m, u, kb, keys, list, s, &first_in, &last_in);
  } else if (kb > 0) {   // every candidate
    for (int i = tid; i < n; i += NT) {
      blk[i] = m.first + i;
      if (list) list[i] = m.first + i;
    }
  }
  // the list is read back, from LDS or from memory
  if (list) lds_barrier();
  else __syncthreads();
  // the chosen blocks' positions within the middle range [sink_end, win_start)
  const int lo_cut = first_in ? m.sink_end - (m.first << a.block_shift) : 0;
  const int hi_cut = last_in ? ((m.first + n) << a.block_shift) - m.win_start : 0;
  const int mid = kb * bs - lo_cut - hi_cut;
  for (int i = tid; i < m.sink_end; i += NT) set[i] = i;
  for (int i = tid; i < mid; i += NT) {
    const int x = i + lo_cut, j = x >> a.block_shift;
    set[m.sink_end + i] = ((list ? list[j] : blk[j]) << a.block_shift) + (x & (bs - 1));
  }
  const int nw = m.n0 - m.win_start;
  for (int i = tid; i < nw; i += NT) set[m.sink_end + mid + i] = m.win_start + i;
  if (tid == 0) {
    a.blk_len[u] = kb;
    a.set_len[u] = m.sink_end + mid + nw;
  }
}

template <typename T, int D, bool PAGED>
__global__ __launch_bounds__(kThreads) void score_blocks(BlockArgs a, int chunks) {
  // LDS: the chunk's keys, then the scorer's
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
  const int u = blockIdx.x / chunks, b = u / a.kv.hkv, g = u - b * a.kv.hkv;
  const MiddleBlocks m = middle_blocks(a, b);
  const int begin = (blockIdx.x - u * chunks) * a.chunk, end = min(m.count, begin + a.chunk);
  if (begin >= end) return;
  const int kb = chosen_blocks(a, m.n0, m.count);
  if (kb == 0 || kb == m.count) return;   // no score decides
  uint32_t* s_keys = (uint32_t*)dyn;
  score_range<T, D, PAGED>(a, m, b, g, begin, end, dyn + (size_t)a.chunk * 4, s_keys - begin);
  lds_barrier();
  uint32_t* keys = a.keys + (size_t)u * a.nbmax;
  for (int i = begin + threadIdx.x; i < end; i += kThreads) keys[i] = s_keys[i - begin];
}

template <int R>
__global__ __launch_bounds__(kPickThreads) void pick_blocks(BlockArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];   // the chosen blocks
  __shared__ PickLds s;
  const int u = blockIdx.x, b = u / a.kv.hkv;
  RowKeys<kPickThreads, R> keys;   // loaded before the row's length is known
  keys.init(a.keys + (size_t)u * a.nbmax, a.nbmax);
  const MiddleBlocks m = middle_blocks(a, b);
  pick_row(a, m, u, chosen_blocks(a, m.n0, m.count), keys, (int32_t*)dyn, s);
}

// LDS: keys, chosen blocks, then the scorer's.
template <typename T, int D, bool PAGED, int R>
__global__ __launch_bounds__(kThreads) void select_blocks(BlockArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char dyn[];
  __shared__ PickLds s;
  const int u = blockIdx.x, b = u / a.kv.hkv, g = u - b * a.kv.hkv;
  const MiddleBlocks m = middle_blocks(a, b);
  const int kb = chosen_blocks(a, m.n0, m.count);
  uint32_t* s_keys = (uint32_t*)dyn;
  int32_t* s_list = (int32_t*)(s_keys + a.nbmax);
  if (kb > 0 && kb < m.count) {
    score_range<T, D, PAGED>(a, m, b, g, 0, m.count, (unsigned char*)(s_list + a.lds_list), s_keys);
    lds_barrier();
  }
  RowKeys<kThreads, R> keys;
  keys.init(s_keys, a.nbmax);
  pick_row(a, m, u, kb, keys, s_list, s);
}

// One launch (us, then in two; d 128 in bf16): where a workgroup reads a row in
// about what the second launch costs (8 rows of 192 KB 9.7 and 10.4, of 256 KB 11.5
// and 10.5), up to as much longer rows as there are more of them (96 of 256 KB 13.0
// and 13.8, of 512 KB 19.5 and 18.0; 160 of 512 KB 22.5 and 23.9, of 1 MB 39.5 and
// 38.9), and where the rows fill the CUs (192 of 1 MB 42.6 and 43.1, 256 of 2 MB 101
// and 107, 512 of 512 KB 52.8 and 59.1, ragged 42.1 and 48.1; 256 of 8 MB 404 and
// 384), but for long rows of a few more units than CUs, which wait for the CUs that
// take two (264 of 512 KB 37.5 and 35.1, 320 of 2 MB 143 and 125; 384 of 512 KB 43.2
// and 46.1, of 2 MB 150 and 148).  The CUs are those of a whole chip; on a part of one
// both forms are as right, but not the faster one is always taken.
bool one_launch(long long units, long long row_bytes) {
  constexpr long long KB = 1024;
  if (row_bytes <= 192 * KB) return true;
  if (units < 192) return row_bytes < 4 * KB * units;
  return row_bytes <= (units > 256 && units < 384 ? 384 * KB : 4096 * KB);
}

// The launches of `units` rows of nbmax keys and row_bytes of bounds: select_blocks,
// or score_blocks in `chunks` workgroups a row, about four workgroups a CU, each of
// whole rounds of its waves' tiles (`round` candidates).
struct Shape {
  bool one;
  int chunk, chunks;
};
Shape launch_shape(long long units, int nbmax, long long row_bytes, int round) {
  if (nbmax <= kLdsKeys && one_launch(units, row_bytes)) return {true, nbmax, 1};
  const long long want = std::max(1LL, 1024 / std::max(1LL, units));
  const long long rounds = ((nbmax + want - 1) / want + round - 1) / round;
  const int chunk = (int)std::min((long long)(kLdsKeys / round), std::max(1LL, rounds)) * round;
  return {false, chunk, (nbmax + chunk - 1) / chunk};
}

// Dynamic LDS beyond the default: always the same bound, so that calls of other
// sizes on other threads do not lower it.
constexpr int kMaxDynamicLds = 144 * 1024;
template <typename F>
hipError_t allow_lds(F* f, size_t bytes) {
  if (bytes <= 49152) return hipSuccess;
  return hipFuncSetAttribute((const void*)f, hipFuncAttributeMaxDynamicSharedMemorySize, kMaxDynamicLds);
}

template <int N>
struct Const {
  static constexpr int value = N;
};

// f(keys a thread): the fewest that hold a row of n keys at once (rows of 3125
// blocks with four 11.65 us, with eight 12.2; of 125 with one 11.0, with two 11.2),
// else the most.
template <typename F>
hipError_t with_keys(int n, int threads, F f) {
  if (n <= threads) return f(Const<1>());
  if (n <= 2 * threads) return f(Const<2>());
  return n <= 4 * threads ? f(Const<4>()) : f(Const<kKeys>());
}

template <typename T, int D, bool PAGED>
hipError_t launch_typed(BlockArgs& a, hipStream_t stream) {
  typedef Scorer<T, D, PAGED> S;
  const int units = a.kv.batch * a.kv.hkv;
  constexpr size_t kScoreLds = S::kLdsQuery + (size_t)kWaves * S::kLdsWave;
  a.lds_list = (std::min(std::min(a.blk_cap, a.nbmax), kListMax) + 3) & ~3;
  const Shape shape = launch_shape(units, a.nbmax, (long long)a.nbmax * 2 * D * sizeof(T), S::kRows * kWaves);
  if (shape.one) {
    const size_t lds = ((size_t)a.nbmax + a.lds_list) * 4 + kScoreLds;
    auto launch = [&](auto r) {
      constexpr int R = decltype(r)::value;
      const hipError_t e = allow_lds(select_blocks<T, D, PAGED, R>, lds);
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL((select_blocks<T, D, PAGED, R>), dim3(units), dim3(kThreads), lds, stream, a);
      return hipGetLastError();
    };
    return with_keys(a.nbmax, kThreads, launch);
  }
  a.chunk = shape.chunk;
  const size_t lds = kScoreLds + (size_t)a.chunk * 4;
  const hipError_t e = allow_lds(score_blocks<T, D, PAGED>, lds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((score_blocks<T, D, PAGED>), dim3((unsigned)(units * shape.chunks)), dim3(kThreads),
                     lds, stream, a, shape.chunks);
  return with_keys(a.nbmax, kPickThreads, [&](auto r) {
    hipLaunchKernelGGL(pick_blocks<decltype(r)::value>, dim3(units), dim3(kPickThreads),
                       (size_t)a.lds_list * 4, stream, a);
    return hipGetLastError();
  });
}

template <typename T, int D>
hipError_t launch_layout(BlockArgs& a, hipStream_t stream) {
  return a.kv.paged ? launch_typed<T, D, true>(a, stream) : launch_typed<T, D, false>(a, stream);
}

}  // namespace

// Keys of a row of the workspace.
static int row_keys(int max_seq_len, int block_shift) {
  return (((max_seq_len + (1 << block_shift) - 1) >> block_shift) + kKeys - 1) / kKeys * kKeys;
}

size_t block_select_workspace_bytes(long long units, int max_seq_len, int block_shift) {
  return (size_t)units * row_keys(max_seq_len, block_shift) * sizeof(uint32_t);
}

// (tiles hold as many rows paged as contiguous)
LaunchSize block_select_size(const KvView& kv, int dtype, int block_shift) {
  const int round = kWaves * (dtype == 1 ? Scorer<__bf16, 128, false>::kRows
                              : kv.d == 128 ? Scorer<float, 128, false>::kRows
                                            : Scorer<float, 64, false>::kRows);
  const int nbmax = row_keys(kv.max_seq_len, block_shift);
  const long long units = (long long)kv.batch * kv.hkv;
  const Shape s = launch_shape(units, nbmax, (long long)nbmax * 2 * kv.d * (dtype == 1 ? 2 : 4), round);
  if (s.one) return {units, kThreads};
  // score_blocks; pick_blocks has twice the threads in a workgroup a row
  return {std::max(units * s.chunks, 2 * units), kThreads};
}

hipError_t launch_block_select(const BlockSelectLaunch& s, hipStream_t stream) {
  BlockArgs a;
  (BlockSelectLaunch&)a = s;
  a.keys = (uint32_t*)s.ws;
  a.nbmax = row_keys(s.kv.max_seq_len, s.block_shift);
  if (s.dtype == 1)
    return s.kv.d == 128 ? launch_layout<__bf16, 128>(a, stream) : launch_layout<__bf16, 64>(a, stream);
  return s.kv.d == 128 ? launch_layout<float, 128>(a, stream) : launch_layout<float, 64>(a, stream);
}

}  // namespace prhs
