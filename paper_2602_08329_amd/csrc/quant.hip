// The 8-bit KV cache's store, and the key bounds of blocks.
//
// quant_store: a team of waves per (kv head, block of tokens, K or V).  With s_old
// the block's scale and amax the largest finite |x| of its new tokens,
//   s_new = 2^e, e = max(-100, min {e : amax <= 448 * 2^e}),
//   s = s_new if the block holds no earlier token, else max(s_old, s_new),
// new elements become rne_e4m3(x / s), and where s > s_old earlier ones
// rne_e4m3(s_old * x8 / s).  A power of two as scale makes every division here
// exact, so the only rounding of an element is the one to 4 significant bits
// (relative 2^-4; below 2^-6 s absolute 2^-10 s), and a block whose scale grows
// while it fills ends as the block stored at once does, but for elements that
// fall below 2^-6 s.  Since e4m3 is itself a floating type, a scale between two
// powers of two would not make it more exact.
//
// A team reads its new elements once, 8 per thread and step, holds them in
// registers while their maximum is taken, and writes their bytes.  Bounds come
// from the same registers.  Moving the bytes bounds both kernels: a 16k prompt of
// 8 heads of d 128 in bf16 (67 MB read, 38 written) is stored in 22.8 us, 4.6 TB/s
// where a large copy reaches 4.9, the bounds of a 32k prompt (67 MB, 2 written)
// take 12.8, 5.4 TB/s; a step of 64 sequences takes 5.0 and 4.9, the time of a
// launch whose loads of lengths, pages and tokens follow each other.
#include "prhs_internal.h"

namespace prhs {
namespace {

constexpr int kThreads = 256;
constexpr int kMinExp = -100;   // exponent of the smallest scale

// Loads of 8 elements; rows of the callers' tensors are aligned to their
// elements only.
typedef uint32_t u32x4_a2_t __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void load8(const __bf16* p, float (&x)[8]) {
  const u32x4_a2_t v = *(const u32x4_a2_t*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(v[i] << 16);
    x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = load_f32x4(p), b = load_f32x4(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// Bits of 2^e for amax given by its bits.
__device__ __forceinline__ uint32_t scale_bits(uint32_t amax) {
  int e = (int)(amax >> 23) - 127 - ((amax & 0x7FFFFFu) <= 0x600000u ? 8 : 7);
  e = max(e, kMinExp);
  return (uint32_t)(e + 127) << 23;
}

// x / s of 8 elements as e4m3 bytes; inv = 1 / s where s is a power of two,
// else 0.
__device__ __forceinline__ u32x2_t to_e4m3(const float (&x)[8], float s, float inv) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = inv != 0.f ? x[i] * inv : x[i] / s;
    if (!(fabsf(x[i]) < INFINITY)) y[i] = __builtin_nanf("");
  }
  u32x2_t w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], v, true);
  }
  return w;
}

__device__ __forceinline__ void from_e4m3(u32x2_t w, float s, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    x[4 * i] = a[0] * s;
    x[4 * i + 1] = a[1] * s;
    x[4 * i + 2] = b[0] * s;
    x[4 * i + 3] = b[1] * s;
  }
}

// The block a workgroup works on: block `j` of sequence b, whose positions
// [at, lo) are earlier ones and [lo, hi) new ones; row: its first row id.
struct Block {
  int b, g, at, lo, hi, t0;   // t0: index of position lo among the new tokens
  int row;
};

// The i-th touched block of unit u; false if there is none or its page lies
// outside the pool.
__device__ __forceinline__ bool find_block(const KvView& kv, const NewTokens& tok, int shift, int u,
                                           int i, Block* k) {
  k->b = u / kv.hkv;
  k->g = u - k->b * kv.hkv;
  const int n = kv_seq_len(kv, k->b);
  const int c = new_tokens(tok, k->b, n);
  const int first = n - c;
  const int j = (first >> shift) + i;
  k->at = j << shift;
  if (c == 0 || k->at >= n) return false;
  k->lo = max(first, k->at);
  k->hi = min(n, k->at + (1 << shift));
  k->t0 = k->lo - first;
  if (!kv.paged) {
    k->row = (k->b * kv.hkv + k->g) * kv.capacity + k->at;
    return true;
  }
  const int phys = kv.table[(int64_t)k->b * kv.max_pages + j];
  if (phys < 0 || phys >= kv.num_pages) return false;
  k->row = (phys * kv.hkv + k->g) << shift;
  return true;
}

// Minimum and maximum over the lanes that hold the same dims (lane mod C), in
// every lane.
template <int C>
__device__ __forceinline__ void wave_bounds(float (&mn)[8], float (&mx)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (C == 8) {
      mn[i] = fminf(mn[i], __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(mn[i]), 0x128, 0xF, 0xF, false)));
      mx[i] = fmaxf(mx[i], __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(mx[i]), 0x128, 0xF, 0xF, false)));
    }
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(mn[i]), __float_as_uint(mn[i]), false, false);
    mn[i] = fminf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(mn[i]), __float_as_uint(mn[i]), false, false);
    mn[i] = fminf(__uint_as_float(b[0]), __uint_as_float(b[1]));
    const auto c = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx[i]), __float_as_uint(mx[i]), false, false);
    mx[i] = fmaxf(__uint_as_float(c[0]), __uint_as_float(c[1]));
    const auto d = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx[i]), __float_as_uint(mx[i]), false, false);
    mx[i] = fmaxf(__uint_as_float(d[0]), __uint_as_float(d[1]));
  }
}

// The same over the W waves of a team, whose first C lanes get it; `lds` holds
// 2 D floats for each wave of the workgroup.  All threads of the workgroup call it.
template <int D, int W>
__device__ __forceinline__ void team_bounds(float (&mn)[8], float (&mx)[8], float* lds) {
  constexpr int C = D / 8;
  wave_bounds<C>(mn, mx);
  if (W == 1) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = wave / W * W;
  if (lane < C)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lds[(wave * 2) * D + lane * 8 + i] = mn[i];
      lds[(wave * 2 + 1) * D + lane * 8 + i] = mx[i];
    }
  __syncthreads();
  if (lane < C)
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mn[i] = fminf(mn[i], lds[((first + w) * 2) * D + lane * 8 + i]);
        mx[i] = fmaxf(mx[i], lds[((first + w) * 2 + 1) * D + lane * 8 + i]);
      }
}

__device__ __forceinline__ void store8(__bf16* p, const float (&x)[8]) {
  typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
  bf16x8_t v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
  *(bf16x8_t*)p = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
  *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// A team of W waves per block, kThreads / (64 W) blocks a workgroup; thread t of
// a team holds the elements 8 v .. 8 v + 7 of the block for v = t + 64 W i.  Rows
// that are not new stand in for the nearest one that is, which changes neither the
// maximum nor the bounds and keeps the loads free of branches.
template <typename T, int D, int W, int VPT>
__global__ __launch_bounds__(kThreads) void quant_store(QuantStoreLaunch a, int nblk, int blocks) {
  constexpr int C = D / 8;
  __shared__ uint32_t s_amax[kThreads / 64];
  __shared__ float s_red[W > 1 ? 2 * (kThreads / 64) * D : 1];
  const int team = blockIdx.x * (kThreads / 64 / W) + (threadIdx.x >> 6) / W, tt = threadIdx.x & (64 * W - 1);
  const bool is_k = blockIdx.y == 0;
  const int u = team / nblk;
  Block k;
  const bool on = team < blocks && find_block(a.kv, a.tok, a.block_shift, u, team - u * nblk, &k);
  if (W == 1 && !on) return;
  float x[VPT][8];
  uint32_t amax = 0u;
  int nold = 0, rows = 0;
  uint8_t* dst = nullptr;
  float* scale = nullptr;
  float s_old = 0.f;
  if (on) {
    nold = k.lo - k.at;
    rows = k.hi - k.at;
    const T* src = (const T*)(is_k ? a.k_new : a.v_new) +
                   ((int64_t)(k.b * a.kv.hkv + k.g) * a.tok.cap + k.t0) * D + (tt % C) * 8;
    dst = (uint8_t*)(is_k ? a.kv.k : a.kv.v) + (int64_t)k.row * D + (tt % C) * 8;
    scale = (is_k ? a.k_scale : a.v_scale) + (k.row >> a.block_shift);
    s_old = *scale;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int r = (tt + i * 64 * W) / C;
      load8(src + (int64_t)(min(max(r, nold), rows - 1) - nold) * D, x[i]);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t m = __float_as_uint(x[i][e]) & 0x7FFFFFFFu;
        amax = max(amax, m < 0x7F800000u ? m : 0u);
      }
  }
  amax = wave_umax(amax);
  if (W > 1) {
    const int wave = threadIdx.x >> 6, first = wave / W * W;
    if ((threadIdx.x & 63) == 0) s_amax[wave] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) amax = max(amax, s_amax[first + w]);
  }
  const float s_new = __uint_as_float(scale_bits(amax));
  const bool grows = nold > 0 && !(s_old >= s_new);
  const float s = nold > 0 && !grows ? s_old : s_new;
  const uint32_t sb = __float_as_uint(s), se = sb >> 23;
  // 1 / s where s and it are normal powers of two
  const float inv = (sb & 0x7FFFFFu) == 0u && se >= 1u && se <= 253u ? __uint_as_float((254u - se) << 23) : 0.f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int r = (tt + i * 64 * W) / C;
    u32x2_t* p = (u32x2_t*)(dst + (int64_t)r * D);
    if (r >= nold && r < rows) {
      *p = to_e4m3(x[i], s, inv);
    } else if (r < nold && grows) {
      float y[8];
      from_e4m3(*p, s_old, y);
      *p = to_e4m3(y, s, inv);
    }
  }
  if (on && tt == 0) *scale = s;
  if (!is_k || !a.k_min) return;

  float mn[8], mx[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    mn[e] = INFINITY;
    mx[e] = -INFINITY;
  }
  if (on)
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        mn[e] = fminf(mn[e], x[i][e]);
        mx[e] = fmaxf(mx[e], x[i][e]);
      }
  team_bounds<D, W>(mn, mx, s_red);
  if (on && tt < C) {
    const int64_t at = (int64_t)(k.row >> a.block_shift) * D + tt * 8;
    if (nold > 0) {
      float lo[8], hi[8];
      load8((const T*)a.k_min + at, lo);
      load8((const T*)a.k_max + at, hi);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        mn[e] = fminf(mn[e], lo[e]);
        mx[e] = fmaxf(mx[e], hi[e]);
      }
    }
    store8((T*)a.k_min + at, mn);
    store8((T*)a.k_max + at, mx);
  }
}

// Bounds of whole blocks from a bf16 or fp32 cache, teams as above.
template <typename T, int D, int W, int VPT>
__global__ __launch_bounds__(kThreads) void block_bounds(BlockBoundsLaunch a, int nblk, int blocks) {
  constexpr int C = D / 8;
  __shared__ float s_red[W > 1 ? 2 * (kThreads / 64) * D : 1];
  const int team = blockIdx.x * (kThreads / 64 / W) + (threadIdx.x >> 6) / W, tt = threadIdx.x & (64 * W - 1);
  const int u = team / nblk;
  Block k;
  const bool on = team < blocks && find_block(a.kv, a.tok, a.block_shift, u, team - u * nblk, &k);
  if (W == 1 && !on) return;
  float mn[8], mx[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    mn[e] = INFINITY;
    mx[e] = -INFINITY;
  }
  if (on) {
    const int rows = k.hi - k.at;
    const T* src = (const T*)a.kv.k + (int64_t)k.row * D + (tt % C) * 8;
    float x[VPT][8];
#pragma unroll
    for (int i = 0; i < VPT; ++i) load8(src + (int64_t)min((tt + i * 64 * W) / C, rows - 1) * D, x[i]);
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        mn[e] = fminf(mn[e], x[i][e]);
        mx[e] = fmaxf(mx[e], x[i][e]);
      }
  }
  team_bounds<D, W>(mn, mx, s_red);
  if (on && tt < C) {
    const int64_t at = (int64_t)(k.row >> a.block_shift) * D + tt * 8;
    store8((T*)a.k_min + at, mn);
    store8((T*)a.k_max + at, mx);
  }
}

// Most blocks that new tokens touch in one sequence: they begin anywhere in a
// block, and there are no more than the cache holds.
int touched_blocks(const KvView& kv, const NewTokens& tok, int shift) {
  const int c = tok.cap < kv.max_seq_len ? tok.cap : kv.max_seq_len;
  const int bs = 1 << shift;
  const int any = (c + bs - 2) / bs + 1, all = (kv.max_seq_len + bs - 1) / bs;
  return any < all ? any : all;
}

// Waves of a team for blocks of vec vectors of 64 x 8 elements: as few as hold them
// at `most` vectors a thread, at most four.  Replayed graphs, 8 heads of d 128 in
// bf16: the store takes at most 4 (a 16k prompt in blocks of 16 20.8 us, two or four
// waves a block 25.2 and 43.5; in blocks of 64 with four waves 20.9, two 23.6, one
// 28.6), bounds, which hold less a thread, 8 (a 32k prompt in blocks of 64 with two
// waves 13.3 us, four 14.1; in blocks of 16 as the store).
constexpr int kStoreVectors = 4, kBoundsVectors = 8;
constexpr int team_waves(int vec, int most) {
  return vec <= most ? 1 : vec / most < 4 ? vec / most : 4;
}

// Workgroups of `blocks` blocks, one a team.
long long team_groups(long long blocks, int shift, int d, int most) {
  const int per = kThreads / 64 / team_waves((d << shift) / 512, most);
  return (blocks + per - 1) / per;
}

// f(waves, vectors a thread) as compile-time numbers.
template <int N>
struct Const {
  static constexpr int value = N;
};
template <int D, int most, typename F>
void with_team(int shift, F f) {
  auto of_block = [&](auto tokens) {
    constexpr int vec = decltype(tokens)::value * D / 512;
    constexpr int W = team_waves(vec, most);
    f(Const<W>(), Const<vec / W>());
  };
  switch (shift) {
    case 4: of_block(Const<16>()); break;
    case 5: of_block(Const<32>()); break;
    case 6: of_block(Const<64>()); break;
    default: of_block(Const<128>());
  }
}

template <typename T, int D>
hipError_t launch_store_typed(const QuantStoreLaunch& a, int nblk, hipStream_t stream) {
  const int blocks = a.kv.batch * a.kv.hkv * nblk;
  const unsigned groups = (unsigned)team_groups(blocks, a.block_shift, D, kStoreVectors);
  with_team<D, kStoreVectors>(a.block_shift, [&](auto w, auto v) {
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    hipLaunchKernelGGL((quant_store<T, D, W, V>), dim3(groups, 2), dim3(kThreads), 0, stream, a, nblk,
                       blocks);
  });
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_bounds_typed(const BlockBoundsLaunch& a, int nblk, hipStream_t stream) {
  const int blocks = a.kv.batch * a.kv.hkv * nblk;
  const unsigned groups = (unsigned)team_groups(blocks, a.block_shift, D, kBoundsVectors);
  with_team<D, kBoundsVectors>(a.block_shift, [&](auto w, auto v) {
    constexpr int W = decltype(w)::value, V = decltype(v)::value;
    hipLaunchKernelGGL((block_bounds<T, D, W, V>), dim3(groups), dim3(kThreads), 0, stream, a, nblk,
                       blocks);
  });
  return hipGetLastError();
}

}  // namespace

LaunchSize quant_store_size(const KvView& kv, const NewTokens& tok, int block_shift) {
  const long long blocks = (long long)kv.batch * kv.hkv * touched_blocks(kv, tok, block_shift);
  return {2 * team_groups(blocks, block_shift, kv.d, kStoreVectors), kThreads};
}

LaunchSize block_bounds_size(const KvView& kv, const NewTokens& tok, int block_shift) {
  const long long blocks = (long long)kv.batch * kv.hkv * touched_blocks(kv, tok, block_shift);
  return {team_groups(blocks, block_shift, kv.d, kBoundsVectors), kThreads};
}

hipError_t launch_quant_store(const QuantStoreLaunch& a, hipStream_t stream) {
  const int nblk = touched_blocks(a.kv, a.tok, a.block_shift);
  if (nblk == 0) return hipSuccess;
  if (a.dtype == 1)
    return a.kv.d == 128 ? launch_store_typed<__bf16, 128>(a, nblk, stream)
                         : launch_store_typed<__bf16, 64>(a, nblk, stream);
  return a.kv.d == 128 ? launch_store_typed<float, 128>(a, nblk, stream)
                       : launch_store_typed<float, 64>(a, nblk, stream);
}

hipError_t launch_block_bounds(const BlockBoundsLaunch& a, hipStream_t stream) {
  const int nblk = touched_blocks(a.kv, a.tok, a.block_shift);
  if (nblk == 0) return hipSuccess;
  if (a.dtype == 1)
    return a.kv.d == 128 ? launch_bounds_typed<__bf16, 128>(a, nblk, stream)
                         : launch_bounds_typed<__bf16, 64>(a, nblk, stream);
  return a.kv.d == 128 ? launch_bounds_typed<float, 128>(a, nblk, stream)
                       : launch_bounds_typed<float, 64>(a, nblk, stream);
}

}  // namespace prhs
