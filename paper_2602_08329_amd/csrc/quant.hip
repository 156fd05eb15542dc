// The 8-bit KV cache's store, and the key bounds of blocks.
//
// quant_store: one workgroup per (kv head, block of tokens, K or V).  With s_old
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
// A workgroup reads its new elements once, 8 per thread and step, holds them in
// registers while their maximum is taken, and writes their bytes.  Bounds come
// from the same registers.
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

// Per-dimension minimum and maximum over a workgroup whose thread t holds those
// of dims 8 (t mod D/8) .. +7 over its rows; thread t < D gets dim t's.
template <int D>
__device__ __forceinline__ void reduce_bounds(float (&mn)[8], float (&mx)[8], float* s_red, float* lo,
                                              float* hi) {
  constexpr int C = D / 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = C; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      mn[i] = fminf(mn[i], __shfl_xor(mn[i], o));
      mx[i] = fmaxf(mx[i], __shfl_xor(mx[i], o));
    }
  if (lane < C)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s_red[(wave * 2) * D + lane * 8 + i] = mn[i];
      s_red[(wave * 2 + 1) * D + lane * 8 + i] = mx[i];
    }
  __syncthreads();
  if (threadIdx.x < D) {
    float a = INFINITY, z = -INFINITY;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      a = fminf(a, s_red[(w * 2) * D + threadIdx.x]);
      z = fmaxf(z, s_red[(w * 2 + 1) * D + threadIdx.x]);
    }
    *lo = a;
    *hi = z;
  }
}

template <typename T, int D, int VPT>
__global__ __launch_bounds__(kThreads) void quant_store(QuantStoreLaunch a, int nblk) {
  constexpr int C = D / 8;
  __shared__ uint32_t s_amax[kThreads / 64];
  __shared__ float s_red[2 * (kThreads / 64) * D];
  const int u = blockIdx.x / nblk;
  const bool is_k = blockIdx.y == 0;
  Block k;
  if (!find_block(a.kv, a.tok, a.block_shift, u, blockIdx.x - u * nblk, &k)) return;
  const int nold = k.lo - k.at, rows = k.hi - k.at;
  const T* src = (const T*)(is_k ? a.k_new : a.v_new) +
                 ((int64_t)(k.b * a.kv.hkv + k.g) * a.tok.cap + k.t0) * D;
  uint8_t* dst = (uint8_t*)(is_k ? a.kv.k : a.kv.v) + (int64_t)k.row * D;
  float* scale = (is_k ? a.k_scale : a.v_scale) + (k.row >> a.block_shift);

  float x[VPT][8];
  uint32_t amax = 0u;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int v = threadIdx.x + i * kThreads, r = v / C, c = v % C;
    if (r < nold || r >= rows) continue;
    load8(src + (int64_t)(r - nold) * D + c * 8, x[i]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t m = __float_as_uint(x[i][e]) & 0x7FFFFFFFu;
      amax = max(amax, m < 0x7F800000u ? m : 0u);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o));
  if ((threadIdx.x & 63) == 0) s_amax[threadIdx.x >> 6] = amax;
  const float s_old = *scale;
  __syncthreads();
  amax = max(max(s_amax[0], s_amax[1]), max(s_amax[2], s_amax[3]));
  const float s_new = __uint_as_float(scale_bits(amax));
  const bool grows = nold > 0 && !(s_old >= s_new);
  const float s = nold > 0 && !grows ? s_old : s_new;
  const uint32_t sb = __float_as_uint(s);
  const uint32_t se = sb >> 23;   // a positive power of two of which 2^-e is normal too
  const float inv = (sb & 0x7FFFFFu) == 0u && se >= 1u && se <= 253u ? __uint_as_float((254u - se) << 23) : 0.f;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int v = threadIdx.x + i * kThreads, r = v / C, c = v % C;
    u32x2_t* p = (u32x2_t*)(dst + (int64_t)r * D + c * 8);
    if (r >= nold && r < rows) {
      *p = to_e4m3(x[i], s, inv);
    } else if (r < nold && grows) {
      float y[8];
      from_e4m3(*p, s_old, y);
      *p = to_e4m3(y, s, inv);
    }
  }
  if (threadIdx.x == 0) *scale = s;
  if (!is_k || !a.k_min) return;

  float mn[8], mx[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    mn[e] = INFINITY;
    mx[e] = -INFINITY;
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int r = (threadIdx.x + i * kThreads) / C;
    if (r < nold || r >= rows) continue;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mn[e] = fminf(mn[e], x[i][e]);
      mx[e] = fmaxf(mx[e], x[i][e]);
    }
  }
  float lo, hi;
  reduce_bounds<D>(mn, mx, s_red, &lo, &hi);
  if (threadIdx.x < D) {
    const int64_t at = (int64_t)(k.row >> a.block_shift) * D + threadIdx.x;
    T* pmin = (T*)a.k_min + at;
    T* pmax = (T*)a.k_max + at;
    if (nold > 0) {
      lo = fminf(lo, (float)*pmin);
      hi = fmaxf(hi, (float)*pmax);
    }
    *pmin = (T)lo;
    *pmax = (T)hi;
  }
}

// One workgroup per (kv head, block).
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void block_bounds(BlockBoundsLaunch a, int nblk) {
  constexpr int C = D / 8, RPI = kThreads / C;
  __shared__ float s_red[2 * (kThreads / 64) * D];
  const int u = blockIdx.x / nblk;
  Block k;
  if (!find_block(a.kv, a.tok, a.block_shift, u, blockIdx.x - u * nblk, &k)) return;
  const int rows = k.hi - k.at;
  const T* src = (const T*)a.kv.k + (int64_t)k.row * D + (threadIdx.x % C) * 8;
  float mn[8], mx[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    mn[e] = INFINITY;
    mx[e] = -INFINITY;
  }
  for (int r = threadIdx.x / C; r < rows; r += RPI) {
    float x[8];
    load8(src + (int64_t)r * D, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mn[e] = fminf(mn[e], x[e]);
      mx[e] = fmaxf(mx[e], x[e]);
    }
  }
  float lo, hi;
  reduce_bounds<D>(mn, mx, s_red, &lo, &hi);
  if (threadIdx.x < D) {
    const int64_t at = (int64_t)(k.row >> a.block_shift) * D + threadIdx.x;
    ((T*)a.k_min)[at] = (T)lo;
    ((T*)a.k_max)[at] = (T)hi;
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

template <typename T, int D>
hipError_t launch_store_typed(const QuantStoreLaunch& a, int nblk, hipStream_t stream) {
  const dim3 grid(a.kv.batch * a.kv.hkv * nblk, 2);
  switch ((D << a.block_shift) / (8 * kThreads)) {
    case 0:
    case 1: hipLaunchKernelGGL((quant_store<T, D, 1>), grid, dim3(kThreads), 0, stream, a, nblk); break;
    case 2: hipLaunchKernelGGL((quant_store<T, D, 2>), grid, dim3(kThreads), 0, stream, a, nblk); break;
    case 4: hipLaunchKernelGGL((quant_store<T, D, 4>), grid, dim3(kThreads), 0, stream, a, nblk); break;
    default: hipLaunchKernelGGL((quant_store<T, D, 8>), grid, dim3(kThreads), 0, stream, a, nblk); break;
  }
  return hipGetLastError();
}

}  // namespace

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
  const dim3 grid(a.kv.batch * a.kv.hkv * nblk), block(kThreads);
  if (a.dtype == 1) {
    if (a.kv.d == 128) hipLaunchKernelGGL((block_bounds<__bf16, 128>), grid, block, 0, stream, a, nblk);
    else hipLaunchKernelGGL((block_bounds<__bf16, 64>), grid, block, 0, stream, a, nblk);
  } else {
    if (a.kv.d == 128) hipLaunchKernelGGL((block_bounds<float, 128>), grid, block, 0, stream, a, nblk);
    else hipLaunchKernelGGL((block_bounds<float, 64>), grid, block, 0, stream, a, nblk);
  }
  return hipGetLastError();
}

}  // namespace prhs
