// Rows of fp32 or bf16 that may start at any multiple of their element's size, as fp32 values in registers, and
// sums over a workgroup in a fixed order: shared by the kernels of the norm and of the expert sorting.
#ifndef DYNB_ROW_ACCESS_H
#define DYNB_ROW_ACCESS_H

#include <hip/hip_runtime.h>

namespace dynb {

typedef __bf16 bf16;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A granule is 8 neighbouring elements of a row.  Vector accesses need no alignment beyond the element's on this
// target: the memory pipeline splits what crosses a line.
constexpr int GRANULE = 8;
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1), may_alias));
typedef uint32_t u32_any __attribute__((aligned(1), may_alias));
typedef uint16_t u16_any __attribute__((aligned(1), may_alias));

// Calls of more bytes than the caches keep until the next one reads them pass them by.  Sorting and combination of 2048
// columns in bf16, 8 choices: 1024 tokens (38 and 42 MB) 30.2 us either way, 2048 tokens 46 us past the caches and 55 through
// them, 16384 tokens 245 and 279; gradients of 4 choices: 1024 tokens (38 and 21 MB) 15.8 and 13.8, 2048 27.0 and 30.2; the norm
// of 16384 x 8192 to fp8 165 and 185.  With a product behind the call that reads what it wrote: norm of 4096 x 2048 with residual
// (67 MB) 51.4 us past the caches and 48.4 through them, 4096 x 4096 57 and 56, 16384 x 4096 (536 MB) 159 and 172; 4096 tokens of
// 2048 columns and 4 choices sorted (83 MB) 56 and 50, 16384 of 8 (603 MB) 275 and 299.
inline bool past_caches(double bytes) { return bytes > 64e6; }

// PAST: the access passes the caches by (data that is used once and is more than they hold).
template <bool PAST = false> __device__ inline u32x4 load16(const void* p) {
  if (PAST) return __builtin_nontemporal_load((const u32x4_any*)p);
  return *(const u32x4_any*)p;
}
template <bool PAST = false> __device__ inline void store16(void* p, const u32x4& v) {
  if (PAST) __builtin_nontemporal_store((u32x4_any)v, (u32x4_any*)p);
  else *(u32x4_any*)p = v;
}

__device__ inline uint32_t two_bf16(float a, float b) {   // round to nearest even
  return (uint32_t)__builtin_bit_cast(unsigned short, (bf16)a) |
         ((uint32_t)__builtin_bit_cast(unsigned short, (bf16)b) << 16);
}

// The first n of 8 elements of a row (n >= 8: all, n <= 0: none) as they are loaded, 4 (bf16) or 8 (fp32) registers: what
// waits for its use between load and arithmetic.  What is left of a row's last granule is 4, 2 and 1 elements, as the
// bits of n say: three accesses at most, which stay apart until unpack() puts them in their places, so that nothing waits
// for them before.  Nothing past the n-th element is touched; zeros stand for the others.
template <typename T> struct Raw;
template <> struct Raw<bf16> { u32x4 a; };
template <> struct Raw<float> { u32x4 a, b; };
template <bool PAST = false> __device__ inline Raw<bf16> load_raw(const bf16* p, int n) {
  Raw<bf16> r = {{0, 0, 0, 0}};
  if (n >= GRANULE) {
    r.a = load16<PAST>(p);
  } else if (n > 0) {
    if (n & 4) {
      const u32x2 four = *(const u32x2_any*)p;
      r.a[0] = four[0];
      r.a[1] = four[1];
    }
    if (n & 2) r.a[2] = *(const u32_any*)(p + (n & 4));
    if (n & 1) r.a[3] = *(const u16_any*)(p + n - 1);
  }
  return r;
}
template <bool PAST = false> __device__ inline Raw<float> load_raw(const float* p, int n) {
  Raw<float> r = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  if (n >= GRANULE) {
    r.a = load16<PAST>(p);
    r.b = load16<PAST>(p + 4);
  } else if (n > 0) {
    if (n & 4) r.a = load16(p);
    if (n & 2) {
      const u32x2 two = *(const u32x2_any*)(p + (n & 4));
      r.b[0] = two[0];
      r.b[1] = two[1];
    }
    if (n & 1) r.b[2] = *(const uint32_t*)(p + n - 1);
  }
  return r;
}
__device__ inline void unpack(Raw<bf16> r, int n, float (&f)[GRANULE]) {
  if (n > 0 && n < GRANULE) {
    const uint32_t first = n & 2 ? r.a[2] : r.a[3], second = n & 2 ? r.a[3] : 0u;   // behind the four
    r.a = n & 4 ? u32x4{r.a[0], r.a[1], first, second} : u32x4{first, second, 0, 0};
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(r.a[e] << 16);
    f[2 * e + 1] = __uint_as_float(r.a[e] & 0xffff0000u);
  }
}
__device__ inline void unpack(Raw<float> r, int n, float (&f)[GRANULE]) {
  if (n > 0 && n < GRANULE) {
    const u32x4 rest = {n & 2 ? r.b[0] : r.b[2], r.b[1], n & 2 ? r.b[2] : 0u, 0};   // behind the four
    r.b = n & 4 ? rest : u32x4{0, 0, 0, 0};
    r.a = n & 4 ? r.a : rest;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = __uint_as_float(r.a[e]);
    f[4 + e] = __uint_as_float(r.b[e]);
  }
}
template <bool PAST = false> __device__ inline void store_packed(bf16* p, int n, const u32x4& a) {   // (8 elements as bits)
  if (n >= GRANULE) {
    store16<PAST>(p, a);
  } else if (n > 0) {
    if (n & 4) *(u32x2_any*)p = u32x2{a[0], a[1]};
    const uint32_t low = n & 4 ? a[2] : a[0], high = n & 4 ? a[3] : a[1];
    if (n & 2) *(u32_any*)(p + (n & 4)) = low;
    if (n & 1) *(u16_any*)(p + n - 1) = (uint16_t)(n & 2 ? high : low);
  }
}
template <bool PAST = false> __device__ inline void store_part(bf16* p, int n, const float (&f)[GRANULE]) {
  u32x4 a;
#pragma unroll
  for (int e = 0; e < 4; ++e) a[e] = two_bf16(f[2 * e], f[2 * e + 1]);
  store_packed<PAST>(p, n, a);
}
template <bool PAST = false> __device__ inline void store_part(float* p, int n, const float (&f)[GRANULE]) {
  u32x4 a, b;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    a[e] = __float_as_uint(f[e]);
    b[e] = __float_as_uint(f[4 + e]);
  }
  if (n >= GRANULE) {
    store16<PAST>(p, a);
    store16<PAST>(p + 4, b);
  } else if (n > 0) {
    if (n & 4) store16(p, a);
    const u32x4 rest = n & 4 ? b : a;
    if (n & 2) *(u32x2_any*)(p + (n & 4)) = u32x2{rest[0], rest[1]};
    if (n & 1) *(uint32_t*)(p + n - 1) = n & 2 ? rest[2] : rest[0];
  }
}
template <typename T> __device__ inline void load_part(const T* p, int n, float (&f)[GRANULE]) { unpack(load_raw(p, n), n, f); }

// Exchanges between lanes that need no LDS: within 2, 4, 8 and 16 lanes (after the step every lane of the group has
// the same value, so that a mirrored partner is as good as the xor-ed one).
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;
template <int CTRL> __device__ inline uint32_t from_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL> __device__ inline float from_lane(float v) { return __uint_as_float(from_lane<CTRL>(__float_as_uint(v))); }
__device__ inline float of_lane(float v, int lane) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}
__device__ inline float wave_sum(float v) {
  v += from_lane<DPP_XOR1>(v);
  v += from_lane<DPP_XOR2>(v);
  v += from_lane<DPP_HALF_MIRROR>(v);
  v += from_lane<DPP_MIRROR>(v);
  return (of_lane(v, 0) + of_lane(v, 16)) + (of_lane(v, 32) + of_lane(v, 48));
}
// Over L neighbouring lanes (8, 16, 32 or 64), the same in all of them.
template <int L> __device__ inline float lanes_sum(float v) {
  if (L == 64) return wave_sum(v);
  v += from_lane<DPP_XOR1>(v);
  v += from_lane<DPP_XOR2>(v);
  v += from_lane<DPP_HALF_MIRROR>(v);
  if (L > 8) v += from_lane<DPP_MIRROR>(v);
  if (L > 16) v += __shfl_xor(v, 16);
  return v;
}
// Over groups of 2, 4, ... 64 neighbouring lanes (`lanes` the same in the whole wave).
__device__ inline uint32_t group_max(uint32_t v, int lanes) {
  if (lanes > 1) v = max(v, from_lane<DPP_XOR1>(v));
  if (lanes > 2) v = max(v, from_lane<DPP_XOR2>(v));
  if (lanes > 4) v = max(v, from_lane<DPP_HALF_MIRROR>(v));
  if (lanes > 8) v = max(v, from_lane<DPP_MIRROR>(v));
  if (lanes > 16) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  if (lanes > 32) v = max(v, (uint32_t)__shfl_xor((int)v, 32));
  return v;
}
__device__ inline uint32_t wave_max(uint32_t v) {
  v = group_max(v, 16);
  uint32_t m = 0;
#pragma unroll
  for (int l = 0; l < 64; l += 16) m = max(m, (uint32_t)__builtin_amdgcn_readlane((int)v, l));
  return m;
}

// Over a workgroup of `waves` <= 16 waves; every thread gets the result.  `red` is workgroup-shared and must not be that of the
// reduction before (the barrier of one is what protects the other).
constexpr int MOST_WAVES = 16;
__device__ inline float block_sum(float v, int waves, float* red) {
  v = wave_sum(v);
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  const int w = threadIdx.x & (MOST_WAVES - 1);
  v = w < waves ? red[w] : 0.f;
  v += from_lane<DPP_XOR1>(v);
  v += from_lane<DPP_XOR2>(v);
  v += from_lane<DPP_HALF_MIRROR>(v);
  return of_lane(v + from_lane<DPP_MIRROR>(v), 0);
}
__device__ inline uint32_t block_max(uint32_t v, int waves, uint32_t* red) {
  v = wave_max(v);
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  const int w = threadIdx.x & (MOST_WAVES - 1);
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)group_max(w < waves ? red[w] : 0u, 16));
}

// Values of 8 bits with a scale: the largest magnitude's bits (a NaN's are above an infinity's) give scale and factor.
// Below 2^-100 a block counts as zeros: the factor could overflow.  (Of a 16th of it: the hardware's reciprocal of values beyond
// 2^126 is 0.)
struct Scale {
  float scale, inv;
};
__device__ inline Scale scale_of(uint32_t amax_bits, float top) {
  if (amax_bits >= 0x7f800000u) return {__uint_as_float(0x7fc00000u), 0.f};
  if (amax_bits < (27u << 23)) return {0.f, 0.f};
  const float a = __uint_as_float(amax_bits);
  return {a * (1.f / top), top * 0x1p-4f * __builtin_amdgcn_rcpf(a * 0x1p-4f)};
}

}  // namespace dynb

#endif
