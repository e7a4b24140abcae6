// AdamW over a list of tensors: the weighted average of the workers' gradients, the step, the states in fp32 or in 8 bits
// and the 16-bit copy of the parameters, in one pass over all of them.
//   g = sum_k lambda_k g_k, m += (1 - beta1) (g - m), v += (1 - beta2) (g^2 - v),
//   p -= lr (decay p + (m / c1) / (sqrt(v / c2) + eps)),  all in fp32.
// Memory bounds it: 54.5 M parameters of 16 workers in fp32 with a 16-bit copy 4.9 GB, 869 us (5.6 TB/s); 235 M parameters, one
// bf16 gradient, 8-bit states 3.76 GB, 638 us (5.9 TB/s), their values read back 232 us (6.0 TB/s); 117 M bf16 parameters, a bf16
// gradient, fp32 states 2.58 GB, 428 us (6.0 TB/s).  A wave takes 256
// neighbouring elements, a scale's block, so that the largest magnitude is an exchange inside it; a table on the device
// says which tensor a workgroup works on, so that one launch does all of up to 256 tensors.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>
#include <vector>

#include "dynb_internal.h"
#include "row_access.h"

namespace dynb {
namespace {

constexpr int BLOCK = DYNB_STATE_BLOCK;   // elements that share a scale: a wave, 4 neighbouring ones per lane
// Blocks of a wave.  8-bit states: two (117 M parameters, a step and its values read back, fp32 gradient 462 us, with one 477,
// bf16 gradient 434 and 437).  fp32 states: one (54.5 M parameters of 16 workers 860 us, with two 890; 532 thousand of 16
// workers 10.8 and 11.5).
constexpr int blocks_of_wave(bool eight) { return eight ? 2 : 1; }
constexpr int chunk_of(bool eight) { return 4 * blocks_of_wave(eight) * BLOCK; }   // elements of a workgroup

struct Tensor {
  void *param, *copy, *s1, *s2;
  float *c1, *c2;
  int64_t n;
  float decay;
  int32_t ordinal;
};
struct Chunk {
  int32_t tensor, at;                     // the at-th chunk of the tensor
};
constexpr int POINTERS = 256;             // tensors of a launch
struct Pointers {
  const void* p[POINTERS];
};
struct Pointers2 {
  void *a[POINTERS / 2], *b[POINTERS / 2];
};
struct Workers {                          // those with rows
  int n;
  float w[DYNB_MAX_WORKERS];
  int32_t index[DYNB_MAX_WORKERS];        // (whole words: read by scalar instructions)
};
struct Rule {
  float lr, eps, beta1, beta2, omb1, omb2, inv_c1, inv_c2;
  uint32_t seed;
};

// ---- 4 neighbouring elements, of which the first n exist ------------------------------------------------------
// Every byte is used once a step: accesses pass the caches by (54.5 M parameters of 16 workers, two
// blocks to a wave: 890 us, 935 through them; nothing behind the step read the copy).
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4), may_alias));
typedef uint32_t u32_half __attribute__((aligned(2), may_alias));
#define GLOBAL __attribute__((address_space(1)))

// As they are stored: what waits for its use between load and arithmetic.
template <typename T> struct Raw4;
template <> struct Raw4<float> { f32x4_any v; };
template <> struct Raw4<bf16> { u32x2 v; };
__device__ inline Raw4<float> load4(const GLOBAL float* p, int n) {
  if (n >= 4) return {__builtin_nontemporal_load((const GLOBAL f32x4_any*)p)};
  Raw4<float> r = {{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) r.v[e] = p[e];
  return r;
}
__device__ inline Raw4<bf16> load4(const GLOBAL bf16* p, int n) {
  if (n >= 4) return {(u32x2)__builtin_nontemporal_load((const GLOBAL u32x2_any*)p)};
  const GLOBAL uint16_t* h = (const GLOBAL uint16_t*)p;
  Raw4<bf16> r = {{0, 0}};               // (written where they belong, so that nothing waits for them here)
  if (n == 1) r.v[0] = *h;
  if (n >= 2) r.v[0] = *(const GLOBAL u32_half*)h;
  if (n == 3) r.v[1] = h[2];
  return r;
}
__device__ inline void unpack(const Raw4<float>& r, float (&f)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f[e] = r.v[e];
}
__device__ inline void unpack(const Raw4<bf16>& r, float (&f)[4]) {
  f[0] = __uint_as_float(r.v[0] << 16);
  f[1] = __uint_as_float(r.v[0] & 0xffff0000u);
  f[2] = __uint_as_float(r.v[1] << 16);
  f[3] = __uint_as_float(r.v[1] & 0xffff0000u);
}
__device__ inline void store4(GLOBAL float* p, int n, const float (&f)[4]) {
  if (n >= 4) {
    const f32x4_any q = {f[0], f[1], f[2], f[3]};
    __builtin_nontemporal_store(q, (GLOBAL f32x4_any*)p);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) p[e] = f[e];
  }
}
__device__ inline void store4(GLOBAL bf16* p, int n, const float (&f)[4]) {
  if (n >= 4) {
    const u32x2_any q = {two_bf16(f[0], f[1]), two_bf16(f[2], f[3])};
    __builtin_nontemporal_store(q, (GLOBAL u32x2_any*)p);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) p[e] = (bf16)f[e];
  }
}
struct Codes {
  uint32_t low, third;                   // the third of three comes apart
};
__device__ inline Codes load_codes(const GLOBAL uint8_t* p, int n) {
  Codes c = {0, 0};
  if (n >= 4) c.low = __builtin_nontemporal_load((const GLOBAL u32_any*)p);
  if (n == 1) c.low = *p;
  if (n == 2 || n == 3) c.low = *(const GLOBAL u16_any*)p;
  if (n == 3) c.third = p[2];
  return c;
}
__device__ inline void store_codes(GLOBAL uint8_t* p, int n, uint32_t q) {
  if (n >= 4) {
    __builtin_nontemporal_store(q, (GLOBAL u32_any*)p);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < n) p[e] = (uint8_t)(q >> (8 * e));
  }
}

// ---- 8-bit states ---------------------------------------------------------------------------------------------
// A magnitude t in [0, top] is coded by the bits of the float t + 2^-15: 16 octaves of equal steps, linear below the
// lowest, and encoding and decoding are an addition and a shift.  MAG magnitude bits: 7 (m, with a sign) or 8 (sqrt v).
constexpr uint32_t LOW_BITS = 112u << 23;           // bits of 2^-15
template <int MAG> struct Code {
  static constexpr int SHIFT = MAG == 7 ? 20 : 19;
  static constexpr float TOP = MAG == 7 ? 1.875f : 1.9375f;
};
// byte `e` of q; low = 2^-15 * scale (a power of two times it, so that the product below rounds once)
template <int MAG> __device__ inline float decode(uint32_t q, int e, float scale, float low) {
  constexpr int SHIFT = Code<MAG>::SHIFT;
  constexpr uint32_t MASK = ((1u << MAG) - 1) << SHIFT;
  const uint32_t bits = (8 * e > SHIFT ? q >> (8 * e - SHIFT) : q << (SHIFT - 8 * e)) & MASK;
  return __builtin_fmaf(__uint_as_float(bits + LOW_BITS), scale, -low);
}
__device__ inline float signed_as(float magnitude, uint32_t q, int e) {       // bit 7 of byte `e`
  return __uint_as_float(__float_as_uint(magnitude) ^ (q << (24 - 8 * e) & 0x80000000u));
}
// u16: 16 random bits, 65536ths of a step.  least: the lowest code that the value may get.  (A factor of 0 gives code 0; of
// a block with an infinity or NaN it does not matter which code: its scale is NaN.)
template <int MAG> __device__ inline uint32_t encode(float magnitude, float inv, uint32_t u16, uint32_t least) {
  const uint32_t bits = __float_as_uint(__builtin_fmaf(magnitude, inv, 0x1p-15f)) - LOW_BITS + (u16 << (Code<MAG>::SHIFT - 16));
  return min(max(bits >> Code<MAG>::SHIFT, least), (1u << MAG) - 1);
}
__device__ inline uint32_t random_bits(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

// The root and the reciprocal are the hardware's (off by a unit in the last place of a term that is small beside the
// parameter): with the correctly rounded ones the 8-bit step is bound by its arithmetic.  The hardware's root takes a v below
// 2^-126 for zero, so where a wave has one, it is taken of 2^64 v.  A v that is zero may stand beside an m that is not (the
// gradient's square is below fp32's range): its root counts as LEAST_ROOT in the division, and such an m is 1 / sqrt(1 - beta2)
// times that at most; its 8-bit code is 0 as well.  (117 M parameters, a bf16 gradient: 8-bit states 317 us,
// fp32 states 554, without any of this 317 and 554.)
constexpr uint32_t LEAST_ROOT = 52u << 23;          // bits of 2^-75 (the smallest v has 2^-74.5)
constexpr int SUBNORMAL = 0x80;                     // of the class test: positive ones

// A wave takes U blocks; all it reads is asked for before anything is used.
template <typename P, typename G, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(const Tensor* tensors, const Chunk* chunks, Pointers grads,
                                                    int first_tensor, int64_t worker_stride, Workers workers,
                                                    Rule rule) {
  constexpr int U = blocks_of_wave(EIGHT), CHUNK = chunk_of(EIGHT);
  const Chunk chunk = chunks[blockIdx.x];
  const Tensor t = tensors[chunk.tensor];
  const GLOBAL G* const grad = (const GLOBAL G*)grads.p[chunk.tensor - first_tensor];
  GLOBAL P* const param = (GLOBAL P*)t.param;
  GLOBAL uint8_t *const codes1 = (GLOBAL uint8_t*)t.s1, *const codes2 = (GLOBAL uint8_t*)t.s2;
  GLOBAL float *const state1 = (GLOBAL float*)t.s1, *const state2 = (GLOBAL float*)t.s2;
  GLOBAL float *const scale1 = (GLOBAL float*)t.c1, *const scale2 = (GLOBAL float*)t.c2;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Raw4<P> p0[U];
  Raw4<float> m0[U], v0[U];
  float p[U][4], m[U][4], v[U][4], g[U][4], c1[U], c2[U];
  Codes q1[U], q2[U];
  int64_t at[U];
  int n[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t begin = (int64_t)chunk.at * CHUNK + (wave * U + u) * BLOCK, left = t.n - begin - 4 * lane;
    at[u] = begin + 4 * lane;
    n[u] = left >= 4 ? 4 : left > 0 ? (int)left : 0;
    p0[u] = load4(param + at[u], n[u]);
    if (EIGHT) {
      c1[u] = begin < t.n ? scale1[begin / BLOCK] : 0.f;
      c2[u] = begin < t.n ? scale2[begin / BLOCK] : 0.f;
      q1[u] = load_codes(codes1 + at[u], n[u]);
      q2[u] = load_codes(codes2 + at[u], n[u]);
    } else {
      m0[u] = load4(state1 + at[u], n[u]);
      v0[u] = load4(state2 + at[u], n[u]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) g[u][e] = 0.f;
  }
  constexpr int KS = 8 / U;               // workers whose gradients are asked for together
  for (int k0 = 0; k0 < workers.n; k0 += KS) {
    Raw4<G> d0[KS][U];
#pragma unroll
    for (int k = 0; k < KS; ++k)
      if (k0 + k < workers.n)
#pragma unroll
        for (int u = 0; u < U; ++u) d0[k][u] = load4(grad + workers.index[k0 + k] * worker_stride + at[u], n[u]);
#pragma unroll
    for (int k = 0; k < KS; ++k)
      if (k0 + k < workers.n)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float d[4];
          unpack(d0[k][u], d);
#pragma unroll
          for (int e = 0; e < 4; ++e) g[u][e] += workers.w[k0 + k] * d[e];
        }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    unpack(p0[u], p[u]);
    if (!EIGHT) {
      unpack(m0[u], m[u]);
      unpack(v0[u], v[u]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t a1 = q1[u].low | q1[u].third << 16, a2 = q2[u].low | q2[u].third << 16;
        const float r = decode<8>(a2, e, c2[u], c2[u] * 0x1p-15f);
        m[u][e] = signed_as(decode<7>(a1, e, c1[u], c1[u] * 0x1p-15f), a1, e);
        v[u][e] = r * r;
      }
    }
    float root[4];
    bool small = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      m[u][e] = rule.beta1 * m[u][e] + rule.omb1 * g[u][e];
      v[u][e] = rule.beta2 * v[u][e] + rule.omb2 * g[u][e] * g[u][e];
      root[e] = __builtin_amdgcn_sqrtf(v[u][e]);
      small |= __builtin_amdgcn_classf(v[u][e], SUBNORMAL);
    }
    if (small)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (__builtin_amdgcn_classf(v[u][e], SUBNORMAL)) root[e] = __builtin_amdgcn_sqrtf(v[u][e] * 0x1p64f) * 0x1p-32f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float r = __uint_as_float(max(__float_as_uint(root[e]), LEAST_ROOT));      // (a NaN's bits are above)
      const float by = __builtin_amdgcn_rcpf(r * rule.inv_c2 + rule.eps);
      // (not p times the rounded 1 - lr decay, which would be off in the same direction on every step)
      p[u][e] = __builtin_fmaf(-rule.lr, __builtin_fmaf(t.decay, p[u][e], m[u][e] * rule.inv_c1 * by), p[u][e]);
    }
    store4(param + at[u], n[u], p[u]);
    if (t.copy) store4((GLOBAL bf16*)t.copy + at[u], n[u], p[u]);
    if (!EIGHT) {
      store4(state1 + at[u], n[u], m[u]);
      store4(state2 + at[u], n[u], v[u]);
      continue;
    }
    uint32_t a1 = 0, a2 = 0;               // (elements that do not exist are zeros)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a1 = max(a1, __float_as_uint(m[u][e]) & 0x7fffffffu);
      a2 = max(a2, __float_as_uint(root[e]));
    }
    const Scale s1 = scale_of(wave_max(a1), Code<7>::TOP), s2 = scale_of(wave_max(a2), Code<8>::TOP);
    uint32_t to1 = 0, to2 = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t r = random_bits((uint32_t)(at[u] + e) * 0x9E3779B1u + t.ordinal * 0x7F4A7C15u + rule.seed);
      const bool some = root[e] > 0.f;
      to1 |= (encode<7>(some ? fabsf(m[u][e]) : 0.f, s1.inv, r >> 16, 0) | (__float_as_uint(m[u][e]) >> 24 & 0x80u)) << (8 * e);
      // (a root below half a step that became 0 beside an m that did not would make a step of m / eps)
      to2 |= encode<8>(root[e], s2.inv, r & 0xffffu, some ? 1 : 0) << (8 * e);
    }
    store_codes(codes1 + at[u], n[u], to1);
    store_codes(codes2 + at[u], n[u], to2);
    if (lane == 0 && n[u] > 0) {
      scale1[at[u] / BLOCK] = s1.scale;
      scale2[at[u] / BLOCK] = s2.scale;
    }
  }
}

// What the codes stand for: m and v.
template <typename T>
__global__ __launch_bounds__(256) void read_states_kernel(const Tensor* tensors, const Chunk* chunks, Pointers2 out,
                                                          int first_tensor) {
  constexpr int U = blocks_of_wave(true), CHUNK = chunk_of(true);
  const Chunk chunk = chunks[blockIdx.x];
  const Tensor t = tensors[chunk.tensor];
  GLOBAL T *const to1 = (GLOBAL T*)out.a[chunk.tensor - first_tensor], *const to2 = (GLOBAL T*)out.b[chunk.tensor - first_tensor];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Codes q1[U], q2[U];
  float c1[U], c2[U];
  int64_t at[U];
  int n[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t begin = (int64_t)chunk.at * CHUNK + (wave * U + u) * BLOCK, left = t.n - begin - 4 * lane;
    at[u] = begin + 4 * lane;
    n[u] = left >= 4 ? 4 : left > 0 ? (int)left : 0;
    c1[u] = begin < t.n ? ((const GLOBAL float*)t.c1)[begin / BLOCK] : 0.f;
    c2[u] = begin < t.n ? ((const GLOBAL float*)t.c2)[begin / BLOCK] : 0.f;
    q1[u] = load_codes((const GLOBAL uint8_t*)t.s1 + at[u], n[u]);
    q2[u] = load_codes((const GLOBAL uint8_t*)t.s2 + at[u], n[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float m[4], v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t a1 = q1[u].low | q1[u].third << 16, a2 = q2[u].low | q2[u].third << 16;
      const float r = decode<8>(a2, e, c2[u], c2[u] * 0x1p-15f);
      m[e] = signed_as(decode<7>(a1, e, c1[u], c1[u] * 0x1p-15f), a1, e);
      v[e] = r * r;
    }
    store4(to1 + at[u], n[u], m);
    store4(to2 + at[u], n[u], v);
  }
}

}  // namespace
}  // namespace dynb

using namespace dynb;

struct dynb_adamw {
  int32_t param_dtype, grad_dtype, state;
  std::vector<Tensor> tensors;
  std::vector<Chunk> chunks;
  std::vector<int64_t> first_chunk;       // [n_tensors + 1]
  const Tensor* d_tensors = nullptr;      // in the bound workspace
  const Chunk* d_chunks = nullptr;
};

namespace {
constexpr int64_t MOST_GRID = 1 << 23;    // workgroups of a launch: fewer than 2^32 threads
size_t tensor_bytes(const dynb_adamw* h) { return (size_t)round_up((int64_t)(h->tensors.size() * sizeof(Tensor)), 16); }

template <typename P, typename G>
void launch_step(const dynb_adamw* h, const Pointers& g, int first, int64_t blocks, int64_t stride, const Workers& w,
                 const Rule& r, hipStream_t st) {
  const Chunk* c = h->d_chunks + h->first_chunk[first];
  for (; blocks > 0; blocks -= MOST_GRID, c += MOST_GRID) {
    const dim3 grid((unsigned)(blocks < MOST_GRID ? blocks : MOST_GRID)), block(256);
    if (h->state == DYNB_STATE_8BIT)
      hipLaunchKernelGGL((adamw_kernel<P, G, true>), grid, block, 0, st, h->d_tensors, c, g, first, stride, w, r);
    else
      hipLaunchKernelGGL((adamw_kernel<P, G, false>), grid, block, 0, st, h->d_tensors, c, g, first, stride, w, r);
  }
}
}  // namespace

extern "C" int dynb_adamw_create(const dynb_adamw_desc* d, dynb_adamw** out) {
  if (!d || !out || !d->tensors) return fail(DYNB_ERR_BADARG, "adamw: null pointer");
  *out = nullptr;
  if ((d->param_dtype != DYNB_F32 && d->param_dtype != DYNB_BF16) ||
      (d->grad_dtype != DYNB_F32 && d->grad_dtype != DYNB_BF16))
    return fail(DYNB_ERR_BADARG, "adamw: unknown dtype");
  if (d->state != DYNB_STATE_F32 && d->state != DYNB_STATE_8BIT) return fail(DYNB_ERR_BADARG, "adamw: unknown state type");
  if (d->n_tensors < 1) return fail(DYNB_ERR_BADARG, "adamw: at least one tensor");
  const bool eight = d->state == DYNB_STATE_8BIT;
  const int64_t chunk = chunk_of(eight);
  int64_t chunks = 0;
  for (int i = 0; i < d->n_tensors; ++i) {
    const dynb_adamw_tensor& t = d->tensors[i];
    if (t.n < 0 || t.n > ((int64_t)1 << 40)) return fail(DYNB_ERR_BADARG, "adamw: tensor %d: size out of range", i);
    if (!(t.weight_decay >= 0.f) || !std::isfinite(t.weight_decay))
      return fail(DYNB_ERR_BADARG, "adamw: tensor %d: weight decay must be finite and not negative", i);
    if (t.copy && d->param_dtype == DYNB_BF16)
      return fail(DYNB_ERR_BADARG, "adamw: tensor %d: a copy of a bf16 parameter", i);
    if (t.n > 0 && (!t.param || !t.state1 || !t.state2 || (eight && (!t.scale1 || !t.scale2))))
      return fail(DYNB_ERR_BADARG, "adamw: tensor %d: null pointer", i);
    if (off_by(t.param, d->param_dtype == DYNB_F32 ? 4 : 2) || off_by(t.copy, 2) ||
        (!eight && (off_by(t.state1, 4) || off_by(t.state2, 4))) || (eight && (off_by(t.scale1, 4) || off_by(t.scale2, 4))))
      return fail(DYNB_ERR_BADARG, "adamw: tensor %d: a pointer is not a multiple of its element's size", i);
    chunks += (t.n + chunk - 1) / chunk;
  }
  if (chunks >= ((int64_t)1 << 35) / chunk) return fail(DYNB_ERR_UNSUPPORTED, "adamw: more than 2^35 elements");
  dynb_adamw* h = new (std::nothrow) dynb_adamw;
  if (!h) return fail(DYNB_ERR_STATE, "adamw: out of host memory");
  try {
    h->param_dtype = d->param_dtype;
    h->grad_dtype = d->grad_dtype;
    h->state = d->state;
    h->chunks.reserve((size_t)chunks);
    for (int i = 0; i < d->n_tensors; ++i) {
      const dynb_adamw_tensor& t = d->tensors[i];
      h->tensors.push_back({t.param, t.copy, t.state1, t.state2, t.scale1, t.scale2, t.n, t.weight_decay, i});
      h->first_chunk.push_back((int64_t)h->chunks.size());
      for (int64_t c = 0; c * chunk < t.n; ++c) h->chunks.push_back({i, (int32_t)c});
    }
    h->first_chunk.push_back((int64_t)h->chunks.size());
  } catch (...) {
    delete h;
    return fail(DYNB_ERR_STATE, "adamw: out of host memory");
  }
  *out = h;
  return DYNB_OK;
}

extern "C" void dynb_adamw_destroy(dynb_adamw* h) { delete h; }

extern "C" size_t dynb_adamw_workspace_bytes(const dynb_adamw* h) {
  return h ? tensor_bytes(h) + (h->chunks.empty() ? 1 : h->chunks.size()) * sizeof(Chunk) : 0;
}

extern "C" int dynb_adamw_bind(dynb_adamw* h, void* workspace, size_t workspace_bytes, void* stream) {
  if (!h || !workspace) return fail(DYNB_ERR_BADARG, "adamw_bind: null pointer");
  if (off_by(workspace, 16)) return fail(DYNB_ERR_BADARG, "adamw_bind: workspace must be 16-byte aligned");
  if (workspace_bytes < dynb_adamw_workspace_bytes(h)) return fail(DYNB_ERR_BADARG, "adamw_bind: workspace too small");
  char* w = (char*)workspace;
  hipStream_t st = (hipStream_t)stream;
  h->d_tensors = nullptr;
  hipError_t e = hipMemcpyAsync(w, h->tensors.data(), h->tensors.size() * sizeof(Tensor), hipMemcpyHostToDevice, st);
  if (e == hipSuccess && !h->chunks.empty())
    e = hipMemcpyAsync(w + tensor_bytes(h), h->chunks.data(), h->chunks.size() * sizeof(Chunk), hipMemcpyHostToDevice, st);
  if (e == hipSuccess) e = hipStreamSynchronize(st);
  if (e != hipSuccess) return fail(DYNB_ERR_HIP, "adamw_bind: %s", hipGetErrorString(e));
  h->d_tensors = (const Tensor*)w;
  h->d_chunks = (const Chunk*)(w + tensor_bytes(h));
  return DYNB_OK;
}

extern "C" int dynb_adamw_step(dynb_adamw* h, const void* const* grads, const int32_t* b, int32_t K,
                               int64_t worker_stride, const dynb_adamw_rule* rule, void* stream) {
  if (!h || !grads || !rule) return fail(DYNB_ERR_BADARG, "adamw_step: null pointer");
  Segs seg;
  if (int rc = segments_of(b, K, "adamw_step", seg)) return rc;
  if (seg.off[K] <= 0) return fail(DYNB_ERR_BADARG, "adamw_step: sum(b) must be positive");
  if (K > 1 && worker_stride < 0) return fail(DYNB_ERR_BADARG, "adamw_step: negative worker_stride");
  if (!(rule->beta1 >= 0.0 && rule->beta1 < 1.0 && rule->beta2 >= 0.0 && rule->beta2 < 1.0))
    return fail(DYNB_ERR_BADARG, "adamw_step: betas must lie in [0, 1)");
  if (rule->step < 1) return fail(DYNB_ERR_BADARG, "adamw_step: steps count from 1");
  if (!std::isfinite(rule->lr) || !(rule->eps >= 0.f) || !std::isfinite(rule->eps))
    return fail(DYNB_ERR_BADARG, "adamw_step: lr and eps must be finite, eps not negative");
  const int n = (int)h->tensors.size();
  for (int i = 0; i < n; ++i)
    if (h->tensors[i].n > 0 && (!grads[i] || off_by(grads[i], h->grad_dtype == DYNB_F32 ? 4 : 2)))
      return fail(DYNB_ERR_BADARG, "adamw_step: gradient %d is null or not a multiple of its element's size", i);
  if (!h->d_tensors) return fail(DYNB_ERR_STATE, "adamw_step: not bound");
  Workers w = {};
  for (int k = 0; k < K; ++k)
    if (b[k] > 0) {
      w.w[w.n] = (float)((double)b[k] / (double)seg.off[K]);
      w.index[w.n++] = k;
    }
  Rule r;
  r.lr = rule->lr;
  r.eps = rule->eps;
  r.beta1 = (float)rule->beta1;
  r.beta2 = (float)rule->beta2;
  r.omb1 = (float)(1.0 - rule->beta1);
  r.omb2 = (float)(1.0 - rule->beta2);
  r.inv_c1 = (float)(1.0 / (1.0 - std::pow(rule->beta1, (double)rule->step)));
  r.inv_c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(rule->beta2, (double)rule->step)));   // (of the root)
  r.seed = rule->seed;
  double elements = 0;
  for (const Tensor& t : h->tensors) elements += (double)t.n;
  const double gs = h->grad_dtype == DYNB_F32 ? 4 : 2, ps = h->param_dtype == DYNB_F32 ? 4 : 2;
  Timed timed(KC_UPDATE, stream, elements * (2.0 * w.n + 14.0),
              elements * (2 * ps + gs * w.n + (h->state == DYNB_STATE_F32 ? 16 : 4)));
  for (int first = 0; first < n; first += POINTERS) {
    const int last = first + POINTERS < n ? first + POINTERS : n;
    const int64_t blocks = h->first_chunk[last] - h->first_chunk[first];
    if (blocks == 0) continue;
    Pointers g = {};
    for (int i = first; i < last; ++i) g.p[i - first] = grads[i];
    const hipStream_t st = (hipStream_t)stream;
    if (h->param_dtype == DYNB_F32 && h->grad_dtype == DYNB_F32) launch_step<float, float>(h, g, first, blocks, worker_stride, w, r, st);
    else if (h->param_dtype == DYNB_F32) launch_step<float, bf16>(h, g, first, blocks, worker_stride, w, r, st);
    else if (h->grad_dtype == DYNB_F32) launch_step<bf16, float>(h, g, first, blocks, worker_stride, w, r, st);
    else launch_step<bf16, bf16>(h, g, first, blocks, worker_stride, w, r, st);
    if (hipGetLastError() != hipSuccess) return fail(DYNB_ERR_HIP, "adamw_step launch failed");
  }
  return DYNB_OK;
}

extern "C" int dynb_adamw_read_states(dynb_adamw* h, void* const* out1, void* const* out2, int32_t out_dtype,
                                      void* stream) {
  if (!h || !out1 || !out2) return fail(DYNB_ERR_BADARG, "adamw_read_states: null pointer");
  if (h->state != DYNB_STATE_8BIT) return fail(DYNB_ERR_BADARG, "adamw_read_states: the states are fp32");
  if (out_dtype != DYNB_F32 && out_dtype != DYNB_BF16) return fail(DYNB_ERR_BADARG, "adamw_read_states: unknown dtype");
  const int n = (int)h->tensors.size();
  const size_t size = out_dtype == DYNB_F32 ? 4 : 2;
  double elements = 0;
  for (int i = 0; i < n; ++i) {
    elements += (double)h->tensors[i].n;
    if (h->tensors[i].n > 0 && (!out1[i] || !out2[i] || off_by(out1[i], size) || off_by(out2[i], size)))
      return fail(DYNB_ERR_BADARG, "adamw_read_states: output %d is null or not a multiple of its element's size", i);
  }
  if (!h->d_tensors) return fail(DYNB_ERR_STATE, "adamw_read_states: not bound");
  Timed timed(KC_UPDATE, stream, 0.0, elements * (2.0 + 2 * size));
  for (int first = 0; first < n; first += POINTERS / 2) {
    const int last = first + POINTERS / 2 < n ? first + POINTERS / 2 : n;
    const int64_t blocks = h->first_chunk[last] - h->first_chunk[first];
    if (blocks == 0) continue;
    Pointers2 o = {};
    for (int i = first; i < last; ++i) {
      o.a[i - first] = out1[i];
      o.b[i - first] = out2[i];
    }
    const Chunk* c = h->d_chunks + h->first_chunk[first];
    if (out_dtype == DYNB_F32)
      hipLaunchKernelGGL(read_states_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream,
                         h->d_tensors, c, o, first);
    else
      hipLaunchKernelGGL(read_states_kernel<bf16>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream,
                         h->d_tensors, c, o, first);
    if (hipGetLastError() != hipSuccess) return fail(DYNB_ERR_HIP, "adamw_read_states launch failed");
  }
  return DYNB_OK;
}
