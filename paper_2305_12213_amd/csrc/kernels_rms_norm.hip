// Root-mean-square norm with the residual's addition, its 8-bit outputs, and its gradients:
//   s = x + residual, rstd = (mean s^2 + eps)^(-1/2), y = s rstd gain;
//   dx = rstd (gain dy - shat mean(gain dy shat)) + dsum, dgain_k = sum over worker k's rows of dy shat, shat = s rstd.
// About 8 and 12 operations per element: memory bounds it, 16384 x 8192 bf16 to fp8 160 us (939 MB, 5.9 TB/s), 4096 x 4096
// forward 25 us (5.4 TB/s), gradients 28 us and 4.7 for the sums over chunks (142 MB in the first); small calls take what a
// launch takes.  Statistics, products and sums are fp32; s, y and dx are rounded once where they are stored, and y comes
// from the s that has not been rounded.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "dynb_internal.h"
#include "row_access.h"

namespace dynb {
namespace {

constexpr float FP8_TOP = 448.f, INT8_TOP = 127.f;
constexpr int MAX_COLS = 1 << 20;
constexpr int WIDEST = 2 * 64 * MOST_WAVES;   // granules of the widest rows that stay in registers
// Rows of up to so many waves take one granule per thread, wider ones two (4096 bf16 columns: one row 3.2 us, with two granules
// 3.8, 4096 rows 25.2 and 26.1; 8192 columns: 53.3 us with one, 49.9 with two).  8-bit outputs, there and back: 4096 x 6000 bf16
// 50.0 us with one, 61.8 with two, 856 x 6437 22.2 and 19.6.
constexpr int one_granule(int out) { return out == DYNB_OUT_SAME ? 8 : 12; }
// Gradients take one granule as far as the waves go (4096 x 8192 bf16: 58.2 us, with two 60.4), then bf16 rows two; fp32 rows do
// not fit in the registers then, and take the two launches of wider ones (4096 x 16384 353 us, with two granules, which spill, 367;
// bf16 107 and with two launches 189).
constexpr int widest_grad(size_t element) { return element == 2 ? WIDEST : WIDEST / 2; }

// A workgroup per row, also of more rows than a grid has workgroups in one direction.
dim3 grid_of_rows(int64_t rows) {
  constexpr int64_t MOST = 1 << 20;
  return dim3((unsigned)std::min(rows, MOST), (unsigned)((rows + MOST - 1) / MOST));
}
__device__ inline int64_t row_of_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// Lanes of a row: 8, 16, 32 or 64, or whole waves.
constexpr int WIDE = 128;
template <int L> __device__ inline int row_in_block() {
  return L == WIDE ? 0 : L == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x / L;
}
template <int L> __device__ inline float row_sum(float v, int waves, float* red) {
  return L < 64 ? lanes_sum<L>(v) : block_sum(v, waves, red);
}

struct NormArgs {
  const void *x, *residual;
  const float* gain;
  void *sum, *y;
  float *scales, *rstd;
  int64_t ld_x, ld_residual, ld_sum, ld_y;
  int rows, cols, scale_block, n_blocks;
  float eps, inv_cols;
  double bytes;                            // of the call
};

// 8 neighbouring values in 8 bits, the first n of them.  (Of a block with an infinity or NaN it does not matter which: its
// scale is NaN.)
template <int OUT, bool PAST>
__device__ inline void store_eight(uint8_t* p, int n, const float (&f)[GRANULE], float inv) {
  u32x2 q;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float *v = f + 4 * h;
    if (OUT == DYNB_OUT_FP8) {
      q[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv,
                                                       __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, 0, false), true);
    } else {                               // the lowest byte of 1.5 * 2^23 + value is the value, rounded to nearest-even
      uint32_t b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = __float_as_uint(__builtin_fmaf(v[e], inv, 12582912.f));
      q[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u),
                                   0x05040100u);
    }
  }
  if (n >= GRANULE) {
    if (PAST) __builtin_nontemporal_store((u32x2_any)q, (u32x2_any*)p);
    else *(u32x2_any*)p = q;
  } else {                                 // 4, 2 and 1 of them, as the bits of n say
    if (n & 4) *(u32_any*)p = q[0];
    const uint32_t rest = n & 4 ? q[1] : q[0];
    if (n & 2) *(u16_any*)(p + (n & 4)) = (uint16_t)rest;
    if (n & 1) p[n - 1] = (uint8_t)(n & 2 ? rest >> 16 : rest);
  }
}

// 1 / sqrt(mean + eps) from the sum of squares, by the hardware's root (one unit in the last place).  Where the sum has
// overflowed, from the squares of the row times 2^-80, which `scaled_sum` gives (eps is nothing beside them; a row with an
// infinity or NaN ends the same either way); where squares may have been lost below fp32's range (eps is below 2^-100 then), of
// the row times 2^80, with eps times 2^160: rows down to a root mean square of 2^-126.
template <typename F> __device__ inline float rstd_of(float ss, float inv_cols, float eps, F scaled_sum) {
  const float m = __builtin_fmaf(ss, inv_cols, eps);
  // (said to be likely, or the other two paths cost the narrow kernels 2 %)
  if (__builtin_expect(m >= 0x1p-100f && m <= 3e38f, 1)) return __builtin_amdgcn_rsqf(m);
  if (m < 1.f) return 0x1p80f / sqrtf(__builtin_fmaf(scaled_sum(0x1p80f), inv_cols, eps * 0x1p80f * 0x1p80f));
  return 0x1p-80f / sqrtf(scaled_sum(0x1p-80f) * inv_cols);
}

// Rows beyond WIDEST granules, and blocks that no group of lanes holds: a workgroup per row goes over it two or three times,
// the later ones in the caches.  group: lanes that share a scale, -1 where it is no power of two up to 64 (then by LDS), 0
// where all threads take a block at a time.  (4096 x 18432 bf16 with a residual 130 us, 4.6 TB/s, element by element 278; one row
// of 20480 6.5 us.  To fp8 4096 x 4096 with a residual: blocks of 96 columns 41 us, of 1024 37; and back 59, a wave per block 121,
// and 55, 57.)
constexpr int MOST_SLOTS = 64 * MOST_WAVES / 12;   // blocks of 96 columns, the narrowest that are no power of two
template <typename T, int OUT>
__global__ __launch_bounds__(64 * MOST_WAVES) void rms_norm_any_kernel(NormArgs p, int group) {
  __shared__ float red[3][MOST_WAVES];
  __shared__ uint32_t redu[2][MOST_WAVES], tops[3][MOST_SLOTS];
  constexpr float TOP = OUT == DYNB_OUT_FP8 ? FP8_TOP : INT8_TOP;
  const int t = threadIdx.x, threads = blockDim.x, waves = threads >> 6;
  int turn = 0, round = 0;
  for (int i = t; i < 3 * MOST_SLOTS; i += threads) (&tops[0][0])[i] = 0;
  __syncthreads();
  for (int64_t r = row_of_block(); r < p.rows; r += (int64_t)gridDim.x * gridDim.y, turn ^= 1) {
    const T* const x = (const T*)p.x + r * p.ld_x;
    const T* const res = p.residual ? (const T*)p.residual + r * p.ld_residual : nullptr;
    auto values = [&](int c, float (&s)[GRANULE]) {
      const Raw<T> a = load_raw(x + c, p.cols - c);
      if (res) {
        float q[GRANULE];
        const Raw<T> b = load_raw(res + c, p.cols - c);
        unpack(a, p.cols - c, s);
        unpack(b, p.cols - c, q);
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) s[e] += q[e];
      } else {
        unpack(a, p.cols - c, s);
      }
    };
    auto sum_of_squares = [&](float factor) {
      float ss = 0.f;
      for (int c = t * GRANULE; c < p.cols; c += threads * GRANULE) {
        float s[GRANULE];
        values(c, s);
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) ss += (s[e] * factor) * (s[e] * factor);
      }
      return ss;
    };
    const float ss = block_sum(sum_of_squares(1.f), waves, red[turn]);
    const float rstd = rstd_of(ss, p.inv_cols, p.eps, [&](float by) { return block_sum(sum_of_squares(by), waves, red[2]); });
    if (t == 0 && p.rstd) p.rstd[r] = rstd;
    auto results = [&](int c, float (&s)[GRANULE]) {
      if (!p.gain) {
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) s[e] *= rstd;
        return;
      }
      float g[GRANULE];
      load_part(p.gain + c, p.cols - c, g);
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) s[e] = s[e] * rstd * g[e];
    };
    auto largest = [&](const float (&y)[GRANULE]) {                   // (elements that do not exist are zeros)
      uint32_t a = 0;
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) a = max(a, __float_as_uint(y[e]) & 0x7fffffffu);
      return a;
    };
    auto keep = [&](int c, const float (&s)[GRANULE]) {
      if (p.sum && c < p.cols) store_part((T*)p.sum + r * p.ld_sum + c, p.cols - c, s);
    };
    // (the lane that reads an element for the block's largest is the one that stores it: outputs may lie on inputs)
    uint8_t* const y = (uint8_t*)p.y + r * p.ld_y;
    if (OUT == DYNB_OUT_SAME) {
      for (int c = t * GRANULE; c < p.cols; c += threads * GRANULE) {
        float s[GRANULE];
        values(c, s);
        keep(c, s);
        results(c, s);
        store_part((T*)p.y + r * p.ld_y + c, p.cols - c, s);
      }
    } else if (group != 0) {              // a granule per thread, whole blocks to a round
      const int lanes = p.scale_block / GRANULE, slots = threads / lanes, slot = t / lanes;
      for (int c0 = 0; c0 < p.cols; c0 += slots * p.scale_block) {
        const int c = c0 + t * GRANULE;
        const bool mine = slot < slots && c < p.cols;
        float s[GRANULE] = {};
        if (mine) {
          values(c, s);
          keep(c, s);
          results(c, s);
        }
        uint32_t a = largest(s);
        if (group > 0) {
          a = group_max(a, group);
        } else {
          if (mine) atomicMax(&tops[round][slot], a);                 // (whole numbers: any order)
          __syncthreads();
          if (mine) a = tops[round][slot];
          if (t < MOST_SLOTS) tops[round == 0 ? 2 : round - 1][t] = 0;  // (read before this barrier, used behind the next)
          round = round == 2 ? 0 : round + 1;
        }
        if (!mine) continue;
        const Scale scale = scale_of(a, TOP);
        if (t == slot * lanes) p.scales[r * p.n_blocks + c / p.scale_block] = scale.scale;
        store_eight<OUT, false>(y + c, p.cols - c, s, scale.inv);
      }
    } else {
      for (int b = 0; b < p.n_blocks; ++b) {
        const int c0 = b * p.scale_block, c1 = min(c0 + p.scale_block, p.cols);
        uint32_t a = 0;
        for (int c = c0 + t * GRANULE; c < c1; c += threads * GRANULE) {
          float s[GRANULE];
          values(c, s);
          results(c, s);
          a = max(a, largest(s));
        }
        const Scale scale = scale_of(block_max(a, waves, redu[b & 1]), TOP);
        if (t == 0) p.scales[r * p.n_blocks + b] = scale.scale;
        for (int c = c0 + t * GRANULE; c < c1; c += threads * GRANULE) {
          float s[GRANULE];
          values(c, s);
          keep(c, s);
          results(c, s);
          store_eight<OUT, false>(y + c, c1 - c, s, scale.inv);
        }
      }
    }
  }
}

// Rows that fit in registers, N granules per thread: one read, one write.  L lanes of a workgroup of four waves take a row at a
// time (16384 x 64 bf16: 8 lanes 3.8 us, 64 9.0; 131072 x 128: 16 lanes 23.5, 64 36.0; x 256: 32 lanes 45.7, 64 49.1), or,
// where L is WIDE, as many waves as a row needs.  A thread keeps its part of the gain over all rows of the
// workgroup, and asks for the next row before it writes the present one in 8 bits.  group: lanes that share a scale (a
// power of two), 0 where the whole row does.
template <typename T, int OUT, int L, int N, bool PAST>
__global__ __launch_bounds__(L == WIDE ? 64 * MOST_WAVES : 256) void rms_norm_kernel(NormArgs p, int group) {
  constexpr int PER = L == WIDE ? 1 : 256 / L;   // rows of a workgroup
  constexpr float TOP = OUT == DYNB_OUT_FP8 ? FP8_TOP : INT8_TOP;
  __shared__ float red[3][MOST_WAVES];
  __shared__ uint32_t redu[2][MOST_WAVES];
  const uint32_t waves = L == WIDE ? blockDim.x >> 6 : 1;
  const uint32_t t = L == WIDE ? threadIdx.x : threadIdx.x % L;
  int64_t r = (int64_t)blockIdx.x * PER + row_in_block<L>();
  int turn = 0;
  Raw<T> x[N], res[N];
  auto ask = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t c = (t + i * 64 * waves) * GRANULE;
      x[i] = load_raw<PAST>((const T*)p.x + row * p.ld_x + c, (int)(p.cols - c));
      if (p.residual) res[i] = load_raw<PAST>((const T*)p.residual + row * p.ld_residual + c, (int)(p.cols - c));
    }
  };
  if (r < p.rows) ask(r);
  Raw<float> gain[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t c = (t + i * 64 * waves) * GRANULE;
    if (p.gain) gain[i] = load_raw(p.gain + c, (int)(p.cols - c));
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) gain[i].a[e] = gain[i].b[e] = 0x3f800000u;
  }
  for (; r < p.rows; r += (int64_t)gridDim.x * PER, turn ^= 1) {
    float s[N][GRANULE], ss = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int n = p.cols - (int)(t + i * 64 * waves) * GRANULE;
      unpack(x[i], n, s[i]);
      if (p.residual) {
        float q[GRANULE];
        unpack(res[i], n, q);
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) s[i][e] += q[e];
      }
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) ss += s[i][e] * s[i][e];
    }
    ss = row_sum<L>(ss, waves, red[turn]);
    const float rstd = rstd_of(ss, p.inv_cols, p.eps, [&](float by) {
      float a = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) a += (s[i][e] * by) * (s[i][e] * by);
      return row_sum<L>(a, waves, red[2]);
    });
    if (t == 0 && p.rstd) p.rstd[r] = rstd;
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t c = (t + i * 64 * waves) * GRANULE;
      if (p.sum && c < (uint32_t)p.cols) store_part<PAST>((T*)p.sum + r * p.ld_sum + c, (int)(p.cols - c), s[i]);
      float g[GRANULE];
      unpack(gain[i], p.gain ? (int)(p.cols - c) : GRANULE, g);
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) s[i][e] = s[i][e] * rstd * g[e];   // (elements that do not exist are zeros)
      if (OUT == DYNB_OUT_SAME && c < (uint32_t)p.cols) store_part<PAST>((T*)p.y + r * p.ld_y + c, (int)(p.cols - c), s[i]);
    }
    const int64_t now = r;
    if (r + (int64_t)gridDim.x * PER < p.rows) ask(r + (int64_t)gridDim.x * PER);
    if (OUT == DYNB_OUT_SAME) continue;
    Scale scale;
    if (group == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) amax = max(amax, __float_as_uint(s[i][e]) & 0x7fffffffu);
      scale = scale_of(L < 64 ? group_max(amax, L) : block_max(amax, waves, redu[turn]), TOP);
      if (t == 0) p.scales[now] = scale.scale;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t c = (t + i * 64 * waves) * GRANULE;
      if (group) {
        amax = 0;
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) amax = max(amax, __float_as_uint(s[i][e]) & 0x7fffffffu);
        scale = scale_of(group_max(amax, group), TOP);
        if ((t & (group - 1)) == 0 && c < (uint32_t)p.cols) p.scales[now * p.n_blocks + c / p.scale_block] = scale.scale;
      }
      if (c < (uint32_t)p.cols) store_eight<OUT, PAST>((uint8_t*)p.y + now * p.ld_y + c, (int)(p.cols - c), s[i], scale.inv);
    }
  }
}

struct NormGradArgs {
  const void* sum;
  const float *rstd, *gain;
  const void *dy, *dsum;
  void* dx;
  float* dgain;
  int64_t ld_sum, ld_dy, ld_dsum, ld_dx, dgain_stride;
  int rows, cols;
  float inv_cols;
};

// A thread takes 8 neighbouring values of a row at a time (16384 x 8192 fp8 to bf16: 74 us, 5.4 TB/s; two at a time 85 us).
template <typename T, bool PAST>
__global__ __launch_bounds__(256) void dequantise_kernel(NormArgs p, int out, T* to, int64_t ld_to) {
  const int granules = (p.cols + GRANULE - 1) / GRANULE;
  const int64_t total = (int64_t)p.rows * granules;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = total < ((int64_t)1 << 32) ? (int64_t)((uint32_t)i / (uint32_t)granules) : i / granules;
    const int c = (int)(i - r * granules) * GRANULE, n = p.cols - c;
    const uint8_t* y = (const uint8_t*)p.y + r * p.ld_y + c;
    const float scale = p.scales[r * p.n_blocks + (p.n_blocks == 1 ? 0 : c / p.scale_block)];
    u32x2 q = {0, 0};
    if (n >= GRANULE) q = PAST ? (u32x2)__builtin_nontemporal_load((const u32x2_any*)y) : (u32x2)*(const u32x2_any*)y;
    else {                                 // 4, 2 and 1 of them, as the bits of n say
      uint32_t rest = 0;
      if (n & 1) rest = y[n - 1];
      if (n & 2) rest = rest << 16 | *(const u16_any*)(y + (n & 4));
      if (n & 4) q[0] = *(const u32_any*)y;
      q[n & 4 ? 1 : 0] = rest;
    }
    float f[GRANULE];
#pragma unroll
    for (int e = 0; e < GRANULE; ++e) {
      const uint32_t b = q[e / 4] >> (8 * (e & 3));
      f[e] = (out == DYNB_OUT_INT8 ? (float)(int8_t)b : __builtin_amdgcn_cvt_f32_fp8(b, 0)) * scale;
    }
    store_part<PAST>(to + r * ld_to + c, n, f);
  }
}

// Checks a description and fills what the kernels take of it.
int describe(const dynb_rms_norm_desc* d, const char* who, NormArgs& a) {
  if (!d) return fail(DYNB_ERR_BADARG, "%s: null pointer", who);
  if (d->dtype != DYNB_F32 && d->dtype != DYNB_BF16) return fail(DYNB_ERR_BADARG, "%s: unknown dtype", who);
  if (d->out < DYNB_OUT_SAME || d->out > DYNB_OUT_INT8) return fail(DYNB_ERR_BADARG, "%s: unknown output type", who);
  if (d->cols < 1 || d->cols > MAX_COLS) return fail(DYNB_ERR_BADARG, "%s: cols out of range", who);
  if (d->out != DYNB_OUT_SAME && (d->scale_block < 0 || d->scale_block % 32))
    return fail(DYNB_ERR_BADARG, "%s: scale_block must be 0 or a positive multiple of 32", who);
  if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return fail(DYNB_ERR_BADARG, "%s: eps must be finite and not negative", who);
  for (int64_t ld : {d->ld_x, d->ld_residual, d->ld_sum, d->ld_y, d->ld_dy, d->ld_dsum, d->ld_dx})
    if (ld != 0 && ld < d->cols) return fail(DYNB_ERR_BADARG, "%s: a row pitch is below cols", who);
  a = {};
  auto pitch = [&](int64_t ld) { return ld ? ld : (int64_t)d->cols; };
  a.ld_x = pitch(d->ld_x);
  a.ld_residual = pitch(d->ld_residual);
  a.ld_sum = pitch(d->ld_sum);
  a.ld_y = pitch(d->ld_y);
  a.cols = d->cols;
  a.eps = d->eps;
  a.inv_cols = 1.f / (float)d->cols;
  a.scale_block = d->scale_block && d->scale_block < d->cols ? d->scale_block : d->cols;
  a.n_blocks = d->out == DYNB_OUT_SAME ? 0 : (d->cols + a.scale_block - 1) / a.scale_block;
  return DYNB_OK;
}

// Workgroups for `units` of work where one has `threads` threads: four times what the chip holds at once, less if there is
// less (16384 x 8192 to fp8: 161 us, as many as it holds 164, one per row 182).
int resident(int64_t units, int threads) {
  const int64_t most = 1024 * (2048 / threads);
  return (int)(units < most ? units : most);
}

template <typename T, int OUT, int L, int N> void launch_norm_as(const NormArgs& a, int waves, int group, hipStream_t st) {
  constexpr int PER = L == WIDE ? 1 : 256 / L;
  const dim3 block(64 * waves), grid(resident(((int64_t)a.rows + PER - 1) / PER, 64 * waves));
  if (past_caches(a.bytes)) hipLaunchKernelGGL((rms_norm_kernel<T, OUT, L, N, true>), grid, block, 0, st, a, group);
  else hipLaunchKernelGGL((rms_norm_kernel<T, OUT, L, N, false>), grid, block, 0, st, a, group);
}

template <typename T, int OUT> void launch_norm_out(const NormArgs& a, hipStream_t st) {
  // lanes that share a scale: a power of two within a wave, or the whole row
  const int granules = (a.cols + GRANULE - 1) / GRANULE, lanes = a.scale_block / GRANULE;
  const bool whole = OUT == DYNB_OUT_SAME || a.n_blocks == 1;
  const int waves = (granules + 63) / 64, threads = 64 * (waves < MOST_WAVES ? waves : MOST_WAVES);
  const int group = whole || lanes > threads ? 0 : lanes > 64 || (lanes & (lanes - 1)) ? -1 : lanes;
  if (granules > WIDEST || group < 0 || (group == 0 && !whole)) {
    // A workgroup per row, or, 8-bit outputs, for as many rows as there are more than the chip holds (16384 x 18432 bf16 461 us,
    // several rows each 504; to fp8 in blocks of 96 columns 574 and 524, 200000 x 200 170 and 150, 16384 x 4096 in blocks of
    // 1024 152 and 131, whole rows of 16384 x 18432 561 and 567).
    const dim3 grid = OUT == DYNB_OUT_SAME ? grid_of_rows(a.rows) : dim3(resident(a.rows, threads));
    hipLaunchKernelGGL((rms_norm_any_kernel<T, OUT>), grid, dim3(threads), 0, st, a, group);
    return;
  }
  if (granules <= 8) launch_norm_as<T, OUT, 8, 1>(a, 4, group, st);
  else if (granules <= 16) launch_norm_as<T, OUT, 16, 1>(a, 4, group, st);
  else if (granules <= 32) launch_norm_as<T, OUT, 32, 1>(a, 4, group, st);
  else if (waves == 1) launch_norm_as<T, OUT, 64, 1>(a, 4, group, st);
  else if (waves == 2) launch_norm_as<T, OUT, 64, 2>(a, 4, group, st);
  else if (waves <= one_granule(OUT)) launch_norm_as<T, OUT, WIDE, 1>(a, waves, group, st);
  else launch_norm_as<T, OUT, WIDE, 2>(a, (waves + 1) / 2, group, st);
}

template <typename T> void launch_norm(const NormArgs& a, int out, hipStream_t st) {
  if (out == DYNB_OUT_SAME) launch_norm_out<T, DYNB_OUT_SAME>(a, st);
  else if (out == DYNB_OUT_FP8) launch_norm_out<T, DYNB_OUT_FP8>(a, st);
  else launch_norm_out<T, DYNB_OUT_INT8>(a, st);
}

// Both gradients of rows that fit in registers, N granules per thread, in one pass: the rows' gradient, and the gain's summed over
// the rows of a chunk (of one worker) in registers, then over the chunks by sum_chunks_kernel.  L lanes take every (256 / L)-th
// row of the chunk and their sums are added by exchanges and in LDS (131072 x 64 bf16: 8 lanes 18.2 us, 64 46.7); WIDE: a
// workgroup of as many waves as a row needs takes a row at a time.  A row's loads are issued while the row before it is
// reduced.
struct Chunks {
  int rows;                               // of a chunk, the last one of a worker may be shorter
  int first[DYNB_MAX_WORKERS + 1];        // of each worker's chunks
};
template <typename T, int L, int N, bool PAST>
__global__ __launch_bounds__(L == WIDE ? 64 * MOST_WAVES : 256) void rms_norm_grad_kernel(NormGradArgs p, Segs seg, Chunks ch,
                                                                             float* partial) {
  constexpr int PER = L == WIDE ? 1 : 256 / L, LANES = L == WIDE ? 64 : L, COLS = LANES * N * GRANULE;
  constexpr bool AHEAD = L != WIDE || N == 1;  // (two granules, up to 16 waves: the next row would spill)
  __shared__ float red[2][MOST_WAVES];
  __shared__ float sums[L == WIDE ? 1 : 3 * COLS];
  const uint32_t waves = L == WIDE ? blockDim.x >> 6 : 1;
  const uint32_t t = L == WIDE ? threadIdx.x : threadIdx.x % L;
  int turn = 0;
  int k = 0;
  while (k + 1 < seg.K && (int)blockIdx.x >= ch.first[k + 1]) ++k;
  const int64_t begin = seg.off[k] + (int64_t)((int)blockIdx.x - ch.first[k]) * ch.rows;
  const int64_t end = begin + ch.rows < seg.off[k + 1] ? begin + ch.rows : seg.off[k + 1];
  Raw<T> s[N], dy[N], ds[N];
  float rstd = 0.f;
  auto ask = [&](int64_t r) {
    rstd = p.rstd[r];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t c = (t + i * 64 * waves) * GRANULE;
      s[i] = load_raw<PAST>((const T*)p.sum + r * p.ld_sum + c, (int)(p.cols - c));
      dy[i] = load_raw<PAST>((const T*)p.dy + r * p.ld_dy + c, (int)(p.cols - c));
      if (p.dsum) ds[i] = load_raw<PAST>((const T*)p.dsum + r * p.ld_dsum + c, (int)(p.cols - c));
    }
  };
  int64_t r = begin + row_in_block<L>();
  if (AHEAD && r < end) ask(r);
  float acc[N][GRANULE];
  Raw<float> gain[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t c = (t + i * 64 * waves) * GRANULE;
    if (p.gain) gain[i] = load_raw(p.gain + c, (int)(p.cols - c));
    else
#pragma unroll
      for (int e = 0; e < 4; ++e) gain[i].a[e] = gain[i].b[e] = 0x3f800000u;
#pragma unroll
    for (int e = 0; e < GRANULE; ++e) acc[i][e] = 0.f;
  }
  for (; r < end; r += PER, turn ^= 1) {
    if (!AHEAD) ask(r);
    float c1 = 0.f;
    Raw<T> s0[N], dy0[N], ds0[N];
    const float rstd0 = rstd;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      s0[i] = s[i];
      dy0[i] = dy[i];
      if (p.dsum) ds0[i] = ds[i];
    }
    if (AHEAD && r + PER < end) ask(r + PER);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int n = p.cols - (int)(t + i * 64 * waves) * GRANULE;
      float a[GRANULE], d[GRANULE], g[GRANULE];
      unpack(s0[i], n, a);
      unpack(dy0[i], n, d);
      unpack(gain[i], p.gain ? n : GRANULE, g);
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) {
        const float q = d[e] * (a[e] * rstd0);
        acc[i][e] += q;
        c1 += g[e] * q;
      }
    }
    c1 = row_sum<L>(c1, waves, red[turn]) * p.inv_cols;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t c = (t + i * 64 * waves) * GRANULE;
      if (c >= (uint32_t)p.cols) continue;
      const int n = p.cols - (int)(t + i * 64 * waves) * GRANULE;
      float a[GRANULE], d[GRANULE], g[GRANULE];
      unpack(s0[i], n, a);
      unpack(dy0[i], n, d);
      unpack(gain[i], p.gain ? n : GRANULE, g);
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) a[e] = rstd0 * (g[e] * d[e] - a[e] * rstd0 * c1);
      if (p.dsum) {
        unpack(ds0[i], n, d);
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) a[e] += d[e];
      }
      store_part<PAST>((T*)p.dx + r * p.ld_dx + c, (int)(p.cols - c), a);
    }
  }
  if (!p.dgain) return;
  if (L != WIDE) {                         // the rows of a wave by exchanges, the waves through LDS
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool mine = L >= 64 || (threadIdx.x & 63) < L;
#pragma unroll
    for (int d = LANES; d < 64; d *= 2)
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) acc[0][e] += __shfl_xor(acc[0][e], d);
    if (wave > 0 && mine)
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) sums[(wave - 1) * COLS + e * LANES * N + i * LANES + t] = acc[i][e];
    __syncthreads();
    if (wave > 0 || !mine) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) acc[i][e] += sums[w * COLS + e * LANES * N + i * LANES + t];
  }
  // a worker's only chunk is its sum
  float* const to = ch.first[k + 1] - ch.first[k] == 1 ? p.dgain + k * p.dgain_stride : partial + (int64_t)blockIdx.x * p.cols;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t c = (t + i * 64 * waves) * GRANULE;
    if (c < (uint32_t)p.cols) store_part(to + c, (int)(p.cols - c), acc[i]);
  }
}

// Gradients of rows beyond widest_grad() granules, in two launches: the rows' by a workgroup per row that goes over it twice, the
// gain's over a chunk's rows by a thread per granule, UNDER rows at a time.  (4096 x 18432 bf16 with dsum 196 us, moving 906 MB;
// a thread per column and worker and single elements 1950.)
template <typename T>
__global__ __launch_bounds__(64 * MOST_WAVES) void rms_norm_grad_any_kernel(NormGradArgs p) {
  __shared__ float red[MOST_WAVES];
  const int threads = blockDim.x;
  const int64_t r = row_of_block();
  if (r >= p.rows) return;
  const T *const s = (const T*)p.sum + r * p.ld_sum, *const dy = (const T*)p.dy + r * p.ld_dy;
  const float rstd = p.rstd[r];
  auto values = [&](int c, float (&a)[GRANULE], float (&gd)[GRANULE]) {        // shat, gain dy
    const int n = p.cols - c;
    const Raw<T> s0 = load_raw(s + c, n), d0 = load_raw(dy + c, n);
    float g[GRANULE];
    if (p.gain) load_part(p.gain + c, n, g);
    unpack(s0, n, a);
    unpack(d0, n, gd);
#pragma unroll
    for (int e = 0; e < GRANULE; ++e) {
      a[e] *= rstd;
      if (p.gain) gd[e] *= g[e];
    }
  };
  float c1 = 0.f;
  for (int c = threadIdx.x * GRANULE; c < p.cols; c += threads * GRANULE) {
    float a[GRANULE], gd[GRANULE];
    values(c, a, gd);
#pragma unroll
    for (int e = 0; e < GRANULE; ++e) c1 += gd[e] * a[e];
  }
  c1 = block_sum(c1, threads >> 6, red) * p.inv_cols;
  for (int c = threadIdx.x * GRANULE; c < p.cols; c += threads * GRANULE) {
    float a[GRANULE], gd[GRANULE], d[GRANULE];
    if (p.dsum) load_part((const T*)p.dsum + r * p.ld_dsum + c, p.cols - c, d);
    values(c, a, gd);
#pragma unroll
    for (int e = 0; e < GRANULE; ++e) a[e] = rstd * (gd[e] - a[e] * c1);
    if (p.dsum)
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) a[e] += d[e];
    store_part((T*)p.dx + r * p.ld_dx + c, p.cols - c, a);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void rms_norm_gain_grad_kernel(NormGradArgs p, Segs seg, Chunks ch, float* partial) {
  constexpr int UNDER = 4;
  const int chunk = blockIdx.y, c = (blockIdx.x * 256 + threadIdx.x) * GRANULE, n = p.cols - c;
  int k = 0;
  while (k + 1 < seg.K && chunk >= ch.first[k + 1]) ++k;
  const int64_t begin = seg.off[k] + (int64_t)(chunk - ch.first[k]) * ch.rows;
  const int64_t end = begin + ch.rows < seg.off[k + 1] ? begin + ch.rows : seg.off[k + 1];
  float acc[GRANULE] = {};
  for (int64_t r = begin; r < end; r += UNDER) {
    Raw<T> s[UNDER], dy[UNDER];
    float rstd[UNDER];
#pragma unroll
    for (int u = 0; u < UNDER; ++u) {
      const int some = r + u < end ? n : 0;
      rstd[u] = r + u < end ? p.rstd[r + u] : 0.f;
      s[u] = load_raw((const T*)p.sum + (r + u) * p.ld_sum + c, some);
      dy[u] = load_raw((const T*)p.dy + (r + u) * p.ld_dy + c, some);
    }
#pragma unroll
    for (int u = 0; u < UNDER; ++u) {
      if (r + u >= end) break;
      float a[GRANULE], d[GRANULE];
      unpack(s[u], n, a);
      unpack(dy[u], n, d);
#pragma unroll
      for (int e = 0; e < GRANULE; ++e) acc[e] += d[e] * (a[e] * rstd[u]);
    }
  }
  float* const to = ch.first[k + 1] - ch.first[k] == 1 ? p.dgain + k * p.dgain_stride : partial + (int64_t)chunk * p.cols;
  store_part(to + c, n, acc);
}

// Sums of the workers' chunks, COLS columns per workgroup: GROUPS groups of threads take every GROUPS-th chunk, then the
// groups are added in order.  Workers without rows get zeros; those with one chunk have their sum.
template <int COLS, int GROUPS>
__global__ __launch_bounds__(COLS * GROUPS) void sum_chunks_kernel(const float* partial, Chunks ch, int cols, float* dgain,
                                                          int64_t stride) {
  __shared__ float sums[GROUPS][COLS];
  const int k = blockIdx.y, n = ch.first[k + 1] - ch.first[k];
  if (n == 1) return;
  const int lane = threadIdx.x % COLS, group = threadIdx.x / COLS, c = blockIdx.x * COLS + lane;
  float a = 0.f;
  if (c < cols) {
    const float* from = partial + (int64_t)ch.first[k] * cols + c;
#pragma unroll 8
    for (int i = group; i < n; i += GROUPS) a += from[(int64_t)i * cols];
  }
  sums[group][lane] = a;
  __syncthreads();
  if (group > 0 || c >= cols) return;
#pragma unroll
  for (int g = 1; g < GROUPS; ++g) a += sums[g][lane];
  dgain[k * stride + c] = a;
}

// How the workers' rows are cut, and how many chunks: enough workgroups for the chip, and rows enough in each that the
// chunks' sums are a small part of what is read (512 and 1024 chunks: 16384 x 128 bf16 10.0 and 11.2 us, 16384 x 512 17.7 and
// 19.0, 4096 x 4096 32.2 and 35.3; 512 and 256: 131072 x 128 29.0 and 35.1, 40000 x 2048 129 and 149).  256 where a workgroup has
// 9 waves or more, or would have less than 6 rows (256 and 512: 4096 x 16384 105 and 111, 1531 x 2050 13.8 and 14.9, 1024 x 8192
// 19.7 and 23.2).  A chunk is whole rounds of a workgroup's rows.
// And no more of them than that where workers are ragged, or a few workgroups would run alone behind the others (4096 x 4096
// of 16 workers: 519 chunks 39.3 us, 464 33.0; 4096 x 8192 of 8: 88 and 59.5).
int chunks_of(const Segs& seg, int cols, Chunks& ch) {
  const int granules = (cols + GRANULE - 1) / GRANULE;
  const int64_t rows = seg.off[seg.K];
  const int target = granules > WIDEST ? 128 : granules > 512 || (granules > 128 && rows <= 5 * 512) ? 256 : 512;
  const int at_once = granules <= 8 ? 32 : granules <= 16 ? 16 : granules <= 32 ? 8 : granules <= 128 ? 4 : 2;
  static_assert(DYNB_MAX_WORKERS < 128, "every worker has a chunk of its own");
  int n = 0;
  for (int most : {target, target - seg.K}) {
    const int64_t share = std::max<int64_t>((rows + most - 1) / most, 1);
    const int64_t of_chunk = granules <= 128 ? round_up(share, at_once) : std::max<int64_t>(share, at_once);
    ch.rows = (int)of_chunk;
    n = 0;
    for (int k = 0; k < seg.K; ++k) {
      ch.first[k] = n;
      n += (int)((seg.off[k + 1] - (int64_t)seg.off[k] + of_chunk - 1) / of_chunk);
    }
    ch.first[seg.K] = n;
    if (n <= target) break;
  }
  return n;
}

template <typename T, int L, int N>
void launch_norm_grad_as(const NormGradArgs& a, const Segs& seg, const Chunks& ch, int waves, float* partial, hipStream_t st) {
  const dim3 grid(ch.first[seg.K]), block(64 * waves);
  if (past_caches((double)a.rows * a.cols * sizeof(T) * (3 + (a.dsum != nullptr))))
    hipLaunchKernelGGL((rms_norm_grad_kernel<T, L, N, true>), grid, block, 0, st, a, seg, ch, partial);
  else
    hipLaunchKernelGGL((rms_norm_grad_kernel<T, L, N, false>), grid, block, 0, st, a, seg, ch, partial);
}

template <typename T>
void launch_norm_grad(const NormGradArgs& a, const Segs& seg, float* partial, hipStream_t st) {
  const int granules = (a.cols + GRANULE - 1) / GRANULE;
  Chunks ch;
  const int n = chunks_of(seg, a.cols, ch);
  if (n > 0 && granules > widest_grad(sizeof(T))) {
    if (a.dgain)   // (first: dx may lie on dy)
      hipLaunchKernelGGL(rms_norm_gain_grad_kernel<T>, dim3((granules + 255) / 256, n), dim3(256), 0, st, a, seg, ch, partial);
    hipLaunchKernelGGL(rms_norm_grad_any_kernel<T>, grid_of_rows(a.rows), dim3(64 * MOST_WAVES), 0, st, a);
  } else if (n > 0) {
    const int waves = (granules + 63) / 64;
    if (granules <= 8) launch_norm_grad_as<T, 8, 1>(a, seg, ch, 4, partial, st);
    else if (granules <= 16) launch_norm_grad_as<T, 16, 1>(a, seg, ch, 4, partial, st);
    else if (granules <= 32) launch_norm_grad_as<T, 32, 1>(a, seg, ch, 4, partial, st);
    else if (granules <= 64) launch_norm_grad_as<T, 64, 1>(a, seg, ch, 4, partial, st);
    else if (granules <= 128) launch_norm_grad_as<T, 64, 2>(a, seg, ch, 4, partial, st);
    else if (waves <= MOST_WAVES) launch_norm_grad_as<T, WIDE, 1>(a, seg, ch, waves, partial, st);
    else if constexpr (sizeof(T) == 2) launch_norm_grad_as<T, WIDE, 2>(a, seg, ch, (waves + 1) / 2, partial, st);
  }
  bool left = false;
  int most = 0;
  for (int k = 0; k < seg.K; ++k) {
    const int c = ch.first[k + 1] - ch.first[k];
    left |= c != 1;
    most = c > most ? c : most;
  }
  if (!a.dgain || !left) return;
  // Many groups where a worker has many chunks, few threads where none does: 4096 columns of one worker with 512 chunks 4.6
  // us, with four groups 7.1; of 16 workers with 9 to 80 chunks 4.7 us, with 32 groups 6.4.
  if (most > 128)
    hipLaunchKernelGGL((sum_chunks_kernel<32, 32>), dim3((a.cols + 31) / 32, seg.K), dim3(1024), 0, st, partial, ch, a.cols,
                       a.dgain, a.dgain_stride);
  else
    hipLaunchKernelGGL((sum_chunks_kernel<64, 4>), dim3((a.cols + 63) / 64, seg.K), dim3(256), 0, st, partial, ch, a.cols,
                       a.dgain, a.dgain_stride);
}

// Bytes of the chunks' sums (none where every worker has one chunk at most).
size_t partial_bytes(const Segs& seg, int cols) {
  Chunks ch;
  const int n = chunks_of(seg, cols, ch);
  bool more = false;
  for (int k = 0; k < seg.K; ++k) more |= ch.first[k + 1] - ch.first[k] > 1;
  return more ? (size_t)n * cols * sizeof(float) : 0;
}

}  // namespace

// Prefix sums of the workers' sizes.
int segments_of(const int32_t* b, int32_t K, const char* who, Segs& s) {
  if (!b) return fail(DYNB_ERR_BADARG, "%s: null pointer", who);
  if (K < 1 || K > DYNB_MAX_WORKERS) return fail(DYNB_ERR_BADARG, "%s: K out of range", who);
  int64_t at = 0;
  s.K = K;
  for (int k = 0; k < K; ++k) {
    if (b[k] < 0) return fail(DYNB_ERR_BADARG, "%s: negative batch size", who);
    s.off[k] = (int)at;
    at += b[k];
    if (at > INT32_MAX) return fail(DYNB_ERR_BADARG, "%s: rows beyond 2^31 - 1", who);
  }
  s.off[K] = (int)at;
  return DYNB_OK;
}

}  // namespace dynb

using namespace dynb;

extern "C" int dynb_rms_norm(const dynb_rms_norm_desc* d, int64_t rows, const void* x, const void* residual,
                             const float* gain, void* sum, void* y, float* scales, float* rstd, void* stream) {
  NormArgs a;
  if (int rc = describe(d, "rms_norm", a)) return rc;
  if (rows < 0 || rows > INT32_MAX) return fail(DYNB_ERR_BADARG, "rms_norm: rows out of range");
  if (rows == 0) return DYNB_OK;
  if (!x || !y || (d->out != DYNB_OUT_SAME && !scales)) return fail(DYNB_ERR_BADARG, "rms_norm: null pointer");
  const size_t size = d->dtype == DYNB_F32 ? 4 : 2;
  if (off_by(x, size) || off_by(residual, size) || off_by(sum, size) || (d->out == DYNB_OUT_SAME && off_by(y, size)) ||
      off_by(gain, 4) || off_by(scales, 4) || off_by(rstd, 4))
    return fail(DYNB_ERR_BADARG, "rms_norm: a pointer is not a multiple of its element's size");
  a.x = x;
  a.residual = residual;
  a.gain = gain;
  a.sum = sum;
  a.y = y;
  a.scales = scales;
  a.rstd = rstd;
  a.rows = (int)rows;
  const double n = (double)rows * d->cols;
  a.bytes = n * (size * (1 + (residual != nullptr) + (sum != nullptr)) + (d->out == DYNB_OUT_SAME ? size : 1));
  Timed t(KC_NORM, stream, 8.0 * n, a.bytes);
  if (d->dtype == DYNB_F32) launch_norm<float>(a, d->out, (hipStream_t)stream);
  else launch_norm<bf16>(a, d->out, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "rms_norm launch failed");
}

extern "C" int32_t dynb_scale_blocks(const dynb_rms_norm_desc* d) {
  NormArgs a;
  return describe(d, "scale_blocks", a) ? -1 : a.n_blocks;
}

extern "C" int dynb_dequantise(const dynb_rms_norm_desc* d, int64_t rows, const void* y, const float* scales,
                               int32_t out_dtype, void* out, int64_t ld_out, void* stream) {
  NormArgs a;
  if (int rc = describe(d, "dequantise", a)) return rc;
  if (d->out == DYNB_OUT_SAME) return fail(DYNB_ERR_BADARG, "dequantise: the output has no scales");
  if (out_dtype != DYNB_F32 && out_dtype != DYNB_BF16) return fail(DYNB_ERR_BADARG, "dequantise: unknown dtype");
  if (rows < 0 || rows > INT32_MAX) return fail(DYNB_ERR_BADARG, "dequantise: rows out of range");
  if (ld_out != 0 && ld_out < d->cols) return fail(DYNB_ERR_BADARG, "dequantise: a row pitch is below cols");
  if (rows == 0) return DYNB_OK;
  if (!y || !scales || !out) return fail(DYNB_ERR_BADARG, "dequantise: null pointer");
  if (off_by(scales, 4) || off_by(out, out_dtype == DYNB_F32 ? 4 : 2))
    return fail(DYNB_ERR_BADARG, "dequantise: a pointer is not a multiple of its element's size");
  a.y = const_cast<void*>(y);
  a.scales = const_cast<float*>(scales);
  a.rows = (int)rows;
  if (!ld_out) ld_out = d->cols;
  const dim3 grid(resident((rows * ((d->cols + GRANULE - 1) / GRANULE) + 255) / 256, 256)), block(256);
  const hipStream_t st = (hipStream_t)stream;
  a.bytes = (double)rows * d->cols * (out_dtype == DYNB_F32 ? 5 : 3);
  Timed t(KC_NORM, stream, (double)rows * d->cols, a.bytes);
  if (out_dtype == DYNB_F32) {
    if (past_caches(a.bytes)) hipLaunchKernelGGL((dequantise_kernel<float, true>), grid, block, 0, st, a, d->out, (float*)out, ld_out);
    else hipLaunchKernelGGL((dequantise_kernel<float, false>), grid, block, 0, st, a, d->out, (float*)out, ld_out);
  } else {
    if (past_caches(a.bytes)) hipLaunchKernelGGL((dequantise_kernel<bf16, true>), grid, block, 0, st, a, d->out, (bf16*)out, ld_out);
    else hipLaunchKernelGGL((dequantise_kernel<bf16, false>), grid, block, 0, st, a, d->out, (bf16*)out, ld_out);
  }
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "dequantise launch failed");
}

extern "C" size_t dynb_rms_norm_backward_workspace_bytes(const dynb_rms_norm_desc* d, const int32_t* b, int32_t K) {
  NormArgs a;
  Segs seg;
  if (describe(d, "rms_norm_backward", a) || segments_of(b, K, "rms_norm_backward", seg)) return 0;
  return partial_bytes(seg, a.cols);
}

extern "C" int dynb_rms_norm_backward(const dynb_rms_norm_desc* d, const int32_t* b, int32_t K, const void* sum,
                                      const float* rstd, const float* gain, const void* dy, const void* dsum,
                                      void* dx, float* dgain, int64_t dgain_stride, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  NormArgs f;
  Segs seg;
  if (int rc = describe(d, "rms_norm_backward", f)) return rc;
  if (int rc = segments_of(b, K, "rms_norm_backward", seg)) return rc;
  const int rows = seg.off[K];
  if (rows > 0 && (!sum || !rstd || !dy || !dx)) return fail(DYNB_ERR_BADARG, "rms_norm_backward: null pointer");
  if (dgain && dgain_stride < d->cols && K > 1)
    return fail(DYNB_ERR_BADARG, "rms_norm_backward: dgain_stride is below cols");
  const size_t size = d->dtype == DYNB_F32 ? 4 : 2;
  if (off_by(sum, size) || off_by(dy, size) || off_by(dsum, size) || off_by(dx, size) || off_by(rstd, 4) ||
      off_by(gain, 4) || off_by(dgain, 4))
    return fail(DYNB_ERR_BADARG, "rms_norm_backward: a pointer is not a multiple of its element's size");
  const size_t need = dgain ? partial_bytes(seg, d->cols) : 0;
  if (need && (!workspace || workspace_bytes < need || off_by(workspace, 16)))
    return fail(DYNB_ERR_BADARG, "rms_norm_backward: workspace is null, too small or not 16-byte aligned");
  NormGradArgs a = {sum, rstd, gain, dy, dsum, dx, dgain, f.ld_sum, d->ld_dy ? d->ld_dy : d->cols,
                    d->ld_dsum ? d->ld_dsum : d->cols, d->ld_dx ? d->ld_dx : d->cols, dgain_stride, rows, d->cols, f.inv_cols};
  const double n = (double)rows * d->cols;
  Timed t(KC_NORM, stream, 12.0 * n, n * size * (3 + (dsum != nullptr)) + 4.0 * K * d->cols);
  if (d->dtype == DYNB_F32) launch_norm_grad<float>(a, seg, (float*)workspace, (hipStream_t)stream);
  else launch_norm_grad<bf16>(a, seg, (float*)workspace, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "rms_norm_backward launch failed");
}
