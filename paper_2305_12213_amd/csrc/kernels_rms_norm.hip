// Root-mean-square norm with the residual's addition, its 8-bit outputs, and its gradients.
#include <hip/hip_runtime.h>

#include <cmath>

#include "dynb_internal.h"
#include "row_access.h"

namespace dynb {
namespace {

constexpr float FP8_TOP = 448.f, INT8_TOP = 127.f;
constexpr int MAX_COLS = 1 << 20;

struct NormArgs {
  const void *x, *residual;
  const float* gain;
  void *sum, *y;
  float *scales, *rstd;
  int64_t ld_x, ld_residual, ld_sum, ld_y;
  int rows, cols, scale_block, n_blocks;
  float eps;
};

// One value in 8 bits.  (An 8-bit block that holds an infinity or NaN has factor 0: 0 * inf is kept out.)
template <int OUT> __device__ inline uint8_t eight_bits(float v, float inv) {
  const float t = inv > 0.f ? v * inv : 0.f;
  if (OUT == DYNB_OUT_INT8) return (uint8_t)(int8_t)rintf(t);
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(t, t, 0, false) & 0xff);
}

// 1 / sqrt(mean + eps) from the sum of squares; where that has overflowed, from the squares of the row times 2^-80,
// which `scaled_sum` gives (eps is nothing beside them; a row with an infinity or NaN ends the same either way).
template <typename F> __device__ inline float rstd_of(float ss, int cols, float eps, F scaled_sum) {
  if (ss <= 3.4e38f) return 1.f / sqrtf(ss / (float)cols + eps);
  return 0x1p-80f / sqrtf(scaled_sum() / (float)cols);
}

// Rows of any width, a workgroup per row that reads it two or three times.
template <typename T, int OUT>
__global__ __launch_bounds__(256) void rms_norm_any_kernel(NormArgs p) {
  __shared__ float red[4];
  __shared__ uint32_t redu[4];
  constexpr float TOP = OUT == DYNB_OUT_FP8 ? FP8_TOP : INT8_TOP;
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* x = (const T*)p.x + r * p.ld_x;
    const T* res = p.residual ? (const T*)p.residual + r * p.ld_residual : nullptr;
    T* sum = p.sum ? (T*)p.sum + r * p.ld_sum : nullptr;
    auto value = [&](int c) { return to_float(x[c]) + (res ? to_float(res[c]) : 0.f); };
    float ss = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += 256) {
      const float s = value(c);
      ss += s * s;
    }
    ss = block_sum<4>(ss, red);
    const float rstd = rstd_of(ss, p.cols, p.eps, [&]() {
      float a = 0.f;
      for (int c = threadIdx.x; c < p.cols; c += 256) {
        const float s = value(c) * 0x1p-80f;
        a += s * s;
      }
      return block_sum<4>(a, red);
    });
    if (threadIdx.x == 0 && p.rstd) p.rstd[r] = rstd;
    auto result = [&](float s, int c) { return s * rstd * (p.gain ? p.gain[c] : 1.f); };
    if (OUT == DYNB_OUT_SAME) {
      for (int c = threadIdx.x; c < p.cols; c += 256) {
        const float s = value(c);
        if (sum) sum[c] = (T)s;
        ((T*)p.y)[r * p.ld_y + c] = (T)result(s, c);
      }
      continue;
    }
    // (the lane that reads an element for the block's largest is the one that stores it: outputs may lie on inputs)
    const bool whole = p.n_blocks == 1;
    const int lane = whole ? threadIdx.x : threadIdx.x & 63, lanes = whole ? 256 : 64;
    for (int b = whole ? 0 : threadIdx.x >> 6; b < p.n_blocks; b += whole ? 1 : 4) {
      const int c0 = b * p.scale_block, c1 = min(c0 + p.scale_block, p.cols);
      uint32_t a = 0;
      for (int c = c0 + lane; c < c1; c += lanes) a = max(a, __float_as_uint(result(value(c), c)) & 0x7fffffffu);
      a = whole ? block_max<4>(a, redu) : wave_max(a);
      const Scale s = scale_of(a, TOP);
      if (lane == 0) p.scales[r * p.n_blocks + b] = s.scale;
      for (int c = c0 + lane; c < c1; c += lanes) {
        const float v = value(c);
        if (sum) sum[c] = (T)v;
        ((uint8_t*)p.y)[r * p.ld_y + c] = eight_bits<OUT>(result(v, c), s.inv);
      }
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
};

template <typename T>
__global__ __launch_bounds__(256) void rms_norm_grad_any_kernel(NormGradArgs p) {
  __shared__ float red[4];
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T *s = (const T*)p.sum + r * p.ld_sum, *dy = (const T*)p.dy + r * p.ld_dy;
    const T* dsum = p.dsum ? (const T*)p.dsum + r * p.ld_dsum : nullptr;
    T* dx = (T*)p.dx + r * p.ld_dx;
    const float rstd = p.rstd[r];
    float c1 = 0.f;
    for (int c = threadIdx.x; c < p.cols; c += 256)
      c1 += (p.gain ? p.gain[c] : 1.f) * to_float(dy[c]) * (to_float(s[c]) * rstd);
    c1 = block_sum<4>(c1, red) / (float)p.cols;
    for (int c = threadIdx.x; c < p.cols; c += 256) {
      const float g = (p.gain ? p.gain[c] : 1.f) * to_float(dy[c]);
      dx[c] = (T)(rstd * (g - to_float(s[c]) * rstd * c1) + (dsum ? to_float(dsum[c]) : 0.f));
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void rms_norm_gain_grad_kernel(NormGradArgs p, Segs seg) {
  const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.y;
  if (c >= p.cols) return;
  float a = 0.f;
  for (int64_t r = seg.off[k]; r < seg.off[k + 1]; ++r)
    a += to_float(((const T*)p.dy)[r * p.ld_dy + c]) * (to_float(((const T*)p.sum)[r * p.ld_sum + c]) * p.rstd[r]);
  p.dgain[k * p.dgain_stride + c] = a;
}

template <typename T>
__global__ __launch_bounds__(256) void dequantise_kernel(NormArgs p, int out, T* to, int64_t ld_to) {
  for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x)
    for (int c = threadIdx.x; c < p.cols; c += 256) {
      const uint8_t q = ((const uint8_t*)p.y)[r * p.ld_y + c];
      const float v = out == DYNB_OUT_INT8 ? (float)(int8_t)q : __builtin_amdgcn_cvt_f32_fp8(q, 0);
      to[r * ld_to + c] = (T)(v * p.scales[r * p.n_blocks + (p.n_blocks == 1 ? 0 : c / p.scale_block)]);
    }
}

int grid_of_rows(int64_t rows) { return (int)(rows < (1 << 20) ? rows : 1 << 20); }

bool off_by(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

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
  a.scale_block = d->scale_block && d->scale_block < d->cols ? d->scale_block : d->cols;
  a.n_blocks = d->out == DYNB_OUT_SAME ? 0 : (d->cols + a.scale_block - 1) / a.scale_block;
  return DYNB_OK;
}

template <typename T> void launch_norm(const NormArgs& a, int out, hipStream_t st) {
  const dim3 grid(grid_of_rows(a.rows)), block(256);
  if (out == DYNB_OUT_SAME) hipLaunchKernelGGL((rms_norm_any_kernel<T, DYNB_OUT_SAME>), grid, block, 0, st, a);
  else if (out == DYNB_OUT_FP8) hipLaunchKernelGGL((rms_norm_any_kernel<T, DYNB_OUT_FP8>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rms_norm_any_kernel<T, DYNB_OUT_INT8>), grid, block, 0, st, a);
}

template <typename T> void launch_norm_grad(const NormGradArgs& a, const Segs& seg, hipStream_t st) {
  if (a.dgain)   // (first: dx may lie on dy)
    hipLaunchKernelGGL(rms_norm_gain_grad_kernel<T>, dim3((a.cols + 255) / 256, seg.K), dim3(256), 0, st, a, seg);
  if (a.rows) hipLaunchKernelGGL(rms_norm_grad_any_kernel<T>, dim3(grid_of_rows(a.rows)), dim3(256), 0, st, a);
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
  Timed t(KC_NORM, stream, 8.0 * n,
          n * (size * (1 + (residual != nullptr) + (sum != nullptr)) + (d->out == DYNB_OUT_SAME ? size : 1)));
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
  const dim3 grid(grid_of_rows(rows)), block(256);
  Timed t(KC_NORM, stream, (double)rows * d->cols, (double)rows * d->cols * (out_dtype == DYNB_F32 ? 5 : 3));
  if (out_dtype == DYNB_F32)
    hipLaunchKernelGGL(dequantise_kernel<float>, grid, block, 0, (hipStream_t)stream, a, d->out, (float*)out, ld_out);
  else
    hipLaunchKernelGGL(dequantise_kernel<bf16>, grid, block, 0, (hipStream_t)stream, a, d->out, (bf16*)out, ld_out);
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "dequantise launch failed");
}

extern "C" size_t dynb_rms_norm_backward_workspace_bytes(const dynb_rms_norm_desc* d, const int32_t* b, int32_t K) {
  NormArgs a;
  Segs seg;
  if (describe(d, "rms_norm_backward", a) || segments_of(b, K, "rms_norm_backward", seg)) return 0;
  return 0;
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
  (void)workspace;
  (void)workspace_bytes;
  NormGradArgs a = {sum, rstd, gain, dy, dsum, dx, dgain, f.ld_sum, d->ld_dy ? d->ld_dy : d->cols,
                    d->ld_dsum ? d->ld_dsum : d->cols, d->ld_dx ? d->ld_dx : d->cols, dgain_stride, rows, d->cols};
  const double n = (double)rows * d->cols;
  Timed t(KC_NORM, stream, 12.0 * n, n * size * (3 + (dsum != nullptr)) + 4.0 * K * d->cols);
  if (d->dtype == DYNB_F32) launch_norm_grad<float>(a, seg, (hipStream_t)stream);
  else launch_norm_grad<bf16>(a, seg, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "rms_norm_backward launch failed");
}
