// What follows the products of dense and gated layers, on 8 neighbouring results of a row, and their launches.
#ifndef DYNB_PRODUCT_EPILOGUES_H
#define DYNB_PRODUCT_EPILOGUES_H

#include "tile_product.h"

namespace dynb {

// act(v) and its derivative, in fp32.
//   silu  v p, p = 1 / (1 + e^-v);             p (1 + v (1 - p))
//   gelu  v P, P = (1 + erf(v / sqrt 2)) / 2;  P + v e^(-v^2 / 2) / sqrt(2 pi)
// (where v's magnitude is beyond an exponential's range p and P are 0 or 1, and the products with 0 vanish.)  Values that are
// rounded to 16 bits take the hardware's exponential and reciprocal and erf by Abramowitz and Stegun 7.1.26
// (off by 1.5e-7 at most), which shares its exponential with gelu's derivative.
template <typename T> struct Curve {
  static constexpr bool SHORT = sizeof(T) == 2;
  static __device__ float power(float v) { return SHORT ? __expf(v) : expf(v); }
  static __device__ float inverse(float v) { return SHORT ? __builtin_amdgcn_rcpf(v) : 1.f / v; }
  // P, and e^(-v^2 / 2)
  static __device__ float normal(float v, float& bell) {
    bell = power(-0.5f * v * v);
    if (!SHORT) return 0.5f + 0.5f * erff(v * 0.70710678f);
    const float t = inverse(1.f + 0.3275911f * 0.70710678f * fabsf(v));
    const float tail = 0.5f * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f)))) * bell;
    return v < 0.f ? tail : 1.f - tail;
  }
  static __device__ float value(int act, float v) {
    float slope;
    return both(act, v, slope);
  }
  static __device__ float both(int act, float v, float& slope) {
    switch (act) {
      case DYNB_ACT_RELU:
        slope = v > 0.f ? 1.f : 0.f;
        return v < 0.f ? 0.f : v;            // (a NaN stays one)
      case DYNB_ACT_SILU: {
        const float p = inverse(1.f + power(-v));
        slope = p * (1.f + v * (1.f - p));
        return v * p;
      }
      case DYNB_ACT_GELU: {
        float bell;
        const float p = normal(v, bell);
        slope = p + v * bell * 0.39894228f;
        return v * p;
      }
      default:
        slope = 1.f;
        return v;
    }
  }
};

// out = act(v + bias) + residual; what the activation is taken of can be kept
template <typename T> struct LinearOut {
  static constexpr int ROWS_AT_ONCE = 4;
  const float* bias;
  const T* residual; int64_t ld_residual;
  T* pre; int64_t ld_pre;
  T* out; int64_t ld_out;
  int act;
  __device__ void row(int, int64_t i, int col, int n, float (&v)[8], float (&)[8]) const {
    if (bias) {
      float b[8];
      load_part(bias + col, n, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += b[e];
    }
    if (pre) store_part(pre + i * ld_pre + col, n, v);
    if (act != DYNB_ACT_NONE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = Curve<T>::value(act, v[e]);
    }
    if (residual) {
      float r[8];
      load_part(residual + i * ld_residual + col, n, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
    store_part(out + i * ld_out + col, n, v);
  }
};

// hidden = act(gate) * up, from the sums before they are rounded
template <typename T> struct GatedOut {
  static constexpr int ROWS_AT_ONCE = 4;
  T* gate; T* up;             // or null: not kept
  int64_t ld_kept;
  T* hidden; int64_t ld_hidden;
  int act;
  __device__ void row(int, int64_t i, int col, int n, float (&v)[8], float (&w)[8]) const {
    if (gate) {
      store_part(gate + i * ld_kept + col, n, v);
      store_part(up + i * ld_kept + col, n, w);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = Curve<T>::value(act, v[e]) * w[e];
    store_part(hidden + i * ld_hidden + col, n, v);
  }
};

// from v = gradient of hidden: dgate = v up act'(gate), dup = v act(gate), and hidden once more
template <typename T> struct GatedGrad {
  static constexpr int ROWS_AT_ONCE = 1;
  const T* gate; const T* up;
  int64_t ld_kept;
  T* dgate; T* dup; T* hidden;
  int64_t ld_hidden;
  int act;
  __device__ void row(int, int64_t i, int col, int n, float (&v)[8], float (&)[8]) const {
    float g[8], u[8], a[8], b[8];
    load_part(gate + i * ld_kept + col, n, g);
    load_part(up + i * ld_kept + col, n, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float slope;
      const float value = Curve<T>::both(act, g[e], slope);
      a[e] = v[e] * u[e] * slope;
      g[e] = value;
      b[e] = v[e] * g[e];
      u[e] *= g[e];
    }
    store_part(dgate + i * ld_hidden + col, n, a);
    store_part(dup + i * ld_hidden + col, n, b);
    store_part(hidden + i * ld_hidden + col, n, u);
  }
};

// gradients of one or two weights: group e * workers + k is worker k's of matrix e
template <typename O> struct WeightOut {
  static constexpr int ROWS_AT_ONCE = 4;
  O* out[2];
  int64_t worker_stride, matrix;
  int workers, cols;
  __device__ void row(int group, int64_t i, int col, int n, float (&v)[8], float (&w)[8]) const {
    const int64_t to = group % workers * worker_stride + group / workers * matrix + i * cols + col;
    store_part(out[0] + to, n, v);
    if (out[1]) store_part(out[1] + to, n, w);
  }
};

// How a product is cut into tiles and its reduction into parts.
enum Tiles { TILES_256, TILES_128, TILES_32 };
struct ProductPlan {
  Tiles tiles;
  int splits;
};

// (instantiated once per type and form: products_*.hip.  T: type of the rows and weights, O: of the weights' gradients)
template <typename T> int launch_linear(const Product& p, Tiles tiles, bool turned, const LinearOut<T>& ep, void* stream);
template <typename T> int launch_gated(const Product& p, Tiles tiles, const GatedOut<T>& ep, void* stream);
template <typename T> int launch_gated_grad(const Product& p, Tiles tiles, const GatedGrad<T>& ep, void* stream);
template <typename T, typename O>
int launch_weights(const Product& p, Tiles tiles, const Segs& s, const WeightOut<O>& ep, void* stream);


namespace {

template <typename T> bool whole_granules(int64_t v) { return v % (16 / (int)sizeof(T)) == 0; }
inline bool near(int64_t ld, size_t size) { return ld * (int64_t)size * 256 < ((int64_t)1 << 31); }

// Whether all of an operand's copies are whole granules at multiples of 16 bytes, and 32-bit offsets reach a stage.
template <typename T> bool direct_ok(const Product& p, int form) {
  for (int q = 0; q < 2; ++q)
    if (off_by(p.A[q], 16) || off_by(p.B[q], 16)) return false;
  return whole_granules<T>(p.lda) && whole_granules<T>(p.ldb) && whole_granules<T>(p.b_stride) && near(p.lda, sizeof(T)) &&
         near(p.ldb, sizeof(T)) && (form == ROWS_NT || whole_granules<T>(p.N)) &&
         (form == WEIGHTS ? whole_granules<T>(p.M) : whole_granules<T>(p.K));
}

template <typename T, int FORM, bool DUAL, int BM, int BN, int WM, int WN, int NB, int SOON, Access ACCESS, class Ep>
int launch_tiles(const Product& p, const Segs& s, const Ep& ep, hipStream_t st) {
  constexpr int BNS = DUAL ? BN / 2 : BN;
  const int64_t tiles_j = (p.N + BNS - 1) / BNS;
  int64_t blocks;
  if (FORM == WEIGHTS) blocks = weight_places((p.M + BM - 1) / BM * tiles_j) * p.groups;
  else blocks = (p.offsets ? p.rows / BM + (p.rows < p.groups ? p.rows : p.groups) : (p.rows + BM - 1) / BM) * tiles_j;
  if (blocks > INT32_MAX / 64) return fail(DYNB_ERR_UNSUPPORTED, "a product of more than 2^25 tiles");
  hipLaunchKernelGGL((product_kernel<T, FORM, DUAL, BM, BN, WM, WN, NB, SOON, ACCESS, Ep>), dim3((unsigned)blocks, p.splits),
                     dim3(WM * WN * 64), 0, st, p, s, ep);
  if (p.splits > 1) {
    const int64_t n = p.partial_rows * ((p.N + 7) / 8);
    hipLaunchKernelGGL((joined_kernel<FORM, DUAL, Ep>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, p, ep);
  }
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "launch of a product failed");
}

template <typename T, int FORM, bool DUAL, class Ep>
int launch_as(const Product& p, Tiles tiles, const Segs& s, const Ep& ep, void* stream) {
  const hipStream_t st = (hipStream_t)stream;
  const bool direct = direct_ok<T>(p, FORM);
  // (rows of less than a granule: nothing to shift)
  const bool singly = (FORM == WEIGHTS ? p.M : p.K) < 16 / (int)sizeof(T) || (FORM != ROWS_NT && p.N < 16 / (int)sizeof(T));
  if constexpr (FORM != WEIGHTS) {
    constexpr int WN = DUAL ? 2 : 4;
    if (singly) return launch_tiles<T, FORM, DUAL, 32, 128, 1, WN, 4, 2, SINGLY>(p, s, ep, st);
    if (tiles == TILES_32)
      return direct ? launch_tiles<T, FORM, DUAL, 32, 128, 1, WN, 4, 2, DIRECT>(p, s, ep, st)
                    : launch_tiles<T, FORM, DUAL, 32, 128, 1, WN, 4, 2, SHIFTED>(p, s, ep, st);
  } else {
    if (singly) return launch_tiles<T, FORM, DUAL, 128, 128, 4, 2, 4, 2, SINGLY>(p, s, ep, st);
  }
  if (!direct) return launch_tiles<T, FORM, DUAL, 128, 128, 4, 2, 4, 2, SHIFTED>(p, s, ep, st);
  if constexpr (sizeof(T) == 2)
    if (tiles == TILES_256) return launch_tiles<T, FORM, DUAL, 256, 256, 2, 4, 2, 4, DIRECT>(p, s, ep, st);
  return launch_tiles<T, FORM, DUAL, 128, 128, 4, 2, 4, 2, DIRECT>(p, s, ep, st);
}

}  // namespace
}  // namespace dynb

#endif
