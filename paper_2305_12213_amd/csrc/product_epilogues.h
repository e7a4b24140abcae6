// What follows the products of dense and gated layers, on 8 neighbouring results of a row, and their launches.  Where memory has to
// take them, epilogues are not hidden: 4096^3 alone 115 us, with bias, GELU, residual and the kept pre-activation (100 MB more) 142.
#ifndef DYNB_PRODUCT_EPILOGUES_H
#define DYNB_PRODUCT_EPILOGUES_H

#include <algorithm>

#include "tile_product.h"

namespace dynb {

// act(v) and its derivative, in fp32.
//   silu  v p, p = 1 / (1 + e^-v);             p (1 + v (1 - p))
//   gelu  v P, P = (1 + erf(v / sqrt 2)) / 2;  P + v e^(-v^2 / 2) / sqrt(2 pi)
// (where v's magnitude is beyond an exponential's range p and P are 0 or 1, and the products with 0 vanish; an infinite v is the
// largest finite one in them, which gives the limits, and a NaN stays one by p and P.)  Values that are
// rounded to 16 bits take the hardware's exponential and reciprocal and erf by Abramowitz and Stegun 7.1.26
// (off by 1.5e-7 at most), which shares its exponential with gelu's derivative.
template <typename T> struct Curve {
  static constexpr bool SHORT = sizeof(T) == 2;
  static constexpr float MOST = 3.40282347e38f;
  static __device__ float finite(float v) { return __builtin_amdgcn_fmed3f(v, -MOST, MOST); }
  static __device__ float bounded_below(float v) { return __builtin_amdgcn_fmed3f(v, -MOST, __builtin_inff()); }
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
        slope = p * (1.f + finite(v) * (1.f - p));
        return bounded_below(v) * p;
      }
      case DYNB_ACT_GELU: {
        float bell;
        const float p = normal(v, bell);
        slope = p + finite(v) * bell * 0.39894228f;
        return bounded_below(v) * p;
      }
      default:
        slope = 1.f;
        return v;
    }
  }
};

// ask() loads what an epilogue reads for 8 results (n of them, none where n <= 0), row() uses it.  PACKS: where packed() says so,
// results are only rounded to 16 bits, and put() stores 8 of them (of the first or the second product).

// out = act(v + bias) + residual; what the activation is taken of can be kept
template <typename T> struct LinearOut {
  static constexpr bool HEAVY = false;
  static constexpr bool PACKS = sizeof(T) == 2;
  const float* bias;
  const T* residual; int64_t ld_residual;
  T* pre; int64_t ld_pre;
  T* out; int64_t ld_out;
  int act;
  struct Held {
    Raw<T> residual;
  };
  __device__ Held ask(int64_t i, int col, int n) const {
    Held h = {};
    if (residual) h.residual = load_raw(residual + i * ld_residual + col, n);
    return h;
  }
  __device__ void row(int, int64_t i, int col, int n, float (&v)[8], float (&)[8], const Held& h) const {
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
      unpack(h.residual, n, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += r[e];
    }
    store_part(out + i * ld_out + col, n, v);
  }
  __device__ bool packed() const { return !bias && !residual && !pre && act == DYNB_ACT_NONE; }
  __device__ void put(int, int64_t i, int col, int n, const u32x4& v, int) const {
    store_packed((bf16*)out + i * ld_out + col, n, v);
  }
};

struct Nothing {};

// hidden = act(gate) * up, from the sums before they are rounded
template <typename T> struct GatedOut {
  static constexpr bool HEAVY = false;
  static constexpr bool PACKS = false;
  T* gate; T* up;             // or null: not kept
  int64_t ld_kept;
  T* hidden; int64_t ld_hidden;
  int act;
  typedef Nothing Held;
  __device__ Held ask(int64_t, int, int) const { return {}; }
  __device__ void row(int, int64_t i, int col, int n, float (&v)[8], float (&w)[8], Held) const {
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
  static constexpr bool HEAVY = true;
  static constexpr bool PACKS = false;
  const T* gate; const T* up;
  int64_t ld_kept;
  T* dgate; T* dup; T* hidden;
  int64_t ld_hidden;
  int act;
  struct Held {
    Raw<T> gate, up;
  };
  __device__ Held ask(int64_t i, int col, int n) const {
    return {load_raw(gate + i * ld_kept + col, n), load_raw(up + i * ld_kept + col, n)};
  }
  __device__ void row(int, int64_t i, int col, int n, float (&v)[8], float (&)[8], const Held& h) const {
    float g[8], u[8], a[8], b[8];
    unpack(h.gate, n, g);
    unpack(h.up, n, u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float slope;
      const float value = Curve<T>::both(act, g[e], slope);
      a[e] = v[e] * u[e] * slope;
      b[e] = v[e] * value;
      u[e] *= value;
    }
    store_part(dgate + i * ld_hidden + col, n, a);
    store_part(dup + i * ld_hidden + col, n, b);
    store_part(hidden + i * ld_hidden + col, n, u);
  }
};

// gradients of one or two weights: group e * workers + k is worker k's of matrix e; the second weight's groups follow (row) or are
// named by `product` (put)
template <typename O> struct WeightOut {
  static constexpr bool HEAVY = false;
  static constexpr bool PACKS = sizeof(O) == 2;
  O* out[2];
  int64_t worker_stride, matrix;
  int workers, cols, groups;
  bool past;                  // more than the caches keep until it is read: past them
  typedef Nothing Held;
  __device__ Held ask(int64_t, int, int) const { return {}; }
  __device__ void row(int group, int64_t i, int col, int n, float (&v)[8], float (&)[8], Held) const {
    O* const to = out[group / groups] + place(group % groups, i, col);
    if (past) store_part<true>(to, n, v);
    else store_part(to, n, v);
  }
  __device__ bool packed() const { return true; }
  __device__ void put(int group, int64_t i, int col, int n, const u32x4& v, int product) const {
    O* const to = out[product] + place(group, i, col);
    if (past) store_packed<true>((bf16*)to, n, v);
    else store_packed((bf16*)to, n, v);
  }
  __device__ int64_t place(int group, int64_t i, int col) const {
    return group % workers * worker_stride + group / workers * matrix + i * cols + col;
  }
};

// How a product is cut into tiles and its reduction into parts.
enum Tiles { TILES_256, TILES_128, TILES_64, TILES_32, TILES_32X64 };
struct ProductPlan {
  Tiles tiles;
  int splits;
};

// Where a product goes.  launch false: it is only asked whether one launch holds it, so that a call of several products is refused
// before the first of them has written anything.
struct Target {
  hipStream_t stream;
  bool launch;
};

// (instantiated once per type and form: products_*.hip.  T: type of the rows and weights, O: of the weights' gradients)
template <typename T> int launch_linear(const Product& p, Tiles tiles, bool turned, const LinearOut<T>& ep, Target to);
template <typename T> int launch_gated(const Product& p, Tiles tiles, const GatedOut<T>& ep, Target to);
template <typename T> int launch_gated_grad(const Product& p, Tiles tiles, const GatedGrad<T>& ep, Target to);
template <typename T, typename O>
int launch_weights(const Product& p, Tiles tiles, const Segs& s, const WeightOut<O>& ep, Target to);

namespace {

template <typename T> bool whole_granules(int64_t v) { return v % (16 / (int)sizeof(T)) == 0; }
inline bool near(int64_t ld, size_t size) { return ld * (int64_t)size * 256 < ((int64_t)1 << 31); }

// Whether 32-bit offsets reach a stage, and whether all of an operand's copies are whole granules at multiples of 16 bytes.
template <typename T> bool copies_ok(const Product& p) { return near(p.lda, sizeof(T)) && near(p.ldb, sizeof(T)); }
template <typename T> bool direct_ok(const Product& p, int form) {
  for (int q = 0; q < 2; ++q)
    if (off_by(p.A[q], 16) || off_by(p.B[q], 16)) return false;
  return copies_ok<T>(p) && whole_granules<T>(p.lda) && whole_granules<T>(p.ldb) && whole_granules<T>(p.b_stride) &&
         (form == ROWS_NT || whole_granules<T>(p.N)) && (form == WEIGHTS ? whole_granules<T>(p.M) : whole_granules<T>(p.K));
}

template <typename T, int FORM, bool DUAL, int BM, int BN, int WM, int WN, int DEPTH, int NB, int SOON, Access ACCESS, class Ep>
int launch_tiles(const Product& p, const Segs& s, const Ep& ep, Target to) {
  constexpr int BNS = DUAL ? BN / 2 : BN;
  const int64_t tiles_j = (p.N + BNS - 1) / BNS;
  int64_t units;
  if (FORM == WEIGHTS) {
    const int64_t tiles = (p.M + BM - 1) / BM * tiles_j;
    units = (tiles < 1 << 24 ? weight_places((int)tiles) : tiles) * (int64_t)p.groups * p.pairs;
  } else {
    units = (p.offsets ? p.rows / BM + (p.rows < p.groups ? p.rows : p.groups) : (p.rows + BM - 1) / BM) * tiles_j;
  }
  if (units * p.splits > INT32_MAX / (WM * WN * 64)) return fail(DYNB_ERR_UNSUPPORTED, "a product of more than 2^22 tiles");
  if (!to.launch) return DYNB_OK;
  hipLaunchKernelGGL((product_kernel<T, FORM, DUAL, BM, BN, WM, WN, DEPTH, NB, SOON, ACCESS, Ep>), dim3((unsigned)units, p.splits),
                     dim3(WM * WN * 64), 0, to.stream, p, s, ep);
  if (p.splits > 1) {
    const int64_t n = p.partial_rows * ((p.N + 7) / 8);
    hipLaunchKernelGGL((joined_kernel<FORM, DUAL, Ep>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, to.stream, p, ep);
  }
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "launch of a product failed");
}

template <typename T, int FORM, bool DUAL, class Ep>
int launch_as(const Product& p, Tiles tiles, const Segs& s, const Ep& ep, Target to) {
  const bool direct = direct_ok<T>(p, FORM);
  // (rows of less than a granule: nothing to shift)
  const bool singly = (FORM == WEIGHTS ? p.M : p.K) < 16 / (int)sizeof(T) || (FORM != ROWS_NT && p.N < 16 / (int)sizeof(T));
  if constexpr (FORM != WEIGHTS) {
    constexpr int WN = DUAL ? 2 : 4;
    if (singly) return launch_tiles<T, FORM, DUAL, 32, 128, 1, WN, 8, 4, 2, SINGLY>(p, s, ep, to);
    if constexpr (!DUAL)
      // (one token through 4096 x 14336: 24.7 us; on tiles of 128 columns, in four parts and joined, 27.4)
      if (tiles == TILES_32X64 && direct) return launch_tiles<T, FORM, DUAL, 32, 64, 1, 2, 8, 6, 2, DIRECT>(p, s, ep, to);
    if (tiles == TILES_32 || tiles == TILES_32X64)
      return direct ? launch_tiles<T, FORM, DUAL, 32, 128, 1, WN, 8, 4, 2, DIRECT>(p, s, ep, to)
                    : launch_tiles<T, FORM, DUAL, 32, 128, 1, WN, 8, 4, 2, SHIFTED>(p, s, ep, to);
  } else {
    if (singly) return launch_tiles<T, FORM, DUAL, 128, 128, 4, 2, 8, 2, 4, SINGLY>(p, s, ep, to);
  }
  // fp32 with few tiles: smaller ones, of which several share a compute unit and leave less of it idle at the end (gradients of
  // 1531 tokens, 3 of 11 experts, 777 x 301: 294 -> 252 us).  Odd widths: single copies, of shorter stages for gradients of weights,
  // took 1 to 12 % less than shifted granules in all of 30 products but one (odd sizes from 768 to 8192; 1531 x 2050 x 777 72 -> 64
  // us, weights of 8192 tokens, 2047 x 2049 704 -> 627, but of 16 workers 786 -> 812)
  if constexpr (sizeof(T) == 4) {
    constexpr int DEPTH = FORM == WEIGHTS ? 4 : 8;
    if (tiles == TILES_64) {
      constexpr int BN = DUAL ? 128 : 64;
      if (direct) return launch_tiles<T, FORM, DUAL, 64, BN, 2, 2, 8, 2, 4, DIRECT>(p, s, ep, to);
      if (copies_ok<T>(p)) return launch_tiles<T, FORM, DUAL, 64, BN, 2, 2, DEPTH, 2, 4, SINGLES>(p, s, ep, to);
    }
    if (!direct && copies_ok<T>(p)) return launch_tiles<T, FORM, DUAL, 128, 128, 2, 2, DEPTH, 2, 4, SINGLES>(p, s, ep, to);
  }
  // (gradients of weights end after a few stages: more and smaller workgroups on a compute unit hide more of their ends; 77 groups of
  // 48 rows, 777 x 301, shifted granules of fp32, two weights: 119 -> 104 us)
  constexpr bool SHORT = FORM == WEIGHTS, F32 = sizeof(T) == 4;
  if (!direct) return launch_tiles<T, FORM, DUAL, 128, 128, SHORT || F32 ? 2 : 4, 2, SHORT ? 4 : 8, 2, 4, SHIFTED>(p, s, ep, to);
  // fp32: two workgroups of four waves on a compute unit, one's matrix instructions in the other's barriers (4096^3 1120 us with one
  // of eight waves and a ring of four stages, 1057)
  if constexpr (F32) return launch_tiles<T, FORM, DUAL, 128, 128, 2, 2, 8, 2, 4, DIRECT>(p, s, ep, to);
  else if (tiles == TILES_256) {
    // (results that come with more bytes than operations: two workgroups to a compute unit, one computes while the other stores.
    // 16384 rows of 8 experts, 2048 x 2048: gradients of hidden 281 us on 256 x 256 tiles, 267; other rows 4 to 20 % slower)
    if constexpr (FORM == WEIGHTS || Ep::HEAVY) return launch_tiles<T, FORM, DUAL, 256, 128, 2, 2, 4, 3, 4, DIRECT>(p, s, ep, to);
    else return launch_tiles<T, FORM, DUAL, 256, 256, 2, 4, 8, 2, 4, DIRECT>(p, s, ep, to);
  } else {
    return launch_tiles<T, FORM, DUAL, 128, 128, 4, 2, 8, 4, 2, DIRECT>(p, s, ep, to);
  }
}

}  // namespace
}  // namespace dynb

#endif
