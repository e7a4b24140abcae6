// Dense layers with what surrounds them (bias, activation, residual) and gated feed-forward blocks of routed experts, and
// their gradients: the calls, how their products are cut, and the passes around the products.
#include <algorithm>

#include "product_epilogues.h"

namespace dynb {
namespace {

constexpr int64_t MOST_COLS = 1 << 20;

// ---- how products are cut -------------------------------------------------------------------------------------
int64_t tiles_of(int64_t n, int64_t size) { return (n + size - 1) / size; }
// Tiles of rows to be expected where groups share `rows`: half a tile more than whole ones for each.
int64_t row_tiles_of(int64_t rows, int groups, int size) {
  return groups == 1 ? tiles_of(rows, size) : rows / size + (std::min<int64_t>(groups, rows) + 1) / 2;
}
// (sizes alone: rows of other pitches or places take the same parts)
bool whole_granules(int dtype, int64_t n) { return n % (dtype == DYNB_F32 ? 4 : 8) == 0; }
// Into how many parts a reduction of `stages` is divided.  A workgroup takes about its share of the stages; where two share a
// compute unit (paired) they take twice as long, one alone there 1.5 times.  `worth`: what a part costs to be written and
// joined, in halves of a stage.  Measured in bf16 with 64 to 512 rows, 1024 to 4096 columns: reductions of 4096 13 to 32 us, in one
// part 29 to 38; of 16384 19 to 91 us, in one part 87 to 151; of 1024, 16 stages, one part is taken, 14 to 16 us, where half of
// `worth` would take two and 11 to 15 us (20 for 512 rows of 4096 columns), and be up to 7 % slower at 16384; twice `worth` is
// up to 19 % slower at 4096 and 16384.  Worst of what was measured: gradients of 1024 x 2048 from 2048 rows, 45 us, in one part 38.
int parts(int64_t tiles, int64_t stages, bool paired, int worth) {
  int best = 1;
  int64_t least = 0;
  for (int n = 1; n <= 16; ++n) {
    const int64_t blocks = tiles * n, share = tiles_of(stages, n);
    const int64_t cost = (paired ? blocks <= 256 ? 3 : 4 * tiles_of(blocks, 512) : 2 * tiles_of(blocks, 256)) * share + (n > 1 ? worth * n : 0);
    if (n == 1 || cost < least) {
      least = cost;
      best = n;
    }
  }
  return best;
}

// The same for fp32 on 64 x 64 tiles (64 x 128 for two products): matrix instructions bound several workgroups on a compute unit
// together, fewer than three leave them waiting.  (128 to 1500 rows, reductions of 1024 and 4096, 512 and 2048 columns: 13 to 204 us,
// in one part 1 to 4.7 times as long; the cost of a part halved 0 to 7 % slower, doubled 0 to 31 %)
int parts_of_small(int64_t tiles, int64_t stages) {
  int best = 1;
  int64_t least = 0;
  for (int n = 1; n <= 8; ++n) {
    const int64_t cost = std::max<int64_t>(tiles_of(tiles * n, 256), 3) * tiles_of(stages, n) + (n > 1 ? 6 * n : 0);
    if (n == 1 || cost < least) {
      least = cost;
      best = n;
    }
  }
  return best;
}
constexpr int64_t FEW_TILES = 768;         // 128 x 128 tiles, three rounds of them: below, smaller ones

// Tiles of 32 rows up to 48 rows a group (memory bounds them; beyond, 64 rows read the weights twice), 256 x 256 where they are
// three quarters of the compute units at least and groups are no smaller than five eighths of a tile (bf16; 2 of 8 experts, 16384 x
// 4096 x 4096: 3.08 ms, on 128 x 128 tiles, two to a compute unit, 4.04), else 128 x 128.
ProductPlan plan_rows(int dtype, int64_t rows, int groups, int N, int64_t reduction, bool dual) {
  const int half = dual ? 2 : 1;
  const int64_t stages = tiles_of(reduction, dtype == DYNB_F32 ? 32 : 64);
  const int64_t each = rows / std::min<int64_t>(groups, std::max<int64_t>(rows, 1));
  // (memory bounds these: parts only until every compute unit has work.  192 narrow tiles and more are not divided: one row of 2048,
  // 4096 and 8192 through 12800 columns 12.7, 24.6 and 47.6 us, in two parts 14.6, 25.8 and 47.6, through 16384 9 to 14 % in favour;
  // with 40 rows it goes either way, 2048, 4096 and 8192 through 6144 columns 13.6, 21.5 and 39.8 us, in two parts 12.4, 16.7 and 37.4)
  if (each <= 48) {
    const int64_t row_tiles = row_tiles_of(rows, groups, 32);
    const bool narrow = !dual && row_tiles * tiles_of(N, 128) < 256;
    const int64_t tiles = row_tiles * tiles_of(N, narrow ? 64 : 128 / half);
    const int n = (int)std::max<int64_t>(1, std::min({512 / std::max<int64_t>(tiles, 1), stages / 4, (int64_t)16}));
    return {narrow ? TILES_32X64 : TILES_32, narrow && tiles >= 192 ? 1 : n};
  }
  if (dtype == DYNB_BF16 && each >= 160 && row_tiles_of(rows, groups, 256) * tiles_of(N, 256 / half) >= 192) return {TILES_256, 1};
  if (dtype == DYNB_F32 && row_tiles_of(rows, groups, 128) * tiles_of(N, 128 / half) < FEW_TILES)
    return {TILES_64, parts_of_small(row_tiles_of(rows, groups, 64) * tiles_of(N, 64), stages)};
  const bool paired = dtype == DYNB_F32 || !whole_granules(dtype, N) || !whole_granules(dtype, reduction);
  return {TILES_128, parts(row_tiles_of(rows, groups, 128) * tiles_of(N, 128 / half), stages, paired, dtype == DYNB_F32 ? groups == 1 ? 6 : 12 : 8)};
}
ProductPlan plan_weights(int dtype, int64_t rows, int groups, int M, int N, int matrices) {
  const int64_t stages = tiles_of(rows / groups, dtype == DYNB_F32 ? 32 : 64);
  if (dtype == DYNB_BF16 && tiles_of(M, 256) * tiles_of(N, 256) * groups * matrices >= 192) return {TILES_256, 1};
  if (dtype == DYNB_F32 && (stages < 8 || tiles_of(M, 128) * tiles_of(N, 128) * groups * matrices < FEW_TILES))
    return {TILES_64, parts_of_small(tiles_of(M, 64) * tiles_of(N, 64) * groups * matrices, stages)};
  const bool paired = dtype == DYNB_F32 || !whole_granules(dtype, N) || !whole_granules(dtype, M);
  return {TILES_128, parts(tiles_of(M, 128) * tiles_of(N, 128) * groups * matrices, stages, paired, dtype == DYNB_F32 ? 6 : 12)};
}
// Bytes of Product::partial (0 where the plan has one part).
size_t partial_bytes(const ProductPlan& plan, int64_t rows, int64_t columns) {
  return plan.splits > 1 ? (size_t)round_up((int64_t)plan.splits * rows * columns * 4, 16) : 0;
}
void cut(Product& p, const ProductPlan& plan, int64_t partial_rows, void* partial) {
  p.splits = plan.splits;
  p.partial = (float*)partial;
  p.partial_rows = partial_rows;
}

// Whether rows of weights' gradients are whole lines: others are not sent past the caches, which put the pieces together.
template <typename O> bool whole_lines(int cols) { return cols * sizeof(O) % 128 == 0; }

size_t size_of(int dtype) { return dtype == DYNB_F32 ? 4 : 2; }
int64_t padded(int64_t cols, int dtype) { return round_up(cols, 16 / (int)size_of(dtype)); }

int check_type(int32_t dtype, int32_t grad, int32_t act, const char* who) {
  if (dtype != DYNB_F32 && dtype != DYNB_BF16) return fail(DYNB_ERR_BADARG, "%s: unknown type of the rows", who);
  if (grad != DYNB_F32 && grad != dtype) return fail(DYNB_ERR_BADARG, "%s: weights' gradients are fp32 or of the rows' type", who);
  if (act < DYNB_ACT_NONE || act > DYNB_ACT_GELU) return fail(DYNB_ERR_BADARG, "%s: unknown activation", who);
  return DYNB_OK;
}
int check_workspace(const void* workspace, size_t bytes, size_t need, const char* who) {
  if (need && (!workspace || bytes < need || off_by(workspace, 16)))
    return fail(DYNB_ERR_BADARG, "%s: workspace is null, too small or not 16-byte aligned", who);
  return DYNB_OK;
}

// A call of several products: all of them are looked at, then all are launched.
template <class Products> int whole_call(void* stream, Products products) {
  if (int rc = products(Target{(hipStream_t)stream, false})) return rc;
  return products(Target{(hipStream_t)stream, true});
}

// ---- gradient of what an activation was taken of, and sums of its columns ------------------------------------------
// dpre = dout act'(pre), and over the rows of each chunk its sums (fp32, the rows in order: four waves take every
// fourth row each, their sums are added in turn).  4096 x 4096 in bf16, 16 workers: 101 MB in 31 us, 3.2 TB/s, 0.64 of a large copy's
// rate: chunks are of 32 rows, so that a wave asks twice for four rows and ends.
constexpr int TOGETHER = 4;
template <typename T>
__global__ __launch_bounds__(256) void dense_grad_kernel(const T* dout, int64_t ld_dout, const T* pre, int64_t ld_pre, int act,
                                                         T* dpre, int64_t ld_dpre, float* sums, int cols, Segs segs,
                                                         RowChunks ch) {
  __shared__ float part[3][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.y * 512 + lane * 8, n = min(cols - col, 8);
  int k = 0;
  while (k + 1 < segs.K && ch.first[k + 1] <= (int)blockIdx.x) ++k;
  const int64_t first = segs.off[k] + (int64_t)((int)blockIdx.x - ch.first[k]) * ch.rows;
  const int64_t last = min((int64_t)segs.off[k + 1], first + ch.rows);
  float s[8] = {};
  for (int64_t r0 = first + wave; r0 < last; r0 += 4 * TOGETHER) {
    Raw<T> d[TOGETHER], z[TOGETHER];                  // (asked for together; rows past the last repeat it)
#pragma unroll
    for (int u = 0; u < TOGETHER; ++u) {
      const int64_t r = min(r0 + 4 * u, last - 1);
      d[u] = load_raw(dout + r * ld_dout + col, n);
      if (act != DYNB_ACT_NONE) z[u] = load_raw(pre + r * ld_pre + col, n);
    }
#pragma unroll
    for (int u = 0; u < TOGETHER; ++u) {
      if (r0 + 4 * u >= last) continue;
      float v[8];
      unpack(d[u], n, v);
      if (act != DYNB_ACT_NONE) {
        float x[8];
        unpack(z[u], n, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float slope;
          Curve<T>::both(act, x[e], slope);
          v[e] *= slope;
        }
        store_part(dpre + (r0 + 4 * u) * ld_dpre + col, n, v);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += v[e];
    }
  }
  if (!sums) return;                       // (uniform)
  if (wave) {
#pragma unroll
    for (int e = 0; e < 8; ++e) part[wave - 1][lane * 8 + e] = s[e];
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = ((s[e] + part[0][lane * 8 + e]) + part[1][lane * 8 + e]) + part[2][lane * 8 + e];
  store_part(sums + (int64_t)blockIdx.x * cols + col, n, s);
}
// dbias[k] = the sums of worker k's chunks, in order
template <typename O>
__global__ __launch_bounds__(256) void chunk_sum_kernel(const float* sums, int cols, RowChunks ch, O* out, int64_t stride) {
  const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.y;
  if (c >= cols) return;
  float s = 0.f;
#pragma unroll 8
  for (int i = ch.first[k]; i < ch.first[k + 1]; ++i) s += sums[(int64_t)i * cols + c];
  out[k * stride + c] = (O)s;
}

RowChunks bias_chunks(const Segs& s) {     // (a hundred or two of them, so that a column's sum is no long chain)
  return make_row_chunks(s, (int)std::max<int64_t>(32, round_up(s.off[s.K] / 128, 16)));
}

// ---- dense layers -----------------------------------------------------------------------------------------------
int check(const dynb_linear_desc* d, const char* who) {
  if (!d) return fail(DYNB_ERR_BADARG, "%s: null description", who);
  if (int rc = check_type(d->dtype, d->grad_dtype, d->activation, who)) return rc;
  if (d->n_in < 1 || d->n_in > MOST_COLS || d->n_out < 1 || d->n_out > MOST_COLS)
    return fail(DYNB_ERR_BADARG, "%s: n_in or n_out out of range", who);
  for (int64_t ld : {d->ld_x, d->ld_dx})
    if (ld != 0 && ld < d->n_in) return fail(DYNB_ERR_BADARG, "%s: a row pitch is below n_in", who);
  for (int64_t ld : {d->ld_residual, d->ld_pre, d->ld_out, d->ld_dout})
    if (ld != 0 && ld < d->n_out) return fail(DYNB_ERR_BADARG, "%s: a row pitch is below n_out", who);
  return DYNB_OK;
}

template <typename T>
int linear_forward(const dynb_linear_desc* d, int64_t rows, const void* x, const void* weight, const float* bias,
                   const void* residual, void* pre, void* out, void* workspace, Target to) {
  Product p = {};
  p.A[0] = p.A[1] = x;
  p.B[0] = p.B[1] = weight;
  p.lda = d->ld_x ? d->ld_x : d->n_in;
  p.ldb = d->n_out;
  p.N = d->n_out;
  p.K = d->n_in;
  p.pairs = p.groups = 1;
  p.rows = rows;
  const ProductPlan plan = plan_rows(d->dtype, rows, 1, p.N, p.K, false);
  cut(p, plan, rows, workspace);
  const int64_t m = d->n_out;
  const LinearOut<T> ep = {bias, (const T*)residual, d->ld_residual ? d->ld_residual : m, (T*)pre, d->ld_pre ? d->ld_pre : m,
                           (T*)out, d->ld_out ? d->ld_out : m, d->activation};
  return launch_linear<T>(p, plan.tiles, false, ep, to);
}

// Where the parts of a backward pass's workspace begin.
struct LinearBackward {
  size_t dpre, sums, partial, end;
};
LinearBackward layout(const dynb_linear_desc* d, const Segs& s) {
  const int64_t T = s.off[s.K];
  LinearBackward w = {};
  size_t at = 0;
  w.dpre = at;
  if (d->activation != DYNB_ACT_NONE) at += (size_t)round_up(T * padded(d->n_out, d->dtype) * (int64_t)size_of(d->dtype), 16);
  w.sums = at;
  at += (size_t)round_up((int64_t)bias_chunks(s).first[s.K] * d->n_out * 4, 16);
  w.partial = at;
  const size_t dx = partial_bytes(plan_rows(d->dtype, T, 1, d->n_in, d->n_out, false), T, d->n_in);
  const size_t dw = partial_bytes(plan_weights(d->dtype, T, s.K, d->n_in, d->n_out, 1), (int64_t)s.K * d->n_in, d->n_out);
  w.end = at + std::max(dx, dw);
  return w;
}

template <typename T, typename O>
int linear_gradients(const dynb_linear_desc* d, const Segs& s, const void* x, const void* weight, const void* pre,
                     const void* dout, void* dx, void* dweight, int64_t dweight_stride, void* dbias, int64_t dbias_stride,
                     char* workspace, Target to) {
  const int64_t rows = s.off[s.K];
  const int n = d->n_in, m = d->n_out;
  const LinearBackward w = layout(d, s);
  const T* g = (const T*)dout;
  int64_t ld_g = d->ld_dout ? d->ld_dout : m;
  const bool act = d->activation != DYNB_ACT_NONE;
  const RowChunks ch = bias_chunks(s);
  float* const sums = (float*)(workspace + w.sums);
  if (rows > 0 && (act || dbias)) {
    T* const dpre = (T*)(workspace + w.dpre);
    if (to.launch)
      hipLaunchKernelGGL(dense_grad_kernel<T>, dim3(ch.first[s.K], (unsigned)tiles_of(m, 512)), dim3(256), 0, to.stream, g, ld_g,
                         (const T*)pre, d->ld_pre ? d->ld_pre : m, d->activation, dpre, padded(m, d->dtype),
                         dbias ? sums : nullptr, m, s, ch);
    if (act) {
      g = dpre;
      ld_g = padded(m, d->dtype);
    }
  }
  if (dbias && to.launch)
    hipLaunchKernelGGL(chunk_sum_kernel<O>, dim3((unsigned)tiles_of(m, 256), s.K), dim3(256), 0, to.stream, sums, m, ch, (O*)dbias,
                       dbias_stride);
  if (to.launch && hipGetLastError() != hipSuccess) return fail(DYNB_ERR_HIP, "linear_backward launch failed");
  if (dx && rows > 0) {
    Product p = {};
    p.A[0] = p.A[1] = g;
    p.B[0] = p.B[1] = weight;
    p.lda = ld_g;
    p.ldb = m;
    p.N = n;
    p.K = m;
    p.pairs = p.groups = 1;
    p.rows = rows;
    const ProductPlan plan = plan_rows(d->dtype, rows, 1, n, m, false);
    cut(p, plan, rows, workspace + w.partial);
    const LinearOut<T> ep = {nullptr, nullptr, 0, nullptr, 0, (T*)dx, d->ld_dx ? d->ld_dx : n, DYNB_ACT_NONE};
    if (int rc = launch_linear<T>(p, plan.tiles, true, ep, to)) return rc;
  }
  if (dweight) {
    Product p = {};
    p.A[0] = p.A[1] = x;
    p.B[0] = p.B[1] = g;
    p.lda = d->ld_x ? d->ld_x : n;
    p.ldb = ld_g;
    p.M = n;
    p.N = m;
    p.pairs = 1;
    p.groups = p.workers = s.K;
    p.rows = rows;
    const ProductPlan plan = plan_weights(d->dtype, rows, s.K, n, m, 1);
    cut(p, plan, (int64_t)s.K * n, workspace + w.partial);
    const WeightOut<O> ep = {{(O*)dweight, nullptr}, dweight_stride, 0, s.K, m, s.K, past_caches((double)sizeof(O) * s.K * n * m) && whole_lines<O>(m)};
    return launch_weights<T, O>(p, plan.tiles, s, ep, to);
  }
  return DYNB_OK;
}

// ---- gated blocks --------------------------------------------------------------------------------------------
int check(const dynb_gated_block_desc* d, const char* who) {
  if (!d) return fail(DYNB_ERR_BADARG, "%s: null description", who);
  if (int rc = check_type(d->dtype, d->grad_dtype, d->activation, who)) return rc;
  if (d->cols < 1 || d->cols > MOST_COLS || d->hidden < 1 || d->hidden > MOST_COLS)
    return fail(DYNB_ERR_BADARG, "%s: cols or hidden out of range", who);
  if (d->n_experts < 1 || d->n_experts > DYNB_MAX_EXPERTS) return fail(DYNB_ERR_BADARG, "%s: n_experts out of range", who);
  if (d->rows < 0 || d->rows > INT32_MAX) return fail(DYNB_ERR_BADARG, "%s: rows out of range", who);
  for (int64_t ld : {d->ld_x, d->ld_y, d->ld_dy, d->ld_dx})
    if (ld != 0 && ld < d->cols) return fail(DYNB_ERR_BADARG, "%s: a row pitch is below cols", who);
  if (d->ld_kept != 0 && d->ld_kept < d->hidden) return fail(DYNB_ERR_BADARG, "%s: a row pitch is below hidden", who);
  return DYNB_OK;
}
int64_t hidden_bytes(const dynb_gated_block_desc* d) {
  return round_up(d->rows * padded(d->hidden, d->dtype) * (int64_t)size_of(d->dtype), 16);
}
ProductPlan plan_up(const dynb_gated_block_desc* d) { return plan_rows(d->dtype, d->rows, d->n_experts, d->hidden, d->cols, true); }
ProductPlan plan_down(const dynb_gated_block_desc* d) { return plan_rows(d->dtype, d->rows, d->n_experts, d->cols, d->hidden, false); }
ProductPlan plan_dhidden(const dynb_gated_block_desc* d) { return plan_rows(d->dtype, d->rows, d->n_experts, d->hidden, d->cols, false); }
ProductPlan plan_dx(const dynb_gated_block_desc* d) {
  return plan_rows(d->dtype, d->rows, d->n_experts, d->cols, 2 * (int64_t)d->hidden, false);
}
ProductPlan plan_dup(const dynb_gated_block_desc* d, int K) {
  return plan_weights(d->dtype, d->rows, d->n_experts * K, d->cols, d->hidden, 2);
}
ProductPlan plan_ddown(const dynb_gated_block_desc* d, int K) {
  return plan_weights(d->dtype, d->rows, d->n_experts * K, d->hidden, d->cols, 1);
}

Product by_expert(const dynb_gated_block_desc* d, const int32_t* offsets) {
  Product p = {};
  p.b_stride = (int64_t)d->cols * d->hidden;
  p.pairs = 1;
  p.rows = d->rows;
  p.offsets = offsets;
  p.groups = d->n_experts;
  return p;
}

template <typename T>
int gated_forward(const dynb_gated_block_desc* d, const int32_t* offsets, const void* x, const void* w_gate, const void* w_up,
                  const void* w_down, void* gate, void* up, void* y, char* workspace, Target to) {
  const int H = d->cols, F = d->hidden;
  const int64_t ld_hidden = padded(F, d->dtype);
  T* const hidden = (T*)workspace;
  char* const partial = workspace + hidden_bytes(d);
  Product p = by_expert(d, offsets);
  p.A[0] = p.A[1] = x;
  p.B[0] = w_gate;
  p.B[1] = w_up;
  p.lda = d->ld_x ? d->ld_x : H;
  p.ldb = F;
  p.N = F;
  p.K = H;
  ProductPlan plan = plan_up(d);
  cut(p, plan, d->rows, partial);
  const GatedOut<T> ep = {(T*)gate, (T*)up, d->ld_kept ? d->ld_kept : F, hidden, ld_hidden, d->activation};
  if (int rc = launch_gated<T>(p, plan.tiles, ep, to)) return rc;
  p.A[0] = p.A[1] = hidden;
  p.B[0] = p.B[1] = w_down;
  p.lda = ld_hidden;
  p.ldb = H;
  p.N = H;
  p.K = F;
  plan = plan_down(d);
  cut(p, plan, d->rows, partial);
  const LinearOut<T> out = {nullptr, nullptr, 0, nullptr, 0, (T*)y, d->ld_y ? d->ld_y : H, DYNB_ACT_NONE};
  return launch_linear<T>(p, plan.tiles, false, out, to);
}

template <typename T, typename O>
int gated_gradients(const dynb_gated_block_desc* d, int K, const int32_t* offsets, const int32_t* segments, const void* x,
                    const void* w_gate, const void* w_up, const void* w_down, const void* gate, const void* up, const void* dy,
                    void* dx, void* dw_gate, void* dw_up, void* dw_down, int64_t worker_stride, char* workspace, Target to) {
  const int H = d->cols, F = d->hidden;
  const int64_t ld_hidden = padded(F, d->dtype), ld_dy = d->ld_dy ? d->ld_dy : H, each = hidden_bytes(d);
  T *const dgate = (T*)workspace, *const dup = (T*)(workspace + each), *const hidden = (T*)(workspace + 2 * each);
  char* const partial = workspace + 3 * each;
  if (d->rows > 0) {
    Product p = by_expert(d, offsets);
    p.A[0] = p.A[1] = dy;
    p.B[0] = p.B[1] = w_down;
    p.lda = ld_dy;
    p.ldb = H;
    p.N = F;
    p.K = H;
    const ProductPlan plan = plan_dhidden(d);
    cut(p, plan, d->rows, partial);
    const GatedGrad<T> ep = {(const T*)gate, (const T*)up, d->ld_kept ? d->ld_kept : F, dgate, dup, hidden, ld_hidden, d->activation};
    if (int rc = launch_gated_grad<T>(p, plan.tiles, ep, to)) return rc;
  }
  if (dx && d->rows > 0) {
    Product p = by_expert(d, offsets);
    p.A[0] = dgate;
    p.A[1] = dup;
    p.B[0] = w_gate;
    p.B[1] = w_up;
    p.lda = ld_hidden;
    p.ldb = F;
    p.N = H;
    p.K = F;
    p.pairs = 2;
    const ProductPlan plan = plan_dx(d);
    cut(p, plan, d->rows, partial);
    const LinearOut<T> ep = {nullptr, nullptr, 0, nullptr, 0, (T*)dx, d->ld_dx ? d->ld_dx : H, DYNB_ACT_NONE};
    if (int rc = launch_linear<T>(p, plan.tiles, true, ep, to)) return rc;
  }
  if (!dw_gate) return DYNB_OK;
  Product p = by_expert(d, offsets);
  Segs whole = {};
  whole.K = 1;
  whole.off[1] = (int)d->rows;
  p.segments = segments;
  p.groups = d->n_experts * K;
  p.workers = K;
  p.b_stride = 0;
  p.A[0] = p.A[1] = x;
  p.B[0] = dgate;
  p.B[1] = dup;
  p.lda = d->ld_x ? d->ld_x : H;
  p.ldb = ld_hidden;
  p.M = H;
  p.N = F;
  ProductPlan plan = plan_dup(d, K);
  p.pairs = 2;
  cut(p, plan, 2 * (int64_t)p.groups * H, partial);
  const int64_t matrix = (int64_t)H * F;
  const bool past = past_caches((double)sizeof(O) * p.groups * matrix);
  const WeightOut<O> ep = {{(O*)dw_gate, (O*)dw_up}, worker_stride, matrix, K, F, p.groups, past && whole_lines<O>(F)};
  if (int rc = launch_weights<T, O>(p, plan.tiles, whole, ep, to)) return rc;
  p.A[0] = p.A[1] = hidden;
  p.B[0] = p.B[1] = dy;
  p.lda = ld_hidden;
  p.ldb = ld_dy;
  p.M = F;
  p.N = H;
  p.pairs = 1;
  plan = plan_ddown(d, K);
  cut(p, plan, (int64_t)p.groups * F, partial);
  const WeightOut<O> down = {{(O*)dw_down, nullptr}, worker_stride, matrix, K, H, p.groups, past && whole_lines<O>(H)};
  return launch_weights<T, O>(p, plan.tiles, whole, down, to);
}

}  // namespace
}  // namespace dynb

using namespace dynb;

extern "C" size_t dynb_linear_workspace_bytes(const dynb_linear_desc* d, int64_t rows) {
  if (check(d, "linear_workspace_bytes") || rows < 1 || rows > INT32_MAX) return 0;
  return partial_bytes(plan_rows(d->dtype, rows, 1, d->n_out, d->n_in, false), rows, d->n_out);
}

extern "C" int dynb_linear(const dynb_linear_desc* d, int64_t rows, const void* x, const void* weight, const float* bias,
                           const void* residual, void* pre, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = check(d, "linear")) return rc;
  if (rows < 0 || rows > INT32_MAX) return fail(DYNB_ERR_BADARG, "linear: rows out of range");
  if (rows == 0) return DYNB_OK;
  if (!x || !weight || !out) return fail(DYNB_ERR_BADARG, "linear: null pointer");
  const size_t size = size_of(d->dtype);
  if (off_by(x, size) || off_by(weight, size) || off_by(bias, 4) || off_by(residual, size) || off_by(pre, size) || off_by(out, size))
    return fail(DYNB_ERR_BADARG, "linear: a pointer is not a multiple of its element's size");
  if (int rc = check_workspace(workspace, workspace_bytes, dynb_linear_workspace_bytes(d, rows), "linear")) return rc;
  const double n = d->n_in, m = d->n_out;
  Timed t(KC_DENSE, stream, 2.0 * rows * n * m, size * (n * m + rows * (n + m * (1 + !!residual + !!pre))));
  const Target to = {(hipStream_t)stream, true};
  return d->dtype == DYNB_F32 ? linear_forward<float>(d, rows, x, weight, bias, residual, pre, out, workspace, to)
                              : linear_forward<bf16>(d, rows, x, weight, bias, residual, pre, out, workspace, to);
}

extern "C" size_t dynb_linear_backward_workspace_bytes(const dynb_linear_desc* d, const int32_t* b, int32_t K) {
  Segs s;
  if (check(d, "linear_backward_workspace_bytes") || segments_of(b, K, "linear_backward_workspace_bytes", s)) return 0;
  return layout(d, s).end;
}

extern "C" int dynb_linear_backward(const dynb_linear_desc* d, const int32_t* b, int32_t K, const void* x, const void* weight,
                                    const void* pre, const void* dout, void* dx, void* dweight, int64_t dweight_stride,
                                    void* dbias, int64_t dbias_stride, void* workspace, size_t workspace_bytes, void* stream) {
  Segs s;
  if (int rc = check(d, "linear_backward")) return rc;
  if (int rc = segments_of(b, K, "linear_backward", s)) return rc;
  const int64_t rows = s.off[K];
  if (rows > 0 && (!dout || (dx && !weight) || (dweight && !x) || (d->activation != DYNB_ACT_NONE && !pre)))
    return fail(DYNB_ERR_BADARG, "linear_backward: null pointer");
  const size_t size = size_of(d->dtype), gsize = size_of(d->grad_dtype);
  if (off_by(x, size) || off_by(weight, size) || off_by(pre, size) || off_by(dout, size) || off_by(dx, size) ||
      off_by(dweight, gsize) || off_by(dbias, gsize))
    return fail(DYNB_ERR_BADARG, "linear_backward: a pointer is not a multiple of its element's size");
  if ((dweight && K > 1 && dweight_stride < (int64_t)d->n_in * d->n_out) || (dbias && K > 1 && dbias_stride < d->n_out))
    return fail(DYNB_ERR_BADARG, "linear_backward: workers' gradients overlap");
  if (int rc = check_workspace(workspace, workspace_bytes, layout(d, s).end, "linear_backward")) return rc;
  const double n = d->n_in, m = d->n_out;
  Timed t(KC_DENSE, stream, 2.0 * rows * n * m * (!!dx + !!dweight),
          size * (n * m + rows * (2 * n + 2 * m)) + gsize * K * n * m);
  auto call = [&](auto type, auto grad) {
    return whole_call(stream, [&](Target to) {
      return linear_gradients<decltype(type), decltype(grad)>(d, s, x, weight, pre, dout, dx, dweight, dweight_stride, dbias,
                                                              dbias_stride, (char*)workspace, to);
    });
  };
  if (d->dtype == DYNB_F32) return call(float(), float());
  return d->grad_dtype == DYNB_F32 ? call(bf16(), float()) : call(bf16(), bf16());
}

extern "C" size_t dynb_gated_block_workspace_bytes(const dynb_gated_block_desc* d) {
  if (check(d, "gated_block_workspace_bytes") || d->rows == 0) return 0;
  return (size_t)hidden_bytes(d) + std::max(partial_bytes(plan_up(d), d->rows, 2 * (int64_t)d->hidden),
                                            partial_bytes(plan_down(d), d->rows, d->cols));
}

extern "C" int dynb_gated_block(const dynb_gated_block_desc* d, const int32_t* offsets, const void* x, const void* w_gate,
                                const void* w_up, const void* w_down, void* gate, void* up, void* y, void* workspace,
                                size_t workspace_bytes, void* stream) {
  if (int rc = check(d, "gated_block")) return rc;
  if (!offsets && d->n_experts > 1) return fail(DYNB_ERR_BADARG, "gated_block: null offsets with more than one expert");
  if (!gate != !up) return fail(DYNB_ERR_BADARG, "gated_block: both pre-activations are kept, or none");
  const size_t size = size_of(d->dtype);
  if (off_by(offsets, 4) || off_by(x, size) || off_by(w_gate, size) || off_by(w_up, size) || off_by(w_down, size) ||
      off_by(gate, size) || off_by(up, size) || off_by(y, size))
    return fail(DYNB_ERR_BADARG, "gated_block: a pointer is not a multiple of its element's size");
  if (d->rows == 0) return DYNB_OK;
  if (!x || !w_gate || !w_up || !w_down || !y) return fail(DYNB_ERR_BADARG, "gated_block: null pointer");
  if (int rc = check_workspace(workspace, workspace_bytes, dynb_gated_block_workspace_bytes(d), "gated_block")) return rc;
  const double n = d->cols, m = d->hidden, rows = (double)d->rows;
  Timed t(KC_DENSE, stream, 6.0 * rows * n * m, size * (3.0 * std::min<double>(d->n_experts, rows) * n * m + rows * (2 * n + (gate ? 2 * m : 0))));
  return whole_call(stream, [&](Target to) {
    return d->dtype == DYNB_F32
               ? gated_forward<float>(d, offsets, x, w_gate, w_up, w_down, gate, up, y, (char*)workspace, to)
               : gated_forward<bf16>(d, offsets, x, w_gate, w_up, w_down, gate, up, y, (char*)workspace, to);
  });
}

extern "C" size_t dynb_gated_block_backward_workspace_bytes(const dynb_gated_block_desc* d, int32_t K) {
  if (check(d, "gated_block_backward_workspace_bytes") || K < 1 || K > DYNB_MAX_WORKERS) return 0;
  const int64_t groups = (int64_t)d->n_experts * K;
  return 3 * (size_t)hidden_bytes(d) +
         std::max({partial_bytes(plan_dhidden(d), d->rows, d->hidden), partial_bytes(plan_dx(d), d->rows, d->cols),
                   partial_bytes(plan_dup(d, K), 2 * groups * d->cols, d->hidden),
                   partial_bytes(plan_ddown(d, K), groups * d->hidden, d->cols)});
}

extern "C" int dynb_gated_block_backward(const dynb_gated_block_desc* d, int32_t K, const int32_t* offsets,
                                         const int32_t* segments, const void* x, const void* w_gate, const void* w_up,
                                         const void* w_down, const void* gate, const void* up, const void* dy, void* dx,
                                         void* dw_gate, void* dw_up, void* dw_down, int64_t worker_stride, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  if (int rc = check(d, "gated_block_backward")) return rc;
  if (K < 1 || K > DYNB_MAX_WORKERS) return fail(DYNB_ERR_BADARG, "gated_block_backward: K out of range");
  if (!offsets && d->n_experts > 1) return fail(DYNB_ERR_BADARG, "gated_block_backward: null offsets with more than one expert");
  if (!segments && K > 1) return fail(DYNB_ERR_BADARG, "gated_block_backward: null segments with more than one worker");
  if (!dw_gate != !dw_up || !dw_gate != !dw_down)
    return fail(DYNB_ERR_BADARG, "gated_block_backward: the gradients of all three weights, or of none");
  const size_t size = size_of(d->dtype), gsize = size_of(d->grad_dtype);
  if (off_by(offsets, 4) || off_by(segments, 4) || off_by(x, size) || off_by(w_gate, size) || off_by(w_up, size) ||
      off_by(w_down, size) || off_by(gate, size) || off_by(up, size) || off_by(dy, size) || off_by(dx, size) ||
      off_by(dw_gate, gsize) || off_by(dw_up, gsize) || off_by(dw_down, gsize))
    return fail(DYNB_ERR_BADARG, "gated_block_backward: a pointer is not a multiple of its element's size");
  if (dw_gate && K > 1 && worker_stride < (int64_t)d->n_experts * d->cols * d->hidden)
    return fail(DYNB_ERR_BADARG, "gated_block_backward: workers' gradients overlap");
  if (d->rows > 0 && (!x || !w_gate || !w_up || !w_down || !gate || !up || !dy))
    return fail(DYNB_ERR_BADARG, "gated_block_backward: null pointer");
  if (int rc = check_workspace(workspace, workspace_bytes, dynb_gated_block_backward_workspace_bytes(d, K), "gated_block_backward"))
    return rc;
  const double n = d->cols, m = d->hidden, rows = (double)d->rows;
  Timed t(KC_DENSE, stream, rows * n * m * (2.0 + (dx ? 4.0 : 0.0) + (dw_gate ? 6.0 : 0.0)),
          size * (3.0 * d->n_experts * n * m + rows * (3 * n + 2 * m)) + (dw_gate ? 3.0 * gsize * K * d->n_experts * n * m : 0.0));
  auto call = [&](auto type, auto grad) {
    return whole_call(stream, [&](Target to) {
      return gated_gradients<decltype(type), decltype(grad)>(d, K, offsets, segments, x, w_gate, w_up, w_down, gate, up, dy, dx,
                                                             dw_gate, dw_up, dw_down, worker_stride, (char*)workspace, to);
    });
  };
  if (d->dtype == DYNB_F32) return call(float(), float());
  return d->grad_dtype == DYNB_F32 ? call(bf16(), float()) : call(bf16(), bf16());
}
