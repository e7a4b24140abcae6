// Tokens sorted by expert and back: the plan (a stable counting sort), the rows' way there, their weighted sum on the
// way back, and the gradients:
//   sorted[slot[t][j]] = x[t];  out[t] = addend[t] + sum_j w[t][j] sorted[slot[t][j]];
//   dsorted[slot[t][j]] = w[t][j] dout[t], dw[t][j] = <dout[t], sorted[slot[t][j]]>, and dx is the sum without weights.
// Memory bounds the rows: 16384 tokens of 2048 bf16 columns, 8 choices each, 604 MB there in 119 us and 671 MB back in 110 us
// (5.1 and 6.1 TB/s), both gradients of 8192 of 4096 columns and 2 choices 335 MB in 60 us and 268 MB in 42 us.  Sums are fp32
// in the order of the choices and rounded once; nothing is added by atomics but whole numbers.
#include <hip/hip_runtime.h>

#include "dynb_internal.h"
#include "row_access.h"

namespace dynb {
namespace {

// ---- the plan -----------------------------------------------------------------------------------------------
// A stable counting sort.  Every wave owns a stretch of the choices; it counts its experts, the counts are summed in the
// order (expert, workgroup, wave), and the wave goes over its stretch again, 64 choices at a time, and hands out the
// places in order.  Up to SMALL choices one workgroup does it all in one launch; beyond, a launch before it counts per
// workgroup, and every workgroup sums those of all of them.  What bounds it are chains: loads, barriers, a round of 64.
constexpr int WAVES = 16, THREADS = WAVES * 64, AHEAD = 2;   // AHEAD: choices per lane that are loaded at once
constexpr int ROUND = THREADS * AHEAD;    // of a workgroup
// Choices of one workgroup alone (128 experts: 4096 choices 7.3 us, in two launches 8.2; 8192 choices 10.4 and 8.3).
constexpr int SMALL = 4096;
constexpr int MOST_BLOCKS = 128;          // whose counts a workgroup sums

// Lanes of the wave with the same key as this one (all lanes take part; keys below 2^bits).
__device__ inline uint64_t same_key(int key, int bits) {
  uint32_t low = ~0u, high = ~0u;
  for (int b = 0; b < bits; ++b) {
    const int mine = -((key >> b) & 1);
    const uint64_t set = __ballot(mine);
    low &= ~((uint32_t)set ^ (uint32_t)mine);
    high &= ~((uint32_t)(set >> 32) ^ (uint32_t)mine);
  }
  return (uint64_t)high << 32 | low;
}

// LDS written by some lanes of a wave and read by others: in order, with nothing moved across.
__device__ inline void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// What one stretch counts: each lane's choices begin + lane + 64 i.
__device__ inline void count_stretch(const int32_t* experts, int64_t begin, int64_t end, int n_experts, int* count) {
  for (int64_t i0 = begin; i0 < end; i0 += 64 * AHEAD) {
    int e[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t i = i0 + 64 * u + (threadIdx.x & 63);
      e[u] = i < end ? experts[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if ((uint32_t)e[u] < (uint32_t)n_experts) atomicAdd(&count[e[u]], 1);   // (whole numbers: any order)
  }
}

__global__ __launch_bounds__(THREADS) void plan_count_kernel(const int32_t* experts, int64_t n, int64_t per_block,
                                                                      int n_experts, int32_t* counts) {
  __shared__ int count[DYNB_MAX_EXPERTS];
  for (int e = threadIdx.x; e < n_experts; e += THREADS) count[e] = 0;
  __syncthreads();
  const int64_t per = per_block / WAVES, begin = blockIdx.x * per_block + (threadIdx.x >> 6) * per;
  count_stretch(experts, begin, begin + per < n ? begin + per : n, n_experts, count);
  __syncthreads();
  for (int e = threadIdx.x; e < n_experts; e += THREADS) counts[(int64_t)blockIdx.x * n_experts + e] = count[e];
}

// counts: [gridDim.x][n_experts] of plan_count_kernel (not read by a single workgroup)
__global__ __launch_bounds__(THREADS) void plan_kernel(const int32_t* experts, int64_t n, int64_t per_block,
                                                          int n_experts, int bits, const int32_t* counts,
                                                          int32_t* offsets, int32_t* slot, int32_t* source) {
  __shared__ int place[WAVES * DYNB_MAX_EXPERTS];     // [wave][expert]: counts, then the next place
  __shared__ int all[DYNB_MAX_EXPERTS];               // choices of an expert, then its first place
  __shared__ int before[DYNB_MAX_EXPERTS];            // ... of the workgroups before this one
  __shared__ int wave_total[WAVES];
  static_assert(DYNB_MAX_EXPERTS <= THREADS, "a thread per expert");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int* const mine = place + wave * n_experts;
  for (int i = threadIdx.x; i < WAVES * n_experts; i += THREADS) place[i] = 0;
  for (int i = threadIdx.x; i < n_experts; i += THREADS) all[i] = before[i] = 0;
  __syncthreads();
  if (gridDim.x > 1) {                   // every thread an expert and some of the workgroups
    int width = 64;
    while (width < n_experts) width *= 2;
    const int e = threadIdx.x % width;
    int total = 0, ahead = 0;
    if (e < n_experts) {
#pragma unroll 8
      for (int b = threadIdx.x / width; b < (int)gridDim.x; b += THREADS / width) {
        const int c = counts[(int64_t)b * n_experts + e];
        ahead += b < (int)blockIdx.x ? c : 0;
        total += c;
      }
      atomicAdd(&all[e], total);
      atomicAdd(&before[e], ahead);
    }
  }
  const int64_t per = per_block / WAVES, begin = blockIdx.x * per_block + wave * per;
  const int64_t end = begin + per < n ? begin + per : n;
  count_stretch(experts, begin, end, n_experts, mine);
  __syncthreads();
  // first places of the waves relative to the workgroup's
  if ((int)threadIdx.x < n_experts) {
    const int e = threadIdx.x;
    int total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int c = place[w * n_experts + e];
      place[w * n_experts + e] = total;
      total += c;
    }
    if (gridDim.x == 1) all[e] = total;
  }
  __syncthreads();
  // first places of the experts: lanes by shuffles, waves through LDS
  const int e0 = threadIdx.x, sum = e0 < n_experts ? all[e0] : 0;
  int upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d);
    upto += lane >= d ? v : 0;
  }
  if (lane == 63) wave_total[wave] = upto;
  __syncthreads();
  int at = upto - sum, kept = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    at += w < wave ? wave_total[w] : 0;
    kept += wave_total[w];
  }
  if (e0 < n_experts) {
    if (blockIdx.x == 0) offsets[e0] = at;
    const int from = at + before[e0];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) place[w * n_experts + e0] += from;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) offsets[n_experts] = kept;
  __syncthreads();
  for (int64_t i0 = begin; i0 < end; i0 += 64 * AHEAD) {
    int next[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t i = i0 + 64 * u + lane;
      next[u] = i < end ? experts[i] : -1;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (i0 + 64 * u >= end) break;
      const int64_t i = i0 + 64 * u + lane;
      const bool is = (uint32_t)next[u] < (uint32_t)n_experts;
      const int e = is ? next[u] : n_experts;
      const uint64_t same = same_key(e, bits);
      const int rank = __popcll(same & ((1ull << lane) - 1));
      const int to = is ? mine[e] + rank : -1;
      wave_fence();                      // every lane has read its expert's place before the first of them moves it on
      if (is && rank == 0) mine[e] += __popcll(same);
      wave_fence();
      if (i < end) slot[i] = to;
      if (is) source[to] = (int)i;
    }
  }
  for (int64_t r = kept + (int64_t)blockIdx.x * THREADS + threadIdx.x; r < n; r += (int64_t)gridDim.x * THREADS)
    source[r] = -1;
}

// segments[e][k]: the first of expert e's rows whose choice is at or behind worker k's first (choices ascend there).  A wave
// per pair looks at 64 places at a time: two rounds up to 4096 rows, where halving takes twelve.
__global__ __launch_bounds__(256) void segments_kernel(const int32_t* offsets, const int32_t* source, Segs seg,
                                                       int top_k, int n_experts, int32_t* segments) {
  const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6), e = i / (seg.K + 1), k = i - e * (seg.K + 1);
  if (e >= n_experts) return;
  int lo = offsets[e], hi = offsets[e + 1];
  if (k == seg.K) lo = hi;
  const int from = k < seg.K ? seg.off[k] * top_k : 0;
  while (lo < hi) {
    const int step = (int)(((int64_t)hi - lo + 63) / 64);
    const int64_t at = lo + (int64_t)lane * step;
    const int below = __popcll(__ballot(at < hi && source[at < hi ? at : lo] < from));   // (a prefix of the lanes)
    if (below == 0) break;
    const int64_t behind = lo + (int64_t)below * step;
    lo = (int)(behind - step) + 1;
    if (behind < hi) hi = (int)behind;
  }
  if (lane == 0) segments[i] = lo;
}

// ---- rows ---------------------------------------------------------------------------------------------------
struct RowArgs {
  const void *in, *addend;        // rows of tokens or choices, and the combination's addend
  void* out;
  const int32_t *slot, *offsets;
  const float* weights;
  float* dweights;
  const void* sorted;             // backward: the experts' outputs
  int64_t ld_in, ld_out, ld_addend, ld_sorted;
  int64_t tokens, choices;
  int cols, granules, top_k, n_experts;
};

// Sorted rows from `from` on, which no choice has: zeros.
template <typename T> __device__ void clear_rows(const RowArgs& p, int64_t from) {
  const float zeros[GRANULE] = {};
  for (int64_t r = from + blockIdx.x; r < p.choices; r += gridDim.x)
    for (int c = threadIdx.x * GRANULE; c < p.cols; c += 256 * GRANULE)
      store_part((T*)p.out + r * p.ld_out + c, p.cols - c, zeros);
}

// What no kernel of a call writes (slots, weights, offsets): where the address is the same in the whole wave, the compiler
// reads it by scalar instructions only if told so.  Both gradients of 8192 tokens of 4096 bf16 columns and 2 choices 60 us,
// by vector loads 64; one token's 8 choices there in 3.3 and 3.7, back in 3.7 and 4.2.  Not so the plain copies and sums of
// calls beyond the caches: 16384 tokens of 2048 bf16 columns, 8 choices there in 122 and 119 us, back in 113 and 110.
template <bool SCALAR = true, typename V> __device__ inline V constant(const V* p, int64_t i) {
  if constexpr (SCALAR) return ((const __attribute__((address_space(4))) V*)p)[i];
  else return p[i];
}

// L lanes take a row, a granule each and another one L granules on; 256 / L rows per workgroup.  From 64 lanes on a row
// is the same in the whole wave, and what belongs to it (slots, weights) can be read by scalar instructions.
template <int L> __device__ inline int64_t row_of_thread() {
  const int64_t r = (int64_t)blockIdx.x * (256 / L);
  return r + (L >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : threadIdx.x / L);
}

// The choices of a token are taken JS at a time: their slots and weights are asked for together, then their rows.
constexpr int JS = 8;

// One load and top_k stores.
template <typename T, int L, bool PAST> __global__ __launch_bounds__(256) void gather_kernel(RowArgs p) {
  const int kept = constant(p.offsets, p.n_experts);
  for (int64_t t = row_of_thread<L>(); t < p.tokens; t += (int64_t)gridDim.x * (256 / L))
    for (int c = threadIdx.x % L * GRANULE; c < p.cols; c += L * GRANULE) {
      const int n = p.cols - c;
      float v[GRANULE];
      unpack(load_raw<PAST>((const T*)p.in + t * p.ld_in + c, n), n, v);
      for (int j0 = 0; j0 < p.top_k; j0 += JS) {
        int s[JS];
#pragma unroll
        for (int u = 0; u < JS; ++u) s[u] = j0 + u < p.top_k ? constant<!PAST>(p.slot, t * p.top_k + j0 + u) : -1;
#pragma unroll
        for (int u = 0; u < JS; ++u)
          if (s[u] >= 0) store_part<PAST>((T*)p.out + (int64_t)s[u] * p.ld_out + c, n, v);
      }
    }
  clear_rows<T>(p, kept);
}

// The sum over a token's choices, j ascending, in fp32.
template <typename T, int L, bool PAST> __global__ __launch_bounds__(256) void combine_kernel(RowArgs p) {
  for (int64_t t = row_of_thread<L>(); t < p.tokens; t += (int64_t)gridDim.x * (256 / L))
    for (int c = threadIdx.x % L * GRANULE; c < p.cols; c += L * GRANULE) {
      const int n = p.cols - c;
      float a[GRANULE] = {};
      Raw<T> add;
      if (p.addend) add = load_raw<PAST>((const T*)p.addend + t * p.ld_addend + c, n);
      for (int j0 = 0; j0 < p.top_k; j0 += JS) {
        int s[JS];
        float w[JS];
        Raw<T> row[JS];
#pragma unroll
        for (int u = 0; u < JS; ++u) {
          const bool is = j0 + u < p.top_k;
          s[u] = is ? constant<!PAST>(p.slot, t * p.top_k + j0 + u) : -1;
          w[u] = is && p.weights ? constant<!PAST>(p.weights, t * p.top_k + j0 + u) : 1.f;
        }
#pragma unroll
        for (int u = 0; u < JS; ++u)
          if (s[u] >= 0) row[u] = load_raw<PAST>((const T*)p.in + (int64_t)s[u] * p.ld_in + c, n);
        if (j0 == 0 && p.addend) unpack(add, n, a);
#pragma unroll
        for (int u = 0; u < JS; ++u) {
          if (s[u] < 0) continue;
          float v[GRANULE];
          unpack(row[u], n, v);
#pragma unroll
          for (int e = 0; e < GRANULE; ++e) a[e] += w[u] * v[e];
        }
      }
      store_part<PAST>((T*)p.out + t * p.ld_out + c, n, a);
    }
}

// L lanes take a choice: its row of dsorted, and the product of the two rows.  For calls that the caches hold, where more and
// shorter chains count (the gradient is read again for each choice): 1024 tokens of 4 choices of 2048 bf16 columns and the
// combination of the rows' gradient behind it 13.8 us, by tokens 16.2.  Such calls have fewer than 2^20 * 256 / L choices.
template <typename T, int L> __global__ __launch_bounds__(256) void choice_grad_kernel(RowArgs p) {
  __shared__ float red[MOST_WAVES];
  const int kept = constant(p.offsets, p.n_experts);
  const int64_t i = row_of_thread<L>();
  if (i < p.choices) {
    const int64_t t = i / p.top_k, s = constant(p.slot, i);
    const float w = constant(p.weights, i);
    float dot = 0.f;
    if (s >= 0) {
      for (int c = threadIdx.x % L * GRANULE; c < p.cols; c += L * GRANULE) {
        float g[GRANULE], y[GRANULE];
        load_part((const T*)p.in + t * p.ld_in + c, p.cols - c, g);
        load_part((const T*)p.sorted + s * p.ld_sorted + c, p.cols - c, y);
#pragma unroll
        for (int e = 0; e < GRANULE; ++e) {
          dot += g[e] * y[e];
          g[e] *= w;
        }
        store_part((T*)p.out + s * p.ld_out + c, p.cols - c, g);
      }
      dot = L > 64 ? block_sum(dot, L / 64, red) : lanes_sum<(L < 64 ? L : 64)>(dot);
    }
    if (threadIdx.x % L == 0) p.dweights[i] = dot;
  }
  clear_rows<T>(p, kept);
}

// A token's rows of dsorted, and the product of its gradient with each of its choices' rows: the gradient is read once for
// JS choices.  For calls beyond the caches: 8192 tokens of 2 choices of 4096 bf16 columns 60 us (5.6 TB/s), by choices 68.
template <typename T, int L, bool PAST> __global__ __launch_bounds__(256) void combine_grad_kernel(RowArgs p) {
  constexpr int WAVES = L > 64 ? L / 64 : 1;          // of a row
  __shared__ float part[4][JS];
  const int kept = constant(p.offsets, p.n_experts);
  const int64_t mine = row_of_thread<L>() - (int64_t)blockIdx.x * (256 / L);
  for (int64_t first = (int64_t)blockIdx.x * (256 / L); first < p.tokens; first += (int64_t)gridDim.x * (256 / L)) {
    const int64_t t = first + mine;
    const bool live = t < p.tokens;
    for (int j0 = 0; j0 < p.top_k; j0 += JS) {
      int s[JS];
      float w[JS], dot[JS];
#pragma unroll
      for (int u = 0; u < JS; ++u) {
        const bool is = live && j0 + u < p.top_k;
        s[u] = is ? constant(p.slot, t * p.top_k + j0 + u) : -1;
        w[u] = is ? constant(p.weights, t * p.top_k + j0 + u) : 0.f;
        dot[u] = 0.f;
      }
      for (int c = threadIdx.x % L * GRANULE; live && c < p.cols; c += L * GRANULE) {
        const int n = p.cols - c;
        Raw<T> row[JS];
        float g[GRANULE];
        const Raw<T> dout = load_raw((const T*)p.in + t * p.ld_in + c, n);
#pragma unroll
        for (int u = 0; u < JS; ++u)
          if (s[u] >= 0) row[u] = load_raw<PAST>((const T*)p.sorted + (int64_t)s[u] * p.ld_sorted + c, n);
        unpack(dout, n, g);
#pragma unroll
        for (int u = 0; u < JS; ++u) {
          if (s[u] < 0) continue;
          float y[GRANULE];
          unpack(row[u], n, y);
#pragma unroll
          for (int e = 0; e < GRANULE; ++e) {
            dot[u] += g[e] * y[e];
            y[e] = w[u] * g[e];
          }
          store_part<PAST>((T*)p.out + (int64_t)s[u] * p.ld_out + c, n, y);
        }
      }
#pragma unroll
      for (int u = 0; u < JS; ++u)
        if (j0 + u < p.top_k) dot[u] = lanes_sum<(L < 64 ? L : 64)>(dot[u]);
      if (WAVES > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
          for (int u = 0; u < JS; ++u) part[wave][u] = dot[u];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < JS; ++u) {
          dot[u] = part[wave / WAVES * WAVES][u];
#pragma unroll
          for (int v = 1; v < WAVES; ++v) dot[u] += part[wave / WAVES * WAVES + v][u];
        }
        __syncthreads();
      }
      if (threadIdx.x % L == 0 && live)
#pragma unroll
        for (int u = 0; u < JS; ++u)
          if (j0 + u < p.top_k) p.dweights[t * p.top_k + j0 + u] = dot[u];
    }
  }
  clear_rows<T>(p, kept);
}

// Workgroups for rows of L lanes.
int grid_of(int64_t rows, int lanes) {
  const int64_t per = 256 / lanes, blocks = (rows + per - 1) / per;
  return (int)(blocks < (1 << 20) ? blocks : 1 << 20);
}

// Lanes of a row (of 8 elements each): as few as hold it up to 32; else the most of 64, 128 and 256 that leave no more than a
// fifth idle over the rounds, or, where rows are too few to fill the chip with waves, those of the fewest rounds.  (70 tokens
// of 8 choices of 3136 bf16 columns, gradients: 256 lanes 10.6 us, 64 20.0; 2000 of 2 of 5300, forward: 256 lanes 43 us, 64 53;
// 3000 of 4 of 1400 fp32: 64 lanes 55.6 us, 256 61.4.)
int lanes_of(int granules, int64_t rows) {
  if (granules <= 32) return granules <= 16 ? 16 : 32;
  if (rows < 1024) return granules <= 64 ? 64 : granules <= 128 ? 128 : 256;
  for (int l : {256, 128})
    if ((granules + l - 1) / l * l * 4 <= granules * 5) return l;
  return 64;
}

#define ROUTE_LAUNCH(name, L) \
  hipLaunchKernelGGL((name##_kernel<T, L, PAST>), dim3(grid_of(a.tokens, L)), dim3(256), 0, st, a)
#define ROUTE_LAUNCHES(name)                                                 \
  template <typename T, bool PAST> void launch_##name(const RowArgs& a, hipStream_t st) { \
    switch (lanes_of(a.granules, a.tokens)) {                                \
      case 16: ROUTE_LAUNCH(name, 16); break;                                \
      case 32: ROUTE_LAUNCH(name, 32); break;                                \
      case 64: ROUTE_LAUNCH(name, 64); break;                                \
      case 128: ROUTE_LAUNCH(name, 128); break;                              \
      default: ROUTE_LAUNCH(name, 256);                                      \
    }                                                                        \
  }
ROUTE_LAUNCHES(gather)
ROUTE_LAUNCHES(combine)
ROUTE_LAUNCHES(combine_grad)
template <typename T, int L> void launch_choice_grad_as(const RowArgs& a, hipStream_t st) {   // (every choice has its lanes)
  hipLaunchKernelGGL((choice_grad_kernel<T, L>), dim3((unsigned)((a.choices + 256 / L - 1) / (256 / L))), dim3(256), 0, st, a);
}
template <typename T> void launch_choice_grad(const RowArgs& a, hipStream_t st) {
  if (a.granules <= 16) launch_choice_grad_as<T, 16>(a, st);
  else if (a.granules <= 32) launch_choice_grad_as<T, 32>(a, st);
  else if (a.granules <= 128 || a.choices >= 1024) launch_choice_grad_as<T, 64>(a, st);
  else launch_choice_grad_as<T, 256>(a, st);
}

int describe(const dynb_route_desc* d, const char* who) {
  if (!d) return fail(DYNB_ERR_BADARG, "%s: null pointer", who);
  if (d->dtype != DYNB_F32 && d->dtype != DYNB_BF16) return fail(DYNB_ERR_BADARG, "%s: unknown dtype", who);
  if (d->cols < 1 || d->cols > (1 << 20)) return fail(DYNB_ERR_BADARG, "%s: cols out of range", who);
  if (d->top_k < 1 || d->top_k > DYNB_MAX_TOP_K) return fail(DYNB_ERR_BADARG, "%s: top_k out of range", who);
  if (d->n_experts < 1 || d->n_experts > DYNB_MAX_EXPERTS) return fail(DYNB_ERR_BADARG, "%s: n_experts out of range", who);
  if (d->tokens < 0 || d->tokens > INT32_MAX / d->top_k) return fail(DYNB_ERR_BADARG, "%s: tokens out of range", who);
  for (int64_t ld : {d->ld_tokens, d->ld_sorted, d->ld_addend, d->ld_out})
    if (ld != 0 && ld < d->cols) return fail(DYNB_ERR_BADARG, "%s: a row pitch is below cols", who);
  return DYNB_OK;
}

RowArgs row_args(const dynb_route_desc* d) {
  RowArgs a = {};
  a.tokens = d->tokens;
  a.choices = d->tokens * d->top_k;
  a.cols = d->cols;
  a.granules = (d->cols + GRANULE - 1) / GRANULE;
  a.top_k = d->top_k;
  a.n_experts = d->n_experts;
  return a;
}
int64_t pitch(const dynb_route_desc* d, int64_t ld) { return ld ? ld : d->cols; }
int launched(const char* what) {
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "%s launch failed", what);
}

}  // namespace
}  // namespace dynb

using namespace dynb;

// Choices of a workgroup of the large plan: whole rounds of all its waves, and no more than MOST_BLOCKS workgroups.
static int64_t choices_per_block(int64_t n) {
  return round_up((n + MOST_BLOCKS - 1) / MOST_BLOCKS, ROUND);
}

extern "C" size_t dynb_route_workspace_bytes(const dynb_route_desc* d) {
  if (describe(d, "route_workspace_bytes")) return 0;
  const int64_t n = d->tokens * d->top_k, per = choices_per_block(n);
  return n <= SMALL ? 0 : (size_t)((n + per - 1) / per * d->n_experts) * sizeof(int32_t);
}

extern "C" int dynb_route_plan(const dynb_route_desc* d, const int32_t* experts, int32_t* offsets, int32_t* slot,
                               int32_t* source, void* workspace, size_t workspace_bytes, void* stream) {
  if (int rc = describe(d, "route_plan")) return rc;
  const int n = (int)(d->tokens * d->top_k);
  if (!offsets || (n > 0 && (!experts || !slot || !source))) return fail(DYNB_ERR_BADARG, "route_plan: null pointer");
  if (off_by(experts, 4) || off_by(offsets, 4) || off_by(slot, 4) || off_by(source, 4))
    return fail(DYNB_ERR_BADARG, "route_plan: a pointer is not a multiple of its element's size");
  const size_t need = dynb_route_workspace_bytes(d);
  if (need && (!workspace || workspace_bytes < need || off_by(workspace, 16)))
    return fail(DYNB_ERR_BADARG, "route_plan: workspace is null, too small or not 16-byte aligned");
  int bits = 0;
  while ((1 << bits) <= d->n_experts) ++bits;      // (keys 0 .. n_experts: the last one stands for a dropped choice)
  const hipStream_t st = (hipStream_t)stream;
  Timed t(KC_ROUTE, stream, 0.0, 12.0 * n);
  if (n <= SMALL) {
    hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(THREADS), 0, st, experts, (int64_t)n,
                       round_up((n + WAVES - 1) / WAVES, 64) * WAVES, d->n_experts, bits,
                       (const int32_t*)nullptr, offsets, slot, source);
  } else {
    const int64_t per = choices_per_block(n);
    const dim3 grid((unsigned)((n + per - 1) / per)), block(THREADS);
    hipLaunchKernelGGL(plan_count_kernel, grid, block, 0, st, experts, (int64_t)n, per, d->n_experts, (int32_t*)workspace);
    hipLaunchKernelGGL(plan_kernel, grid, block, 0, st, experts, (int64_t)n, per, d->n_experts, bits,
                       (const int32_t*)workspace, offsets, slot, source);
  }
  return launched("route_plan");
}

extern "C" int dynb_route_segments(const dynb_route_desc* d, const int32_t* offsets, const int32_t* source,
                                   const int32_t* b, int32_t K, int32_t* segments, void* stream) {
  Segs seg;
  if (int rc = describe(d, "route_segments")) return rc;
  if (int rc = segments_of(b, K, "route_segments", seg)) return rc;
  if (seg.off[K] != d->tokens) return fail(DYNB_ERR_BADARG, "route_segments: sum(b) is not the number of tokens");
  if (!offsets || !segments || (d->tokens > 0 && !source)) return fail(DYNB_ERR_BADARG, "route_segments: null pointer");
  if (off_by(offsets, 4) || off_by(source, 4) || off_by(segments, 4))
    return fail(DYNB_ERR_BADARG, "route_segments: a pointer is not a multiple of its element's size");
  Timed t(KC_ROUTE, stream, 0.0, 4.0 * d->n_experts * (K + 1));
  hipLaunchKernelGGL(segments_kernel, dim3((d->n_experts * (K + 1) + 3) / 4), dim3(256), 0, (hipStream_t)stream,
                     offsets, source, seg, d->top_k, d->n_experts, segments);
  return launched("route_segments");
}

extern "C" int dynb_route_gather(const dynb_route_desc* d, const void* x, const int32_t* offsets, const int32_t* slot,
                                 void* sorted, void* stream) {
  if (int rc = describe(d, "route_gather")) return rc;
  if (d->tokens == 0) return DYNB_OK;
  if (!x || !offsets || !slot || !sorted) return fail(DYNB_ERR_BADARG, "route_gather: null pointer");
  const size_t size = d->dtype == DYNB_F32 ? 4 : 2;
  if (off_by(x, size) || off_by(sorted, size) || off_by(offsets, 4) || off_by(slot, 4))
    return fail(DYNB_ERR_BADARG, "route_gather: a pointer is not a multiple of its element's size");
  RowArgs a = row_args(d);
  a.in = x;
  a.ld_in = pitch(d, d->ld_tokens);
  a.out = sorted;
  a.ld_out = pitch(d, d->ld_sorted);
  a.offsets = offsets;
  a.slot = slot;
  const double bytes = (double)size * d->cols * (a.tokens + a.choices);
  const bool past = past_caches(bytes);
  Timed t(KC_ROUTE, stream, 0.0, bytes);
  const hipStream_t st = (hipStream_t)stream;
  if (d->dtype == DYNB_F32) past ? launch_gather<float, true>(a, st) : launch_gather<float, false>(a, st);
  else past ? launch_gather<bf16, true>(a, st) : launch_gather<bf16, false>(a, st);
  return launched("route_gather");
}

extern "C" int dynb_route_combine(const dynb_route_desc* d, const void* sorted, const int32_t* slot,
                                  const float* weights, const void* addend, void* out, void* stream) {
  if (int rc = describe(d, "route_combine")) return rc;
  if (d->tokens == 0) return DYNB_OK;
  if (!sorted || !slot || !out) return fail(DYNB_ERR_BADARG, "route_combine: null pointer");
  const size_t size = d->dtype == DYNB_F32 ? 4 : 2;
  if (off_by(sorted, size) || off_by(addend, size) || off_by(out, size) || off_by(slot, 4) || off_by(weights, 4))
    return fail(DYNB_ERR_BADARG, "route_combine: a pointer is not a multiple of its element's size");
  RowArgs a = row_args(d);
  a.in = sorted;
  a.ld_in = pitch(d, d->ld_sorted);
  a.slot = slot;
  a.weights = weights;
  a.addend = addend;
  a.ld_addend = pitch(d, d->ld_addend);
  a.out = out;
  a.ld_out = pitch(d, d->ld_out);
  const double bytes = (double)size * d->cols * (a.choices + a.tokens * (1 + (addend != nullptr)));
  const bool past = past_caches(bytes);
  Timed t(KC_ROUTE, stream, 2.0 * a.choices * d->cols, bytes);
  const hipStream_t st = (hipStream_t)stream;
  if (d->dtype == DYNB_F32) past ? launch_combine<float, true>(a, st) : launch_combine<float, false>(a, st);
  else past ? launch_combine<bf16, true>(a, st) : launch_combine<bf16, false>(a, st);
  return launched("route_combine");
}

extern "C" int dynb_route_combine_backward(const dynb_route_desc* d, const void* dout, const void* sorted,
                                           const int32_t* offsets, const int32_t* slot, const float* weights,
                                           void* dsorted, float* dweights, void* stream) {
  if (int rc = describe(d, "route_combine_backward")) return rc;
  if (d->tokens == 0) return DYNB_OK;
  if (!dout || !sorted || !offsets || !slot || !weights || !dsorted || !dweights)
    return fail(DYNB_ERR_BADARG, "route_combine_backward: null pointer");
  const size_t size = d->dtype == DYNB_F32 ? 4 : 2;
  if (off_by(dout, size) || off_by(sorted, size) || off_by(dsorted, size) || off_by(offsets, 4) || off_by(slot, 4) ||
      off_by(weights, 4) || off_by(dweights, 4))
    return fail(DYNB_ERR_BADARG, "route_combine_backward: a pointer is not a multiple of its element's size");
  RowArgs a = row_args(d);
  a.in = dout;
  a.ld_in = pitch(d, d->ld_tokens);
  a.sorted = sorted;
  a.ld_sorted = a.ld_out = pitch(d, d->ld_sorted);
  a.out = dsorted;
  a.offsets = offsets;
  a.slot = slot;
  a.weights = weights;
  a.dweights = dweights;
  const double bytes = (double)size * d->cols * (a.tokens + 2 * a.choices);
  const bool past = past_caches(bytes);
  Timed t(KC_ROUTE, stream, 3.0 * a.choices * d->cols, bytes);
  const hipStream_t st = (hipStream_t)stream;
  if (d->dtype == DYNB_F32) past ? launch_combine_grad<float, true>(a, st) : launch_choice_grad<float>(a, st);
  else past ? launch_combine_grad<bf16, true>(a, st) : launch_choice_grad<bf16>(a, st);
  return launched("route_combine_backward");
}
