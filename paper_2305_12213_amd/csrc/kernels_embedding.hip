// Rows of a table by token, and the table's gradient for every worker:
//   out[t] = scale * table[ids[t]];   dtable[k][v] = scale * sum over worker k's tokens t with ids[t] = v of dout[t].
// The gradient's tokens are sorted by (worker, id) first, so that every row of it is one sum in a fixed order, written
// once, and nothing is added by atomics but whole numbers.  What bounds it is the table, most of whose rows are zeros: 4 workers,
// 16384 tokens of 32000 x 2048, 1.05 GB in 210 us (5.0 TB/s) behind 25 us of sorting; a small one (7 workers, 1531 tokens of
// 1009 x 301) is three launches of 9, 6 and 9 us, chains of a few loads each.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "dynb_internal.h"
#include "row_access.h"

namespace dynb {
namespace {

// ---- lookup ----------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void lookup_kernel(const int32_t* ids, const T* table, int64_t ld_table, int64_t vocabulary,
                                                     T* out, int64_t ld_out, int64_t tokens, int cols, int granules, float scale) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, t = at / granules;
  if (t >= tokens) return;
  const int c = (int)(at % granules) * GRANULE, n = min(cols - c, GRANULE);
  const int64_t id = ids[t];
  float v[GRANULE] = {};
  if (id >= 0 && id < vocabulary) {
    load_part(table + id * ld_table + c, n, v);
#pragma unroll
    for (int e = 0; e < GRANULE; ++e) v[e] *= scale;
  }
  store_part(out + t * ld_out + c, n, v);
}

// ---- the sort ----------------------------------------------------------------------------------------------------
// By the lowest digit first, every pass stable.  Key: worker * vocabulary + id, and workers * vocabulary for what is no
// token of the vocabulary.  Every wave owns a stretch; it counts its digits, the counts are summed in the order (digit,
// workgroup, wave), and the wave goes over its stretch again, 64 tokens at a time, and hands out the places in order.
constexpr int WAVES = 16, THREADS = WAVES * 64, MOST_BITS = 9, DIGITS = 1 << MOST_BITS;
constexpr int64_t ALONE = 4096;           // so many tokens are sorted by one workgroup
constexpr int64_t MOST_BLOCKS = 128;      // whose counts a workgroup sums

struct SortPass {
  const int32_t* ids;                     // first pass: the tokens as they are
  const int32_t* keys; const int32_t* tokens;
  int32_t* keys_out; int32_t* tokens_out;
  int64_t n, per_block;
  int64_t vocabulary;
  int shift, bits;
  int32_t* counts;                        // [workgroups][digits]
};

__device__ inline int key_of(const SortPass& p, const Segs& s, int64_t i) {
  if (!p.ids) return p.keys[i];
  int k = 0;                              // the worker whose rows have i: the last one that begins at or before it
  for (int low = 0, high = s.K; low < high;) {
    const int mid = (low + high) / 2;
    if (s.off[mid] <= i) k = mid, low = mid + 1;
    else high = mid;
  }
  const int64_t id = p.ids[i];
  return (int)(id >= 0 && id < p.vocabulary ? k * p.vocabulary + id : s.K * p.vocabulary);
}

__global__ __launch_bounds__(THREADS) void digit_count_kernel(SortPass p, Segs s) {
  __shared__ int count[DIGITS];
  for (int e = threadIdx.x; e < DIGITS; e += THREADS) count[e] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * p.per_block, end = min(begin + p.per_block, p.n);
  for (int64_t i = begin + threadIdx.x; i < end; i += THREADS)
    atomicAdd(&count[(key_of(p, s, i) >> p.shift) & ((1 << p.bits) - 1)], 1);
  __syncthreads();
  for (int e = threadIdx.x; e < 1 << p.bits; e += THREADS) p.counts[((int64_t)blockIdx.x << p.bits) + e] = count[e];
}

__device__ inline void place_digits(const SortPass& p, const Segs& s, int (*place)[DIGITS], int* wave_total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, digits = 1 << p.bits, mask = digits - 1;
  for (int i = threadIdx.x; i < WAVES * DIGITS; i += THREADS) ((int*)place)[i] = 0;
  __syncthreads();
  const int64_t per = p.per_block / WAVES;          // (a multiple of 64)
  const int64_t begin = min(blockIdx.x * p.per_block + wave * per, p.n), end = min(begin + per, p.n);
  for (int64_t i = begin + lane; i < end; i += 64) atomicAdd(&place[wave][(key_of(p, s, i) >> p.shift) & mask], 1);
  __syncthreads();
  // first place of each digit, of this workgroup in it, of each wave in that
  const int d = threadIdx.x;
  int total = 0, ahead = 0;
  if (d < digits) {
    if (gridDim.x == 1) {
#pragma unroll
      for (int w = 0; w < WAVES; ++w) total += place[w][d];
    } else {
#pragma unroll 8
      for (int b = 0; b < (int)gridDim.x; ++b) {
        const int c = p.counts[((int64_t)b << p.bits) + d];
        ahead += b < (int)blockIdx.x ? c : 0;
        total += c;
      }
    }
  }
  int upto = total;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int v = __shfl_up(upto, o);
    upto += lane >= o ? v : 0;
  }
  if (lane == 63 && wave < DIGITS / 64) wave_total[wave] = upto;
  __syncthreads();
  if (d < digits) {
    int at = upto - total + ahead;
    for (int w = 0; w < wave; ++w) at += wave_total[w];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int c = place[w][d];
      place[w][d] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int64_t i0 = begin; i0 < end; i0 += 64) {
    const int64_t i = i0 + lane;
    const bool live = i < end;
    const int key = live ? key_of(p, s, i) : 0, digit = (key >> p.shift) & mask;
    uint64_t same = __ballot(live);
    for (int b = 0; b < p.bits; ++b) {
      const uint64_t set = __ballot((digit >> b) & 1);
      same &= (digit >> b) & 1 ? set : ~set;
    }
    const int before = __builtin_popcountll(same & (((uint64_t)1 << lane) - 1));
    const int to = live ? place[wave][digit] + before : 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (live) {
      if (before == 0) place[wave][digit] = to + __builtin_popcountll(same);
      p.keys_out[to] = key;
      p.tokens_out[to] = p.ids ? (int)i : p.tokens[i];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// (one workgroup alone goes on with `more` further passes, from what it wrote to where it read)
__global__ __launch_bounds__(THREADS) void digit_place_kernel(SortPass p, Segs s, int more, int all_bits) {
  __shared__ int place[WAVES][DIGITS];    // counts, then the next places
  __shared__ int wave_total[DIGITS / 64];
  for (;; --more) {
    place_digits(p, s, place, wave_total);
    if (more == 0) return;
    __syncthreads();
    int32_t *const keys = p.keys_out, *const tokens = p.tokens_out;
    p.keys_out = const_cast<int32_t*>(p.keys);
    p.tokens_out = const_cast<int32_t*>(p.tokens);
    p.keys = keys;
    p.tokens = tokens;
    p.ids = nullptr;
    p.shift += p.bits;
    p.bits = min(p.bits, all_bits - p.shift);
  }
}

// ---- the sums ----------------------------------------------------------------------------------------------------
// A token that appears often (a padding token may be all of them) would be one wave's long chain, and one fp32 sum whose
// roundings add up: the sorted tokens are cut into chunks of 16, and one whose tokens are all the same is summed beforehand; while
// a level has more than MOST_SUMS sums, 64 neighbouring ones of the same token are summed to one of the next.  A run is then its first
// tokens up to a chunk's end, its whole chunks up to the end of a sum of the next level and so on, and what is left of each level on
// the way back: every term goes through less than 1500 additions, whatever the run's length (2^22 equal rows in bf16 were off by 4e-3
// in one sum of their chunks).  131072 tokens of 32000 x 512, half of them one token: 127 us, 529 with chunks alone.  A level costs
// 2 to 9 us, which is why 1024 sums go without (16384 tokens of 32000 x 2048: 74 us, 83 with one; all of them one token: 166, 93).
// A lane has four neighbouring columns twice, 256 apart, so that every access of a
// wave is one stretch of memory; the numbers of 64 tokens are loaded at once and AHEAD of their rows are asked for together.
constexpr int CHUNK = 16, QUAD = 4, HALF = 64 * QUAD, SPAN = 2 * HALF;   // SPAN: columns of a wave
constexpr int AHEAD = 8, EACH = 64, MOST_SUMS = 1024;
// Sums of a level over n tokens, each over 16 * 64^level of them, and levels.  All sums are in one array, level by level.
__host__ __device__ constexpr int level_bits(int level) { return 4 + 6 * level; }
__host__ __device__ inline int64_t sums_of_level(int64_t n, int level) { return n >> level_bits(level); }
static_assert(1 << level_bits(0) == CHUNK && 1 << level_bits(1) == CHUNK * EACH, "bits of a level");
int levels_of(int64_t n) {
  int levels = 1;
  while (sums_of_level(n, levels - 1) > MOST_SUMS) ++levels;
  return levels;
}
int64_t sums_of(int64_t n) {
  int64_t sums = 0;
  for (int l = 0; l < levels_of(n); ++l) sums += sums_of_level(n, l);
  return sums;
}
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

struct TableGrad {
  const int32_t* keys; const int32_t* tokens;    // sorted
  const void* dout; int64_t ld_dout;
  float* sums;                                   // [levels: sums][cols]
  float* dtable; int64_t worker_stride;
  int64_t n; int vocabulary;
  int cols, workers, per, levels;
  float scale;
};

// The first n of four elements (n <= 0: none is read), zeros for the others; as loaded, and as values.
template <typename T> struct Quad;
template <> struct Quad<float> { u32x4 v; };
template <> struct Quad<bf16> { u32x2 v; };
__device__ inline Quad<float> load_quad(const float* p, int n) {
  Quad<float> q = {{0, 0, 0, 0}};
  if (n >= QUAD) {
    q.v = load16(p);
  } else if (n > 0) {
#pragma unroll
    for (int e = 0; e < QUAD - 1; ++e)
      if (e < n) q.v[e] = __float_as_uint(p[e]);
  }
  return q;
}
__device__ inline Quad<bf16> load_quad(const bf16* p, int n) {
  Quad<bf16> q = {{0, 0}};
  if (n >= QUAD) {
    q.v = *(const u32x2_any*)p;
  } else if (n > 0) {
    q.v[0] = ((const uint16_t*)p)[0];
    if (n > 1) q.v[0] |= (uint32_t)((const uint16_t*)p)[1] << 16;
    if (n > 2) q.v[1] = ((const uint16_t*)p)[2];
  }
  return q;
}
__device__ inline f32x4_any values(const Quad<float>& q) {
  return f32x4_any{__uint_as_float(q.v[0]), __uint_as_float(q.v[1]), __uint_as_float(q.v[2]), __uint_as_float(q.v[3])};
}
__device__ inline f32x4_any values(const Quad<bf16>& q) {
  return f32x4_any{__uint_as_float(q.v[0] << 16), __uint_as_float(q.v[0] & 0xffff0000u), __uint_as_float(q.v[1] << 16),
                   __uint_as_float(q.v[1] & 0xffff0000u)};
}
template <bool PAST> __device__ inline void store_quad(float* p, int n, const f32x4_any& v) {
  if (n >= QUAD) {
    if (PAST) __builtin_nontemporal_store(v, (f32x4_any*)p);
    else *(f32x4_any*)p = v;
  } else if (n > 0) {
#pragma unroll
    for (int e = 0; e < QUAD - 1; ++e)
      if (e < n) p[e] = v[e];
  }
}

// s += the rows of sorted tokens [from, to), in order (from and to the same in the whole wave)
template <typename T>
__device__ inline void add_rows(const TableGrad& p, int64_t from, int64_t to, int c, f32x4_any (&s)[2]) {
  const int n0 = p.cols - c, n1 = n0 - HALF;
  for (int64_t i0 = from; i0 < to; i0 += 64) {
    const int count = (int)min((int64_t)64, to - i0), lane = threadIdx.x & 63;
    const int mine = p.tokens[i0 + (lane < count ? lane : count - 1)];
    for (int i = 0; i < count; i += AHEAD) {
      Quad<T> q[AHEAD][2];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (i + u >= count) continue;                  // (uniform)
        const T* const row = (const T*)p.dout + (int64_t)__builtin_amdgcn_readlane(mine, i + u) * p.ld_dout + c;
        q[u][0] = load_quad(row, n0);
        q[u][1] = load_quad(row + HALF, n1);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (i + u >= count) continue;
        s[0] += values(q[u][0]);
        s[1] += values(q[u][1]);
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void chunk_rows_kernel(TableGrad p) {
  const int c = blockIdx.y * SPAN + (threadIdx.x & 63) * QUAD;
  for (int64_t chunk = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); (chunk + 1) * CHUNK <= p.n;
       chunk += (int64_t)gridDim.x * 4) {
    const int64_t first = chunk * CHUNK;
    const int key = p.keys[first];
    if (key != p.keys[first + CHUNK - 1] || key >= p.workers * p.vocabulary) continue;
    f32x4_any s[2] = {};
    add_rows<T>(p, first, first + CHUNK, c, s);
    float* const to = p.sums + chunk * p.cols + c;
    store_quad<false>(to, p.cols - c, s[0]);
    store_quad<false>(to + HALF, p.cols - c - HALF, s[1]);
  }
}

// s += the sums [from, to) of all levels' (from and to the same in the whole wave)
__device__ inline void add_sums(const TableGrad& p, int64_t from, int64_t to, int c, f32x4_any (&s)[2]) {
  const int n0 = p.cols - c, n1 = n0 - HALF;
#pragma unroll 8
  for (int64_t q = from; q < to; ++q) {
    const float* const at = p.sums + q * p.cols + c;
    s[0] += values(load_quad(at, n0));
    s[1] += values(load_quad(at + HALF, n1));
  }
}

// The sums of a level from those of the one below, which begin at `below`, where all their tokens are the same.
__global__ __launch_bounds__(256) void level_kernel(TableGrad p, int level, int64_t below) {
  const int c = blockIdx.y * SPAN + (threadIdx.x & 63) * QUAD, bits = level_bits(level);
  const int64_t i = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (i >= sums_of_level(p.n, level)) return;
  const int key = p.keys[i << bits];
  if (key != p.keys[((i + 1) << bits) - 1] || key >= p.workers * p.vocabulary) return;
  f32x4_any s[2] = {};
  add_sums(p, below + i * EACH, below + (i + 1) * EACH, c, s);
  float* const to = p.sums + (below + sums_of_level(p.n, level - 1) + i) * p.cols + c;
  store_quad<false>(to, p.cols - c, s[0]);
  store_quad<false>(to + HALF, p.cols - c - HALF, s[1]);
}

// Sorted tokens with keys below `key` (the whole wave takes part): 64 places at a time.
__device__ inline int64_t keys_below(const int32_t* keys, int64_t n, int key) {
  const int lane = threadIdx.x & 63;
  int64_t low = 0, high = n;                     // the answer is in [low, high]
  while (high > low) {
    const int64_t step = (high - low + 63) / 64, at = low + lane * step;
    const int less = __builtin_popcountll(__ballot(at < high && keys[at < high ? at : low] < key));
    if (less == 0) return low;
    const int64_t from = low + (less - 1) * step + 1;
    high = min(high, low + less * step);
    low = from;
  }
  return low;
}

// p.per neighbouring rows of the gradients to a wave: MOST_PER, which share a search, or fewer where waves are few (the
// first rows of a vocabulary are often those of its most frequent tokens), or more where a launch of MOST_GRID workgroups would not
// hold the table otherwise.
constexpr int MOST_PER = 8, ENOUGH_WAVES = 8192, MOST_GRID = 1 << 23;
template <typename T, bool PAST>
__global__ __launch_bounds__(256) void table_grad_kernel(TableGrad p) {
  const int lane = threadIdx.x & 63, all = p.workers * p.vocabulary;
  // (the spans of a row are neighbours in time too: as another dimension of the grid, each pass over the table met a part of the
  // memory channels, 237 us instead of 210)
  const int spans = (p.cols + SPAN - 1) / SPAN;
  const int first = (blockIdx.x / spans * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * p.per;
  if (first >= all) return;
  const int c = blockIdx.x % spans * SPAN + lane * QUAD, n0 = p.cols - c, n1 = n0 - HALF;
  int64_t at = keys_below(p.keys, p.n, first);
  int mine = at + lane < p.n ? p.keys[at + lane] : 0x7fffffff;      // the 64 keys from `at` on
  int worker = first / p.vocabulary, id = first % p.vocabulary;
  for (int row = first; row < first + p.per && row < all; ++row) {
    // this row's run begins at `begin`, the first of the 64 that is not below it
    const int less = __builtin_popcountll(__ballot(mine < row)), same = __builtin_popcountll(__ballot(mine == row));
    int64_t begin = at + less, end = begin + same;
    if (less + same == 64) {                                        // it may go on behind them
      end = keys_below(p.keys, p.n, row + 1);
      begin = less == 64 ? keys_below(p.keys, p.n, row) : begin;
      at = end;
      mine = at + lane < p.n ? p.keys[at + lane] : 0x7fffffff;
    }
    f32x4_any s[2] = {};
    if (begin < end) {
      int64_t sum = (begin + CHUNK - 1) / CHUNK;                    // the next sum of the level, of those in the run
      if (sum < end / CHUNK) {
        add_rows<T>(p, begin, sum * CHUNK, c, s);
        int level = 0;
        int64_t base = 0;                                           // where the level's sums begin
        for (; level + 1 < p.levels; ++level) {
          const int64_t above = (sum + EACH - 1) / EACH;
          if (above >= end >> level_bits(level + 1)) break;
          add_sums(p, base + sum, base + above * EACH, c, s);
          base += sums_of_level(p.n, level);
          sum = above;
        }
        for (;;) {
          add_sums(p, base + sum, base + (end >> level_bits(level)), c, s);
          if (level == 0) break;
          sum = (end >> level_bits(level)) * EACH;
          base -= sums_of_level(p.n, --level);
        }
        add_rows<T>(p, end / CHUNK * CHUNK, end, c, s);
      } else {
        add_rows<T>(p, begin, end, c, s);
      }
      s[0] *= p.scale;
      s[1] *= p.scale;
    }
    float* const to = p.dtable + worker * p.worker_stride + (int64_t)id * p.cols + c;
    store_quad<PAST>(to, n0, s[0]);
    store_quad<PAST>(to + HALF, n1, s[1]);
    if (++id == p.vocabulary) {
      id = 0;
      ++worker;
    }
  }
}

int check(const dynb_embedding_desc* d, const char* who) {
  if (!d) return fail(DYNB_ERR_BADARG, "%s: null description", who);
  if (d->dtype != DYNB_F32 && d->dtype != DYNB_BF16) return fail(DYNB_ERR_BADARG, "%s: unknown type of the rows", who);
  if (d->cols < 1 || d->cols > 1 << 20) return fail(DYNB_ERR_BADARG, "%s: cols out of range", who);
  if (d->vocabulary < 1 || d->vocabulary > 1 << 24) return fail(DYNB_ERR_BADARG, "%s: vocabulary out of range", who);
  if (d->tokens < 0 || d->tokens > INT32_MAX) return fail(DYNB_ERR_BADARG, "%s: tokens out of range", who);
  if (!std::isfinite(d->scale)) return fail(DYNB_ERR_BADARG, "%s: scale is not finite", who);
  for (int64_t ld : {d->ld_table, d->ld_out, d->ld_dout})
    if (ld != 0 && ld < d->cols) return fail(DYNB_ERR_BADARG, "%s: a row pitch is below cols", who);
  return DYNB_OK;
}

int64_t sort_blocks(int64_t n) { return n <= ALONE ? 1 : std::min<int64_t>((n + THREADS * 2 - 1) / (THREADS * 2), MOST_BLOCKS); }

// Where the parts of the workspace begin: keys and tokens twice, counts, the sums.
struct Parts {
  int64_t keys, tokens, counts, sums, end;       // (keys, tokens: the second ones follow the first)
};
Parts parts_of(const dynb_embedding_desc* d) {
  Parts w;
  const int64_t each = round_up(d->tokens * 4, 16), B = sort_blocks(d->tokens);
  w.keys = 0;
  w.tokens = 2 * each;
  w.counts = 4 * each;
  w.sums = w.counts + (B > 1 ? B * DIGITS * 4 : 0);
  w.end = w.sums + round_up(sums_of(d->tokens) * d->cols * 4, 16);
  return w;
}

int64_t table_grad_blocks(const TableGrad& p) {
  return ((int64_t)p.workers * p.vocabulary + 4 * p.per - 1) / (4 * p.per) * ((p.cols + SPAN - 1) / SPAN);
}

template <typename T>
void launch_table_grad(const TableGrad& p, hipStream_t st) {
  if (p.n >= CHUNK)
    hipLaunchKernelGGL(chunk_rows_kernel<T>, dim3((unsigned)std::min<int64_t>((p.n / CHUNK + 3) / 4, 1 << 20), (p.cols + SPAN - 1) / SPAN), dim3(256), 0, st, p);
  int64_t below = 0;
  for (int l = 1; l < p.levels; below += sums_of_level(p.n, l - 1), ++l)
    hipLaunchKernelGGL(level_kernel, dim3((unsigned)((sums_of_level(p.n, l) + 3) / 4), (p.cols + SPAN - 1) / SPAN), dim3(256), 0, st, p, l, below);
  const dim3 grid((unsigned)table_grad_blocks(p));
  if (past_caches(4.0 * p.workers * p.vocabulary * p.cols)) hipLaunchKernelGGL((table_grad_kernel<T, true>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((table_grad_kernel<T, false>), grid, dim3(256), 0, st, p);
}

}  // namespace
}  // namespace dynb

using namespace dynb;

extern "C" int dynb_embedding(const dynb_embedding_desc* d, const int32_t* ids, const void* table, void* out, void* stream) {
  if (int rc = check(d, "embedding")) return rc;
  const size_t size = d->dtype == DYNB_F32 ? 4 : 2;
  if (off_by(ids, 4) || off_by(table, size) || off_by(out, size))
    return fail(DYNB_ERR_BADARG, "embedding: a pointer is not a multiple of its element's size");
  if (d->tokens == 0) return DYNB_OK;
  if (!ids || !table || !out) return fail(DYNB_ERR_BADARG, "embedding: null pointer");
  const int granules = (d->cols + GRANULE - 1) / GRANULE;
  const int64_t blocks = (d->tokens * granules + 255) / 256;
  if (blocks > INT32_MAX / 256) return fail(DYNB_ERR_UNSUPPORTED, "embedding: rows of more than 2^31 - 256 pieces of 8 columns");
  const int64_t lt = d->ld_table ? d->ld_table : d->cols, lo = d->ld_out ? d->ld_out : d->cols;
  Timed t(KC_EMBEDDING, stream, (double)d->tokens * d->cols, 2.0 * size * d->tokens * d->cols);
  if (d->dtype == DYNB_F32)
    hipLaunchKernelGGL(lookup_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, ids, (const float*)table,
                       lt, d->vocabulary, (float*)out, lo, d->tokens, d->cols, granules, d->scale);
  else
    hipLaunchKernelGGL(lookup_kernel<bf16>, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, ids, (const bf16*)table,
                       lt, d->vocabulary, (bf16*)out, lo, d->tokens, d->cols, granules, d->scale);
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "embedding launch failed");
}

extern "C" size_t dynb_embedding_backward_workspace_bytes(const dynb_embedding_desc* d, int32_t K) {
  if (check(d, "embedding_backward_workspace_bytes") || K < 1 || K > DYNB_MAX_WORKERS) return 0;
  return (size_t)parts_of(d).end;
}

extern "C" int dynb_embedding_backward(const dynb_embedding_desc* d, const int32_t* b, int32_t K, const int32_t* ids,
                                       const void* dout, float* dtable, int64_t worker_stride, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  Segs s;
  if (int rc = check(d, "embedding_backward")) return rc;
  if (int rc = segments_of(b, K, "embedding_backward", s)) return rc;
  if (s.off[K] != d->tokens) return fail(DYNB_ERR_BADARG, "embedding_backward: sum(b) is not the number of tokens");
  const size_t size = d->dtype == DYNB_F32 ? 4 : 2;
  if (off_by(ids, 4) || off_by(dout, size) || off_by(dtable, 4))
    return fail(DYNB_ERR_BADARG, "embedding_backward: a pointer is not a multiple of its element's size");
  if (!dtable || (d->tokens > 0 && (!ids || !dout))) return fail(DYNB_ERR_BADARG, "embedding_backward: null pointer");
  if (K > 1 && worker_stride < d->vocabulary * d->cols)
    return fail(DYNB_ERR_BADARG, "embedding_backward: workers' gradients overlap");
  const Parts w = parts_of(d);
  if (w.end && (!workspace || workspace_bytes < (size_t)w.end || off_by(workspace, 16)))
    return fail(DYNB_ERR_BADARG, "embedding_backward: workspace is null, too small or not 16-byte aligned");
  const int64_t table_rows = K * d->vocabulary, at_once = (int64_t)4 * (MOST_GRID / ((d->cols + SPAN - 1) / SPAN));
  const int per = (int)std::max({(int64_t)1, std::min<int64_t>(MOST_PER, table_rows / ENOUGH_WAVES), (table_rows + at_once - 1) / at_once});
  TableGrad grad = {nullptr, nullptr, dout, d->ld_dout ? d->ld_dout : d->cols, (float*)((char*)workspace + w.sums), dtable,
                       worker_stride, d->tokens, (int)d->vocabulary, d->cols, K, per, levels_of(d->tokens), d->scale};
  const hipStream_t st = (hipStream_t)stream;
  Timed t(KC_EMBEDDING, stream, (double)d->tokens * d->cols,
          4.0 * K * d->vocabulary * d->cols + (double)size * d->tokens * d->cols);
  char* const ws = (char*)workspace;
  const int64_t each = round_up(d->tokens * 4, 16);
  int32_t *keys[2] = {(int32_t*)(ws + w.keys), (int32_t*)(ws + w.keys + each)};
  int32_t *tokens[2] = {(int32_t*)(ws + w.tokens), (int32_t*)(ws + w.tokens + each)};
  int cur = 0;
  if (d->tokens > 0) {
    int bits = 1;                                 // of the keys 0 .. K * vocabulary
    while (((int64_t)1 << bits) <= K * d->vocabulary) ++bits;
    const int passes = (bits + MOST_BITS - 1) / MOST_BITS, per_pass = (bits + passes - 1) / passes;
    const int64_t B = sort_blocks(d->tokens), per = round_up((d->tokens + B - 1) / B, THREADS);
    const dim3 grid((unsigned)((d->tokens + per - 1) / per));
    for (int i = 0; i < passes; ++i) {
      SortPass p = {i ? nullptr : ids, keys[cur], tokens[cur], keys[1 - cur], tokens[1 - cur], d->tokens, per, d->vocabulary,
                    i * per_pass, std::min(per_pass, bits - i * per_pass), (int32_t*)(ws + w.counts)};
      if (grid.x == 1) {
        hipLaunchKernelGGL(digit_place_kernel, grid, dim3(THREADS), 0, st, p, s, passes - 1, bits);
        cur = passes & 1;
        break;
      }
      hipLaunchKernelGGL(digit_count_kernel, grid, dim3(THREADS), 0, st, p, s);
      hipLaunchKernelGGL(digit_place_kernel, grid, dim3(THREADS), 0, st, p, s, 0, bits);
      cur = 1 - cur;
    }
  }
  grad.keys = keys[cur];
  grad.tokens = tokens[cur];
  if (d->dtype == DYNB_F32) launch_table_grad<float>(grad, st);
  else launch_table_grad<bf16>(grad, st);
  return hipGetLastError() == hipSuccess ? DYNB_OK : fail(DYNB_ERR_HIP, "embedding_backward launch failed");
}
