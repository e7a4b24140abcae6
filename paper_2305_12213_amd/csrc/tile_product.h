// Matrix products over groups of rows, with what follows a product computed on its results while they are in registers:
//   ROWS_NN   out[i] = sum_k x[i][k] W[e][k][j]          rows i of group e (an expert's rows, or all of a dense layer)
//   ROWS_NT   out[i] = sum_k x[i][k] W[e][j][k]          ... against the weight turned: gradients of the rows
//   WEIGHTS   out[g][i][j] = sum_r x[r][i] y[r][j]       over the rows r of group g: gradients of the weights
// Where a group begins and ends stands in device memory, so nothing waits for the host: a workgroup finds its group by
// itself, the grid is the largest that the sizes allow, and workgroups past the last tile end at once.
//
// A stage is 128 bytes of reduction per row (64 bf16, 32 fp32), in LDS as memory has it.  An operand whose rows run
// along the reduction is read in granules of 16 bytes; of one whose rows run across it ("turned") bf16 is fetched by the LDS
// transpose reads, fp32 element by element.  One step is two granules: a 32 x 32 x 16 matrix instruction in bf16, four of
// 32 x 32 x 2 in fp32, whose k are numbered so that both operands' lanes hold the same ones.
//
// Copies go from memory straight to LDS, a ring of NB stages, a step's fragments are fetched one step ahead, and
// fetches and copies stand between the matrix instructions (as in the dense layers' products).  Rows that are no
// multiple of 16 bytes are copied element by element in fp32, and in bf16 pass through registers, which can fill up
// partial granules with zeros.
//
// What bounds it.  Long reductions in bf16: the matrix instructions at the clock that they leave (8192^3 915 us, 1200 TFLOP/s; the clock
// falls to 1.8 GHz).  Short ones (gradients of weights from a few hundred rows): the stores, which all workgroups come to
// at about the same time -- 16 workers of 256 rows, 4096 x 4096 in bf16: 220 us, of which 115 are products and 140 would be the stores
// alone.  Workgroups that stay and copy the next tile's stages while they store were measured too, on tiles of 256 x 256 with eight
// waves of 128 sums a lane: 8 % slower where
// tiles are many (registers run out around the longer code, and wait counters are in order, so that the next stage waits for the
// stores all the same), equal where reductions are short; not with smaller tiles to a wave.  fp32: the matrix instructions, 4096^3 982 to 1060 us, 130 to 140 TFLOP/s.
// Few rows: the weights' way from memory (64 experts of 3 x 2048 x 1024 in bf16, two rows each: 130 us, 6.2 TB/s).
#ifndef DYNB_TILE_PRODUCT_H
#define DYNB_TILE_PRODUCT_H

#include <hip/hip_runtime.h>

#include "device_rows.h"
#include "dynb_internal.h"
#include "lds_async.h"
#include "row_access.h"

namespace dynb {

enum Form { ROWS_NN, ROWS_NT, WEIGHTS };

struct Product {
  const void* A[2];
  const void* B[2];          // of two products that share A (dual), or see pairs
  int64_t lda, ldb;          // elements
  int64_t b_stride;          // elements from one group's B to the next (ROWS_*)
  int M, N;                  // WEIGHTS: output rows; output columns of one product
  int K;                     // ROWS_*: reduction length of one pair
  int pairs;                 // 2: both A and both B (ROWS_*); both B, each with a result of its own (WEIGHTS)
  int64_t rows;              // rows there are (ROWS_*: of A; WEIGHTS: of both)
  const int32_t* offsets;    // ROWS_*: device [groups + 1], or null: one group of all rows.  WEIGHTS: see `segments`
  const int32_t* segments;   // WEIGHTS: device [groups / workers][workers + 1]; null: `offsets`, or the launch's Segs
  int groups, workers;
  int splits;                // parts that the reduction is divided into; > 1: sums of the parts go to `partial`
  float* partial;            // fp32 [splits][partial_rows][columns of all products]
  int64_t partial_rows;
};

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t PARKED = 0x80000000u;   // an offset past the end of a buffer: the copy writes zeros

// Workgroup -> place in the tile sequence: consecutive workgroups go round the 8 XCDs, each of which gets a run of it.
__device__ inline int run_of_xcd(int pid, int total) {
  if (total < 16) return pid;
  const int per = total / 8, extra = total % 8, xcd = pid % 8;
  return xcd * per + (xcd < extra ? xcd : extra) + pid / 8;
}
// Gradients of weights: every group's tiles are spread over all XCDs (groups differ in their rows, so that whole groups to
// an XCD left seven of them waiting: 32 groups of 16384 rows, 2048 x 2048, 545 us), in runs where there are enough of them: places
// for a multiple of 8 tiles, some of them empty.
constexpr int XCD_RUNS = 32;
__host__ __device__ inline int weight_places(int tiles) { return tiles < XCD_RUNS ? tiles : (tiles + 7) / 8 * 8; }
// Place -> tile, in bands of 8 tile rows, so that a run covers a compact rectangle.
__device__ inline void tile_of_place(int t, int tiles_i, int tiles_j, int& ti, int& tj) {
  const int bsz = 8 * tiles_j, b0 = t / bsz, r = t % bsz;
  const int rows = tiles_i - b0 * 8 < 8 ? tiles_i - b0 * 8 : 8;
  ti = b0 * 8 + r % rows;
  tj = r / rows;
}

__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Rows [first, last) of a group, whatever stands in memory kept inside [0, rows).
__device__ inline void group_rows(const int32_t* bounds, int64_t rows, int64_t& first, int64_t& last) {
  const int64_t a = bounds[0], b = bounds[1];
  first = a < 0 ? 0 : a > rows ? rows : a;
  last = b < first ? first : b > rows ? rows : b;
}
// Sum over the wave's lanes up to this one.
__device__ inline int sum_upto(int v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    v += (int)(threadIdx.x & 63) >= d ? o : 0;
  }
  return v;
}
// The groups' tiles of BM rows: how many there are, and which group has tile `ti`, with its rows from that tile on.  The bounds of
// up to 256 groups are asked for at once and stay in registers, those of more are read again in the search.
struct RowTiles {
  static constexpr int HELD = 4;
  int first[HELD], last[HELD];            // rows of group 64 c + lane
  int total;
};
__device__ inline void rows_of(const Product& p, int e, int& first, int& last) {
  int64_t f = 0, l = 0;
  if (e < p.groups) group_rows(p.offsets + e, p.rows, f, l);
  first = (int)f;
  last = (int)l;
}
__device__ inline int tiles_between(int first, int last, int BM) { return (int)(((uint32_t)(last - first) + BM - 1) / BM); }
__device__ inline void count_tiles(const Product& p, int BM, RowTiles& t) {
  t.total = (int)((p.rows + BM - 1) / BM);
  if (!p.offsets) return;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int c = 0; c < RowTiles::HELD; ++c) rows_of(p, 64 * c + lane, t.first[c], t.last[c]);
  int mine = 0;
#pragma unroll
  for (int c = 0; c < RowTiles::HELD; ++c) mine += tiles_between(t.first[c], t.last[c], BM);
  for (int e = 64 * RowTiles::HELD + lane; e < p.groups; e += 64) {
    int f, l;
    rows_of(p, e, f, l);
    mine += tiles_between(f, l, BM);
  }
  t.total = __builtin_amdgcn_readlane(sum_upto(mine), 63);
}
__device__ inline void find_group(const Product& p, int BM, const RowTiles& t, int ti, int& group, int64_t& first, int64_t& last) {
  group = 0;
  first = (int64_t)ti * BM;
  last = p.rows;
  if (!p.offsets) return;
  int before = 0;
  auto look = [&](int c, int f, int l) {
    const int mine = tiles_between(f, l, BM), upto = before + sum_upto(mine);
    const uint64_t has = __ballot(ti >= upto - mine && ti < upto);
    before = __builtin_amdgcn_readlane(upto, 63);
    if (!has) return false;
    const int lane = __builtin_ctzll(has);
    group = 64 * c + lane;
    first = __builtin_amdgcn_readlane(f, lane) + (int64_t)(ti - __builtin_amdgcn_readlane(upto - mine, lane)) * BM;
    last = __builtin_amdgcn_readlane(l, lane);
    return true;
  };
#pragma unroll
  for (int c = 0; c < RowTiles::HELD; ++c)
    if (64 * c < p.groups && look(c, t.first[c], t.last[c])) return;
  for (int c = RowTiles::HELD; 64 * c < p.groups; ++c) {
    int f, l;
    rows_of(p, 64 * c + (threadIdx.x & 63), f, l);
    if (look(c, f, l)) return;
  }
  last = first = 0;       // (not reached: ti is below the number of tiles)
}

// How an operand's granules reach LDS.  DIRECT: copied, all of them whole and at multiples of 16 bytes.  SINGLES (fp32): copied
// element by element, four times the copies, wherever rows begin and end.  SHIFTED: through registers; the last granule of a row is
// loaded so that it ends with the row and shifted into its place, which needs rows of a granule at least and keeps every load
// unconditional and in flight until it is stored.  SINGLY: element by element.
enum Access { DIRECT, SHIFTED, SINGLY, SINGLES };

template <typename T> __device__ inline u32x4 load_singly(const T* p, int n) {
  u32x4 r = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 16 / (int)sizeof(T); ++e) {
    if (e >= n) continue;
    if (sizeof(T) == 4) r[e] = ((const uint32_t*)p)[e];
    else r[e / 2] |= (uint32_t)((const uint16_t*)p)[e] << (16 * (e & 1));
  }
  return r;
}
// The last n of a granule's elements first, zeros behind them (n <= 0: zeros).
template <typename T> __device__ inline u32x4 shifted(u32x4 v, int n) {
  constexpr int G = 16 / (int)sizeof(T);
  if (n >= G) return v;
  const int bytes = (G - max(n, 0)) * (int)sizeof(T);
  if (bytes & 8) v = u32x4{v[2], v[3], 0, 0};
  if (bytes & 4) v = u32x4{v[1], v[2], v[3], 0};
  if (bytes & 2) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
  return n > 0 ? v : u32x4{0, 0, 0, 0};
}

// Slot of granule g in reduction row k of a turned tile with rows of `pitch` bytes: the rows that one read touches
// at once fall into different banks (bf16: four neighbouring ones, 64 bytes of each; fp32: rows 4 apart, 128 bytes of each).
template <typename T> __device__ constexpr int turned_swizzle(int k, int pitch) {
  return sizeof(T) == 4 ? ((k >> 2) & 1) << 3 : pitch >= 256 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
}

// ... of granule g of row r of a tile whose rows run along the reduction, DEPTH granules each: 16 neighbouring rows, read at one
// granule, fall into 64 different banks.
template <int DEPTH> __device__ constexpr int along_swizzle(int r) {
  return DEPTH == 8 ? (((r >> 1) & 3) << 1) | ((r >> 3) & 1) : (((r >> 2) & 1) << 1) | ((r >> 3) & 1);
}

// LDS written by some lanes of a wave and read by others.
__device__ inline void patch_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A tile of BM x BN results, WM x WN waves.  DUAL: two products with BN / 2 columns each, which share A; a wave has the same
// columns of both.  Ep: what is done with 8 neighbouring results of a row.  SOON: of a stage's copies, eighths that are
// issued in the last step of the stage that releases its buffer, and in the first step of the next.
template <typename T, int FORM, bool DUAL, int BM, int BN, int WM, int WN, int DEPTH, int NB, int SOON, Access ACCESS, class Ep>
__global__ __launch_bounds__(WM * WN * 64, WM * WN == 8 ? 1 : (ACCESS == SHIFTED || ACCESS == SINGLES) && DEPTH == 4 ? 3 : 2) void product_kernel(Product p, Segs segs, Ep ep) {
  constexpr bool TA = FORM == WEIGHTS, TB = FORM != ROWS_NT;
  constexpr int G = 16 / sizeof(T), BK = DEPTH * G, STEPS = DEPTH / 2, NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  constexpr bool COPIED = ACCESS == DIRECT || ACCESS == SINGLES;
  constexpr int BNS = DUAL ? BN / 2 : BN, NBUF = COPIED ? NB : 2;
  constexpr int CA = BM * DEPTH / 64 / NW, CB = BN * DEPTH / 64 / NW, NC = CA + CB;   // copies of 1 KB per wave and stage
  constexpr uint32_t STAGE_A = BM * DEPTH * 16, STAGE = (BM + BN) * DEPTH * 16;
  constexpr int CW = 32 * TN, EP = CW + 4;                          // a wave's columns, row pitch of its patch
  static_assert(BM * DEPTH % (64 * NW) == 0 && BN * DEPTH % (64 * NW) == 0 && (DEPTH == 4 || DEPTH == 8), "whole copies");
  static_assert(!DUAL || TN % 2 == 0, "a wave has columns of both products");
  constexpr uint32_t AREA = NBUF * STAGE > NW * 32 * EP * 4 ? NBUF * STAGE : NW * 32 * EP * 4;   // (the patches come last)
  static_assert(!TA || BM * (int)sizeof(T) >= 256, "a turned A has the wide swizzle");
  __shared__ uint4 ring[AREA / 16];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN, l31 = lane & 31, h = lane >> 5;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)&ring[0];

  // ---- which tile
  int group, tj, depth, second = 0;
  int64_t i0, i_end, r0 = 0;              // output rows; WEIGHTS: first reduction row
  const int tiles_j = (p.N + BNS - 1) / BNS;
  if constexpr (FORM == WEIGHTS) {
    const int tiles_i = (p.M + BM - 1) / BM;
    const int tiles = tiles_i * tiles_j, places = weight_places(tiles);
    int place = blockIdx.x % places, ti;
    group = blockIdx.x / places;
    second = group / p.groups;            // (pairs = 2: the other B, the other result)
    group %= p.groups;
    if (places >= XCD_RUNS) {
      // (every XCD at other groups: tiles of one are stored while those of another are computed)
      group = (group + place % 8 * p.groups / 8) % p.groups;
      place = place % 8 * (places / 8) + place / 8;
    }
    if (place >= tiles) return;
    tile_of_place(place, tiles_i, tiles_j, ti, tj);
    i0 = (int64_t)ti * BM;
    i_end = p.M;
    int64_t last;
    if (p.segments) group_rows(p.segments + (int64_t)(group / p.workers) * (p.workers + 1) + group % p.workers, p.rows, r0, last);
    else if (p.offsets) group_rows(p.offsets + group, p.rows, r0, last);
    else r0 = segs.off[group], last = segs.off[group + 1];
    r0 = uniform((int)r0);
    depth = uniform((int)(last - r0));
  } else {
    RowTiles rt;
    count_tiles(p, BM, rt);
    const int tiles_i = uniform(rt.total);
    const int total = tiles_i * tiles_j;
    if ((int)blockIdx.x >= total) return;
    int ti;
    tile_of_place(run_of_xcd(blockIdx.x, total), tiles_i, tiles_j, ti, tj);
    find_group(p, BM, rt, ti, group, i0, i_end);
    group = uniform(group);
    i0 = uniform((int)i0);
    i_end = uniform((int)i_end);
    depth = p.K;
  }
  const int j0 = tj * BNS;

  // ---- the stages of this workgroup
  const int per_pair = (int)(((uint32_t)depth + BK - 1) / BK), all = FORM == WEIGHTS ? per_pair : per_pair * p.pairs;
  const int part = (all + p.splits - 1) / p.splits;
  const int s_begin = p.splits > 1 ? min((int)blockIdx.y * part, all) : 0;
  const int s_end = p.splits > 1 ? min(s_begin + part, all) : all;
  const int64_t stepA = TA ? (int64_t)BK * p.lda * sizeof(T) : DEPTH * 16, stepB = TB ? (int64_t)BK * p.ldb * sizeof(T) : DEPTH * 16;
  // first byte of the tile in the operands of pair q
  auto base_a = [&](int q) {
    return (uint64_t)(uintptr_t)p.A[q] + (TA ? r0 * p.lda + i0 : i0 * p.lda) * sizeof(T);
  };
  auto base_b = [&](int q) {
    return (uint64_t)(uintptr_t)p.B[FORM == WEIGHTS ? second : q] +
           (FORM == WEIGHTS ? r0 * p.ldb + j0 : group * p.b_stride + (TB ? (int64_t)j0 : j0 * p.ldb)) * sizeof(T);
  };
  int next = s_begin;                     // the stage that is copied next, where it stands, and what is left of the reduction
  uint64_t from[3];                       // A, B, the other product's B
  int left;
  auto enter = [&](int q, int s) {        // stage s of pair q
    from[0] = base_a(q) + s * stepA;
    from[1] = base_b(q) + s * stepB;
    if (DUAL) from[2] = base_b(1) + s * stepB;
    left = depth - s * BK;
  };
  const int turn_at = FORM != WEIGHTS && !DUAL && p.pairs == 2 ? per_pair : -1;      // where the second pair begins
  const uint64_t other[2] = {base_a(1), base_b(1)};
  if (turn_at >= 0 && next >= turn_at) enter(1, next - turn_at);
  else enter(0, next);
  if (next >= s_end) left = 0;
  auto next_stage = [&]() {
    ++next;
    from[0] += stepA;
    from[1] += stepB;
    if (DUAL) from[2] += stepB;
    left -= BK;
    if (FORM != WEIGHTS && !DUAL) {       // (selects: no branch in the inner loop)
      const bool turn = next == turn_at;
      from[0] = turn ? other[0] : from[0];
      from[1] = turn ? other[1] : from[1];
      left = turn ? depth : left;
    }
    left = next >= s_end ? 0 : left;      // (copies past the last stage keep the waits constant: zeros)
  };

  // ---- copies: block c of a tile is 64 granules, lane l's lands in slot 64 c + l.  SINGLES: a quarter of a block at a time, an
  // element per lane.
  constexpr int PER = ACCESS == SINGLES ? 4 : 1, NP = NC * PER, WIDTH = ACCESS == SINGLES ? 1 : G;   // WIDTH: elements of a lane
  static_assert(ACCESS != SINGLES || sizeof(T) == 4, "copies of 4 bytes");
  int64_t off[NP];                        // bytes from the stage's first (copied: below 2^31)
  int need[NP];                           // a granule (SINGLES: an element) is there where more than this is left of the reduction
  int have[NP];                           // ... and so many of its elements (turned operands; the others: all or none)
#pragma unroll
  for (int v = 0; v < NP; ++v) {
    const int u = v / PER;
    const bool isA = u < CA;
    const int c = isA ? CA * wave + u : (CB * wave + u - CA) % (BNS * DEPTH / 64);      // (dual: block within its product's half)
    const int in = PER == 1 ? lane : 16 * (v % PER) + lane / 4, e = PER == 1 ? 0 : lane % 4;   // granule of the block, element of it
    const bool turned = isA ? TA : TB;
    const int64_t ld = isA ? p.lda : p.ldb, limit = isA ? i_end - i0 : p.N - j0;
    if (turned) {
      const int row = isA ? BM / G : BNS / G, s = 64 * c + in, k = s / row;
      const int g = (s % row) ^ turned_swizzle<T>(k, row * 16);
      off[v] = k * ld * (int64_t)sizeof(T) + g * 16 + e * 4;
      need[v] = k;
      have[v] = (int)max((int64_t)0, min((int64_t)WIDTH, limit - g * G - e));
    } else {
      const int r = 64 / DEPTH * c + in / DEPTH, g = in % DEPTH ^ along_swizzle<DEPTH>(r);
      off[v] = r * ld * (int64_t)sizeof(T) + g * 16 + e * 4;
      need[v] = g * G + e;
      have[v] = r < limit ? WIDTH : 0;
    }
    if (COPIED && have[v] == 0) need[v] = 0x7fffffff;
  }
  auto source = [&](int u) { return u < CA ? 0 : DUAL && (CB * wave + u - CA) >= BNS * DEPTH / 64 ? 2 : 1; };
  auto slot_of = [&](int u) { return u < CA ? (CA * wave + u) * 1024u : STAGE_A + (CB * wave + u - CA) * 1024u; };
  auto copy_one = [&](uint32_t buf, int v) {
    const int u = v / PER;
    const uint64_t a = from[source(u)];
    const i32x4 r = {(int)(uint32_t)a, (int)((uint32_t)(a >> 32) & 0xffffu), (int)PARKED, BUFFER_32BIT};
    const uint32_t at = need[v] < left ? (uint32_t)off[v] : PARKED, to = lds + buf + slot_of(u);
    if constexpr (ACCESS == SINGLES) async_copy_256_buffer(r, at, to + v % PER * 256);
    else async_copy_1k_buffer(r, at, to);
  };

  // ---- fragments: element (row or column l31, k of half h) of two granules
  const char* const base = (const char*)&ring[0];
  constexpr int PA = BM * sizeof(T), PB = BNS * sizeof(T);          // pitches of turned tiles
  // turned bf16: 16 lanes fetch 4 reduction rows x 16 features with a transpose read (lane r supplies the address of
  // features 4 (r % 4) .. of row r / 4 and receives feature r of the 4 rows)
  const int tg = lane >> 4, tr = lane & 15;
  auto turned_at = [&](int feat0, int pitch) {
    if (sizeof(T) == 4) {
      const int f = feat0 + l31;
      return 4 * h * pitch + (((f >> 2) ^ (h << 3)) * 16) + (f & 3) * 4;
    }
    const int f = feat0 + 16 * (tg & 1) + 4 * (tr & 3), k = 8 * (tg >> 1) + (tr >> 2);
    return k * pitch + (((f >> 3) ^ turned_swizzle<T>(k, pitch)) * 16) + (f & 7) * 2;
  };
  int at[STEPS], atA[TA ? TM : 1], atB[TB ? TN : 1];
#pragma unroll
  for (int kk = 0; kk < STEPS; ++kk) at[kk] = (l31 * DEPTH + ((2 * kk + h) ^ along_swizzle<DEPTH>(l31))) * 16;
  if constexpr (TA) {
#pragma unroll
    for (int a = 0; a < TM; ++a) atA[a] = turned_at(wm * (BM / WM) + a * 32, PA);
  }
  auto sub_column = [&](int b) { return DUAL ? wn * (CW / 2) + b % (TN / 2 ? TN / 2 : 1) * 32 : wn * CW + b * 32; };
  if constexpr (TB) {
#pragma unroll
    for (int b = 0; b < TN; ++b)
      atB[b] = STAGE_A + (DUAL && b >= TN / 2 ? BNS * DEPTH * 16 : 0) + turned_at(sub_column(b), PB);
  }
  auto turned_fragment = [&](uint32_t where, int kk, int pitch) {
    if constexpr (sizeof(T) == 4) {
      f32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const float*)(base + where + (kk * 8 + j) * pitch);
      return __builtin_bit_cast(u32x4, v);
    } else {
      const s16x4 lo = lds_read_tr(lds + where + kk * 16 * pitch), hi = lds_read_tr(lds + where + (kk * 16 + 4) * pitch);
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(u32x4, v);
    }
  };
  u32x4 fa[2][TM], fb[2][TN];             // [register set: the step's parity]
  auto fetch_one = [&](uint32_t buf, int kk, int f) {
    if (f < TM) {
      if constexpr (TA) fa[kk & 1][f] = turned_fragment(buf + atA[f], kk, PA);
      else fa[kk & 1][f] = *(const u32x4*)(base + buf + (wm * (BM / WM) + f * 32) * DEPTH * 16 + at[kk]);
    } else {
      const int b = f - TM;
      if constexpr (TB) fb[kk & 1][b] = turned_fragment(buf + atB[b], kk, PB);
      else fb[kk & 1][b] = *(const u32x4*)(base + buf + (BM + wn * CW + b * 32) * DEPTH * 16 + at[kk]);
    }
  };
  static_assert(TB || !DUAL, "two products at a time: B turned");
  f32x16 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.f;
  // B's columns as the instruction's rows: a lane then has 4 neighbouring columns of the output.  fp32: the four instructions of a
  // step go round the tiles, so that neighbours do not wait for each other's sums.
  constexpr int NM = TM * TN * (sizeof(T) == 4 ? 4 : 1), NF = TM + TN;
  auto mma_one = [&](int set, int m) {
    const int a = m % TM, b = m / TM % TN;
    if constexpr (sizeof(T) == 4) {
      const int j = m / (TM * TN);
      const f32x4 x = __builtin_bit_cast(f32x4, fa[set][a]), w = __builtin_bit_cast(f32x4, fb[set][b]);
      acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[j], x[j], acc[a][b], 0, 0, 0);
    } else {
      acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fb[set][b]),
                                                          __builtin_bit_cast(bf16x8, fa[set][a]), acc[a][b], 0, 0, 0);
    }
  };

  if constexpr (COPIED) {
    // copies behind the last step of the stage before, the first, the second ...: up to Q[1], Q[2], ...
    constexpr int Q[5] = {0, SOON * NP / 8, STEPS == 2 ? NP : 2 * SOON * NP / 8, SOON * NP / 4 + (NP - SOON * NP / 4) / 2, NP};
    static_assert((NB - 2) * NP + Q[1] <= 63, "the counter of copies");
#pragma unroll 1
    for (int s = 0; s < NB - 1; ++s) {
#pragma unroll
      for (int u = 0; u < NP; ++u) copy_one(s * STAGE, u);
      next_stage();
    }
#pragma unroll
    for (int u = 0; u < Q[1]; ++u) copy_one((NB - 1) * STAGE, u);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 2) * NP + Q[1]) : "memory");
    __syncthreads();
    uint32_t slot = 0, fill = (NB - 1) * STAGE;
    if (WM > 1 && i0 + wm * (BM / WM) >= i_end) {
      // a wave without rows copies and waits alike, and leaves the matrix instructions to the others, one of which is on each SIMD (64
      // experts of 320 rows on average, 2048 x 2048: forward 772 -> 710 us, gradients of rows 826 -> 812; 384 rows 798 -> 781, 873 -> 866)
#pragma unroll 1
      for (int s = s_begin; s < s_end; ++s) {
        const uint32_t after = slot + STAGE == NB * STAGE ? 0 : slot + STAGE;
#pragma unroll
        for (int u = Q[1]; u < NP; ++u) copy_one(fill, u);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 2) * NP) : "memory");
        __syncthreads();
        next_stage();
#pragma unroll
        for (int u = 0; u < Q[1]; ++u) copy_one(slot, u);
        fill = slot;
        slot = after;
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      return;
    }
#pragma unroll
    for (int f = 0; f < NF; ++f) fetch_one(0, 0, f);
#pragma unroll 1
    for (int s = s_begin; s < s_end; ++s) {
      const uint32_t after = slot + STAGE == NB * STAGE ? 0 : slot + STAGE;
#pragma unroll
      for (int kk = 0; kk < STEPS; ++kk) {
        constexpr int LAST = STEPS - 1;
        if (kk == LAST) {
          // this wave's copies of the next stage have landed (behind them, NB - 2 stages) and its reads of this one have
          // returned, and so for every wave
          asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NB - 2) * NP) : "memory");
          __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0), the other counters at their limits
          __syncthreads();
          next_stage();
          __builtin_amdgcn_sched_barrier(0);
        }
        const int step = (kk + 1) % STEPS;
#pragma unroll
        for (int m = 0; m < NM; ++m) {
          mma_one(kk & 1, m);
          __builtin_amdgcn_sched_barrier(0);
          const int first = Q[step], items = NF + Q[step + 1] - first;
#pragma unroll
          for (int it = m * items / NM; it < (m + 1) * items / NM; ++it) {
            if (it < NF) fetch_one(kk < LAST ? slot : after, step, it);
            else copy_one(kk < LAST ? fill : slot, first + it - NF);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      fill = slot;
      slot = after;
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);      // (fetches past the last stage)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (no copy may land in the patches, or after the LDS has been given back)
    __syncthreads();
  } else {
    u32x4 held[NC];
    auto count_of = [&](int u, int l) {    // elements of granule u where l are left of the reduction
      return have[u] == 0 || need[u] >= l ? 0 : (u < CA ? TA : TB) ? have[u] : min(G, l - need[u]);
    };
    int left_held;
    auto load_stage = [&]() {
      left_held = left;
#pragma unroll
      for (int u = 0; u < NC; ++u) {
        const int n = count_of(u, left);
        const uint64_t at = from[source(u)] + off[u];
        if constexpr (ACCESS == SINGLY) {
          held[u] = load_singly((const T*)(uintptr_t)at, n);
        } else {
          const uint64_t back = (uint64_t)(n < G ? G - n : 0) * sizeof(T);
          held[u] = load16((const void*)(uintptr_t)(n > 0 ? at - back : (uint64_t)(uintptr_t)(u < CA ? p.A[0] : p.B[0])));
        }
      }
    };
    auto store_stage = [&](uint32_t buf) {
#pragma unroll
      for (int u = 0; u < NC; ++u) {
        if constexpr (ACCESS == SHIFTED) {
          const int n = count_of(u, left_held);
          if (__any(n < G)) held[u] = shifted<T>(held[u], n);
        }
        *(u32x4*)((char*)&ring[0] + buf + slot_of(u) + lane * 16) = held[u];
      }
    };
    if (s_begin < s_end) {                 // (no rows: there may be no memory either)
      load_stage();
      store_stage(0);
    }
    __syncthreads();
    uint32_t slot = 0;
#pragma unroll 1
    for (int s = s_begin; s < s_end; ++s) {
      next_stage();
      load_stage();
#pragma unroll
      for (int kk = 0; kk < STEPS; ++kk) {
#pragma unroll
        for (int f = 0; f < NF; ++f) fetch_one(slot, kk, f);
#pragma unroll
        for (int m = 0; m < NM; ++m) mma_one(kk & 1, m);
      }
      // (the other buffer: every wave has read it before the last barrier)
      store_stage(STAGE - slot);
      slot = STAGE - slot;
      __syncthreads();
    }
  }

  // ---- results, through a private patch of LDS, so that one access of the wave covers whole lines
  if constexpr (CW == 64 && Ep::PACKS) {
    if (p.splits == 1 && ep.packed()) {
      // nothing but a rounding, done before the patches: all of the wave's results at once, 4 KB for 32 rows.  Granule g of row r
      // is at g ^ (r / 2): two rows share a pass over the banks.
      static_assert(NW * TM * 4096 <= AREA, "the patches fit in the ring");
      char* const bits = (char*)&ring[0] + wave * TM * 4096;
      const int c = lane & 7, product = DUAL ? c / 4 : 0;
      const int col = j0 + wn * (BNS / WN) + (DUAL ? c % 4 : c) * 8, n = min(p.N - col, 8);
#pragma unroll
      for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *(u32x2*)(bits + a * 4096 + l31 * 128 + ((4 * b + q) ^ (l31 / 2 & 7)) * 16 + h * 8) =
                u32x2{two_bf16(acc[a][b][4 * q], acc[a][b][4 * q + 1]), two_bf16(acc[a][b][4 * q + 2], acc[a][b][4 * q + 3])};
      patch_fence();
#pragma unroll
      for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int r = u * 8 + lane / 8;
          const int64_t i = i0 + wm * (BM / WM) + a * 32 + r;
          const u32x4 v = *(const u32x4*)(bits + a * 4096 + r * 128 + (c ^ (r / 2 & 7)) * 16);
          if (i < i_end) ep.put(group, i, col, n, v, FORM == WEIGHTS ? second : product);
        }
      return;
    }
  }
  // 32 rows in fp32 at a time
  constexpr int LPR = BNS / WN / 8, RPI = 64 / LPR, TIMES = 32 / RPI;
  float* const patch = (float*)&ring[0] + wave * 32 * EP;
  const int rrow = lane / LPR, rcol = (lane % LPR) * 8, hi4 = 4 * h;
  const int col = j0 + wn * (BNS / WN) + rcol, n = min(p.N - col, 8);
  const int wide = DUAL ? 2 * p.N : p.N;
#pragma unroll
  for (int a = 0; a < TM; ++a) {
    const int64_t first = i0 + wm * (BM / WM) + a * 32 + rrow;
    typename Ep::Held held[TIMES];
    if (p.splits == 1) {
#pragma unroll
      for (int t = 0; t < TIMES; ++t) held[t] = ep.ask(first + RPI * t, col, first + RPI * t < i_end ? n : 0);
    }
#pragma unroll
    for (int b = 0; b < TN; ++b)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 o = {acc[a][b][4 * q], acc[a][b][4 * q + 1], acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]};
        *(f32x4*)&patch[l31 * EP + b * 32 + 8 * q + hi4] = o;
      }
    patch_fence();
#pragma unroll
    for (int t = 0; t < TIMES; ++t) {
      const int r = rrow + RPI * t;
      const int64_t i = first + RPI * t;
      float v[8], w[8];
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const f32x4 x = *(const f32x4*)&patch[r * EP + rcol + 4 * g], y = *(const f32x4*)&patch[r * EP + (DUAL ? CW / 2 : 0) + rcol + 4 * g];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[4 * g + e] = x[e];
          w[4 * g + e] = DUAL ? y[e] : 0.f;
        }
      }
      if (i >= i_end || n <= 0) continue;
      if (p.splits > 1) {
        float* const to = p.partial + ((int64_t)blockIdx.y * p.partial_rows + (FORM == WEIGHTS ? (int64_t)(second * p.groups + group) * p.M : 0) + i) * wide + col;
        store_part(to, n, v);
        if (DUAL) store_part(to + p.N, n, w);
      } else {
        ep.row(FORM == WEIGHTS ? second * p.groups + group : group, i, col, n, v, w, held[t]);
      }
    }
    patch_fence();
    __builtin_amdgcn_sched_barrier(0);      // (or registers run out)
  }
}

// The parts of a divided reduction, in order, and what follows the product.
template <int FORM, bool DUAL, class Ep>
__global__ __launch_bounds__(256) void joined_kernel(Product p, Ep ep) {
  const int chunks = (p.N + 7) / 8, wide = DUAL ? 2 * p.N : p.N;
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / chunks;
  int64_t first = 0, rows = p.partial_rows;
  if (FORM != WEIGHTS && p.offsets) {     // rows outside the groups have no parts
    const int64_t end = p.offsets[p.groups];
    rows = end < rows ? end : rows;
    first = p.offsets[0];
  }
  if (row < first || row >= rows) return;
  const int col = (int)(at % chunks) * 8, n = min(p.N - col, 8);
  float v[8] = {}, w[8] = {}, x[8];
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
    const float* const from = p.partial + (s * p.partial_rows + row) * wide + col;
    load_part(from, n, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += x[e];
    if (DUAL) {
      load_part(from + p.N, n, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] += x[e];
    }
  }
  const int64_t i = FORM == WEIGHTS ? row % p.M : row;
  ep.row(FORM == WEIGHTS ? (int)(row / p.M) : 0, i, col, n, v, w, ep.ask(i, col, n));
}

}  // namespace
}  // namespace dynb

#endif
