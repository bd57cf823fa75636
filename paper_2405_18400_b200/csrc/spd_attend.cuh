// Attention for sequences that share prefixes (one pass over keys and values with the running maximum and sum of
// the softmax), in two launches: partial results of pieces of the positions, then their join per row.
//
// Mathematics.  A piece of the positions gives a row (m, l, O) = (max s, sum e^(s-m), sum e^(s-m) v); pieces join by
// m = max m_j, l = sum l_j e^(m_j-m), O = sum O_j e^(m_j-m), whatever the pieces are.  So the positions of a group's prefix are read
// once for all rows of the group (their queries stacked into the 16 to 64 rows of a tile), a sequence's own positions for its
// rows alone, both split where it suits the machine.
//
// What bounds it.  With r rows per key head a position costs 4 r D operations against 4 D bytes (bf16): with 16 rows
// the stream of the cache from device memory bounds it, with 64 the instructions (mma.sync at a third of its rate), and small calls the chain lengths -
// page numbers - rows - join.  So everything is laid out for the stream, in as little code as possible:
//  * Two kinds of blocks stand side by side on each SM.  A block of the prefix kind puts all its warps on one tile of 16, 32 or 64 rows (row tiles x
//    shares of a step's positions); a block of the own kind has a tile (one sequence, one key head, up to 16 rows) per warp, because own
//    parts are short and many.
//  * Each kind's work, laid end to end in steps, is cut into equal runs, one per block (or warp): no block idles, whatever the lengths are.  A run
//    that crosses into another tile starts that tile's partial result; run r's part of tile t is number r + t, so parts need no table.  Lengths are
//    read on the device, by every warp for itself.
//  * Keys and values travel by cp.async into a ring of stages (per block or per warp); page numbers of later positions are asked for a step
//    ahead of their copies, which zero the places behind a length (so that 0 x rubbish is never formed).
//  * Scores and weighted values on mma.sync, operands by ldmatrix from 16-byte columns exchanged by row (no bank conflicts).
//  * An instruction has 16 rows, and float32 operands are sums of two or three terms.  Where a tile has few rows their terms are rows of the same
//    operand: one instruction does the work of three (up to four rows over a bf16 cache), or two do (up to eight), the rows' sums
//    being taken once at the end; a lane has one row instead of two, and the registers that are left make a third block per SM.
//  * One copy of each piece of code: loops that begin before their first step instead of prologues, masks under a branch instead of a
//    second instance.  Unrolled twice and thrice the paths pushed one another out of the instruction cache (64 requests 54 us instead of 44, weights of one term).
//
// Measured (B200, 128 dimensions, lengths as in perf/operators.py): 4 x 8 beams behind 16384 positions of 8 key heads, bf16, 68 us for 277 MB (4.1 TB/s of the
// copy's 6.46); 8 rows behind 4 x 4096 positions of 32 heads 50 us for 268 MB; 64 requests behind 2048 positions with 50 to 200 of their own 48 us for 165 MB;
// three float32 rows behind 2048 positions 14.6 us for 34 MB, eight times as many 51 for 266; 31 float32 rows over 1001 positions of a float32 cache, 40 heads, 33 us for 52 MB.
//
// Roundings.  bf16 queries and cache: products exact, sums float32, the softmax weights e^(s-m) <= 1 as two bf16 terms (the first by truncation, exact; the
// second to 2^-16 of the weight), so that the output's own rounding is all that shows (error 1.66e-3, as float32 arithmetic rounded once; with weights
// of one term, 2^-9 each, it was 2.21e-3.  The second term's products are
// half as many again behind the softmax: 64 requests 44 -> 48 us, four long prompts 59 -> 68, 64 rows behind each of 4 x 4096 positions of 32 heads 107 -> 130.)  float32 queries with a
// bf16 cache: queries and weights as three exact bf16 terms.  float32 cache: both sides of both products as two tf32 terms (11 + 11
// bits), three products.
#pragma once
#include <math_constants.h>

#include <atomic>
#include <type_traits>

#include "spd_ops.h"
#include "spd_prefill_tc.h"
#include "spd_ptx.cuh"

namespace spd {

// What a step and a tile of either kind cost, in units of an own step (a prefix step by a block, an own one by a warp).
struct Weights {
  float step, tile, own_step, own_tile;
};
// Division by a number that is 2^shift (shift < 0: any).
struct Divisor {
  int size, shift;
#ifdef __CUDACC__
  __device__ __forceinline__ int operator()(int v) const { return shift >= 0 ? v >> shift : (int)((unsigned)v / (unsigned)size); }
#endif
};
struct Attend {
  spd_attention_args a;
  int ratio, rows_o;            // query heads per key head; rows of an own part's place (at most 16)
  int q_whole;                  // head_dim is the kernel's, and queries may be read two (bf16, terms) or four (float32 cache) at a time
  float scale_log2;
  float *prefix_o, *own_o;      // parts: [part][rows][head_dim]
  float2 *prefix_ml, *own_ml;   // [part][rows]: maximum (in powers of two), sum
  long long prefix_parts, own_parts;  // that the workspace holds: all of them, unless the arrays change under the kernel
  int blocks;                   // of the first launch
  int prefix_room, own_room;    // places of a table's row
  int many_parts;               // a row's prefix comes in six parts and more (1), in sixteen and more (2)
  int out_fours;                // out may be written four at a time
  Weights weights;
  Divisor prefix_pages, own_pages, by_ratio;
};

// (x, kv): (bf16, bf16), (f32, bf16), (f32, f32); then (f32, bf16) with four rows to a tile, (f32, f32) and (f32, bf16) with eight: a
// row's terms are rows of one operand there, or of two instead of three.
enum { kAttBf16 = 0, kAttTerms = 1, kAttFloat = 2, kAttFew = 3, kAttFewFloat = 4, kAttEight = 5 };
template <int MODE> constexpr int kRows = MODE == kAttFew ? 4 : MODE == kAttFewFloat || MODE == kAttEight ? 8 : 16;   // rows of a warp's tile
template <int MODE> constexpr bool kTf32 = MODE == kAttFloat || MODE == kAttFewFloat;            // a float32 cache
// Positions that a warp takes at a step: the depth of a bf16 instruction, or of a tf32 one (so that eight warps' stages of a float32
// cache fit the shared memory: with 16 positions and four warps it is the latency of one warp per scheduler that bounds).
template <int MODE> constexpr int kPositions = kTf32<MODE> ? 8 : 16;

// ---- work: how many steps and tiles a group's prefix and a sequence's own part are, and who does them.  Every warp works it out
// for itself (32 segments at a time, no barrier); the host has made sure that all steps fit 31 bits.
struct Cost {
  int steps, tiles;                // steps < 0: the segment ends before it begins
};
struct Totals {
  int steps, tiles;                // all of them
  int before, tiles_before;        // those of the segments in front of `mark`
  bool falls;                      // the segments are no partition
};

// (Bounded, so that no entry leads outside the queries; entries that do not fall are then a partition, whose steps the host has bounded.)
__device__ __forceinline__ int within(int v, int most) { return v < 0 ? 0 : v < most ? v : most; }
__device__ __forceinline__ int first_row(const Attend &p, int seq) { return p.a.q_start ? within(p.a.q_start[seq], p.a.n) : seq; }
__device__ __forceinline__ int first_seq(const Attend &p, int g) { return p.a.group_start ? within(p.a.group_start[g], p.a.b) : g * p.a.b; }
__device__ __forceinline__ int tiles_of(int rows, int height) { return rows > 0 ? (rows + height - 1) / height : 0; }
__device__ __forceinline__ int prefix_length(const Attend &p, int g) { return within(p.a.prefix_len[g], p.prefix_room); }
__device__ __forceinline__ int own_length(const Attend &p, int s) { return within(p.a.own_len[s], p.own_room); }

// (No early return: the lengths are asked for together with the segments' ends.)
template <int HEIGHT, int STEP>
__device__ __forceinline__ Cost prefix_cost(const Attend &p, int g) {
  const int first = first_seq(p, g), end = first_seq(p, g + 1);
  const int steps = (int)(((unsigned)prefix_length(p, g) + STEP - 1) / STEP);
  const int rows = (first_row(p, end) - first_row(p, first)) * p.ratio;
  const int tiles = steps ? tiles_of(rows, HEIGHT) * p.a.n_kv_heads : 0;
  return {end < first ? -1 : tiles * steps, tiles};
}
template <int STEP, int HEIGHT>
__device__ __forceinline__ Cost own_cost(const Attend &p, int s) {
  const int steps = (int)(((unsigned)own_length(p, s) + STEP - 1) / STEP);
  const int rows = (first_row(p, s + 1) - first_row(p, s)) * p.ratio;
  const int tiles = steps ? tiles_of(rows, HEIGHT) * p.a.n_kv_heads : 0;
  return {rows < 0 ? -1 : tiles * steps, tiles};
}

template <typename F>
__device__ __forceinline__ Totals sum_segments(int n, int mark, F cost) {
  const int lane = threadIdx.x & 31;
  Totals t = {0, 0, 0, 0, false};
#pragma unroll 1
  for (int base = 0; base < n; base += 32) {
    const int i = base + lane;
    const Cost c = i < n ? cost(i) : Cost{0, 0};
    t.steps += __reduce_add_sync(~0u, c.steps);
    t.tiles += __reduce_add_sync(~0u, c.tiles);
    t.falls |= __any_sync(~0u, c.steps < 0);
    if (base < mark) {
      t.before += __reduce_add_sync(~0u, i < mark ? c.steps : 0);
      t.tiles_before += __reduce_add_sync(~0u, i < mark ? c.tiles : 0);
    }
  }
  return t;
}
// Nothing is attended to where q_start or group_start falls: the sums above say nothing then.
__device__ __forceinline__ bool no_partition(Totals &pre, Totals &own) {
  const bool falls = pre.falls || own.falls;
  if (falls) pre.steps = own.steps = 0;
  return falls;
}

// The segment that holds a step.
struct Place {
  int segment;
  int before, tiles_before;  // steps and tiles of the segments in front of it
};
template <typename F>
__device__ __forceinline__ Place find_segment(int n, int step, F cost) {
  const int lane = threadIdx.x & 31;
  if (n == 1) return {0, 0, 0};
  Place at = {n, 0, 0};
#pragma unroll 1
  for (int base = 0; base < n; base += 32) {
    const Cost c = base + lane < n ? cost(base + lane) : Cost{0, 0};
    int s = c.steps, t = c.tiles;
#pragma unroll 1
    for (int j = 1; j < 32; j <<= 1) {
      const int us = __shfl_up_sync(~0u, s, j), ut = __shfl_up_sync(~0u, t, j);
      if (lane >= j) s += us, t += ut;
    }
    const unsigned past = __ballot_sync(~0u, at.before + s > step);
    if (past) {
      const int k = __ffs(past) - 1;
      at.segment = base + k;
      at.before += __shfl_sync(~0u, s - c.steps, k);
      at.tiles_before += __shfl_sync(~0u, t - c.tiles, k);
      return at;
    }
    at.before += __shfl_sync(~0u, s, 31);
    at.tiles_before += __shfl_sync(~0u, t, 31);
  }
  return at;
}

// How the blocks are shared out: in proportion to the time that either kind takes alone.
struct Split {
  int prefix_blocks, own_warps;
};
__device__ __forceinline__ Split split_blocks(int blocks, int warps, const Weights &w, const Totals &pre, const Totals &own) {
  // (each operation is one instruction, so that both kernels come to the same numbers)
  const float wp = __fadd_rn(__fmul_rn(w.step, pre.steps), __fmul_rn(w.tile, pre.tiles));
  const float wo = __fadd_rn(__fmul_rn(w.own_step, own.steps), __fmul_rn(w.own_tile, own.tiles));
  float part;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(part) : "f"(__fadd_rn(__fmul_rn(wp, warps), wo)));
  int n = pre.steps ? __float2int_rn(__fmul_rn(blocks, __fmul_rn(__fmul_rn(wp, warps), part))) : 0;
  // As many runs for a tile as for another, where that costs no more than a sixth of the blocks: a block that crosses into a second tile
  // fills its ring anew and writes a second part (four prompts of 8 key heads on 294 blocks 65 us, on 288 60, weights of one term).
  if (n > pre.tiles && pre.tiles > 0) {
    const int even = n / pre.tiles * pre.tiles;
    if (n - even <= n / 6) n = even;
  }
  if (pre.steps && n < 1) n = 1;
  if (own.steps && n > blocks - 1) n = blocks - 1;
  if (n > pre.steps) n = pre.steps;  // no run is empty
  const int rest = (blocks - n) * warps;
  return {n, rest < own.steps ? rest : own.steps};
}
// Run i of n over `steps` begins at step floor(i steps / n): all runs alike but for one step, and whole numbers of them to tiles that
// are alike.  run_of: the run that has a step.  (In 64 bits only where 32 do not hold n steps, which no product here passes.)
static __host__ __device__ __noinline__ int wide_ratio(unsigned a, unsigned b, unsigned minus, unsigned by) { return (int)(((unsigned long long)a * b - minus) / by); }
__host__ __device__ __forceinline__ bool wide(int n, int steps) { return ((unsigned long long)(unsigned)n * (unsigned)steps) >> 32 != 0; }
__host__ __device__ __forceinline__ int run_start(int i, int n, int steps) {
  return !wide(n, steps) ? (int)((unsigned)i * (unsigned)steps / (unsigned)n) : wide_ratio(i, steps, 0, n);
}
__host__ __device__ __forceinline__ int run_of(int step, int n, int steps) {
  return !wide(n, steps) ? (int)((((unsigned)step + 1) * (unsigned)n - 1) / (unsigned)steps) : wide_ratio(step + 1, n, 1, steps);
}

// ---- instructions
__device__ __forceinline__ void cp16(uint32_t dst, const void *src, int size) {  // zeros behind `size` bytes
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldm4(uint32_t *r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t *r, uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ float4 lds4(uint32_t at) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void mma_bf16(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// v = hi + lo, hi the nearest value of 11 significant bits, lo the rest, of whose 12 bits the instruction takes 11.  |lo| <= 2^-11 |v|,
// so that the product of two lows, which is left out, is 2^-22 of the whole at most (with hi by truncation it is 2^-20 and has a
// sign).  The rounding is an addition: cvt.rna.tf32 has a quarter of its rate and took 1001 positions of a float32 cache from 60 to 82 us.
__device__ __forceinline__ void split_tf32(float v, uint32_t &hi, uint32_t &lo) {
  hi = (__float_as_uint(v) + 0x1000u) & 0xffffe000u;
  lo = __float_as_uint(v - __uint_as_float(hi));
}
// The three exact bf16 terms (by truncation) of a pair of values, packed: x in the low half.
__device__ __forceinline__ void split_terms(float x, float y, uint32_t *t) {
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const uint32_t bx = __float_as_uint(x), by = __float_as_uint(y);
    t[k] = __byte_perm(bx, by, 0x7632);
    x -= __uint_as_float(bx & 0xffff0000u);
    y -= __uint_as_float(by & 0xffff0000u);
  }
}
// A pair of values as two bf16 terms, packed: the first by truncation (exact), what it leaves to the nearest.  The rest is 2^-16 of a value at most.
__device__ __forceinline__ void split_weights(float x, float y, uint32_t &high, uint32_t &low) {
  const uint32_t bx = __float_as_uint(x), by = __float_as_uint(y);
  high = __byte_perm(bx, by, 0x7632);
  low = pack_bf16(x - __uint_as_float(bx & 0xffff0000u), y - __uint_as_float(by & 0xffff0000u));
}

// ---- one tile's piece
template <int MODE, int DT, int NW, int STAGES>
struct AttendShape {
  static constexpr int kThreads = 32 * NW;
  static constexpr int kElem = kTf32<MODE> ? 4 : 2;
  static constexpr int kRow = DT * kElem;                // bytes of a position's key or value
  static constexpr int kChunks = kRow / 16;
  static constexpr int kPos = kPositions<MODE>;        // positions of a warp and stage
  static constexpr int kWarpStage = kPos * kRow * 2;
  static constexpr int kRing = STAGES * NW * kWarpStage;
  static constexpr bool kQueriesInShared = MODE == kAttFewFloat ? DT > 128 : MODE == kAttFew || MODE == kAttEight ? false : kTf32<MODE> || DT > 128;  // else in registers
  static constexpr int kQueryTile = DT / 16 * (MODE == kAttBf16 ? 512 : MODE == kAttTerms ? 3 * 512 : 1024);
  static constexpr int kQueries = kQueriesInShared ? NW * kQueryTile : 0;
  static constexpr int kOutRow = DT + (kTf32<MODE> ? 4 : 8);  // floats of a row of the merge area: no bank conflicts
  static constexpr int kSlots = STAGES * NW * kPos * 16;   // a position's key and value offsets
  static constexpr int kTiles = MODE == kAttFloat && DT <= 128 ? 2 : 1;  // row tiles of a warp, at most
  static constexpr int kMl = NW * (STAGES * 32 > kTiles * 16 * 8 ? STAGES * 32 : kTiles * 16 * 8);  // maxima and sums to be merged, or the stages' tiles
  static constexpr int kShared = kRing + kQueries + kSlots + kMl;
  static_assert(NW * kTiles * 16 * kOutRow * 4 <= kRing + kQueries, "the merge area lies in the ring, and where the queries were");
};

template <int MODE, int DT, int NW, int STAGES>
struct Attending {
  using S = AttendShape<MODE, DT, NW, STAGES>;
  static constexpr int kBlocks16 = DT / 16;  // blocks of 16 dimensions
  static constexpr int kP = S::kPos;
  // times kP positions that a warp scores at a time: what registers hold
  static constexpr int kAtOnce = MODE == kAttBf16 || MODE == kAttFew ? (DT > 128 ? 1 : 4) : MODE == kAttTerms ? (DT > 64 ? 1 : 2) : (DT > 128 ? 1 : 2);
  static constexpr int kQRegs = S::kQueriesInShared ? 1 : kBlocks16 * (MODE == kAttTerms ? 12 : MODE == kAttFewFloat ? 8 : MODE == kAttEight ? 6 : 4);
  static constexpr bool kFew = MODE == kAttFew, kFewFloat = MODE == kAttFewFloat, kEight = MODE == kAttEight;
  static constexpr int kHalves = kRows<MODE> < 16 ? 1 : 2;   // rows of a lane: lane / 4 and lane / 4 + 8, or one alone (lane / 4 % 4, lane / 4)

  const Attend &p;
  uint32_t ring, queries, slots, ml;  // shared-memory addresses
  int lane, warp;
  uint32_t q[kQRegs];
  // Row tiles that a warp may have: two over a float32 cache, whose keys and values it then splits into their terms once for both.
  static constexpr int kMR = S::kTiles;
  float o[kMR][DT / 8][4];
  float m[kMR][2], l[kMR][2];         // of rows lane / 4 and lane / 4 + 8: largest score (before the scale), the lane's columns' sum
  uint32_t key_lane, value_lane;      // the lane's place in 16 positions, blocks of dimensions by XOR or addition

  __device__ __forceinline__ Attending(const Attend &p_, uint32_t base) : p(p_) {
    ring = base;
    queries = base + S::kRing;
    slots = queries + S::kQueries;
    ml = slots + S::kSlots;
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3, mat = lane >> 3;
    if constexpr (kTf32<MODE>) {
      key_lane = key_at(g, t);
      value_lane = value_at(2 * t, g);
    } else {
      key_lane = key_at(((mat >> 1) << 3) + (lane & 7), mat & 1);
      value_lane = value_at(((mat & 1) << 3) + (lane & 7), mat >> 1);
    }
  }

  // Columns of 16 bytes change places by the row, so that the lanes of one access meet different banks: ldmatrix reads eight rows of one column;
  // a float32 key is read by two rows x four columns at a time, a value by rows 2t x two columns.
  static __device__ __forceinline__ uint32_t key_at(int row, int chunk) {
    const int c = kTf32<MODE> ? chunk ^ ((row & 1) << 2) : chunk ^ (row & 7);
    return row * S::kRow + c * 16;
  }
  static __device__ __forceinline__ uint32_t value_at(int row, int chunk) {
    const int c = kTf32<MODE> ? chunk ^ (((row >> 1) & 3) << 1) : chunk ^ (row & 7);
    return row * S::kRow + c * 16;
  }

  // Queries of the warp's 16 rows: flat row `row` + 0..15 of (token from `token0`, query head of key head h), `valid` of them (at least
  // one).  Rows behind them repeat the first: nothing of theirs is stored.  Asked for before the copies of keys and values (which they would
  // otherwise wait behind), made ready by finish_queries.
  template <bool SPLIT = false>
  __device__ __forceinline__ void load_queries(int token0, int row, int valid, int h, int tile) {
    const spd_attention_args &a = p.a;
    const int g = lane >> 2, t = lane & 3;
    int64_t at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int f = row + (g + 8 * i < valid ? g + 8 * i : 0);
      const int token = p.by_ratio(f);
      at[i] = (int64_t)(token0 + token) * a.q_row + (int64_t)(h * p.ratio + f - token * p.ratio) * a.q_head;
    }
    const bool whole = p.q_whole;   // all dimensions there, and on addresses that may be read two or four at a time
    if constexpr (MODE == kAttBf16) {
      const uint16_t *x[2] = {static_cast<const uint16_t *>(a.q) + at[0] + 2 * t, static_cast<const uint16_t *>(a.q) + at[1] + 2 * t};
      const auto pair = [&](int k, int j) {   // rows g, g + 8; columns 2t, 2t + 8
        const int d = 16 * k + 8 * (j >> 1);
        if (whole) return *reinterpret_cast<const uint32_t *>(x[j & 1] + d);
        return d + 2 * t < a.head_dim ? x[j & 1][d] | ((uint32_t)x[j & 1][d + 1] << 16) : 0u;
      };
      if constexpr (S::kQueriesInShared) {
        uint32_t v[kBlocks16 * 4];   // (all asked for before the first is stored)
#pragma unroll
        for (int k = 0; k < kBlocks16 * 4; ++k) v[k] = pair(k / 4, k % 4);
#pragma unroll
        for (int k = 0; k < kBlocks16; ++k)
          asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(queries + tile * S::kQueryTile + (k * 32 + lane) * 16), "r"(v[4 * k]), "r"(v[4 * k + 1]), "r"(v[4 * k + 2]), "r"(v[4 * k + 3]) : "memory");
      } else {
#pragma unroll
        for (int k = 0; k < kBlocks16; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) q[k * 4 + j] = pair(k, j);
      }
    } else if constexpr (kFew) {
      // A row's three terms are rows r, r + 4 and r + 8 of the operand, so that one instruction does the work of three.  A lane holds row
      // lane / 4 % 4 (until finish_queries, all of it: two columns and the two eight further).
      const int f = row + ((g & 3) < valid ? g & 3 : 0), token = p.by_ratio(f);
      const float *x = static_cast<const float *>(a.q) + (int64_t)(token0 + token) * a.q_row + (int64_t)(h * p.ratio + f - token * p.ratio) * a.q_head + 2 * t;
#pragma unroll
      for (int k = 0; k < kBlocks16; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 v = query_pair(x, 16 * k + 8 * j, whole);
          q[k * 4 + 2 * j] = __float_as_uint(v.x), q[k * 4 + 2 * j + 1] = __float_as_uint(v.y);
        }
    } else if constexpr (kEight) {
      // Row g's first two terms are rows g and g + 8 of one operand, its third row g of another (until finish_queries, the row's values).
      const float *x = static_cast<const float *>(a.q) + at[0] + 2 * t;
#pragma unroll
      for (int k = 0; k < kBlocks16; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 v = query_pair(x, 16 * k + 8 * j, whole);
          q[k * 6 + 2 * j] = __float_as_uint(v.x), q[k * 6 + 2 * j + 1] = __float_as_uint(v.y);
        }
    } else if constexpr (MODE == kAttTerms) {
      const float *x[2] = {static_cast<const float *>(a.q) + at[0] + 2 * t, static_cast<const float *>(a.q) + at[1] + 2 * t};
      if constexpr (S::kQueriesInShared) {
        float2 v[kBlocks16 * 4];
#pragma unroll
        for (int k = 0; k < kBlocks16 * 4; ++k) v[k] = query_pair(x[k & 1], 16 * (k / 4) + 8 * ((k >> 1) & 1), whole);
#pragma unroll
        for (int k = 0; k < kBlocks16; ++k) {
          uint32_t w[4][3];
#pragma unroll
          for (int j = 0; j < 4; ++j) split_terms(v[4 * k + j].x, v[4 * k + j].y, w[j]);
#pragma unroll
          for (int n = 0; n < 3; ++n)
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(queries + tile * S::kQueryTile + ((k * 3 + n) * 32 + lane) * 16), "r"(w[0][n]), "r"(w[1][n]),
                         "r"(w[2][n]), "r"(w[3][n])
                         : "memory");
        }
      } else {
        // (a row's values wait where two of the three terms will be)
#pragma unroll
        for (int k = 0; k < kBlocks16; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 v = query_pair(x[j & 1], 16 * k + 8 * (j >> 1), whole);
            q[k * 12 + j] = __float_as_uint(v.x), q[k * 12 + 4 + j] = __float_as_uint(v.y);
          }
      }
    } else if constexpr (kFewFloat) {
      // Row g's leading part is row g of the operand, what it leaves row g + 8: two instructions, by the keys' two parts, do the work of three.
      const float *x = static_cast<const float *>(a.q) + at[0] + 4 * t;
      float4 v[kBlocks16];
#pragma unroll
      for (int k = 0; k < kBlocks16; ++k) {
        const float *e = x + 16 * k;
        if (whole) v[k] = *reinterpret_cast<const float4 *>(e);
        else v[k] = 16 * k + 4 * t < a.head_dim ? make_float4(e[0], e[1], e[2], e[3]) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < kBlocks16; ++k) {
        if constexpr (S::kQueriesInShared) {
          uint32_t w[8];
          stack_query(v[k], w);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(queries + tile * S::kQueryTile + ((k * 2 + i) * 32 + lane) * 16), "r"(w[4 * i]), "r"(w[4 * i + 1]), "r"(w[4 * i + 2]),
                         "r"(w[4 * i + 3])
                         : "memory");
        } else {
          q[8 * k] = __float_as_uint(v[k].x), q[8 * k + 1] = __float_as_uint(v[k].y), q[8 * k + 2] = __float_as_uint(v[k].z), q[8 * k + 3] = __float_as_uint(v[k].w);
        }
      }
    } else {
      const float *x[2] = {static_cast<const float *>(a.q) + at[0] + 4 * t, static_cast<const float *>(a.q) + at[1] + 4 * t};
      float4 v[kBlocks16 * 2];
#pragma unroll
      for (int k = 0; k < kBlocks16 * 2; ++k) {  // rows g, g + 8; dimensions 16 (k / 2) + 4 t .. + 3
        const float *e = x[k & 1] + 16 * (k / 2);
        if (whole) v[k] = *reinterpret_cast<const float4 *>(e);
        else v[k] = 16 * (k / 2) + 4 * t < a.head_dim ? make_float4(e[0], e[1], e[2], e[3]) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      if constexpr (SPLIT) {
#pragma unroll
        for (int k = 0; k < kBlocks16; ++k) {
          uint32_t term[2][2][4];  // high ones, low ones
          split_queries(v[2 * k], v[2 * k + 1], term[0], term[1]);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(queries + tile * (2 * S::kQueryTile) + ((k * 4 + i) * 32 + lane) * 16), "r"(term[i / 2][i % 2][0]),
                         "r"(term[i / 2][i % 2][1]), "r"(term[i / 2][i % 2][2]), "r"(term[i / 2][i % 2][3])
                         : "memory");
        }
        return;
      }
#pragma unroll
      for (int k = 0; k < kBlocks16 * 2; ++k)
        asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(queries + tile * S::kQueryTile + (k * 32 + lane) * 16), "f"(v[k].x), "f"(v[k].y), "f"(v[k].z), "f"(v[k].w) : "memory");
    }
  }
  // Four dimensions as two operands whose rows g + 8 hold what rows g leave: dimensions 4t + 2i and 4t + 2i + 1 are columns t and t + 4 of operand i.
  static __device__ __forceinline__ void stack_query(const float4 &v, uint32_t *w) {
    split_tf32(v.x, w[0], w[1]), split_tf32(v.y, w[2], w[3]), split_tf32(v.z, w[4], w[5]), split_tf32(v.w, w[6], w[7]);
  }
  // Terms of a pair as rows g and g + 8 of an operand whose rows are stacked.
  __device__ __forceinline__ void stack_terms(float x, float y, uint32_t &low, uint32_t &high) const {
    uint32_t term[3];
    split_terms(x, y, term);
    low = lane < 16 ? term[0] : term[1], high = lane < 16 ? term[2] : 0u;
  }
  // The sum of a row's terms, in all lanes that have a part of it.
  static __device__ __forceinline__ float unstack(float low, float high) {
    const float v = low + high;
    if constexpr (kFew) return v + __shfl_xor_sync(~0u, v, 16);
    return v;
  }
  __device__ __forceinline__ void finish_queries() {
    if constexpr (kFewFloat && !S::kQueriesInShared) {
#pragma unroll
      for (int k = 0; k < kBlocks16; ++k)
        stack_query(make_float4(__uint_as_float(q[8 * k]), __uint_as_float(q[8 * k + 1]), __uint_as_float(q[8 * k + 2]), __uint_as_float(q[8 * k + 3])), q + 8 * k);
    }
    if constexpr (kEight) {
#pragma unroll
      for (int k = 0; k < kBlocks16; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t term[3];
          split_terms(__uint_as_float(q[k * 6 + 2 * j]), __uint_as_float(q[k * 6 + 2 * j + 1]), term);
          q[k * 6 + 2 * j] = term[0], q[k * 6 + 2 * j + 1] = term[1], q[k * 6 + 4 + j] = term[2];
        }
    }
    if constexpr (kFew) {
#pragma unroll
      for (int k = 0; k < kBlocks16 * 2; ++k) stack_terms(__uint_as_float(q[2 * k]), __uint_as_float(q[2 * k + 1]), q[2 * k], q[2 * k + 1]);
    }
    if constexpr (MODE == kAttTerms && !S::kQueriesInShared) {
#pragma unroll
      for (int k = 0; k < kBlocks16; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t term[3];
          split_terms(__uint_as_float(q[k * 12 + j]), __uint_as_float(q[k * 12 + 4 + j]), term);
          q[k * 12 + j] = term[0], q[k * 12 + 4 + j] = term[1], q[k * 12 + 8 + j] = term[2];
        }
    }
  }
  __device__ __forceinline__ float2 query_pair(const float *x, int d, bool whole) const {
    if (whole) return *reinterpret_cast<const float2 *>(x + d);
    return d + 2 * (lane & 3) < p.a.head_dim ? make_float2(x[d], x[d + 1]) : make_float2(0.f, 0.f);
  }

  template <int MR = 1>
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int r = 0; r < MR; ++r) {
      m[r][0] = m[r][1] = -CUDART_INF_F;
      l[r][0] = l[r][1] = 0.f;
#pragma unroll
      for (int j = 0; j < DT / 8; ++j) o[r][j][0] = o[r][j][1] = o[r][j][2] = o[r][j][3] = 0.f;
    }
  }

  // Where a position's key and value lie: a page number's slot, bytes from the caches' starts.  Negative (the top bit alone) where
  // there is nothing to copy: behind the length, or where the table names no slot.
  static constexpr unsigned long long kNowhere = 1ull << 63;
  __device__ __forceinline__ ulonglong2 offsets_of(int page_number, int in_page, int page, int h) const {
    const int64_t s = (int64_t)page_number * page + in_page;
    if (s >= 0 && s < p.a.slots) {
      const unsigned slot = (unsigned)s;
      return make_ulonglong2((slot * (unsigned long long)p.a.kc_slot + h * (unsigned long long)p.a.kc_head) * S::kElem,
                             (slot * (unsigned long long)p.a.vc_slot + h * (unsigned long long)p.a.vc_head) * S::kElem);
    }
    if (p.a.status) *p.a.status = SPD_ERANGE;
    return make_ulonglong2(kNowhere, kNowhere);
  }
  __device__ __forceinline__ void put_offsets(int i, const ulonglong2 &v) {
    asm volatile("st.shared.v2.u64 [%0], {%1,%2};" ::"r"(slots + i * 16), "l"(v.x), "l"(v.y) : "memory");
  }

  // Copies of kP x WARPS positions by 32 x WARPS threads (t of them): keys, then values.
  template <int WARPS>
  __device__ __forceinline__ void copy_stage(uint32_t stage, uint32_t offsets, int t) {
    constexpr int kThreads = 32 * WARPS;
    constexpr int kPer = kP * WARPS * S::kChunks / kThreads;
    const char *const kc = static_cast<const char *>(p.a.k_cache), *const vc = static_cast<const char *>(p.a.v_cache);
    const int width = p.a.head_dim * S::kElem;
    // (all the offsets first: a load from shared memory is not moved in front of a copy into it)
    unsigned long long ko[kPer], vo[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      asm volatile("ld.shared.v2.u64 {%0,%1}, [%2];" : "=l"(ko[i]), "=l"(vo[i]) : "r"(offsets + (i * kThreads + t) / S::kChunks * 16) : "memory");
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int n = i * kThreads + t;
      const int row = n / S::kChunks, chunk = n % S::kChunks;
      const int live = chunk * 16 < width ? 16 : 0, at = live ? chunk * 16 : 0;   // (the same for all rows, where a row has no more chunks than the threads)
      const int size = live & ~((int)(ko[i] >> 32) >> 31);
      cp16(stage + key_at(row, chunk), kc + (ko[i] & ~kNowhere) + at, size);
      cp16(stage + kP * WARPS * S::kRow + value_at(row, chunk), vc + (vo[i] & ~kNowhere) + at, size);
    }
  }

  static __device__ __forceinline__ void split_queries(const float4 &qa, const float4 &qb, uint32_t (*hi)[4], uint32_t (*lo)[4]) {
    split_tf32(qa.x, hi[0][0], lo[0][0]), split_tf32(qb.x, hi[0][1], lo[0][1]), split_tf32(qa.y, hi[0][2], lo[0][2]), split_tf32(qb.y, hi[0][3], lo[0][3]);
    split_tf32(qa.z, hi[1][0], lo[1][0]), split_tf32(qb.z, hi[1][1], lo[1][1]), split_tf32(qa.w, hi[1][2], lo[1][2]), split_tf32(qb.w, hi[1][3], lo[1][3]);
  }

  // kP x NT positions: keys and values from these addresses on; first: their first position; seen[i]: positions that rows g and g + 8 see.
  // CAUSAL: rows may see different numbers, of the `loaded` ones (behind those there are zeros); all see least_seen.
  // SPLIT: the float32 queries lie in shared memory as their two terms.  MR: row tiles, from `tile` on.
  template <bool CAUSAL, int NT, bool SPLIT, int MR>
  __device__ __forceinline__ void positions(uint32_t keys, uint32_t values, int first, const int *seen, int tile, int least_seen, int loaded) {
    const int t = lane & 3;
    constexpr int N8 = kP / 8 * NT;      // eights of positions
    constexpr int kUnroll = S::kQueriesInShared ? 2 : kBlocks16;  // (code that does not fit the instruction cache costs more than a loop)
    float s[MR][N8][4], small[MR][N8][4];  // small: what is added apart (low terms; with 16 positions every other block), for shorter chains
#pragma unroll
    for (int r = 0; r < MR; ++r)
#pragma unroll
      for (int j = 0; j < N8; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[r][j][c] = small[r][j][c] = 0.f;
    if constexpr (kFewFloat) {
      float other[N8][4] = {};   // every other instruction's: the tensor cores truncate when they add, so short chains
#pragma unroll kUnroll
      for (int k = 0; k < kBlocks16; ++k) {
        uint32_t w[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if constexpr (S::kQueriesInShared) {
            const float4 x = lds4(queries + tile * S::kQueryTile + ((k * 2 + i) * 32 + lane) * 16);
            w[i][0] = __float_as_uint(x.x), w[i][1] = __float_as_uint(x.y), w[i][2] = __float_as_uint(x.z), w[i][3] = __float_as_uint(x.w);
          } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) w[i][c] = q[8 * k + 4 * i + c];
          }
        }
#pragma unroll
        for (int j = 0; j < N8; ++j) {
          const float4 kv = lds4(((keys + key_lane) ^ (64 * k)) + 8 * j * S::kRow);
          uint32_t h[4], l[4];
          split_tf32(kv.x, h[0], l[0]), split_tf32(kv.y, h[1], l[1]), split_tf32(kv.z, h[2], l[2]), split_tf32(kv.w, h[3], l[3]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            mma_tf32(i ? other[j] : s[0][j], w[i], h[2 * i], h[2 * i + 1]);
            mma_tf32(small[0][j], w[i], l[2 * i], l[2 * i + 1]);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < N8; ++j)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          s[0][j][c] += other[j][c];
          // (an infinite sum of the leading parts stands as it is: the small ones may have overflowed the other way)
          if (fabsf(s[0][j][c]) != CUDART_INF_F) s[0][j][c] += (small[0][j][2 + c] + small[0][j][c]) + (s[0][j][2 + c] + other[j][2 + c]);
        }
    } else if constexpr (kTf32<MODE>) {
      float other[MR == 1 ? N8 : 1][4] = {};
#pragma unroll kUnroll
      for (int k = 0; k < kBlocks16; ++k) {
        uint32_t hi[MR][2][4], lo[MR][2][4];  // dimensions (4t, 4t + 1) and (4t + 2, 4t + 3) as an instruction's columns t and t + 4
#pragma unroll
        for (int r = 0; r < MR; ++r) {
          if constexpr (SPLIT) {
            const uint32_t at = queries + (tile + r) * (2 * S::kQueryTile) + (k * 128 + lane) * 16;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float4 x = lds4(at + i * 512), y = lds4(at + (2 + i) * 512);
              hi[r][i][0] = __float_as_uint(x.x), hi[r][i][1] = __float_as_uint(x.y), hi[r][i][2] = __float_as_uint(x.z), hi[r][i][3] = __float_as_uint(x.w);
              lo[r][i][0] = __float_as_uint(y.x), lo[r][i][1] = __float_as_uint(y.y), lo[r][i][2] = __float_as_uint(y.z), lo[r][i][3] = __float_as_uint(y.w);
            }
          } else {
            const uint32_t at = queries + (tile + r) * S::kQueryTile + (k * 64 + lane) * 16;
            split_queries(lds4(at), lds4(at + 512), hi[r], lo[r]);
          }
        }
#pragma unroll
        for (int j = 0; j < N8; ++j) {
          const float4 kv = lds4(((keys + key_lane) ^ (64 * k)) + 8 * j * S::kRow);
          uint32_t h[4], w[4];
          split_tf32(kv.x, h[0], w[0]), split_tf32(kv.y, h[1], w[1]), split_tf32(kv.z, h[2], w[2]), split_tf32(kv.w, h[3], w[3]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int r = 0; r < MR; ++r) mma_tf32(small[r][j], lo[r][i], h[2 * i], h[2 * i + 1]);
#pragma unroll
            for (int r = 0; r < MR; ++r) mma_tf32(MR == 1 && i ? other[MR == 1 ? j : 0] : s[r][j], hi[r][i], h[2 * i], h[2 * i + 1]);
#pragma unroll
            for (int r = 0; r < MR; ++r) mma_tf32(small[r][j], hi[r][i], w[2 * i], w[2 * i + 1]);
          }
        }
      }
#pragma unroll
      for (int r = 0; r < MR; ++r)
#pragma unroll
        for (int j = 0; j < N8; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if constexpr (MR == 1) s[r][j][c] += other[j][c];
            // (an infinite sum of the leading parts stands as it is: the small ones may have overflowed the other way)
            if (fabsf(s[r][j][c]) != CUDART_INF_F) s[r][j][c] += small[r][j][c];
          }
    } else {
#pragma unroll kUnroll
      for (int k = 0; k < kBlocks16; ++k) {
        uint32_t w[3][4];
        if constexpr (MODE == kAttBf16 || kFew) {
          if constexpr (S::kQueriesInShared) {
            const float4 v = lds4(queries + tile * S::kQueryTile + (k * 32 + lane) * 16);
            w[0][0] = __float_as_uint(v.x), w[0][1] = __float_as_uint(v.y), w[0][2] = __float_as_uint(v.z), w[0][3] = __float_as_uint(v.w);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[0][j] = q[k * 4 + j];
          }
        } else if constexpr (kEight) {
#pragma unroll
          for (int j = 0; j < 4; ++j) w[0][j] = q[k * 6 + j];
          w[1][0] = q[k * 6 + 4], w[1][1] = 0, w[1][2] = q[k * 6 + 5], w[1][3] = 0;
        } else {
#pragma unroll
          for (int n = 0; n < 3; ++n) {
            if constexpr (S::kQueriesInShared) {
              const float4 v = lds4(queries + tile * S::kQueryTile + ((k * 3 + n) * 32 + lane) * 16);
              w[n][0] = __float_as_uint(v.x), w[n][1] = __float_as_uint(v.y), w[n][2] = __float_as_uint(v.z), w[n][3] = __float_as_uint(v.w);
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) w[n][j] = q[(k * 3 + n) * 4 + j];
            }
          }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          uint32_t b[4];
          ldm4(b, ((keys + key_lane) ^ (32 * k)) + 16 * j * S::kRow);
          if constexpr (MODE == kAttBf16 || kFew) {
            mma_bf16(NT == 1 && (k & 1) ? small[0][0] : s[0][2 * j], w[0], b[0], b[1]);
            mma_bf16(NT == 1 && (k & 1) ? small[0][1] : s[0][2 * j + 1], w[0], b[2], b[3]);
          } else if constexpr (kEight) {
            mma_bf16(small[0][2 * j], w[1], b[0], b[1]);
            mma_bf16(small[0][2 * j + 1], w[1], b[2], b[3]);
            mma_bf16(s[0][2 * j], w[0], b[0], b[1]);
            mma_bf16(s[0][2 * j + 1], w[0], b[2], b[3]);
          } else {
            mma_bf16(small[0][2 * j], w[2], b[0], b[1]);
            mma_bf16(small[0][2 * j + 1], w[2], b[2], b[3]);
            mma_bf16(s[0][2 * j], w[0], b[0], b[1]);
            mma_bf16(s[0][2 * j + 1], w[0], b[2], b[3]);
            mma_bf16(small[0][2 * j], w[1], b[0], b[1]);
            mma_bf16(small[0][2 * j + 1], w[1], b[2], b[3]);
          }
        }
      }
      if constexpr (MODE == kAttTerms || NT == 1) {
#pragma unroll
        for (int j = 0; j < N8; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[0][j][c] += small[0][j][c];
      }
      if constexpr (kFew || kEight) {
#pragma unroll
        for (int j = 0; j < N8; ++j)
#pragma unroll
          for (int c = 0; c < 2; ++c) s[0][j][c] = unstack(s[0][j][c], s[0][j][2 + c]);
      }
    }
    if (first + kP * NT > least_seen) {
#pragma unroll
      for (int j = 0; j < N8; ++j)
#pragma unroll
        for (int c = 0; c < 2 * kHalves; ++c)
          if (first + 2 * t + 8 * j + (c & 1) >= seen[c >> 1])
#pragma unroll
            for (int r = 0; r < MR; ++r) s[r][j][c] = -CUDART_INF_F;
    }
    float f[MR][2];
#pragma unroll
    for (int r = 0; r < MR; ++r) {
      float top[2] = {m[r][0], m[r][1]};
#pragma unroll
      for (int j = 0; j < N8; ++j)
#pragma unroll
        for (int c = 0; c < 2 * kHalves; ++c) top[c >> 1] = fmaxf(top[c >> 1], s[r][j][c]);
#pragma unroll
      for (int i = 0; i < kHalves; ++i) {
        top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 1));
        top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 2));
        f[r][i] = 1.f;
      }
      if (__any_sync(~0u, top[0] > m[r][0] || top[1] > m[r][1])) {
#pragma unroll
        for (int i = 0; i < kHalves; ++i) {
          f[r][i] = m[r][i] > -CUDART_INF_F ? power2((m[r][i] - top[i]) * p.scale_log2) : 0.f;  // nothing so far: nothing to scale
          m[r][i] = top[i];
          l[r][i] *= f[r][i];
          if constexpr (!kTf32<MODE>) {
#pragma unroll
            for (int j = 0; j < DT / 8; ++j)
#pragma unroll
              for (int c = 0; c < 4 / kHalves; ++c) o[r][j][2 * i + c] *= f[r][i];
          }
        }
      }
      // a score of minus infinity has no weight (also where all are), a NaN one makes the row NaN
      float zero[2];
#pragma unroll
      for (int i = 0; i < kHalves; ++i) zero[i] = m[r][i] > -CUDART_INF_F ? -m[r][i] * p.scale_log2 : 0.f;
#pragma unroll
      for (int j = 0; j < N8; ++j)
#pragma unroll
        for (int c = 0; c < 2 * kHalves; ++c) {
          s[r][j][c] = power2(fmaf(s[r][j][c], p.scale_log2, zero[c >> 1]));
          l[r][c >> 1] += s[r][j][c];
        }
    }
    if constexpr (CAUSAL) {
      if (first + kP > least_seen && loaded > least_seen && rubbish(values)) {
        if constexpr (kTf32<MODE>) {
#pragma unroll
          for (int j = 0; j < DT / 8; ++j)
#pragma unroll
            for (int c = 0; c < 2 * kHalves; ++c) o[0][j][c] *= f[0][c >> 1];
        }
        plain_values(values, first, seen, s[0]);
        return;
      }
    }
    if constexpr (kFewFloat) {
      uint32_t w[N8][4];  // positions 2t, 2t + 1 of each eight as columns t, t + 4; what rows g leave in rows g + 8
#pragma unroll
      for (int j = 0; j < N8; ++j) split_tf32(s[0][j][0], w[j][0], w[j][1]), split_tf32(s[0][j][1], w[j][2], w[j][3]);
#pragma unroll
      for (int jj = 0; jj < DT / 32; ++jj) {   // (a step's sum by itself, as below)
        float sum[4][4] = {};
#pragma unroll
        for (int j = 0; j < N8; ++j) {
          const float4 va = lds4(values + value_lane + 8 * j * S::kRow + 128 * jj);
          const float4 vb = lds4(values + value_lane + (8 * j + 1) * S::kRow + 128 * jj);
          const float x[4] = {va.x, va.y, va.z, va.w}, y[4] = {vb.x, vb.y, vb.z, vb.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t xh, xl, yh, yl;
            split_tf32(x[i], xh, xl);
            split_tf32(y[i], yh, yl);
            mma_tf32(sum[i], w[j], xl, yl);
            mma_tf32(sum[i], w[j], xh, yh);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < 2; ++c) o[0][4 * jj + i][c] = fmaf(o[0][4 * jj + i][c], f[0][0], sum[i][c] + sum[i][2 + c]);
      }
    } else if constexpr (kTf32<MODE>) {
      uint32_t hi[MR][N8][4], lo[MR][N8][4];  // positions 2t, 2t + 1 of each eight as columns t, t + 4
#pragma unroll
      for (int r = 0; r < MR; ++r)
#pragma unroll
        for (int j = 0; j < N8; ++j) {
          split_tf32(s[r][j][0], hi[r][j][0], lo[r][j][0]), split_tf32(s[r][j][2], hi[r][j][1], lo[r][j][1]);
          split_tf32(s[r][j][1], hi[r][j][2], lo[r][j][2]), split_tf32(s[r][j][3], hi[r][j][3], lo[r][j][3]);
        }
      // The step's sum is formed by itself and added in float32 (with the rescaling): the tensor cores truncate when they add, and
      // in one chain over a thousand positions that came to twice the error of plain float32.
#pragma unroll
      for (int jj = 0; jj < DT / 32; ++jj) {
        float sum[MR][4][4] = {};
#pragma unroll
        for (int j = 0; j < N8; ++j) {
          // column g of tiles 4 jj + i is dimension 32 jj + 4 g + i
          const float4 va = lds4(values + value_lane + 8 * j * S::kRow + 128 * jj);
          const float4 vb = lds4(values + value_lane + (8 * j + 1) * S::kRow + 128 * jj);
          const float x[4] = {va.x, va.y, va.z, va.w}, y[4] = {vb.x, vb.y, vb.z, vb.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t xh, xl, yh, yl;
            split_tf32(x[i], xh, xl);
            split_tf32(y[i], yh, yl);
#pragma unroll
            for (int r = 0; r < MR; ++r) mma_tf32(sum[r][i], lo[r][j], xh, yh);
#pragma unroll
            for (int r = 0; r < MR; ++r) mma_tf32(sum[r][i], hi[r][j], xl, yl);
#pragma unroll
            for (int r = 0; r < MR; ++r) mma_tf32(sum[r][i], hi[r][j], xh, yh);
          }
        }
#pragma unroll
        for (int r = 0; r < MR; ++r)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[r][4 * jj + i][c] = fmaf(o[r][4 * jj + i][c], f[r][c >> 1], sum[r][i][c]);
      }
    } else {
      constexpr int kTerms = MODE == kAttTerms ? 3 : kEight || MODE == kAttBf16 ? 2 : 1;
      uint32_t w[NT][kTerms][4];
      if constexpr (kFew) {
#pragma unroll
        for (int j = 0; j < 2 * NT; ++j) stack_terms(s[0][j][0], s[0][j][1], w[j / 2][0][2 * (j & 1)], w[j / 2][0][2 * (j & 1) + 1]);
      }
      if constexpr (kEight) {
#pragma unroll
        for (int j = 0; j < 2 * NT; ++j) {
          uint32_t term[3];
          split_terms(s[0][j][0], s[0][j][1], term);
          w[j / 2][0][2 * (j & 1)] = term[0], w[j / 2][0][2 * (j & 1) + 1] = term[1];
          w[j / 2][kTerms - 1][2 * (j & 1)] = term[2], w[j / 2][kTerms - 1][2 * (j & 1) + 1] = 0;
        }
      }
#pragma unroll
      for (int n = 0; n < (kFew || kEight ? 0 : NT); ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // rows g, g + 8 of positions 2t, then of 2t + 8
          const float x = s[0][2 * n + (j >> 1)][2 * (j & 1)], y = s[0][2 * n + (j >> 1)][2 * (j & 1) + 1];
          if constexpr (MODE == kAttBf16) {
            split_weights(x, y, w[n][0][j], w[n][kTerms - 1][j]);
          } else {
            uint32_t term[3];
            split_terms(x, y, term);
#pragma unroll
            for (int i = 0; i < kTerms; ++i) w[n][i][j] = term[i];
          }
        }
#pragma unroll
      for (int k = 0; k < kBlocks16; ++k)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          uint32_t b[4];
          ldm4t(b, ((values + value_lane) ^ (32 * k)) + 16 * n * S::kRow);
#pragma unroll
          for (int i = kTerms - 1; i >= 0; --i) {
            mma_bf16(o[0][2 * k], w[n][i], b[0], b[1]);
            mma_bf16(o[0][2 * k + 1], w[n][i], b[2], b[3]);
          }
        }
    }
  }

  // Whether any of the values of kP positions is not finite.
  static __device__ __noinline__ bool rubbish(uint32_t values) {
    const int lane = threadIdx.x & 31;
    bool bad = false;
#pragma unroll 1
    for (int i = lane; i < kP * S::kChunks; i += 32) {
      const float4 v = lds4(values + value_at(i / S::kChunks, i % S::kChunks));
      const uint32_t w[4] = {__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
      for (int j = 0; j < 4; ++j) {
        if constexpr (kTf32<MODE>) bad |= (w[j] & 0x7f800000u) == 0x7f800000u;
        else bad |= (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
      }
    }
    return __any_sync(~0u, bad);
  }
  // The weighted values of 16 positions for rows that see different ones, where a value that some row must not see is not
  // finite: 0 x NaN must not reach that row, so each row takes only what it sees.
  __device__ __forceinline__ void plain_values(uint32_t values, int first, const int *seen, const float (*e)[4]) {
    const int t = lane & 3;
#pragma unroll 1
    for (int j = 0; j < kP; ++j) {
      float w[2];
#pragma unroll
      for (int i = 0; i < kHalves; ++i) {
        const float x = kP == 8 || j < 8 ? e[0][2 * i] : e[kP / 8 - 1][2 * i], y = kP == 8 || j < 8 ? e[0][2 * i + 1] : e[kP / 8 - 1][2 * i + 1];
        const int from = (lane & ~3) | ((j & 7) >> 1);
        const float wx = __shfl_sync(~0u, x, from), wy = __shfl_sync(~0u, y, from);
        w[i] = j & 1 ? wy : wx;
      }
#pragma unroll
      for (int n = 0; n < DT / 8; ++n)
#pragma unroll
        for (int c = 0; c < 2 * kHalves; ++c) {
          const int d = column(n, t, c & 1);
          float v;
          if constexpr (kTf32<MODE>) {
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(values + value_at(j, d / 4) + (d % 4) * 4) : "memory");
          } else {
            unsigned short u;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(u) : "r"(values + value_at(j, d / 8) + (d % 8) * 2) : "memory");
            v = __uint_as_float((uint32_t)u << 16);
          }
          if (first + j < seen[c >> 1] && (!kFew || lane < 16)) o[0][n][c] += w[c >> 1] * v;   // (a row of stacked terms: to one of them)
        }
    }
  }
  // Dimension of accumulator column 2t + i of tile n.
  static __device__ __forceinline__ int column(int n, int t, int i) {
    return kTf32<MODE> ? (n / 4) * 32 + 8 * t + 4 * i + (n & 3) : 8 * n + 2 * t + i;
  }

  template <int MR = 1>
  __device__ __forceinline__ void sum_columns() {
    if constexpr (kFew || kEight) {
#pragma unroll
      for (int j = 0; j < DT / 8; ++j)
#pragma unroll
        for (int c = 0; c < 2; ++c) o[0][j][c] = unstack(o[0][j][c], o[0][j][2 + c]);
    }
#pragma unroll
    for (int i = 0; i < 2 * MR; ++i) {
      l[i / 2][i % 2] += __shfl_xor_sync(~0u, l[i / 2][i % 2], 1);
      l[i / 2][i % 2] += __shfl_xor_sync(~0u, l[i / 2][i % 2], 2);
    }
  }
  // The warp's part, from registers: `valid` rows to out[row][head_dim], ml[row].
  __device__ __forceinline__ void store_part(float *out, float2 *part_ml, int valid) const {
    const int g = lane >> 2, t = lane & 3, D = p.a.head_dim;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = g + 8 * i;
      if (r >= valid) continue;
      if (t == 0) part_ml[r] = make_float2(m[0][i] * p.scale_log2, l[0][i]);
      float *dst = out + r * D;
#pragma unroll
      for (int j = 0; j < DT / 8; ++j) {
        if constexpr (kTf32<MODE>) {
          if ((j & 3) == 0) {  // eight neighbouring dimensions, four tiles' columns
            const int d = column(j, t, 0);
            if (d < D) *reinterpret_cast<float4 *>(dst + d) = make_float4(o[0][j][2 * i], o[0][j + 1][2 * i], o[0][j + 2][2 * i], o[0][j + 3][2 * i]);
            if (d + 4 < D) *reinterpret_cast<float4 *>(dst + d + 4) = make_float4(o[0][j][2 * i + 1], o[0][j + 1][2 * i + 1], o[0][j + 2][2 * i + 1], o[0][j + 3][2 * i + 1]);
          }
        } else {
          const int d = column(j, t, 0);
          if (d < D) *reinterpret_cast<float2 *>(dst + d) = make_float2(o[0][j][2 * i], o[0][j][2 * i + 1]);
        }
      }
    }
  }

  // ---- the prefix kind: steps s0 .. s1 of the tile of `valid` rows from `row` on, key head h; all warps.  RT row tiles, MR
  // of them to a warp, x NW MR / RT shares of the positions.
  template <int RT>
  __device__ void prefix_piece(int token0, int row, int valid, int h, int len, const int32_t *table, int s0, int s1, int64_t part) {
    constexpr int kHeight = kRows<MODE> * RT, kStep = kP * NW, MR = RT == 4 ? kMR : 1, kGroups = RT / MR, kPos = kP * kGroups, kNT = kGroups < kAtOnce ? kGroups : kAtOnce;
    constexpr uint32_t kStage = NW * S::kWarpStage;
    const int rt = warp % kGroups * MR, share = warp / kGroups, t = threadIdx.x;  // the warp's first row tile, its share of the positions
    const bool busy = rt * 16 < valid;
    const int n = s1 - s0;
    // a step's page numbers are asked for while the step before is worked on, and turned into offsets after it
    const Divisor pages = p.prefix_pages;
    const auto entry = [&](int i) {
      const int pos = (s0 + i) * kStep + t;
      return t < kStep && i < n && pos < len ? table[pages(pos)] : -1;
    };
    const auto put = [&](int i, int number, int at) {
      const int pos = (s0 + i) * kStep + t;
      if (t < kStep) put_offsets(at * kStep + t, i < n && pos < len ? offsets_of(number, pos - pages(pos) * pages.size, pages.size, h) : make_ulonglong2(kNowhere, kNowhere));
    };
    constexpr bool kSplit = MODE == kAttFloat && 2 * RT <= NW;   // (twice the room; the warps' own tiles leave no more)
#pragma unroll
    for (int r = 0; r < MR; ++r)
      if (rt * 16 + r * 16 < valid) load_queries<kSplit>(token0, row + rt * 16 + r * 16, valid - rt * 16 - r * 16, h, rt + r);
    constexpr int kLooked = S::kThreads / kStep;   // steps that the threads look up at once
#pragma unroll 1
    for (int i = 0; i < STAGES; i += kLooked) {
      const int pos = (s0 + i) * kStep + t, last = (s0 + n) * kStep < len ? (s0 + n) * kStep : len;
      if (i + t / kStep < STAGES) put_offsets(i * kStep + t, pos < last ? offsets_of(table[pages(pos)], pos - pages(pos) * pages.size, pages.size, h) : make_ulonglong2(kNowhere, kNowhere));
    }
    __syncthreads();
    const int seen[2] = {len, len};
    int stage = 0, fill = 0;
#pragma unroll 1
    for (int i = 1 - STAGES; i < n; ++i) {
      if (i >= 0) {
        cp_wait<STAGES - 2>();
        __syncthreads();
      }
      if (i + STAGES - 1 < n) copy_stage<NW>(ring + fill * kStage, slots + fill * kStep * 16, t);
      cp_commit();
      fill = fill + 1 == STAGES ? 0 : fill + 1;
      if (i < 0) {
        if (i == -1) {
          finish_queries();
          clear<MR>();
        }
        continue;
      }
      const int number = entry(i + STAGES);
      if (busy) {
        const uint32_t keys = ring + stage * kStage + share * kPos * S::kRow, values = keys + kStep * S::kRow;
        const int first = (s0 + i) * kStep + share * kPos;
#pragma unroll 1
        for (int j = 0; j < kGroups; j += kNT)
          if (first + kP * j < len) positions<false, kNT, kSplit, MR>(keys + kP * j * S::kRow, values + kP * j * S::kRow, first + kP * j, seen, rt, len, 0);
      }
      put(i + STAGES, number, stage);
      stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    cp_wait<0>();
    sum_columns<MR>();
    if constexpr (kGroups == NW && MR == 1) {
      if (busy && part < p.prefix_parts)
        store_part(p.prefix_o + (part * kHeight + rt * 16) * p.a.head_dim, p.prefix_ml + part * kHeight + rt * 16, valid - rt * 16);
      __syncthreads();
      return;
    }
    __syncthreads();
    // the warps' results meet in the ring: rows of the same tile of the shares of the positions
    const int g = lane >> 2, tt = lane & 3;
#pragma unroll
    for (int i = 0; i < 2 * MR; ++i) {
      const int r = i / 2, at = (warp * MR + r) * 16 + g + 8 * (i % 2);
      if (rt * 16 + r * 16 + g + 8 * (i % 2) >= valid) continue;
      if (tt == 0) asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(ml + at * 8), "f"(m[r][i % 2] * p.scale_log2), "f"(l[r][i % 2]) : "memory");
      const uint32_t to = ring + at * S::kOutRow * 4 + column(0, tt, 0) * 4;
#pragma unroll
      for (int j = 0; j < DT / 8; ++j) {
        if constexpr (kTf32<MODE>) {
          if ((j & 3) == 0)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int e = 2 * (i % 2) + c;
              asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(to + (32 * (j / 4) + 4 * c) * 4), "f"(o[r][j][e]), "f"(o[r][j + 1][e]), "f"(o[r][j + 2][e]), "f"(o[r][j + 3][e]) : "memory");
            }
        } else {
          asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(to + 32 * j), "f"(o[r][j][2 * (i % 2)]), "f"(o[r][j][2 * (i % 2) + 1]) : "memory");
        }
      }
    }
    __syncthreads();
    const int D = p.a.head_dim, d = t % (DT / 4) * 4;
    const int rows = part < p.prefix_parts && d < D ? valid : 0;
#pragma unroll 2
    for (int r = t / (DT / 4); r < rows; r += S::kThreads / (DT / 4)) {
      const int tile = r / 16, rr = r & 15;
      float mm[NW / kGroups], w[NW / kGroups], top = -CUDART_INF_F, sum = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < NW / kGroups; ++k) {
        asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(mm[k]), "=f"(w[k]) : "r"(ml + ((k * RT + tile) * 16 + rr) * 8) : "memory");
        top = fmaxf(top, mm[k]);
      }
#pragma unroll
      for (int k = 0; k < NW / kGroups; ++k) {
        const float f = mm[k] > -CUDART_INF_F ? power2(mm[k] - top) : 0.f;
        const float4 u = lds4(ring + (((k * RT + tile) * 16 + rr) * S::kOutRow + d) * 4);
        sum += f * w[k];
        v.x += f * u.x, v.y += f * u.y, v.z += f * u.z, v.w += f * u.w;
      }
      const int64_t at = part * kHeight + r;
      *reinterpret_cast<float4 *>(p.prefix_o + at * D + d) = v;
      if (d == 0) p.prefix_ml[at] = make_float2(top, sum);
    }
    __syncthreads();
  }

  // ---- the own kind: the warp's run of steps at .. end, across tiles and sequences without a pause: what the copies need is worked
  // out STAGES steps ahead, and each stage of the ring carries its tile along.
  struct Tile {
    int token0, count, len, row;   // first query token of the sequence and how many it has, length, first flat row
    int h, step, part, last;       // last: the tile's (or the run's) last step
  };
  template <typename F>
  __device__ void own_run(int run, int at, int end, const F &cost) {
    const spd_attention_args &a = p.a;
    const uint32_t my_ring = ring + warp * (STAGES * S::kWarpStage);
    const int mine = warp * (STAGES * kP);
    const uint32_t tiles_at = ml + warp * (STAGES * 32);
    const int g = lane >> 2;
    const Divisor pages = p.own_pages;
    // the place of the next step to be looked up
    Place place = find_segment(a.b, at, cost);
    int token0 = 0, count = 0, len = 0, steps = 0, high = 0, tiles = 0;
    const auto enter = [&]() {   // the segment's numbers; empty ones are passed over
#pragma unroll 1
      for (;;) {
        if (place.segment >= a.b) {   // (only if the arrays change under the kernel: one tile of no rows and no positions to the run's end)
          token0 = count = 0, len = -0x7fffffff, steps = 0x7fffffff, high = tiles = 1;
          place.before = at, place.segment = a.b - 1;
          return;
        }
        token0 = first_row(p, place.segment);
        count = first_row(p, place.segment + 1) - token0;
        len = own_length(p, place.segment);
        steps = (int)(((unsigned)len + kP - 1) / kP);
        high = tiles_of(count * p.ratio, kRows<MODE>);
        tiles = steps ? high * a.n_kv_heads : 0;
        if (at < place.before + tiles * steps) return;
        place.before += tiles * steps;
        place.tiles_before += tiles;
        ++place.segment;
      }
    };
    enter();
    int tile = (at - place.before) / steps, step = at - place.before - tile * steps, h = tile / high, row = tile - h * high;
    const int n = end - at;
    int ahead = 0;               // steps looked up
    int number = -1;
    const auto entry = [&]() {
      const int pos = step * kP + lane;
      number = ahead < n && lane < kP && pos < len ? a.own_table[place.segment * a.own_row + pages(pos)] : -1;
    };
    const auto put = [&](int to) {
      if (ahead >= n) return;
      const int pos = step * kP + lane;
      if (lane < kP) put_offsets(mine + to * kP + lane, pos < len ? offsets_of(number, pos - pages(pos) * pages.size, pages.size, h) : make_ulonglong2(kNowhere, kNowhere));
      const bool last = step + 1 == steps || ahead + 1 == n;
      if (lane == 0) {
        asm volatile("st.shared.v4.s32 [%0], {%1,%2,%3,%4};" ::"r"(tiles_at + to * 32), "r"(token0), "r"(count), "r"(len), "r"(row * kRows<MODE>) : "memory");
        asm volatile("st.shared.v4.s32 [%0], {%1,%2,%3,%4};" ::"r"(tiles_at + to * 32 + 16), "r"(h), "r"(step), "r"(run + place.tiles_before + tile), "r"((int)last) : "memory");
      }
      if (ahead && step == 0) prefetch_queries(token0, row * kRows<MODE>, count * p.ratio - row * kRows<MODE>, h);
      ++ahead, ++step, ++at;
      if (step == steps) {
        step = 0, ++tile;
        if (++row == high) row = 0, ++h;
        if (tile == tiles && ahead < n) {
          enter();
          tile = h = row = 0;
        }
      }
    };
    int stage = 0, fill = 0, valid = 0, least = 0, most = 0, seen[2] = {0, 0};
    bool fresh = true;
#pragma unroll 1
    for (int i = -STAGES; i < n; ++i) {
      if (i >= 0) cp_wait<STAGES - 2>();
      __syncwarp();
      if (i > -STAGES) {
        if (i + STAGES - 1 < n) copy_stage<1>(my_ring + fill * S::kWarpStage, slots + (mine + fill * kP) * 16, lane);
        cp_commit();
        fill = fill + 1 == STAGES ? 0 : fill + 1;
      }
      entry();
      if (i >= 0) {
        Tile x;
        asm volatile("ld.shared.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(x.token0), "=r"(x.count), "=r"(x.len), "=r"(x.row) : "r"(tiles_at + stage * 32) : "memory");
        asm volatile("ld.shared.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(x.h), "=r"(x.step), "=r"(x.part), "=r"(x.last) : "r"(tiles_at + stage * 32 + 16) : "memory");
        if (fresh) {
          valid = x.count * p.ratio - x.row;
          if (valid > kRows<MODE>) valid = kRows<MODE>;
          load_queries(x.token0, x.row, valid, x.h, warp);
          clear();
          finish_queries();
          seen[0] = seen[1] = least = most = x.len;
          if (a.q_start) {
#pragma unroll
            for (int k = 0; k < kHalves; ++k) {
              const int r = kFew ? g & 3 : g + 8 * k;
              seen[k] = x.len - (x.count - 1 - (x.row + (r < valid ? r : 0)) / p.ratio);
            }
            least = x.len - (x.count - 1 - x.row / p.ratio), most = x.len - (x.count - 1 - (x.row + valid - 1) / p.ratio);
          }
          if constexpr (S::kQueriesInShared) __syncwarp();
        }
        const uint32_t keys = my_ring + stage * S::kWarpStage;
        if (x.step * kP < most) positions<true, 1, false, 1>(keys, keys + kP * S::kRow, x.step * kP, seen, warp, least, x.len);
        fresh = x.last;
        if (x.last) {
          sum_columns();
          if (x.part < p.own_parts) store_part(p.own_o + (int64_t)x.part * p.rows_o * a.head_dim, p.own_ml + (int64_t)x.part * p.rows_o, valid);
        }
      }
      __syncwarp();  // (all lanes have read the stage's tile)
      put(stage);    // step i + STAGES into the stage that is done (before the first, into stages 0, 1, ..)
      stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    cp_wait<0>();
  }
  // Asks a tile's queries into L2.
  __device__ __forceinline__ void prefetch_queries(int token0, int row, int valid, int h) const {
    const int r = lane >> 1;
    if (r >= valid) return;
    const int f = row + r, token = p.by_ratio(f);
    const int bytes = p.a.head_dim * (MODE == kAttBf16 ? 2 : 4);
    const char *at = static_cast<const char *>(p.a.q) +
                     ((int64_t)(token0 + token) * p.a.q_row + (int64_t)(h * p.ratio + f - token * p.ratio) * p.a.q_head) * (MODE == kAttBf16 ? 2 : 4);
#pragma unroll 1
    for (int c = (lane & 1) * 128; c < bytes; c += 256) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + c));
  }
};

template <int MODE, int DT, int NW, int STAGES, int RT, int PER_SM>
__global__ void __launch_bounds__(32 * NW, PER_SM) spd_attend_kernel(const __grid_constant__ Attend p) {
  extern __shared__ __align__(1024) char dyn[];  // (rows are exchanged by XOR of address bits)
  using A = Attending<MODE, DT, NW, STAGES>;
  constexpr int kHeight = kRows<MODE> * RT, kStep = kPositions<MODE> * NW;
  dep_launch();
  const spd_attention_args &a = p.a;
  const auto prefix = [&](int g) { return prefix_cost<kHeight, kStep>(p, g); };
  const auto own = [&](int s) { return own_cost<kPositions<MODE>, kRows<MODE>>(p, s); };
  Totals pre = sum_segments(a.g, 0, prefix), mine = sum_segments(a.b, 0, own);
  if (no_partition(pre, mine)) return;
  const Split split = split_blocks(gridDim.x, NW, p.weights, pre, mine);
  A w(p, smem_u32(dyn));
  if ((int)blockIdx.x < split.prefix_blocks) {
    int at = run_start(blockIdx.x, split.prefix_blocks, pre.steps);
    const int end = run_start(blockIdx.x + 1, split.prefix_blocks, pre.steps);
    if (at >= end) return;
    Place place = find_segment(a.g, at, prefix);
#pragma unroll 1
    while (at < end) {
      const int g = place.segment;
      if (g >= a.g) return;
      const int first = first_seq(p, g), token0 = first_row(p, first);
      const int rows = (first_row(p, first_seq(p, g + 1)) - token0) * p.ratio;
      const int len = prefix_length(p, g), steps = (int)(((unsigned)len + kStep - 1) / kStep);
      const int high = tiles_of(rows, kHeight), tiles = steps ? high * a.n_kv_heads : 0;
      if (at >= place.before + tiles * steps) {  // (an empty one, or done)
        place.before += tiles * steps;
        place.tiles_before += tiles;
        ++place.segment;
        continue;
      }
      const int tile = (at - place.before) / steps;
      const int s0 = at - place.before - tile * steps;
      const int s1 = end - at < steps - s0 ? s0 + (end - at) : steps;
      const int h = tile / high, row = (tile - h * high) * kHeight;
      w.template prefix_piece<RT>(token0, row, rows - row < kHeight ? rows - row : kHeight, h, len, a.prefix_table + g * a.prefix_row, s0, s1,
                                  (int64_t)blockIdx.x + place.tiles_before + tile);
      at += s1 - s0;
    }
  } else if (mine.steps) {
    const int run = (blockIdx.x - split.prefix_blocks) * NW + w.warp;
    if (run >= split.own_warps) return;
    const int at = run_start(run, split.own_warps, mine.steps), end = run_start(run + 1, split.own_warps, mine.steps);
    w.own_run(run, at, end, own);
  }
}

__device__ __forceinline__ bool past_table(int len, int room) { return len < 0 || len > room; }

// The join: a warp per (token, query head), or WIDE: a block, whose warps share the parts.  Every warp works out for itself which parts its row has, while the first kernel still runs.
constexpr int kJoinThreads = 128;
template <typename X, int DT, int HEIGHT, int OWN, int NW, int POS, int AHEAD, bool WIDE>
__global__ void __launch_bounds__(kJoinThreads) spd_attend_join_kernel(const __grid_constant__ Attend p) {
  const spd_attention_args &a = p.a;
  const int token = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = a.head_dim;
  constexpr int kWarps = kJoinThreads / 32;
  const int head = WIDE ? blockIdx.y : blockIdx.y * kWarps + warp;
  int seq = a.q_start ? -1 : token, group = a.group_start ? -1 : 0;
  if (a.q_start)
#pragma unroll 1
    for (int base = 0; base < a.b; base += 32) {
      const int s = base + lane;
      const unsigned hit = __ballot_sync(~0u, s < a.b && a.q_start[s < a.b ? s : 0] <= token && token < a.q_start[s < a.b ? s + 1 : 0]);
      if (hit) seq = base + __ffs(hit) - 1;
    }
  if (a.group_start)
#pragma unroll 1
    for (int base = 0; base < a.g; base += 32) {
      const int g = base + lane;
      const unsigned hit = __ballot_sync(~0u, g < a.g && a.group_start[g < a.g ? g : 0] <= seq && seq < a.group_start[g < a.g ? g + 1 : 0]);
      if (hit) group = base + __ffs(hit) - 1;
    }
  Totals pre = sum_segments(a.g, group, [&](int g) { return prefix_cost<HEIGHT, POS * NW>(p, g); });
  Totals own = sum_segments(a.b, seq, [&](int s) { return own_cost<POS, OWN>(p, s); });
  const bool falls = no_partition(pre, own);
  const Split split = split_blocks(p.blocks, NW, p.weights, pre, own);
  const int h = p.by_ratio(head), hr = head - h * p.ratio;
  // pieces: prefix parts first .. first + np - 1 at row `prow`, own parts at `orow`
  long long pfirst = 0, ofirst = 0;
  int np = 0, no = 0, prow = 0, orow = 0;
  if (pre.steps > 0 && seq >= 0 && group >= 0) {
    const int token0 = first_row(p, first_seq(p, group)), rows = (first_row(p, first_seq(p, group + 1)) - token0) * p.ratio;
    const int steps = (int)(((unsigned)prefix_length(p, group) + POS * NW - 1) / (POS * NW)), high = tiles_of(rows, HEIGHT);
    if (steps > 0) {
      const int f = (token - token0) * p.ratio + hr;
      const int tile = h * high + f / HEIGHT;
      prow = f % HEIGHT;
      const int from = pre.before + tile * steps;
      const int r0 = run_of(from, split.prefix_blocks, pre.steps), r1 = run_of(from + steps - 1, split.prefix_blocks, pre.steps);
      pfirst = (long long)r0 + pre.tiles_before + tile;
      np = r1 - r0 + 1;
    }
  }
  if (seq >= 0 && own.steps > 0) {
    const int token0 = first_row(p, seq), rows = (first_row(p, seq + 1) - token0) * p.ratio;
    const int steps = (int)(((unsigned)own_length(p, seq) + POS - 1) / POS), high = tiles_of(rows, OWN);
    if (steps > 0) {
      const int f = (token - token0) * p.ratio + hr;
      const int tile = h * high + f / OWN;
      orow = f % OWN;
      const int from = own.before + tile * steps;
      const int r0 = run_of(from, split.own_warps, own.steps), r1 = run_of(from + steps - 1, split.own_warps, own.steps);
      ofirst = (long long)r0 + own.tiles_before + tile;
      no = r1 - r0 + 1;
    }
  }
  if (pfirst + np > p.prefix_parts) np = pfirst < p.prefix_parts ? (int)(p.prefix_parts - pfirst) : 0;
  if (ofirst + no > p.own_parts) no = ofirst < p.own_parts ? (int)(p.own_parts - ofirst) : 0;
  if (a.status && lane == 0 && (falls || seq < 0 || past_table(a.own_len[seq], p.own_room) || (group >= 0 && a.g > 0 && past_table(a.prefix_len[group], p.prefix_room))))
    *a.status = SPD_ERANGE;
  dep_wait();
  if (head >= a.n_heads) return;
  const int n = WIDE ? (np + no - warp + kWarps - 1) / kWarps : np + no;   // parts of this warp: every one, or every fourth from its own on
  const auto nth = [&](int i) { return WIDE ? warp + i * kWarps : i; };
  const float2 *const pml = p.prefix_ml + pfirst * HEIGHT + prow, *const oml = p.own_ml + ofirst * p.rows_o + orow;
  const float *const po = p.prefix_o + (pfirst * HEIGHT + prow) * D + lane * 4, *const oo = p.own_o + (ofirst * p.rows_o + orow) * D + lane * 4;
  const auto part_ml = [&](int k) {
    const int i = nth(k);
    return __ldcg(i < np ? pml + i * HEIGHT : oml + (i - np) * p.rows_o);
  };
  constexpr int kVec = DT > 128 ? 2 : 1;  // fours of dimensions of a lane
  float4 o[AHEAD][kVec];                  // parts under way; the first of them are asked for together with the maxima
  const auto ask = [&](int first) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = nth(first + k);
      const float *src = i < np ? po + (int64_t)i * (HEIGHT * D) : oo + (int64_t)(i - np) * (p.rows_o * D);
#pragma unroll
      for (int c = 0; c < kVec; ++c)
        o[k][c] = first + k < n && c * 128 + lane * 4 < D ? __ldcg(reinterpret_cast<const float4 *>(src + c * 128)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  ask(0);
  float2 v = make_float2(-CUDART_INF_F, 0.f);
  if (lane < n) v = part_ml(lane);
  float top = v.x, sum = 0.f;
#pragma unroll 1
  for (int i = lane + 32; i < n; i += 32) top = fmaxf(top, part_ml(i).x);
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, j));
  float acc[4 * kVec] = {};
  float f = 0.f;
#pragma unroll 1
  for (int i = 0; i < n; i += AHEAD) {
    if ((i & 31) == 0) {   // the weights of the next 32 parts, a lane each
      if (i) v = i + lane < n ? part_ml(i + lane) : make_float2(-CUDART_INF_F, 0.f);
      f = v.x > -CUDART_INF_F ? power2(v.x - top) : 0.f;
      sum += f * v.y;
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const float w = __shfl_sync(~0u, f, (i + k) & 31);
#pragma unroll
      for (int c = 0; c < kVec; ++c) {
        const float4 x = o[k][c];
        acc[4 * c] += w * x.x, acc[4 * c + 1] += w * x.y, acc[4 * c + 2] += w * x.z, acc[4 * c + 3] += w * x.w;
      }
    }
    if (i + AHEAD < n) ask(i + AHEAD);
  }
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) sum += __shfl_xor_sync(~0u, sum, j);
  if constexpr (WIDE) {
    __shared__ float all[kWarps][4 * 32 * kVec];
    __shared__ float2 all_ml[kWarps];
#pragma unroll
    for (int c = 0; c < 4 * kVec; ++c) all[warp][c * 32 + lane] = acc[c];
    if (lane == 0) all_ml[warp] = make_float2(top, sum);
    __syncthreads();
    if (warp) return;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, all_ml[w].x);
    sum = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * kVec; ++c) acc[c] = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float2 x = all_ml[w];
      const float f = x.x > -CUDART_INF_F ? power2(x.x - top) : 0.f;
      sum += f * x.y;
#pragma unroll
      for (int c = 0; c < 4 * kVec; ++c) acc[c] += f * all[w][c * 32 + lane];
    }
  }
  const bool none = top == -CUDART_INF_F && !(sum != sum);
  const float inv = none ? 0.f : 1.f / sum;
  X *out = static_cast<X *>(a.out) + (int64_t)token * a.o_row + (int64_t)head * a.o_head;
#pragma unroll
  for (int c = 0; c < kVec; ++c) {
    const int d = c * 128 + lane * 4;
    if (d >= D) continue;
    const float4 v = make_float4(acc[4 * c] * inv, acc[4 * c + 1] * inv, acc[4 * c + 2] * inv, acc[4 * c + 3] * inv);
    if (p.out_fours) {
      store4(out + d, v);
    } else {
      out[d] = from_float<X>(v.x), out[d + 1] = from_float<X>(v.y), out[d + 2] = from_float<X>(v.z), out[d + 3] = from_float<X>(v.w);
    }
  }
  if (lane == 0 && a.lse) a.lse[(int64_t)token * a.n_heads + head] = none ? -CUDART_INF_F : (top + log2f(sum)) * 0.6931471805599453f;
}

// ---- launch.  Dimensions a kernel is built for, warps, stages and blocks per SM: as many stages as 227 KB hold for the blocks
// that 65536 registers allow.  (Four float32 rows, 128 dimensions, 3 rows behind 2048 positions: 14.6 us with three blocks of two stages, 15.9 with two of
// three, 16.6 with one of eight warps; 256 dimensions 18.3 with two stages, 20.5 with three; eight rows: 17.1 with two blocks, 20.0 with three, which spill.)
template <int MODE, int DT> struct AttendTune;
template <> struct AttendTune<kAttBf16, 64> { static constexpr int nw = 4, stages = 4, per_sm = 3; };
template <> struct AttendTune<kAttBf16, 128> { static constexpr int nw = 4, stages = 3, per_sm = 2; };
template <> struct AttendTune<kAttBf16, 256> { static constexpr int nw = 4, stages = 2, per_sm = 1; };
template <> struct AttendTune<kAttTerms, 64> { static constexpr int nw = 4, stages = 4, per_sm = 3; };
template <> struct AttendTune<kAttTerms, 128> { static constexpr int nw = 4, stages = 3, per_sm = 2; };
template <> struct AttendTune<kAttTerms, 256> { static constexpr int nw = 4, stages = 2, per_sm = 1; };
template <> struct AttendTune<kAttFloat, 64> { static constexpr int nw = 4, stages = 3, per_sm = 3; };
template <> struct AttendTune<kAttFloat, 128> { static constexpr int nw = 8, stages = 2, per_sm = 1; };
template <> struct AttendTune<kAttFloat, 256> { static constexpr int nw = 4, stages = 2, per_sm = 1; };

template <> struct AttendTune<kAttFewFloat, 64> { static constexpr int nw = 4, stages = 3, per_sm = 4; };
template <> struct AttendTune<kAttFewFloat, 128> { static constexpr int nw = 4, stages = 2, per_sm = 3; };
template <> struct AttendTune<kAttFewFloat, 256> { static constexpr int nw = 4, stages = 2, per_sm = 1; };
template <> struct AttendTune<kAttEight, 64> { static constexpr int nw = 4, stages = 4, per_sm = 3; };
template <> struct AttendTune<kAttEight, 128> { static constexpr int nw = 4, stages = 3, per_sm = 2; };
template <> struct AttendTune<kAttFew, 64> { static constexpr int nw = 4, stages = 3, per_sm = 4; };
template <> struct AttendTune<kAttFew, 128> { static constexpr int nw = 4, stages = 2, per_sm = 3; };
template <> struct AttendTune<kAttFew, 256> { static constexpr int nw = 4, stages = 2, per_sm = 1; };

template <int MODE, int DT, int RT>
cudaError_t attend_launch(const Attend &p, int device, cudaStream_t s) {
  using T = AttendTune<MODE, DT>;
  constexpr size_t smem = AttendShape<MODE, DT, T::nw, T::stages>::kShared;
  static_assert((smem + 1024) * T::per_sm <= 228 * 1024, "the blocks of an SM fit its shared memory");
  const auto kernel = spd_attend_kernel<MODE, DT, T::nw, T::stages, RT, T::per_sm>;
  static std::atomic<bool> prepared[64];  // per device; setting it twice does no harm
  if (device >= 64 || !prepared[device].load(std::memory_order_relaxed)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    if (device < 64) prepared[device].store(true, std::memory_order_relaxed);
  }
  kernel<<<p.blocks, 32 * T::nw, smem, s>>>(p);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  constexpr int kWarps = kJoinThreads / 32;
  const dim3 grid(p.a.n, (p.a.n_heads + kWarps - 1) / kWarps);
  using X = typename std::conditional<MODE == kAttBf16, __nv_bfloat16, float>::type;
  // Few rows of many parts each keep eight parts under way (32 rows of 60 parts: 17.5 us in all instead of 19.8), with 16 and more their blocks' warps
  // share them (28 rows of 130 parts: 12.4 instead of 21.5); many rows of few parts keep four, with more rows on an SM (128 rows of 32 heads: 34 instead of 38).
  if (p.many_parts > 1)
    return launch_dep(spd_attend_join_kernel<X, DT, kRows<MODE> * RT, kRows<MODE>, T::nw, kPositions<MODE>, (DT > 128 ? 4 : 8), true>, dim3(p.a.n, p.a.n_heads), dim3(kJoinThreads), 0, s, p);
  if (p.many_parts)
    return launch_dep(spd_attend_join_kernel<X, DT, kRows<MODE> * RT, kRows<MODE>, T::nw, kPositions<MODE>, (DT > 128 ? 4 : 8), false>, grid, dim3(kJoinThreads), 0, s, p);
  return launch_dep(spd_attend_join_kernel<X, DT, kRows<MODE> * RT, kRows<MODE>, T::nw, kPositions<MODE>, (DT > 128 ? 2 : 4), false>, grid, dim3(kJoinThreads), 0, s, p);
}
template <int MODE, int DT>
cudaError_t attend_launch(const Attend &p, int rt, int device, cudaStream_t s) {
  if constexpr (kRows<MODE> == 16) {
    if (rt == 2) return attend_launch<MODE, DT, 2>(p, device, s);
    if (rt == 4) return attend_launch<MODE, DT, 4>(p, device, s);
  }
  return attend_launch<MODE, DT, 1>(p, device, s);
}
template <int MODE>
cudaError_t attend_launch(const Attend &p, int rt, int device, cudaStream_t s) {
  if (p.a.head_dim <= 64) return attend_launch<MODE, 64>(p, rt, device, s);
  if constexpr (MODE != kAttEight) {   // (whose registers do not hold more dimensions)
    if (p.a.head_dim > 128) return attend_launch<MODE, 256>(p, rt, device, s);
  }
  return attend_launch<MODE, 128>(p, rt, device, s);
}

cudaError_t attend_bf16(const Attend &p, int rt, int device, cudaStream_t s);
cudaError_t attend_terms(const Attend &p, int rt, int device, cudaStream_t s);
cudaError_t attend_float(const Attend &p, int rt, int device, cudaStream_t s);
cudaError_t attend_few(const Attend &p, int rt, int device, cudaStream_t s);
cudaError_t attend_few_float(const Attend &p, int rt, int device, cudaStream_t s);
cudaError_t attend_eight(const Attend &p, int rt, int device, cudaStream_t s);

}  // namespace spd
