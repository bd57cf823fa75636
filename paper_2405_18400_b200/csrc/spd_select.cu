// Beam search's selection: the best `beams` of beams x vocab options of each request, in one launch.
//
// The rank of an option inside its beam is that of its logit, so the logits are read once, into registers: a block takes a slice of one
// beam's row, finds its largest logit and sum of exponentials, and its `beams` best logits; the block of a request that arrives
// last joins the slices' sums, gives the few options that are left their scores in 64 bits and ranks them.  What bounds it is
// the chain load - threshold - list - arrive - join, each 1 to 2 us (3 beams of 4096 tokens 5.8 us), and with many rows the phases of two blocks an SM
// one after the other (16 x 8 beams of 32000 tokens 13.5 us: logits there 3, lists written 7, joined 11, from the first block's start; the logits' bytes are 1.9).
//
// No rank is found by a sort.  Of n lists without equal keys, exactly w have a head among the w best heads; nothing outside
// these w lists can be among the w best of all.  So with four lanes' logits as a list, the w-th best head is a threshold, and
// what passes it (a few more than w on random rows) is ranked by counting the greater ones.  Sorted lists are then merged, by counting too where
// they are few, else by taking the best head w times.  A key holds value and index, so that no two are equal and ties fall to the lower index.
#include <cfloat>
#include <cmath>

#include <math_constants.h>

#include "spd_ops.h"
#include "spd_ptx.cuh"

namespace spd {
namespace {

constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelGroups = kSelThreads / 4;
constexpr int kSelMaxBeams = 32;
constexpr int kSelMaxSlices = 32;   // a lane each when their sums are joined
constexpr int kSelMaxVocab = 262144;
constexpr int kSelMaxRequests = 65535;
// The counters have their place to themselves whatever the call's sizes are, so that a workspace may serve calls of different sizes in turn.
constexpr size_t kSelCounters = ((size_t)kSelMaxRequests * 4 + 255) / 256 * 256;
constexpr int kSelJoinBytes = 44 * 1024;

struct Select {
  spd_select_args a;
  int slices;
  unsigned *arrived;               // [requests]
  float2 *stats;                   // [requests][beams][slices]: largest logit, sum of exponentials
  unsigned long long *keys;        // [requests][beams][slices][beams]: best logits, best first, 0 = none
  double2 *per;                    // [requests][beams]: length^alpha and its inverse
  double inv_tau;
  float scale;                     // log2 e / tau
  int keys_fit;                    // all lists of a request have room in shared memory
};

// Order-preserving words: larger value, larger word; nothing real maps to 0.  Within equal values the lower index is the larger key.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t w) { return __uint_as_float(w & 0x80000000u ? w ^ 0x80000000u : ~w); }
__device__ __forceinline__ unsigned long long ordered(double v) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(v);
  return b ^ ((unsigned long long)((long long)b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ unsigned long long logit_key(float z, int index) {
  return z > -CUDART_INF_F ? ((unsigned long long)ordered(z + 0.f) << 32) | (uint32_t)~index : 0ull;  // -0 and 0 are one value
}

// The lanes' keys, largest first.
__device__ __forceinline__ unsigned long long sort_lanes(unsigned long long v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1) {
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      const unsigned long long o = __shfl_xor_sync(~0u, v, j);
      const bool keep_max = ((lane & k) == 0) == ((lane & j) == 0);
      v = (v > o) == keep_max ? v : o;
    }
  }
  return v;
}

struct Option {
  unsigned long long rank;  // ordered score per length, 0 = none
  uint32_t flat;            // beam * vocab + token
};

// Ranks of n things by all threads of the block: as many neighbouring lanes to a thing as n leaves, each counting its share of the
// others.  count(k, first, step): how many of the things first, first + step, .. come before thing k; done(k, rank): by one lane.
template <typename C, typename D>
__device__ __forceinline__ void rank_all(int n, C count, D done) {
  const int log2 = n <= 8 ? 5 : n <= 16 ? 4 : n <= 32 ? 3 : n <= 64 ? 2 : n <= 128 ? 1 : 0;
  const int lanes = 1 << log2, part = threadIdx.x & (lanes - 1);
  for (int base = 0; base < n; base += kSelThreads >> log2) {   // (all lanes of a warp take part)
    const int k = base + (threadIdx.x >> log2);
    int rank = k < n ? count(k, part, lanes) : 0;
    for (int j = lanes >> 1; j > 0; j >>= 1) rank += __shfl_xor_sync(~0u, rank, j);
    if (part == 0 && k < n) done(k, rank);
  }
}

template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int n = 4;
  __device__ static void load(const float *p, float *z) {
    const float4 v = *reinterpret_cast<const float4 *>(p);
    z[0] = v.x, z[1] = v.y, z[2] = v.z, z[3] = v.w;
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  __device__ static void load(const __nv_bfloat16 *p, float *z) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    z[0] = low_bf16(v.x), z[1] = high_bf16(v.x), z[2] = low_bf16(v.y), z[3] = high_bf16(v.y);
    z[4] = low_bf16(v.z), z[5] = high_bf16(v.z), z[6] = low_bf16(v.w), z[7] = high_bf16(v.w);
  }
};

struct Shared {
  alignas(16) float group[kSelGroups];                     // largest logits
  unsigned long long best_keys[kSelWarps * kSelMaxBeams];  // the warps' best heads
  unsigned long long threshold;
  float limit_value, wsum[kSelWarps];
  int count, last;
  double at[kSelMaxBeams];                                 // of a beam: score - log sum, the value of its largest logit
  float most[kSelMaxBeams];                                // that logit
  double per[kSelMaxBeams], inv_per[kSelMaxBeams];         // length^alpha and its inverse
  float score[kSelMaxBeams];
  int length[kSelMaxBeams];
  bool ended[kSelMaxBeams], in_use[kSelMaxBeams];
};

// The slice's keys that can be among its best, where too many values are equal for the quick way: the threshold is a key, which no two
// share, so that at most beams x elements of a thread pass it.
// (It reads the logits again: the caller's stay in registers.)
template <typename T, int N>
__device__ __noinline__ void collect_by_key(const T *row, int vocab, int first, int W, Shared &sh, unsigned long long *list) {
  constexpr int E = Vec<T>::n;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const auto key_of = [&](int j) {
    const int e = first + (j / E) * kSelThreads * E + j % E;
    return e >= 0 && e < vocab ? logit_key(to_float(row[e]), e) : 0ull;
  };
  unsigned long long head = 0;
  for (int j = 0; j < N; ++j) {
    const unsigned long long key = key_of(j);
    if (key > head) head = key;
  }
  const unsigned long long sorted = sort_lanes(head);
  if (lane < W) sh.best_keys[warp * W + lane] = sorted;
  if (tid == 0) sh.threshold = 1, sh.count = 0;
  __syncthreads();
  if (tid < kSelWarps * W) {
    const unsigned long long mine = sh.best_keys[tid];
    int greater = 0;
    for (int k = 0; k < kSelWarps * W; ++k) greater += sh.best_keys[k] > mine;
    if (mine && greater == W - 1) sh.threshold = mine;
  }
  __syncthreads();
  const unsigned long long threshold = sh.threshold;
  if (head >= threshold)
    for (int j = 0; j < N; ++j) {
      const unsigned long long key = key_of(j);
      if (key >= threshold) list[atomicAdd(&sh.count, 1)] = key;
    }
  __syncthreads();
}

// A slice of a beam's row.  list: room for beams * elements of a thread.  What it finds is left out where the beam is not `live`.
template <typename T, int NV>
__device__ __forceinline__ void select_slice(const Select &p, Shared &sh, unsigned long long *list, int r, int i, int slice) {
  constexpr int E = Vec<T>::n, N = NV * E;
  const spd_select_args &a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, W = a.beams;
  const int64_t beam = (int64_t)r * W + i;
  const T *row = static_cast<const T *>(a.logits) + r * a.request_stride + i * a.beam_stride;
  // Vectors lie on 16 bytes; the row may begin inside one.
  const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  const int first = slice * (kSelThreads * N) - skew + tid * E;
  const bool live = a.score[beam] > -CUDART_INF_F && !(a.ended && a.ended[beam]);  // (asked for together with the logits)
  float z[N];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int e = first + v * kSelThreads * E;
    if (e >= 0 && e + E <= a.vocab) {
      Vec<T>::load(row + e, z + v * E);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) z[v * E + j] = e + j >= 0 && e + j < a.vocab ? to_float(row[e + j]) : -CUDART_INF_F;
    }
  }
  if (slice == 0 && tid == kSelThreads - 1) {
    // the beam's divisor, worked out while the logits travel
    const int length = (a.length ? a.length[beam] : 0) + (a.ended && a.ended[beam] ? 0 : 1);
    const double per = a.alpha == 0.f ? 1.0 : pow((double)(length > 1 ? length : 1), (double)a.alpha);
    p.per[beam] = make_double2(per, 1.0 / per);
  }
  if (!live) return;
  float head = -CUDART_INF_F;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    z[j] = fmaxf(z[j], -CUDART_INF_F);  // not a number: no option
    head = fmaxf(head, z[j]);
  }
  float mine = fmaxf(head, __shfl_xor_sync(~0u, head, 1));
  mine = fmaxf(mine, __shfl_xor_sync(~0u, mine, 2));
  if ((lane & 3) == 0) sh.group[tid >> 2] = mine;
  if (tid == 0) sh.count = 0, sh.limit_value = -CUDART_INF_F;
  __syncthreads();
  // the W-th largest of the groups' largest logits, equal ones counted as often as they are there: the group's four lanes count a quarter
  // each (greater ones in the low half of a count, equal ones in the high)
  float m = -CUDART_INF_F;
  int c = 0;
#pragma unroll
  for (int j = 0; j < kSelGroups / 16; ++j) {
    const float4 v = reinterpret_cast<const float4 *>(sh.group)[4 * j + (lane & 3)];
    m = fmaxf(m, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
    c += (v.x > mine) + (v.y > mine) + (v.z > mine) + (v.w > mine) + (((v.x == mine) + (v.y == mine) + (v.z == mine) + (v.w == mine)) << 16);
  }
#pragma unroll
  for (int j = 1; j < 4; j *= 2) {
    m = fmaxf(m, __shfl_xor_sync(~0u, m, j));
    c += __shfl_xor_sync(~0u, c, j);
  }
  if ((lane & 3) == 0 && mine > -CUDART_INF_F && (c & 0xffff) < W && (c & 0xffff) + (c >> 16) >= W) sh.limit_value = mine;
  const float scale = p.scale;
  float sum = 0.f;
  if (m > -CUDART_INF_F) {
#pragma unroll
    for (int j = 0; j < N; ++j) sum += power2((z[j] - m) * scale);
  }
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) sum += __shfl_xor_sync(~0u, sum, j);
  if (lane == 0) sh.wsum[warp] = sum;
  __syncthreads();
  const float limit = sh.limit_value;
  const int room = W * N;
  if (head >= limit && head > -CUDART_INF_F) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (z[j] >= limit && z[j] > -CUDART_INF_F) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < room) list[at] = logit_key(z[j], first + (j / E) * kSelThreads * E + j % E);
      }
  }
  __syncthreads();
  int n = sh.count;
  if (n > room) {
    __syncthreads();
    collect_by_key<T, N>(row, a.vocab, first, W, sh, list);
    n = sh.count;
  }
  const int64_t at = beam * p.slices + slice;
  unsigned long long *out = p.keys + at * W;
  if (n <= 32) {   // as good as always: a lane to a logit
    if (warp == 0) {
      const unsigned long long mine = lane < n ? list[lane] : 0;
      int greater = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) greater += list[j] > mine;
      if (lane < n && greater < W) out[greater] = mine;
      if (lane >= n && lane < W) out[lane] = 0;
    }
  } else {
    rank_all(
        n,
        [&](int k, int from, int step) {
          const unsigned long long mine = list[k];
          int greater = 0;
          for (int j = from; j < n; j += step) greater += list[j] > mine;
          return greater;
        },
        [&](int k, int greater) {
          if (greater < W) out[greater] = list[k];
        });
  }
  if (tid == 32) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) s += sh.wsum[w];
    p.stats[at] = make_float2(m, s);
  }
}

// log v, v > 0 and normal, to 2^-24 of ln 2: the exponent's part in 64 bits, the logarithm of what lies in [1, 2) in 32.  (log() in 64 bits
// is a microsecond of the request's last block.)
__device__ __forceinline__ double log_of_sum(float v) {
  const uint32_t b = __float_as_uint(v);
  const float f = __uint_as_float((b & 0x007fffffu) | 0x3f800000u);
  const double l = (double)((int)(b >> 23) - 127) * 0.69314718055994530942 + (double)logf(f);
  return b - 0x00800000u < 0x7f000000u ? l : (double)CUDART_NAN_F;  // (a sum of exponentials is 1 at least)
}

// Of 64-bit words the lanes' largest.
__device__ __forceinline__ unsigned long long largest(unsigned long long w) {
  const uint32_t high = __reduce_max_sync(~0u, (uint32_t)(w >> 32));
  const uint32_t low = __reduce_max_sync(~0u, (uint32_t)(w >> 32) == high ? (uint32_t)w : 0u);
  return ((unsigned long long)high << 32) | low;
}

// The request's best options from its slices' lists.  First the lists of each beam become one, which needs no scores; then, by one warp, the
// beams': a lane holds the head of a list, the best head of all leaves its list, W times (for 64 entries as fast as counting by all warps; binary
// searches by all warps took 16 beams 6 us longer).  all: beams * beams; best: as many; keys: the lists where they fit there (else null).
__device__ __forceinline__ void select_join(const Select &p, Shared &sh, Option *all, unsigned long long *best, unsigned long long *keys, int r) {
  const spd_select_args &a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, W = a.beams, S = p.slices;
  const int64_t row0 = (int64_t)r * W;
  const unsigned long long *const from = p.keys + row0 * S * W;
  // Few entries of a beam are counted against one another (16 x 8 beams of 4 lists 13.5 us, merged 14.6; 3 beams of 4 lists 6.0 and 6.3; but 2 beams of 32
  // lists 8.5 and 7.9).  (Such lists fit.)  More are merged, by as many neighbouring lanes as the beam has slices, and a power of two; by a warp
  // where every beam has one (8 beams: 9.9 us, 10.6 by the fewest lanes).
  const bool few = S * W <= 64 && S <= 16;
  const int log2 = W <= kSelWarps && !few ? 5 : S > 1 ? 32 - __clz(S - 1) : 0, lanes = 1 << log2, list = lane & (lanes - 1);
  const float scale = p.scale;
#pragma unroll 1
  for (int base = warp; base < W; base += (32 >> log2) * kSelWarps) {
    const int i = base + (lane >> log2) * kSelWarps;
    const bool here = i < W && list < S;
    const float score = i < W ? a.score[row0 + i] : 0.f;
    const bool ended = i < W && a.ended && a.ended[row0 + i];
    const int length = i < W && a.length ? a.length[row0 + i] : 0;
    const double2 per = i < W ? __ldcg(p.per + row0 + i) : make_double2(1.0, 1.0);
    const float2 st = here ? __ldcg(p.stats + (row0 + i) * S + list) : make_float2(-CUDART_INF_F, 0.f);
    if (keys && base == warp) {   // (all that the warp asks for is under way together; a beam that is over has whatever lies there)
      for (int b = warp; b < W; b += kSelWarps)
        for (int k = lane; k < S * W; k += 32) keys[b * S * W + k] = __ldcg(from + b * S * W + k);
      __syncwarp();
    }
    const bool live = here && !ended && score > -CUDART_INF_F;
    float m = live ? st.x : -CUDART_INF_F;
    const float mine = m;
    for (int j = lanes >> 1; j > 0; j >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, j));
    float s = mine > -CUDART_INF_F ? st.y * power2((mine - m) * scale) : 0.f;
    for (int j = lanes >> 1; j > 0; j >>= 1) s += __shfl_xor_sync(~0u, s, j);
    if (here && list == 0) {
      // A row whose largest logit is not finite, or a sum that is not, gives no number here and has no options.
      sh.at[i] = ended ? (double)score : (double)score - log_of_sum(s);
      sh.most[i] = m;
      sh.per[i] = per.x, sh.inv_per[i] = per.y;
      sh.score[i] = score, sh.length[i] = length, sh.ended[i] = ended, sh.in_use[i] = score > -CUDART_INF_F;
    }
    if (few) continue;
    const int at = (i * S + list) * W;
    const auto entry = [&](int e) { return live && e < W ? (keys ? keys[at + e] : __ldcg(from + at + e)) : 0ull; };
    unsigned long long head = entry(0), next = entry(1);
    int e = 1;
#pragma unroll 1
    for (int w = 0; w < W; ++w) {
      unsigned long long top = head;
      if (log2 == 5)
        top = largest(head);
      else
#pragma unroll 1
        for (int j = lanes >> 1; j > 0; j >>= 1) {
          const unsigned long long other = __shfl_xor_sync(~0u, top, j);
          if (other > top) top = other;
        }
      if (here && list == 0) best[i * W + w] = top;
      if (head == top) head = next, next = entry(++e);
    }
  }
  __syncwarp();
#pragma unroll 1
  for (int i = warp; i < W; i += kSelWarps) {
    if (few) {   // an entry counts those before it
      if (lane < W) best[i * W + lane] = 0;
      __syncwarp();
      if (sh.in_use[i] && !sh.ended[i]) {
        const unsigned long long *const l = keys + i * S * W;
        const unsigned long long low = lane < S * W ? l[lane] : 0, high = lane + 32 < S * W ? l[lane + 32] : 0;
        int before_low = 0, before_high = 0;
#pragma unroll 4
        for (int j = 0; j < S * W; ++j) before_low += l[j] > low, before_high += l[j] > high;
        if (low && before_low < W) best[i * W + before_low] = low;
        if (high && before_high < W) best[i * W + before_high] = high;
      }
      __syncwarp();
    }
    Option o = {0, 0};
    if (sh.in_use[i] && lane < W) {
      const bool ended = sh.ended[i];
      const unsigned long long key = best[i * W + lane];
      if (ended ? lane == 0 : key != 0) {
        // (the difference is exact: a score does not vanish beside logits of any size over any tau)
        const double z = ended ? 0.0 : ((double)unordered((uint32_t)(key >> 32)) - (double)sh.most[i]) * p.inv_tau, rank = (sh.at[i] + z) * sh.inv_per[i];
        if (rank > -CUDART_INF) o.rank = ordered(rank), o.flat = (uint32_t)i * a.vocab + (ended ? max(a.eos_id, 0) : ~(uint32_t)key);
      }
    }
    if (lane < W) all[i * W + lane] = o;
  }
  __syncthreads();
  if (warp) return;
  const auto entry = [&](int e) { return lane < W && e < W ? all[lane * W + e] : Option{0, 0}; };
  Option head = entry(0), next = entry(1), mine = {0, 0};
  int e = 1;
#pragma unroll 1
  for (int w = 0; w < W; ++w) {
    const unsigned long long rank = largest(head.rank);
    if (!rank) break;
    const uint32_t flat = __reduce_min_sync(~0u, head.rank == rank ? head.flat : ~0u);
    if (lane == w) mine = {rank, flat};
    if (head.rank == rank && head.flat == flat) head = next, next = entry(++e);
  }
  if (lane >= W) return;
  int token = -1, parent = lane, length = 0;
  float score = -CUDART_INF_F;
  bool ended = false;
  if (mine.rank) {
    parent = mine.flat / (uint32_t)a.vocab;
    ended = sh.ended[parent];
    token = ended ? a.eos_id : (int)(mine.flat - (uint32_t)parent * a.vocab);
    length = sh.length[parent] + (ended ? 0 : 1);
    const unsigned long long w = mine.rank;   // back from the rank to the value
    const double rank = __longlong_as_double((long long)(w & 0x8000000000000000ull ? w ^ 0x8000000000000000ull : ~w));
    score = ended ? sh.score[parent] : (float)(rank * sh.per[parent]);
    ended |= a.eos_id >= 0 && token == a.eos_id;
  }
  a.new_token[row0 + lane] = token;
  a.new_parent[row0 + lane] = parent;
  a.new_score[row0 + lane] = score;
  if (a.new_length) a.new_length[row0 + lane] = length;
  if (a.new_ended) a.new_ended[row0 + lane] = ended;
}

template <typename T, int NV>
__global__ void __launch_bounds__(kSelThreads) spd_select_kernel(const __grid_constant__ Select p) {
  extern __shared__ unsigned long long dyn[];
  __shared__ Shared sh;
  const int slice = blockIdx.x, i = blockIdx.y, r = blockIdx.z, W = p.a.beams;
  select_slice<T, NV>(p, sh, dyn, r, i, slice);
  __syncthreads();
  if (threadIdx.x == 0) {
    // (one thread's release and acquire stand for the block's stores and loads, which the barriers put in front of it and behind it)
    unsigned before;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(p.arrived + r) : "memory");
    sh.last = before == gridDim.x * gridDim.y - 1;
    if (sh.last) p.arrived[r] = 0;   // for the next call
  }
  __syncthreads();
  if (!sh.last) return;
  Option *const all = reinterpret_cast<Option *>(dyn);
  unsigned long long *const best = reinterpret_cast<unsigned long long *>(all + W * W);
  select_join(p, sh, all, best, p.keys_fit ? best + W * W : nullptr, r);
}

// Vectors of 16 bytes a thread takes: what gives the fullest SM the least to do, a block being worth some 6 logits a thread beside its own
// (16 x 8 beams of 32000: 13.4 us in 256 blocks, 14.3 in 512, 14.9 in 1024; 32 x 3 beams of as many, bf16: 11.8 in 192, 10.3 in 384, 11.2 in 768); but
// no more lists than a request's last block merges quickly (64): 16 beams of one request in 512 lists took 73 us, in 64 12.
int64_t slices_of(int nv, int vocab, int per_vector, int skew) {
  const int64_t slice = (int64_t)kSelThreads * nv * per_vector;
  return (vocab + skew + slice - 1) / slice;
}
bool few_lists(int64_t slices, int beams) { return slices <= kSelMaxSlices && slices * beams <= 64; }
int vectors(int64_t rows, int beams, int vocab, int per_vector, int skew) {
  int best = 64 / per_vector;
  int64_t least = INT64_MAX;
  for (int nv = best; nv >= 1; nv /= 2) {
    const int64_t slices = slices_of(nv, vocab, per_vector, skew);
    const int64_t work = (rows * slices + 147) / 148 * (nv * per_vector + 6);
    if (!few_lists(slices, beams) || work >= least) continue;
    least = work;
    best = nv;
  }
  return best;
}
// The most slices that any number of requests is given.
int64_t most_slices(int beams, int vocab, int per_vector, int skew) {
  int64_t most = slices_of(64 / per_vector, vocab, per_vector, skew);
  for (int nv = 64 / per_vector; nv >= 1; nv /= 2) {
    const int64_t slices = slices_of(nv, vocab, per_vector, skew);
    if (few_lists(slices, beams) && slices > most) most = slices;
  }
  return most;
}
struct SelectPlan {
  int nv, slices, keys_fit;
  size_t stats, keys, per, bytes, smem;
};
void select_layout(SelectPlan *l, int64_t rows, int beams, int64_t slices) {
  l->stats = kSelCounters;
  l->keys = l->stats + ((size_t)rows * slices * 8 + 255) / 256 * 256;
  l->per = l->keys + ((size_t)rows * slices * beams * 8 + 255) / 256 * 256;
  l->bytes = l->per + (size_t)rows * 16;
}
SelectPlan select_plan(const spd_select_args &a, bool on_vectors) {
  SelectPlan l;
  const int per = 16 / (int)type_bytes(a.x_dtype);
  const int skew = on_vectors ? 0 : per - 1;
  const int64_t rows = (int64_t)a.requests * a.beams;
  l.nv = vectors(rows, a.beams, a.vocab, per, skew);
  l.slices = (int)slices_of(l.nv, a.vocab, per, skew);
  select_layout(&l, rows, a.beams, l.slices);
  const size_t slice_list = (size_t)a.beams * l.nv * per * 8;
  size_t join = (size_t)a.beams * a.beams * (sizeof(Option) + 8);
  const size_t lists = (size_t)a.beams * l.slices * a.beams * 8;
  l.keys_fit = join + lists <= kSelJoinBytes;   // (four blocks of an SM still have it)
  if (l.keys_fit) join += lists;
  l.smem = slice_list > join ? slice_list : join;
  return l;
}

template <typename T, int NV>
int select_launch(const Select &p, const SelectPlan &l) {
  static_assert(kSelMaxBeams * kSelMaxBeams * (sizeof(Option) + 8) <= kSelJoinBytes && kSelMaxBeams * 64 * 8 <= kSelJoinBytes &&
                kSelJoinBytes + sizeof(Shared) <= 48 * 1024, "lists fit a block's shared memory");
  spd_select_kernel<T, NV><<<dim3(l.slices, p.a.beams, p.a.requests), kSelThreads, l.smem, static_cast<cudaStream_t>(p.a.stream)>>>(p);
  return launched("beam selection launch");
}
template <typename T>
int select_launch(const Select &p, const SelectPlan &l) {
  switch (l.nv) {
    case 1: return select_launch<T, 1>(p, l);
    case 2: return select_launch<T, 2>(p, l);
    case 4: return select_launch<T, 4>(p, l);
    case 8: return select_launch<T, 8>(p, l);
    default: return select_launch<T, 64 / Vec<T>::n>(p, l);
  }
}

int select_check(const spd_select_args *a) {
  if (!a || a->requests < 0 || a->beams < 1 || a->vocab < 1 || !known_type(a->x_dtype)) return SPD_EINVAL;
  if (a->beams > kSelMaxBeams || a->vocab > kSelMaxVocab || a->requests > kSelMaxRequests) return SPD_ERANGE;
  return SPD_OK;
}

}  // namespace
}  // namespace spd

extern "C" int spd_beam_select_bytes(const spd_select_args *args, size_t *bytes) {
  using namespace spd;
  const int rc = select_check(args);
  if (rc || !bytes) return rc ? rc : SPD_EINVAL;
  // The most that these requests or fewer need, whether rows begin on a vector or not: the number of slices goes by both.
  const int per = 16 / (int)type_bytes(args->x_dtype);
  SelectPlan l;
  select_layout(&l, (int64_t)args->requests * args->beams, args->beams, most_slices(args->beams, args->vocab, per, per - 1));
  *bytes = l.bytes;
  return SPD_OK;
}

extern "C" int spd_beam_select(const spd_select_args *args) {
  using namespace spd;
  const int rc = select_check(args);
  if (rc) return rc;
  const spd_select_args &a = *args;
  if (a.requests == 0) return SPD_OK;
  if (!a.logits || !a.score || !a.new_token || !a.new_parent || !a.new_score || !a.workspace || !aligned(a.workspace, 256)) return SPD_EINVAL;
  if (!(a.tau > 0.f) || !(a.alpha >= 0.f) || std::isinf(a.alpha) || a.eos_id < -1 || a.eos_id >= a.vocab || !aligned(a.logits, type_bytes(a.x_dtype))) return SPD_EINVAL;
  if (!all_aligned(4, {a.score, a.length, a.new_token, a.new_parent, a.new_score, a.new_length})) return SPD_EINVAL;
  const SelectPlan l = select_plan(a, aligned(a.logits, 16) && (a.request_stride | a.beam_stride) % (16 / (int64_t)type_bytes(a.x_dtype)) == 0);
  if (a.workspace_bytes < (int64_t)l.bytes) return SPD_ENOMEM;
  Select p;
  p.a = a;
  p.slices = l.slices;
  p.keys_fit = l.keys_fit;
  p.inv_tau = 1.0 / (double)a.tau;
  // (kept finite and off zero: what is largest has weight 1 whatever tau is, what is masked none)
  const double scale = 1.4426950408889634 / (double)a.tau;
  p.scale = scale > (double)FLT_MAX ? FLT_MAX : scale < (double)FLT_TRUE_MIN ? FLT_TRUE_MIN : (float)scale;
  char *ws = static_cast<char *>(a.workspace);
  p.arrived = reinterpret_cast<unsigned *>(ws);
  p.stats = reinterpret_cast<float2 *>(ws + l.stats);
  p.keys = reinterpret_cast<unsigned long long *>(ws + l.keys);
  p.per = reinterpret_cast<double2 *>(ws + l.per);
  return a.x_dtype == SPD_F32 ? select_launch<float>(p, l) : select_launch<__nv_bfloat16>(p, l);
}
