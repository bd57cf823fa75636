// The beams' states follow their parents, in place.
//
// A thread owns a column (one vector of up to 16 bytes at one place of the rows) of all beams of a request: it loads what
// every beam that changes will hold, then stores.  Nobody else touches the column, so the permutation, with
// parents that several beams share, needs neither a second copy of the state nor a barrier: each parent that is
// needed is read from memory once (a second child's load finds it in L1), each row that changes is written once, and that is
// the floor.  Device memory bounds it: 235 MB of dense caches (8 layers, 4 x 5 beams, K and V) 46 us, 0.79 of the copy's rate; slot tables and histories of
// 128 beams 2.4 us.
#include "spd_ops.h"

namespace spd {
namespace {

constexpr int kReorderThreads = 128;

struct ReorderState {
  char *base;
  int64_t outer_stride, request_stride, beam_stride;
  int vec_log2;         // log2 of the bytes of a vector
  int64_t vecs;         // vectors of a row
  int64_t col_blocks;   // blocks along a row
  int64_t first_block;  // of the launch
};
struct Reorder {
  ReorderState st[SPD_MAX_STATES];
  const int32_t *parent;
  int32_t *status;
  int n_states, requests, beams;
};

template <typename V, int BEAMS>
__device__ __forceinline__ void reorder_column(char *at, int64_t stride, const int *parent, int beams) {
  V v[BEAMS];
#pragma unroll
  for (int j = 0; j < BEAMS; ++j)
    if (j < beams && parent[j] != j) v[j] = *reinterpret_cast<const V *>(at + parent[j] * stride);
#pragma unroll
  for (int j = 0; j < BEAMS; ++j)
    if (j < beams && parent[j] != j) *reinterpret_cast<V *>(at + j * stride) = v[j];
}

template <int BEAMS>
__global__ void __launch_bounds__(kReorderThreads) spd_reorder_kernel(const __grid_constant__ Reorder p) {
  __shared__ int parent[BEAMS];
  int k = 0;
  while (k + 1 < p.n_states && blockIdx.x >= p.st[k + 1].first_block) ++k;
  const ReorderState &st = p.st[k];
  const int64_t block = blockIdx.x - st.first_block;
  const int64_t row = block / st.col_blocks;
  const int64_t col = (block - row * st.col_blocks) * kReorderThreads + threadIdx.x;
  const int64_t o = row / p.requests;
  const int r = (int)(row - o * p.requests);
  if (threadIdx.x < BEAMS && threadIdx.x < p.beams) {
    int j = p.parent[(int64_t)r * p.beams + threadIdx.x];
    if (j < 0 || j >= p.beams) {  // no such beam: the row stays
      j = threadIdx.x;
      if (p.status) *p.status = SPD_ERANGE;
    }
    parent[threadIdx.x] = j;
  }
  __syncthreads();
  if (col >= st.vecs) return;
  char *at = st.base + o * st.outer_stride + r * st.request_stride + (col << st.vec_log2);
  switch (st.vec_log2) {
    case 4: reorder_column<uint4, BEAMS>(at, st.beam_stride, parent, p.beams); break;
    case 2: reorder_column<uint32_t, BEAMS>(at, st.beam_stride, parent, p.beams); break;
    default: reorder_column<uint8_t, BEAMS>(at, st.beam_stride, parent, p.beams); break;
  }
}

}  // namespace
}  // namespace spd

extern "C" int spd_beam_reorder(const spd_reorder_args *args) {
  using namespace spd;
  if (!args) return SPD_EINVAL;
  const spd_reorder_args &a = *args;
  if (a.n_states < 0 || a.n_states > SPD_MAX_STATES || a.requests < 0 || a.beams < 1) return SPD_EINVAL;
  if (a.beams > 32) return SPD_ERANGE;
  if (a.requests == 0) return SPD_OK;
  if (!a.parent || !all_aligned(4, {a.parent, a.status})) return SPD_EINVAL;
  Reorder p;
  p.parent = a.parent;
  p.status = a.status;
  p.n_states = 0;
  p.requests = a.requests;
  p.beams = a.beams;
  int64_t blocks = 0;
  for (int i = 0; i < a.n_states; ++i) {
    if (a.outer[i] == 0 || a.row_bytes[i] == 0) continue;
    if (!a.state[i] || a.outer[i] < 0 || a.row_bytes[i] < 0) return SPD_EINVAL;
    const auto apart = [&](int64_t stride) { return (stride < 0 ? -stride : stride) >= a.row_bytes[i]; };
    if (a.beams > 1 && !apart(a.beam_stride[i])) return SPD_EINVAL;
    ReorderState &s = p.st[p.n_states++];
    s.base = static_cast<char *>(a.state[i]);
    s.outer_stride = a.outer_stride[i];
    s.request_stride = a.request_stride[i];
    s.beam_stride = a.beam_stride[i];
    const int64_t all = (int64_t)reinterpret_cast<uintptr_t>(s.base) | s.outer_stride | s.request_stride | s.beam_stride | a.row_bytes[i];
    s.vec_log2 = all % 16 == 0 ? 4 : all % 4 == 0 ? 2 : 0;
    s.vecs = a.row_bytes[i] >> s.vec_log2;
    s.col_blocks = (s.vecs + kReorderThreads - 1) / kReorderThreads;
    s.first_block = blocks;
    const __int128 more = (__int128)s.col_blocks * a.outer[i] * a.requests;
    if (more + blocks > 0x7fffffff) return SPD_ERANGE;
    // Blocks that write the same rows would read what one another wrote.
    if (a.beams > 1 && ((a.requests > 1 && !apart(a.request_stride[i])) || (a.outer[i] > 1 && !apart(a.outer_stride[i])))) return SPD_EINVAL;
    for (int j = 0; a.beams > 1 && j + 1 < p.n_states; ++j)
      if (p.st[j].base == s.base) return SPD_EINVAL;
    blocks += (int64_t)more;
  }
  if (blocks == 0 || a.beams == 1) return SPD_OK;
  const cudaStream_t s = static_cast<cudaStream_t>(a.stream);
  const unsigned grid = (unsigned)blocks;
  if (a.beams <= 4) spd_reorder_kernel<4><<<grid, kReorderThreads, 0, s>>>(p);
  else if (a.beams <= 8) spd_reorder_kernel<8><<<grid, kReorderThreads, 0, s>>>(p);
  else if (a.beams <= 16) spd_reorder_kernel<16><<<grid, kReorderThreads, 0, s>>>(p);
  else spd_reorder_kernel<32><<<grid, kReorderThreads, 0, s>>>(p);
  return launched("beam reorder launch");
}
