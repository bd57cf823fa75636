// Appending keys and values to a paged cache, with the rotary embedding on the way.
//
// Every element is read once and written once: 5 flops per pair against 12 to 24 bytes, so device memory (long prefixes) or the
// launch itself (a timestep's few tokens) bounds it.  A thread takes 2 E elements of a head as two pieces of E: neighbours, or the two
// halves' partners when pairs lie rot_dim / 2 apart, so that an angle (c, s) is fetched by the one thread that needs it
// for both of its elements; and the same place of several heads, so that it is fetched once for them all (for each head anew, the
// angles are twice the bytes of bf16 data: 2048 tokens of 32 heads took 48 us, now 22.9 for 102 MB, 0.69 of the copy's rate; 64 tokens 3.3 us, 3 tokens 1.8).
#include "spd_ops.h"

namespace spd {
namespace {

struct Append {
  spd_append_args a;
  int units;       // pairs of pieces per head
  int at_once;     // heads that the threads of a block take together
  int heads;       // of q, k and v
};

// Small blocks: what an SM works on is finer, and fewer threads find no head left (2048 tokens of 32 heads: 22.6 us with 64 threads of two heads, 23.3
// with 128, 34 with 256; one, three and four heads a thread 24 to 29).
constexpr int kAppendThreads = 64, kAppendHeads = 2;

// E elements as they lie in memory (bf16 ones take half the registers that way while they are under way).
template <typename T, int E> struct Raw {
  static constexpr int kWords = E * (int)sizeof(T) / 4;
  uint32_t w[kWords];
};
template <typename T, int E, bool VEC>
__device__ __forceinline__ Raw<T, E> load_piece(const T *p) {
  Raw<T, E> r;
  if constexpr (VEC && Raw<T, E>::kWords % 4 == 0) {
#pragma unroll
    for (int i = 0; i < Raw<T, E>::kWords; i += 4) {
      const uint4 v = reinterpret_cast<const uint4 *>(p)[i / 4];
      r.w[i] = v.x, r.w[i + 1] = v.y, r.w[i + 2] = v.z, r.w[i + 3] = v.w;
    }
  } else if constexpr (VEC) {
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    r.w[0] = v.x, r.w[1] = v.y;
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < E; ++i) r.w[i] = __float_as_uint(p[i]);
  } else {
    const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
    for (int i = 0; i < E; i += 2) r.w[i / 2] = h[i] | ((uint32_t)h[i + 1] << 16);
  }
  return r;
}
template <typename T, int E>
__device__ __forceinline__ void widen(const Raw<T, E> &r, float *v) {
#pragma unroll
  for (int i = 0; i < E; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(r.w[i]);
    else v[i] = i & 1 ? high_bf16(r.w[i / 2]) : low_bf16(r.w[i / 2]);
  }
}
template <typename T, int E, bool VEC>
__device__ __forceinline__ void store_piece(T *p, const float *v) {
  if constexpr (VEC && sizeof(T) == 2 && E == 8) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  } else if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < E; i += 4) store4(p + i, make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]));
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) p[i] = from_float<T>(v[i]);
  }
}

template <typename X, typename C, int E, bool VEC, int HEADS>
__global__ void __launch_bounds__(kAppendThreads) spd_append_kernel(const __grid_constant__ Append p) {
  const spd_append_args &a = p.a;
  const int sub = threadIdx.x / p.units, u = threadIdx.x - sub * p.units;
  if (sub >= p.at_once) return;
  const int half = a.rot_dim / 2;
  const bool turned = u * 2 * E < a.rot_dim, apart = turned && a.pairs != 0;
  const int r0 = apart ? E * u : 2 * E * u, r1 = apart ? half + E * u : 2 * E * u + E;  // where q and k have their pieces
  for (int64_t t = blockIdx.y; t < a.n; t += gridDim.y) {
    const int pos = a.rot_dim ? a.pos[t] : 0;
    const int index = a.n_kv_heads ? (a.index ? a.index : a.pos)[t] : 0;
    const int seq = a.seq ? a.seq[t] : (int)t;
    Raw<X, E> x0[HEADS], x1[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      const int h = (blockIdx.x * HEADS + i) * p.at_once + sub;
      if (h >= p.heads) continue;
      const bool is_q = h < a.n_heads, is_k = !is_q && h < a.n_heads + a.n_kv_heads;
      const X *row = is_q ? static_cast<const X *>(a.q) + t * a.q_row + h * a.q_head
                     : is_k ? static_cast<const X *>(a.k) + t * a.k_row + (h - a.n_heads) * a.k_head
                            : static_cast<const X *>(a.v) + t * a.v_row + (h - a.n_heads - a.n_kv_heads) * a.v_head;
      x0[i] = load_piece<X, E, VEC>(row + (is_q || is_k ? r0 : 2 * E * u));
      x1[i] = load_piece<X, E, VEC>(row + (is_q || is_k ? r1 : 2 * E * u + E));
    }
    const bool angle = !a.rot_dim || (pos >= 0 && pos < a.rope_rows);
    Raw<float, 2 * E> cs;   // (c, s) of the thread's pairs
    if (turned && angle) cs = load_piece<float, 2 * E, true>(a.rope + ((int64_t)pos * half + E * u) * 2);
    int64_t slot = index;
    if (a.table && index >= 0) {
      const int col = index / a.page;
      slot = seq >= 0 && seq < a.table_rows && col < a.table_cols ? (int64_t)a.table[seq * a.table_row + col] * a.page + (index - col * a.page) : -1;
    }
    const bool stored = index >= 0 && slot >= 0 && slot < a.slots;
    // (padding may hold any position, and no slot is wanted for it)
    if (a.status && threadIdx.x == 0 && ((a.n_kv_heads && index >= 0 && (!stored || !angle)) || (!a.n_kv_heads && !angle))) *a.status = SPD_ERANGE;
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      const int h = (blockIdx.x * HEADS + i) * p.at_once + sub;
      if (h >= p.heads) continue;
      const bool is_q = h < a.n_heads, is_k = !is_q && h < a.n_heads + a.n_kv_heads;
      if ((is_q || is_k) && !angle) continue;
      if (!is_q && !stored) continue;
      float y0[E], y1[E];
      widen<X, E>(x0[i], y0);
      widen<X, E>(x1[i], y1);
      if ((is_q || is_k) && turned) {
        const auto angle_at = [&](int j) { return make_float2(__uint_as_float(cs.w[2 * j]), __uint_as_float(cs.w[2 * j + 1])); };
        if (apart) {
#pragma unroll
          for (int j = 0; j < E; ++j) {
            const float2 r = angle_at(j);
            const float v = y0[j], w = y1[j];
            y0[j] = v * r.x - w * r.y, y1[j] = v * r.y + w * r.x;
          }
        } else {
#pragma unroll
          for (int j = 0; j < E; j += 2) {
            const float2 r = angle_at(j / 2), q = angle_at(E / 2 + j / 2);
            const float v = y0[j], w = y0[j + 1], v1 = y1[j], w1 = y1[j + 1];
            y0[j] = v * r.x - w * r.y, y0[j + 1] = v * r.y + w * r.x;
            y1[j] = v1 * q.x - w1 * q.y, y1[j + 1] = v1 * q.y + w1 * q.x;
          }
        }
      }
      if (is_q) {
        X *dst = static_cast<X *>(a.q_out) + t * a.qo_row + h * a.qo_head;
        store_piece<X, E, VEC>(dst + r0, y0);
        store_piece<X, E, VEC>(dst + r1, y1);
      } else {
        C *dst = is_k ? static_cast<C *>(a.k_cache) + slot * a.kc_slot + (h - a.n_heads) * a.kc_head
                      : static_cast<C *>(a.v_cache) + slot * a.vc_slot + (h - a.n_heads - a.n_kv_heads) * a.vc_head;
        store_piece<C, E, VEC>(dst + (is_k ? r0 : 2 * E * u), y0);
        store_piece<C, E, VEC>(dst + (is_k ? r1 : 2 * E * u + E), y1);
      }
    }
  }
}

template <typename X, typename C, int E, bool VEC>
void append_launch(Append &p, cudaStream_t s) {
  p.units = p.a.head_dim / (2 * E);
  p.at_once = kAppendThreads / p.units < p.heads ? kAppendThreads / p.units : p.heads;
  const int passes = (p.heads + p.at_once - 1) / p.at_once;
  const int rows = p.a.n < 65535 ? p.a.n : 65535;
  // Two heads per thread once there are blocks enough to fill the SMs without (148 x 8): few tokens are spread over more threads.
  if (VEC && passes > 1 && (int64_t)passes * p.a.n > 148 * 8) {
    spd_append_kernel<X, C, E, VEC, kAppendHeads><<<dim3((passes + kAppendHeads - 1) / kAppendHeads, rows), kAppendThreads, 0, s>>>(p);
  } else {
    spd_append_kernel<X, C, E, VEC, 1><<<dim3(passes, rows), kAppendThreads, 0, s>>>(p);
  }
}
// Pieces of 16 bytes where everything lies on them, of four elements, or one by one.
template <typename X, typename C>
void append_launch(Append &p, bool eights, bool fours, cudaStream_t s) {
  if (sizeof(X) == 2 && eights) append_launch<X, C, sizeof(X) == 2 ? 8 : 4, true>(p, s);
  else if (fours) append_launch<X, C, 4, true>(p, s);
  else append_launch<X, C, 4, false>(p, s);
}

bool in_groups(const spd_append_args &a, int64_t n) {
  const int64_t all = a.q_row | a.q_head | a.qo_row | a.qo_head | a.k_row | a.k_head | a.v_row | a.v_head | a.kc_slot | a.kc_head | a.vc_slot | a.vc_head;
  const size_t x = n * type_bytes(a.x_dtype), c = n * type_bytes(a.kv_dtype) < 16 ? n * type_bytes(a.kv_dtype) : 16;
  return all % n == 0 && aligned(a.q, x) && aligned(a.q_out, x) && aligned(a.k, x) && aligned(a.v, x) && aligned(a.k_cache, c) && aligned(a.v_cache, c);
}

}  // namespace
}  // namespace spd

extern "C" int spd_cache_append(const spd_append_args *args) {
  using namespace spd;
  if (!args) return SPD_EINVAL;
  const spd_append_args &a = *args;
  if (a.n == 0) return SPD_OK;
  const bool kv = a.k || a.v;
  if (a.n < 0 || a.head_dim < 8 || a.head_dim % 8 || a.head_dim > 256 || a.rot_dim < 0 || a.rot_dim % 8 || a.rot_dim > a.head_dim) return SPD_EINVAL;
  if (a.pairs < 0 || a.pairs > 1 || !known_type(a.x_dtype) || !known_type(a.kv_dtype)) return SPD_EINVAL;
  if ((!kv && !a.q) || (kv && (!a.k || !a.v || !a.k_cache || !a.v_cache || a.n_kv_heads < 1 || a.slots < 1 || (!a.index && !a.pos)))) return SPD_EINVAL;
  if (a.q && (!a.q_out || a.n_heads < 1)) return SPD_EINVAL;
  if (a.rot_dim && (!a.rope || !a.pos || a.rope_rows < 1 || !aligned(a.rope, 16))) return SPD_EINVAL;
  if (kv && a.table && (a.page < 1 || a.table_rows < 1 || a.table_cols < 1)) return SPD_EINVAL;
  if (!all_aligned(type_bytes(a.x_dtype), {a.q, a.k, a.v, a.q_out}) || !all_aligned(type_bytes(a.kv_dtype), {a.k_cache, a.v_cache})) return SPD_EINVAL;
  if (!all_aligned(4, {a.pos, a.index, a.seq, a.table, a.status})) return SPD_EINVAL;
  if (a.n_heads > 1 << 16 || a.n_kv_heads > 1 << 16) return SPD_ERANGE;
  Append p;
  p.a = a;
  if (!a.q) p.a.n_heads = 0;
  if (!kv) p.a.n_kv_heads = 0;
  p.heads = p.a.n_heads + 2 * p.a.n_kv_heads;
  const bool eights = a.head_dim % 16 == 0 && a.rot_dim % 16 == 0 && in_groups(a, 8), fours = in_groups(a, 4);
  const cudaStream_t s = static_cast<cudaStream_t>(a.stream);
  if (a.x_dtype == SPD_F32) {
    if (a.kv_dtype == SPD_F32) append_launch<float, float>(p, eights, fours, s);
    else append_launch<float, __nv_bfloat16>(p, eights, fours, s);
  } else {
    if (a.kv_dtype == SPD_F32) append_launch<__nv_bfloat16, float>(p, eights, fours, s);
    else append_launch<__nv_bfloat16, __nv_bfloat16>(p, eights, fours, s);
  }
  return launched("cache append launch");
}
