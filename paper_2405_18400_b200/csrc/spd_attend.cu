// Host side of the attention over shared prefixes (spd_attend.cuh): argument checks, workspace, which kernel.
#include <cmath>

#include "spd_attend.cuh"

namespace spd {
namespace {

int mode_of(const spd_attention_args &a) {
  // Tiles of four or eight float32 rows where the mean group (without prefixes: sequence) has no more (larger groups among them have several, and
  // read their prefix as often).  Against tiles of 16, bf16 cache: 3 rows behind 2048 positions 14.6 and 17.3 us, 8 x 3 rows 51 and 66, 4 x 8 rows 37.5 and 42;
  // float32 cache: 3 rows 22 and 29, 2 x 7 rows behind 8000 positions of 8 key heads 35 and 44.  Uneven groups gain as well: one of 64 rows
  // beside 63 of one, 8 key heads, 2048 positions each, 93 and 113 us, float32 cache 200 and 282.  (256 dimensions of eight rows leave no registers.)
  const long long rows = (long long)a.n * (a.n_heads / a.n_kv_heads), groups = a.g ? a.g : a.b;
  if (a.x_dtype == SPD_BF16 && a.kv_dtype == SPD_BF16) return kAttBf16;
  if (a.x_dtype == SPD_F32 && a.kv_dtype == SPD_BF16) return rows <= 4 * groups ? kAttFew : rows <= 8 * groups && a.head_dim <= 128 ? kAttEight : kAttTerms;
  if (a.x_dtype == SPD_F32 && a.kv_dtype == SPD_F32) return rows <= 8 * groups ? kAttFewFloat : kAttFloat;
  return -1;
}
// Whether a call of these types and dimensions may go to a kernel, by its counts.
bool serves(int mode, const spd_attention_args &a) {
  if (a.x_dtype == SPD_BF16) return mode == kAttBf16;
  if (a.kv_dtype == SPD_F32) return mode == kAttFloat || mode == kAttFewFloat;
  return mode == kAttTerms || mode == kAttFew || (mode == kAttEight && a.head_dim <= 128);
}
template <int MODE> void tuning(int d, int *warps, int *per_sm) {
  if constexpr (MODE != kAttEight) {
    if (d > 128) *warps = AttendTune<MODE, 256>::nw, *per_sm = AttendTune<MODE, 256>::per_sm;
  }
  if (d <= 128) *warps = AttendTune<MODE, 128>::nw, *per_sm = AttendTune<MODE, 128>::per_sm;
  if (d <= 64) *warps = AttendTune<MODE, 64>::nw, *per_sm = AttendTune<MODE, 64>::per_sm;
}

// Microseconds of a step among others, 128 dimensions: of a prefix tile of 16, 32 and 64 (of few) rows by a block, of an own tile by a warp; by mode.
constexpr float kStepCost[6][3] = {{1.55f, 2.2f, 3.5f}, {2.1f, 3.5f, 6.2f}, {2.7f, 3.8f, 6.4f}, {2.4f}, {2.5f}, {2.6f}};
constexpr float kOwnStepCost[6] = {1.8f, 2.2f, 2.7f, 3.2f, 3.4f, 3.4f};

struct AttendPlan {
  int rt, many_parts, blocks, warps, rows_o, device;
  long long prefix_parts, own_parts;
  size_t prefix_ml, own_o, own_ml, bytes;  // prefix_o lies at 0
};
Divisor divisor(int size) {
  Divisor p = {size, -1};
  for (int i = 0; i < 31; ++i)
    if (size == 1 << i) p.shift = i;
  return p;
}
size_t up(size_t v) { return (v + 255) / 256 * 256; }

int attend_check(const spd_attention_args *a) {
  if (!a || a->n < 0 || a->b < 0 || a->g < 0 || a->n_kv_heads < 1 || a->n_heads < 1 || a->n_heads % a->n_kv_heads || mode_of(*a) < 0) return SPD_EINVAL;
  if (a->head_dim < 1 || a->head_dim > 256 || a->head_dim * type_bytes(a->kv_dtype) % 16) return SPD_EINVAL;
  if (a->b > 4096 || a->g > a->b || a->n > 1 << 24 || a->n_heads > 4 * 65535 || (int64_t)a->n * a->n_heads / a->n_kv_heads > 1 << 30) return SPD_ERANGE;
  return SPD_OK;
}

int attend_plan(const spd_attention_args &a, int mode, AttendPlan *l) {
  int warps = 0, per_sm = 0, sms = 0;
  if (mode == kAttBf16) tuning<kAttBf16>(a.head_dim, &warps, &per_sm);
  else if (mode == kAttTerms) tuning<kAttTerms>(a.head_dim, &warps, &per_sm);
  else if (mode == kAttFew) tuning<kAttFew>(a.head_dim, &warps, &per_sm);
  else if (mode == kAttEight) tuning<kAttEight>(a.head_dim, &warps, &per_sm);
  else if (mode == kAttFewFloat) tuning<kAttFewFloat>(a.head_dim, &warps, &per_sm);
  else tuning<kAttFloat>(a.head_dim, &warps, &per_sm);
  cudaError_t e = cudaGetDevice(&l->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, l->device);
  if (e != cudaSuccess) return spd_internal_cuda_fail(e, "attention: device");
  l->blocks = sms * per_sm;
  l->warps = warps;
  const long long ratio = a.n_heads / a.n_kv_heads, rows = a.n * ratio;
  // The height of a tile (16, 32 or 64 rows of the mean group): what needs the least time if the blocks take equal runs of the tiles' steps, each
  // step at its measured cost (us of a block among others, 128 dimensions).  Higher tiles read a prefix less often and use operands more often,
  // lower ones make more runs: 80 float32 rows behind 490 positions of 2 key heads 26 us at 64 rows, 14 at 16; 64 rows behind each of 4 x 4096
  // positions of 32 heads (bf16) 130 us at 64, 196 at 16.  The lengths are the device's, so the tables' room stands for them.
  const long long mean = a.g ? (rows + a.g - 1) / a.g : 0, step = (a.kv_dtype == SPD_F32 ? kPositions<kAttFloat> : kPositions<kAttBf16>) * warps;
  const double steps = std::ceil((double)a.prefix_cols * a.prefix_page / step);
  l->rt = 1;
  double least = 0;
  const int rows_of = mode == kAttFew ? kRows<kAttFew> : mode == kAttFewFloat || mode == kAttEight ? kRows<kAttEight> : 16;
  for (int i = 0; i < (rows_of < 16 ? 1 : 3); ++i) {
    const long long high = rows_of << i, tiles = (mean + high - 1) / high * a.g * a.n_kv_heads;
    const double time = std::ceil(tiles * steps / l->blocks) * kStepCost[mode][i];
    if (i == 0 || (time < least && mean > high / 2)) {
      least = time, l->rt = 1 << i;
      const double parts = tiles > 0 && (double)l->blocks / tiles < steps ? (double)l->blocks / tiles : steps;   // of a row's prefix
      l->many_parts = parts >= 16 && a.n_heads <= 65535 ? 2 : parts >= 6;
    }
  }
  l->rows_o = a.q_start || ratio > rows_of ? rows_of : (int)ratio;
  l->prefix_parts = a.g ? l->blocks + a.n_kv_heads * (rows / (rows_of * l->rt) + a.g) : 0;
  l->own_parts = (long long)l->blocks * warps + a.n_kv_heads * (rows / rows_of + a.b);
  // (room for the highest tiles that the kernel has, so that the need does not hang on the tables)
  const size_t highest = rows_of < 16 ? rows_of : 64;
  const size_t part_rows = a.g ? highest * ((size_t)l->blocks + a.n_kv_heads * (size_t)a.g) + (size_t)a.n_kv_heads * rows : 0;
  l->prefix_ml = up(part_rows * a.head_dim * 4);
  l->own_o = l->prefix_ml + up(part_rows * 8);
  l->own_ml = l->own_o + up((size_t)l->own_parts * l->rows_o * a.head_dim * 4);
  l->bytes = l->own_ml + up((size_t)l->own_parts * l->rows_o * 8);
  return SPD_OK;
}

}  // namespace
}  // namespace spd

extern "C" int spd_shared_attention_bytes(const spd_attention_args *args, size_t *bytes) {
  using namespace spd;
  int rc = attend_check(args);
  if (rc || !bytes) return rc ? rc : SPD_EINVAL;
  // Each kernel's need grows with the counts, but fewer rows or prefixes may go to another kernel: the most that one of these types needs.
  *bytes = 0;
  for (const int mode : {kAttBf16, kAttTerms, kAttFloat, kAttFew, kAttFewFloat, kAttEight}) {
    AttendPlan l;
    if (!serves(mode, *args)) continue;
    if ((rc = attend_plan(*args, mode, &l))) return rc;
    if (l.bytes > *bytes) *bytes = l.bytes;
  }
  return SPD_OK;
}

extern "C" int spd_shared_attention(const spd_attention_args *args) {
  using namespace spd;
  int rc = attend_check(args);
  if (rc) return rc;
  const spd_attention_args &a = *args;
  if (a.n == 0) return SPD_OK;
  const size_t kv = type_bytes(a.kv_dtype), x = type_bytes(a.x_dtype);
  if (!a.q || !a.k_cache || !a.v_cache || !a.out || !a.own_len || !a.workspace || !aligned(a.workspace, 256) || a.slots < 1) return SPD_EINVAL;
  if (!aligned(a.q, x) || !aligned(a.out, x) || !aligned(a.k_cache, 16) || !aligned(a.v_cache, 16)) return SPD_EINVAL;
  if (!all_aligned(4, {a.lse, a.q_start, a.group_start, a.prefix_table, a.prefix_len, a.own_table, a.own_len, a.status})) return SPD_EINVAL;
  // (offsets into the caches are unsigned)
  if ((a.kc_slot | a.kc_head | a.vc_slot | a.vc_head) % (int64_t)(16 / kv) || (a.kc_slot | a.kc_head | a.vc_slot | a.vc_head) < 0) return SPD_EINVAL;
  if (a.own_page < 1 || a.own_cols < 0 || (a.own_cols && !a.own_table) || !(a.scale > 0.f) || std::isinf(a.scale)) return SPD_EINVAL;
  if (a.g && (a.prefix_page < 1 || a.prefix_cols < 0 || (a.prefix_cols && !a.prefix_table) || !a.prefix_len || (a.g > 1 && !a.group_start))) return SPD_EINVAL;
  if (a.b < 1 || (!a.q_start && a.n != a.b)) return SPD_EINVAL;
  if (a.slots > 0x7fffffff) return SPD_ERANGE;
  AttendPlan l;
  if ((rc = attend_plan(a, mode_of(a), &l))) return rc;
  if (a.workspace_bytes < (int64_t)l.bytes) return SPD_ENOMEM;
  // steps in 31 bits
  const int step = a.kv_dtype == SPD_F32 ? kPositions<kAttFloat> : kPositions<kAttBf16>;
  const double room_p = (double)a.prefix_cols * a.prefix_page, room_o = (double)a.own_cols * a.own_page, most = 2147483647.0;
  const double steps_p = (a.g ? l.prefix_parts : 0) * ((room_p < most ? room_p : most) / (step * l.warps) + 1), steps_o = l.own_parts * ((room_o < most ? room_o : most) / step + 1);
  if (steps_p > most || steps_o > most) return SPD_ERANGE;
  Attend p;
  p.a = a;
  p.ratio = a.n_heads / a.n_kv_heads;
  p.rows_o = l.rows_o;
  const int group = a.kv_dtype == SPD_F32 ? 4 : 2;
  p.q_whole = aligned(a.q, group * x) && (a.q_row | a.q_head) % group == 0 && (a.head_dim == 64 || a.head_dim == 128 || a.head_dim == 256);
  p.out_fours = aligned(a.out, 4 * x) && (a.o_row | a.o_head) % 4 == 0;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  const float own_step = kOwnStepCost[mode_of(a)];
  p.weights = {kStepCost[mode_of(a)][l.rt == 1 ? 0 : l.rt == 2 ? 1 : 2] / own_step, 3.f, 1.f, 2.f};
  p.prefix_pages = divisor(a.prefix_page);
  p.own_pages = divisor(a.own_page);
  p.by_ratio = divisor(p.ratio);
  char *ws = static_cast<char *>(a.workspace);
  p.prefix_o = reinterpret_cast<float *>(ws);
  p.prefix_ml = reinterpret_cast<float2 *>(ws + l.prefix_ml);
  p.own_o = reinterpret_cast<float *>(ws + l.own_o);
  p.own_ml = reinterpret_cast<float2 *>(ws + l.own_ml);
  p.prefix_parts = l.prefix_parts;
  p.own_parts = l.own_parts;
  p.blocks = l.blocks;
  p.many_parts = l.many_parts;
  p.prefix_room = (int)(room_p < most ? room_p : most);
  p.own_room = (int)(room_o < most ? room_o : most);
  const cudaStream_t s = static_cast<cudaStream_t>(a.stream);
  const int mode = mode_of(a);
  decltype(&attend_bf16) const launch[] = {attend_bf16, attend_terms, attend_float, attend_few, attend_few_float, attend_eight};   // by mode
  const cudaError_t e = launch[mode](p, l.rt, l.device, s);
  return e == cudaSuccess ? SPD_OK : spd_internal_cuda_fail(e, "attention launch");
}
