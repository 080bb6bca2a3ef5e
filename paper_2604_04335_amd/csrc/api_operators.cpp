// C ABI of the operators around the attention and of attention with masks: argument checks, split of the keys, launch.
#include "../../include/dit_attn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>
#include <vector>

#include "context.h"
#include "masked_attn.h"
#include "qk_norm_rope.h"

namespace {

using dit::fail;
using dit::fail_hip;

bool misaligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// No exception leaves a C entry.
template <class F>
int guarded(dit_attn_ctx* ctx, F&& body) {
  if (!ctx) return DIT_ATTN_ERR_NULL;
  try {
    ctx->error.clear();
    return body();
  } catch (...) {
    return DIT_ATTN_ERR_HIP;  // out of host memory
  }
}

// ---------------------------------------------------------------- rotation table

// Radians per position of pair j of an axis.
double rope_frequency(const dit_attn_rope& r, int axis, int j) {
  const double d = r.axis_dim[axis], theta = r.theta[axis], s = r.factor[axis];
  double f = std::pow(theta, -2.0 * j / d);
  if (r.scaling == DIT_ATTN_ROPE_LINEAR) return f / s;
  if (r.scaling == DIT_ATTN_ROPE_BASE && d > 2) return std::pow(theta * std::pow(s, d / (d - 2.0)), -2.0 * j / d);
  if (r.scaling == DIT_ATTN_ROPE_BANDS) {
    const double turns = r.original_length[axis] * f / (2.0 * 3.14159265358979323846);
    const double g = std::min(1.0, std::max(0.0, (turns - r.low) / (r.high - r.low)));
    return f * (g + (1.0 - g) / s);
  }
  return f;
}

int rope_table(dit_attn_ctx* ctx, const int32_t* positions, int64_t n_rows, const dit_attn_rope* r, float* table, void* stream) {
  if (!r) return fail(ctx, DIT_ATTN_ERR_NULL, "rope is NULL");
  if (r->n_axes < 1 || r->n_axes > 4) return fail(ctx, DIT_ATTN_ERR_ROPE, "n_axes must be in 1..4");
  if (r->scaling < DIT_ATTN_ROPE_PLAIN || r->scaling > DIT_ATTN_ROPE_BANDS) return fail(ctx, DIT_ATTN_ERR_ROPE, "no such scaling");
  if (!std::isfinite(r->magnitude) || std::fabs(r->magnitude) > 1e30) return fail(ctx, DIT_ATTN_ERR_ROPE, "magnitude must be finite");
  int total = 0;
  for (int a = 0; a < r->n_axes; ++a) {
    if (r->axis_dim[a] < 2 || r->axis_dim[a] % 2 != 0 || r->axis_dim[a] > 2 * dit::kMaxRopePairs)
      return fail(ctx, DIT_ATTN_ERR_ROPE, "axis_dim must be even and in 2..128");
    total += r->axis_dim[a];
    if (!(r->theta[a] >= 1.0) || !std::isfinite(r->theta[a])) return fail(ctx, DIT_ATTN_ERR_ROPE, "theta must be finite and at least 1");
    if (r->scaling != DIT_ATTN_ROPE_PLAIN && (!(r->factor[a] >= 1.0) || !std::isfinite(r->factor[a])))
      return fail(ctx, DIT_ATTN_ERR_ROPE, "factor must be finite and at least 1");
    if (r->scaling == DIT_ATTN_ROPE_BANDS && (!(r->original_length[a] > 0.0) || !std::isfinite(r->original_length[a])))
      return fail(ctx, DIT_ATTN_ERR_ROPE, "original_length must be positive");
  }
  if (total > 2 * dit::kMaxRopePairs) return fail(ctx, DIT_ATTN_ERR_ROPE, "the axes have more than 128 elements together");
  if (r->scaling == DIT_ATTN_ROPE_BANDS && !(r->low < r->high && std::isfinite(r->low) && std::isfinite(r->high)))
    return fail(ctx, DIT_ATTN_ERR_ROPE, "low must be under high");
  if (n_rows < 0) return fail(ctx, DIT_ATTN_ERR_CU_SEQLENS, "n_rows must be >= 0");
  if (n_rows == 0) return DIT_ATTN_OK;
  if (!positions || !table) return fail(ctx, DIT_ATTN_ERR_NULL, "positions and table must be non-NULL");
  if (misaligned(positions, 4) || misaligned(table, 16))
    return fail(ctx, DIT_ATTN_ERR_ALIGN, "positions must be 4-byte, table 16-byte aligned");

  dit::RopeTableParams p{};
  p.positions = positions;
  p.table = table;
  p.n_rows = n_rows;
  p.n_axes = r->n_axes;
  p.n_pairs = total / 2;
  p.magnitude = static_cast<float>(r->magnitude);
  if (n_rows > (int64_t{1} << 34) || dit::rope_table_blocks(p) > dit::kMaxRowBlocks) return fail(ctx, DIT_ATTN_ERR_LIMIT, "too many rows");
  int pair = 0;
  for (int a = 0; a < r->n_axes; ++a)
    for (int j = 0; j < r->axis_dim[a] / 2; ++j, ++pair) {
      const long double quarters = static_cast<long double>(rope_frequency(*r, a, j)) / 1.5707963267948966192313216916398L;
      p.quarters_hi[pair] = static_cast<double>(quarters);
      p.quarters_lo[pair] = static_cast<double>(quarters - static_cast<long double>(p.quarters_hi[pair]));
      p.axis[pair] = static_cast<uint8_t>(a);
    }
  dit::DeviceGuard guard;
  hipError_t e = guard.enter(ctx->device);
  if (e != hipSuccess) return fail_hip(ctx, e, "hipSetDevice");
  e = dit::rope_table_launch(p, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DIT_ATTN_OK : fail_hip(ctx, e, "rotation table kernel launch");
}

// ---------------------------------------------------------------- norm and rotation

int check_norm_heads(dit_attn_ctx* ctx, const dit_attn_norm_heads& s, const char* name, int64_t n_rows, int32_t head_dim, int32_t norm,
                     dit::NormHeadsParams& out) {
  const std::string who = std::string(name) + ": ";
  if (s.n_heads < 1 || s.n_heads > 65535) return fail(ctx, DIT_ATTN_ERR_N_HEADS, who + "n_heads must be in 1..65535");
  const int64_t row = static_cast<int64_t>(s.n_heads) * head_dim;
  const int64_t in_stride = s.row_stride ? s.row_stride : row, out_stride = s.out_row_stride ? s.out_row_stride : row;
  for (const int64_t st : {in_stride, out_stride})
    if (st < row || st % 8 != 0 || st > (int64_t{1} << 40))
      return fail(ctx, DIT_ATTN_ERR_STRIDE, who + "row strides must be multiples of 8 elements and hold n_heads * head_dim");
  if (norm == DIT_ATTN_NORM_NONE && (s.weight || s.bias)) return fail(ctx, DIT_ATTN_ERR_NORM, who + "weight and bias belong to a norm");
  if (n_rows == 0) return DIT_ATTN_OK;
  if (!s.x || !s.out) return fail(ctx, DIT_ATTN_ERR_NULL, who + "x and out must be non-NULL");
  if (misaligned(s.x, 16) || misaligned(s.out, 16) || misaligned(s.weight, 16) || misaligned(s.bias, 16))
    return fail(ctx, DIT_ATTN_ERR_ALIGN, who + "x, out, weight and bias must be 16-byte aligned");
  if (s.x == s.out && in_stride != out_stride) return fail(ctx, DIT_ATTN_ERR_STRIDE, who + "in place, both row strides must be equal");
  out.x = static_cast<const char*>(s.x);
  out.out = static_cast<char*>(s.out);
  out.row_stride_b = 2 * in_stride;
  out.out_stride_b = 2 * out_stride;
  out.weight = s.weight;
  out.bias = s.bias;
  out.n_heads = s.n_heads;
  return DIT_ATTN_OK;
}

int qk_norm_rope(dit_attn_ctx* ctx, const dit_attn_norm_heads* q, const dit_attn_norm_heads* k, int64_t n_rows, int32_t head_dim,
                 int32_t norm, float eps, const float* table, int32_t rot_dim, int32_t layout, void* stream) {
  if (!q && !k) return fail(ctx, DIT_ATTN_ERR_NULL, "q and k are both NULL");
  if (head_dim != 64 && head_dim != 128) return fail(ctx, DIT_ATTN_ERR_HEAD_DIM, "head_dim must be 64 or 128");
  if (norm < DIT_ATTN_NORM_NONE || norm > DIT_ATTN_NORM_LAYER) return fail(ctx, DIT_ATTN_ERR_NORM, "no such norm");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(ctx, DIT_ATTN_ERR_NORM, "eps must be finite and not negative");
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 8 != 0)
    return fail(ctx, DIT_ATTN_ERR_ROPE, "rot_dim must be a multiple of 8 in 0..head_dim");
  if (layout != DIT_ATTN_ROPE_INTERLEAVED && layout != DIT_ATTN_ROPE_HALF) return fail(ctx, DIT_ATTN_ERR_ROPE, "no such layout");
  if (n_rows < 0) return fail(ctx, DIT_ATTN_ERR_CU_SEQLENS, "n_rows must be >= 0");
  dit::QkNormRopeParams p{};
  if (q) {
    const int rc = check_norm_heads(ctx, *q, "q", n_rows, head_dim, norm, p.side[0]);
    if (rc != DIT_ATTN_OK) return rc;
  }
  if (k) {
    const int rc = check_norm_heads(ctx, *k, "k", n_rows, head_dim, norm, p.side[1]);
    if (rc != DIT_ATTN_OK) return rc;
  }
  if (n_rows == 0) return DIT_ATTN_OK;
  if (q && k && (q->out == k->out || q->out == k->x || k->out == q->x))
    return fail(ctx, DIT_ATTN_ERR_STRIDE, "the output of one side is the other side's input or output");
  if (rot_dim > 0 && !table) return fail(ctx, DIT_ATTN_ERR_NULL, "table is NULL");
  if (rot_dim > 0 && misaligned(table, 16)) return fail(ctx, DIT_ATTN_ERR_ALIGN, "table must be 16-byte aligned");
  p.table = table;
  p.n_rows = n_rows;
  p.rot_dim = rot_dim;
  p.half = layout == DIT_ATTN_ROPE_HALF ? 1 : 0;
  p.eps = eps;
  if (n_rows > (int64_t{1} << 34) || dit::qk_norm_rope_blocks(p, head_dim) > dit::kMaxRowBlocks)
    return fail(ctx, DIT_ATTN_ERR_LIMIT, "too many rows");
  dit::DeviceGuard guard;
  hipError_t e = guard.enter(ctx->device);
  if (e != hipSuccess) return fail_hip(ctx, e, "hipSetDevice");
  e = dit::qk_norm_rope_launch(p, static_cast<dit::HeadNorm>(norm), head_dim, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? DIT_ATTN_OK : fail_hip(ctx, e, "norm and rotation kernel launch");
}

// ---------------------------------------------------------------- masked attention

int64_t tiles_of(int64_t keys) { return (keys + 63) / 64; }

// Tiles of a part: the keys of a sequence are split into parts of so many 64-key tiles, as few as still make no more work items
// than there are compute units (two to each where parts have 32 tiles even so), or not at all where that is no quicker.
// Measured on MI355X, us:
//   one item to a compute unit or two  512 x 4 heads against 40000 keys (head dimension 64) 34.6 / 42.8, 1570 x 5 20.8 / 27.0, 4951 x
//     3 50.2 / 51.0;  226 rows x 24 heads against 20506 keys 90 / 94 on the same keys over and over, 107 / 101 on changing ones: a
//     workgroup by itself waits for its tiles to come from HBM;  parts of at least 6 tiles or 16  77 x 24 against 4352 20.5 / 24.3.
//   unsplit / split, the unsplit call taking 0.65 us a tile (few rows 0.33, at head dimension 64 0.19), the join 4 us and the
//     partial results 0.33 us a megabyte:  1024 x 8 17.1 / 19.0, 2048 x 4 28.0 / 24.6, 33 x 8 against 1024 17.0 / 14.4, 410 x 24
//     (64) 9.6 / 14.5;  one row of 8 heads against 768 keys 8.8 / 9.7, 1024 10.1 / 9.9, 2048 15.6 / 9.5, 20506 131 / 22.5;  at head
//     dimension 64, 24 heads, 1024 7.5 / 8.6, 1536 9.1 / 9.2, 2048 10.6 / 8.1.
// Few rows: parts of at least 4 tiles (2 to 8: level).
// All of these are calls whose rows see all keys.  Keys are counted whatever a causal mask or ids leave of them, so that there parts
// may have little to do or nothing.
struct SeqWork {
  int64_t items, tiles, rows;  // items unsplit, key tiles, query rows
};
int64_t parts_of(int64_t tiles, int64_t part_tiles) { return std::max<int64_t>((tiles + part_tiles - 1) / part_tiles, 1); }

int64_t choose_part_tiles(const std::vector<SeqWork>& seqs, bool few_rows, int32_t n_heads, int32_t head_dim, int n_cus) {
  int64_t max_tiles = 1;
  for (const SeqWork& s : seqs) max_tiles = std::max(max_tiles, s.tiles);
  const int64_t least = std::max<int64_t>(few_rows ? 4 : 6, (max_tiles + dit::kMaskedMaxParts - 1) / dit::kMaskedMaxParts);
  const auto fit = [&](int64_t places) {
    int64_t lo = least, hi = std::max(max_tiles, least);
    while (lo < hi) {  // the least of [lo, hi] that fits; hi splits nothing
      const int64_t mid = (lo + hi) / 2;
      int64_t n = 0;
      for (const SeqWork& s : seqs) n += s.items * parts_of(s.tiles, mid);
      if (n <= places) hi = mid;
      else lo = mid + 1;
    }
    return lo;
  };
  int64_t lo = fit(n_cus);
  if (!few_rows && lo >= 32) {
    const int64_t two = fit(2 * static_cast<int64_t>(n_cus));
    if (two >= 32) lo = two;
  }
  double part_mb = 0;
  for (const SeqWork& s : seqs)
    if (s.tiles > lo) part_mb += static_cast<double>(s.rows * parts_of(s.tiles, lo)) * n_heads * head_dim * 4e-6;
  const double tile_us = !few_rows ? 0.65 : head_dim == 64 ? 0.19 : 0.33;
  return tile_us * static_cast<double>(max_tiles - lo) > 4.0 + 0.33 * part_mb ? lo : max_tiles;
}

// Sequences of a call that one kernel takes, in launch order, and how their keys are split.
struct MaskedBatch {
  bool few_rows;
  std::vector<int32_t> order;  // with query rows; the most keys first, once planned: their items take longest
  std::vector<SeqWork> seqs;
  int64_t part_tiles = 1, items = 0, tiles = 0, part_rows = 0;  // part_rows: of the partial results

  size_t doc_bytes() const { return (static_cast<size_t>(tiles) * sizeof(dit::DocTile) + 255) / 256 * 256; }
  size_t workspace_bytes(int32_t n_heads, int32_t head_dim, bool docs) const {
    return (docs ? doc_bytes() : 0) +
           static_cast<size_t>(part_rows) * static_cast<size_t>(n_heads) * (static_cast<size_t>(head_dim) + 1) * sizeof(float);
  }
};

// Whether the sequences with few rows get a kernel of their own beside the others: where, as items of 128 rows, they would take
// longer than its launch, by their work (0.65 us a tile and compute unit) or because their keys are the longest.  us, all as
// items of 128 rows / in two kernels, D 128, 24 heads:  2 x 512 rows and 32 single rows against 4352 keys (8 key heads) 265 / 120, 4352
// rows and one against 20506 keys 404 / 170;  D 64  4 x 1024 rows and 16 against 2000 keys (8) 55 / 43;  not worth one: 2 x 512 and
// 4 against 1280 (8) 27 either way.
bool worth_a_kernel(const MaskedBatch& few, const MaskedBatch& others, const int32_t* cu_k, int32_t n_heads, int n_cus) {
  if (few.order.empty() || others.order.empty()) return true;
  int64_t tiles = 0, longest = 0, longest_other = 0;
  for (const int32_t i : few.order) {
    tiles += tiles_of(cu_k[i + 1] - cu_k[i]);
    longest = std::max(longest, tiles_of(cu_k[i + 1] - cu_k[i]));
  }
  for (const int32_t i : others.order) longest_other = std::max(longest_other, tiles_of(cu_k[i + 1] - cu_k[i]));
  return 0.65 * static_cast<double>(tiles * n_heads) > 8.0 * n_cus || longest > longest_other + 16;
}

void plan_batch(MaskedBatch& b, const int32_t* cu_q, const int32_t* cu_k, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int n_cus) {
  std::stable_sort(b.order.begin(), b.order.end(), [&](int32_t x, int32_t y) { return cu_k[x + 1] - cu_k[x] > cu_k[y + 1] - cu_k[y]; });
  for (const int32_t i : b.order) {
    const int64_t lq = cu_q[i + 1] - cu_q[i], tiles = tiles_of(cu_k[i + 1] - cu_k[i]);
    b.seqs.push_back({b.few_rows ? n_kv_heads : (lq + dit::kMaskedBlockM - 1) / dit::kMaskedBlockM * n_heads, tiles, lq});
    b.tiles += tiles;
  }
  if (b.seqs.empty()) return;
  b.part_tiles = choose_part_tiles(b.seqs, b.few_rows, n_heads, head_dim, n_cus);
  for (const SeqWork& w : b.seqs) {
    const int64_t parts = parts_of(w.tiles, b.part_tiles);
    b.items += w.items * parts;
    if (parts > 1) b.part_rows += parts * w.rows;
  }
}

int masked_forward(dit_attn_ctx* ctx, const void* q, const void* k, const void* v, const int64_t* row_strides, const int32_t* cu_q,
                   const int32_t* cu_k, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                   const dit_attn_mask* mask, void* out, float* lse, void* stream) {
  std::string msg;
  int rc = dit::check_shape_args(cu_q, n_seqs, n_heads, head_dim, msg);
  if (rc != DIT_ATTN_OK) return fail(ctx, rc, msg);
  if (cu_k && dit::plan_validate(cu_k, n_seqs) != 0)
    return fail(ctx, DIT_ATTN_ERR_CU_SEQLENS, "cu_seqlens_k must start at 0 and be non-decreasing");
  if (!cu_k) cu_k = cu_q;
  if (n_kv_heads < 1 || n_heads % n_kv_heads != 0) return fail(ctx, DIT_ATTN_ERR_N_HEADS, "n_kv_heads must be >= 1 and divide n_heads");
  if (!std::isfinite(scale)) return fail(ctx, DIT_ATTN_ERR_SCALE, "scale must be finite");
  const dit_attn_mask no_mask{};
  const dit_attn_mask& m = mask ? *mask : no_mask;
  if (m.causal != 0 && m.causal != 1) return fail(ctx, DIT_ATTN_ERR_MASK, "causal must be 0 or 1");
  if (!(m.softcap >= 0.f) || !std::isfinite(m.softcap)) return fail(ctx, DIT_ATTN_ERR_MASK, "softcap must be finite and not negative");
  if (m.prefix && !m.causal) return fail(ctx, DIT_ATTN_ERR_MASK, "prefix belongs to a causal mask");
  if (m.prefix)
    for (int32_t i = 0; i < n_seqs; ++i)
      if (m.prefix[i] < 0) return fail(ctx, DIT_ATTN_ERR_MASK, "prefix must not be negative");
  const int64_t total_q = n_seqs > 0 ? cu_q[n_seqs] : 0, total_k = n_seqs > 0 ? cu_k[n_seqs] : 0;
  // (An array of no ids may have no address.)
  if ((m.q_doc || m.k_doc) && ((!m.q_doc && total_q > 0) || (!m.k_doc && total_k > 0)))
    return fail(ctx, DIT_ATTN_ERR_MASK, "q_doc and k_doc come together");
  int64_t strides[3];
  for (int i = 0; i < 3; ++i) {
    const int64_t row = static_cast<int64_t>(i == 0 ? n_heads : n_kv_heads) * head_dim;
    strides[i] = row_strides && row_strides[i] != 0 ? row_strides[i] : row;
    if (strides[i] < row || strides[i] % 8 != 0 || strides[i] > (int64_t{1} << 24))
      return fail(ctx, DIT_ATTN_ERR_STRIDE, "row strides must be multiples of 8 elements, hold a row's heads and be at most 2^24");
  }
  if (total_q == 0) return DIT_ATTN_OK;
  if (!q || !out || (total_k > 0 && (!k || !v))) return fail(ctx, DIT_ATTN_ERR_NULL, "q, k, v and out must be non-NULL");
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16))
    return fail(ctx, DIT_ATTN_ERR_ALIGN, "q, k, v and out must be 16-byte aligned");
  if (misaligned(lse, 4) || misaligned(m.slopes, 4) || misaligned(m.q_doc, 4) || misaligned(m.k_doc, 4))
    return fail(ctx, DIT_ATTN_ERR_ALIGN, "lse, slopes, q_doc and k_doc must be 4-byte aligned");

  const int32_t group = n_heads / n_kv_heads;
  MaskedBatch batches[2];
  batches[0].few_rows = true;
  batches[1].few_rows = false;
  for (int32_t i = 0; i < n_seqs; ++i) {
    const int64_t lq = cu_q[i + 1] - cu_q[i];
    if (lq > 0) batches[lq * group <= dit::kMaskedFewRows ? 0 : 1].order.push_back(i);
  }
  if (!worth_a_kernel(batches[0], batches[1], cu_k, n_heads, ctx->n_cus)) {
    batches[1].order.insert(batches[1].order.end(), batches[0].order.begin(), batches[0].order.end());
    std::sort(batches[1].order.begin(), batches[1].order.end());
    batches[0].order.clear();
  }
  const bool docs = m.q_doc != nullptr;
  size_t need = 0;
  for (MaskedBatch& b : batches) {
    plan_batch(b, cu_q, cu_k, n_heads, n_kv_heads, head_dim, ctx->n_cus);
    if (b.items > 0x7FFFFFFF) return fail(ctx, DIT_ATTN_ERR_LIMIT, "pack has too many work items");
    need = std::max(need, b.workspace_bytes(n_heads, head_dim, docs));
  }

  dit::DeviceGuard guard;
  hipError_t e = guard.enter(ctx->device);
  if (e != hipSuccess) return fail_hip(ctx, e, "hipSetDevice");
  hipStream_t s = static_cast<hipStream_t>(stream);

  if (need > 0) {  // the second batch comes behind the first one on the stream and takes the same workspace
    rc = dit::ensure_workspace(ctx, need, dit::stream_capturing(s), "masked attention");
    if (rc != DIT_ATTN_OK) return rc;
  }
  dit::MaskedParams p{};
  p.q = q;
  p.k = k;
  p.v = v;
  p.out = out;
  p.lse = lse;
  p.n_heads = n_heads;
  p.group = group;
  // Never 0, so that a dead score of -inf times it stays -inf; with a bias, whose slopes are divided by it, further from 0.
  p.c_log2 = std::max(std::fabs(scale) * 1.44269504088896340736f, m.slopes ? 1e-20f : 1e-30f);
  p.negate = scale < 0.f ? 1 : 0;
  if (m.softcap > 0.f) {
    // Finite, so that a score of 0 times it is 0.
    p.tanh_in = static_cast<float>(std::min(2.0 * 1.44269504088896340736 * std::fabs(static_cast<double>(scale)) / m.softcap, 3e38));
    p.cap_log2 = static_cast<float>(std::min(m.softcap * 1.44269504088896340736, 3e38));
    // tanh(x) / x as a polynomial in x^2, off by at most 4e-7 relative for |x| <= 0.25 (a fit of least maximal error), no more than
    // the exponential form beyond.  A term more would be off by 1e-7 up to 0.4 and take an instruction a score: 5229 us and not 5008 at
    // 20506 rows x 24 heads with a cap of 50.
    const double a[3] = {0.9999996043443452, -0.33321908223103114, 0.12841613400294474};
    const double k = std::fabs(static_cast<double>(scale)) / m.softcap;
    // (Finite with scale 0, so that an infinite score is not among them, and with a finite square.)
    p.poly_up_to = static_cast<float>(std::min(0.25 / k, 1e18));
    // Exponents of at most 30 either way.
    p.small = static_cast<float>(std::min<double>(p.poly_up_to, 30.0 / (1.44269504088896340736 * std::fabs(static_cast<double>(scale)))));
    for (int i = 0; i < 3; ++i) {
      const double coefficient = a[i] * m.softcap * 1.44269504088896340736 * std::pow(k, 2 * i + 1);
      if (std::fabs(coefficient) < 3e38) p.poly[i] = static_cast<float>(coefficient);
      else p.small = p.poly_up_to = -1.f;  // never
    }
  }
  p.q_stride_b = 2 * strides[0];
  p.k_stride_b = 2 * strides[1];
  p.v_stride_b = 2 * strides[2];
  p.q_doc = m.q_doc;
  p.k_doc = m.k_doc;
  p.slopes = m.slopes;
  p.causal = m.causal;
  for (const MaskedBatch& b : batches) {
    const size_t doc_bytes = docs ? b.doc_bytes() : 0;
    p.part_tiles = static_cast<int32_t>(b.part_tiles);
    p.doc_tiles = docs ? reinterpret_cast<dit::DocTile*>(ctx->workspace) : nullptr;
    p.part_out = b.part_rows > 0 ? ctx->workspace + doc_bytes / sizeof(float) : nullptr;
    p.part_lse = b.part_rows > 0 ? p.part_out + static_cast<size_t>(b.part_rows) * static_cast<size_t>(n_heads) * static_cast<size_t>(head_dim) : nullptr;
    const dit::MaskedKind kind = {head_dim, b.few_rows, m.softcap > 0.f, m.slopes != nullptr, lse != nullptr || b.part_rows > 0};
    int64_t part_row = 0;
    for (size_t first = 0; first < b.order.size(); first += dit::kMaskedSeqs) {
      p.n = static_cast<int32_t>(std::min<size_t>(b.order.size() - first, dit::kMaskedSeqs));
      uint32_t item = 0, tile = 0, join = 0;
      int32_t n_join = 0;  // sequences with several parts come first: they have the most tiles
      for (int32_t i = 0; i < p.n; ++i) {
        const size_t at = first + static_cast<size_t>(i);
        const int32_t sq = b.order[at];
        const int64_t parts = parts_of(b.seqs[at].tiles, b.part_tiles);
        dit::MaskedSeq& d = p.seq[i];
        d.part_row = part_row;
        d.first = item;
        d.tile0 = tile;
        d.join0 = join;
        d.q_start = cu_q[sq];
        d.q_len = cu_q[sq + 1] - cu_q[sq];
        d.kv_start = cu_k[sq];
        d.kv_len = cu_k[sq + 1] - cu_k[sq];
        d.prefix = m.prefix ? m.prefix[sq] : 0;
        d.parts = static_cast<int32_t>(parts);
        item += static_cast<uint32_t>(b.seqs[at].items * parts);
        tile += static_cast<uint32_t>(b.seqs[at].tiles);
        if (parts > 1) {
          part_row += parts * d.q_len;
          join += dit::masked_join_blocks(d, n_heads);
          ++n_join;
        }
      }
      p.n_items = item;
      e = dit::masked_attn_launch(p, kind, docs ? tile : 0, s);
      if (e != hipSuccess) return fail_hip(ctx, e, "masked attention kernel launch");
      e = dit::masked_join_launch(p, n_join, join, head_dim, s);
      if (e != hipSuccess) return fail_hip(ctx, e, "join kernel launch");
    }
  }
  return DIT_ATTN_OK;
}

}  // namespace

extern "C" {

int dit_attn_rope_table(dit_attn_ctx* ctx, const int32_t* positions, int64_t n_rows, const dit_attn_rope* rope, float* table, void* stream) {
  return guarded(ctx, [&] { return rope_table(ctx, positions, n_rows, rope, table, stream); });
}

int dit_attn_qk_norm_rope(dit_attn_ctx* ctx, const dit_attn_norm_heads* q, const dit_attn_norm_heads* k, int64_t n_rows, int32_t head_dim,
                          int32_t norm, float eps, const float* table, int32_t rot_dim, int32_t layout, void* stream) {
  return guarded(ctx, [&] { return qk_norm_rope(ctx, q, k, n_rows, head_dim, norm, eps, table, rot_dim, layout, stream); });
}

int dit_attn_masked_varlen_fwd(dit_attn_ctx* ctx, const void* q, const void* k, const void* v, const int64_t* row_strides,
                               const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t n_seqs, int32_t n_heads,
                               int32_t n_kv_heads, int32_t head_dim, float scale, const dit_attn_mask* mask, void* out, float* lse,
                               void* stream) {
  return guarded(ctx, [&] {
    return masked_forward(ctx, q, k, v, row_strides, cu_seqlens_q, cu_seqlens_k, n_seqs, n_heads, n_kv_heads, head_dim, scale, mask, out,
                          lse, stream);
  });
}

}  // extern "C"
