// The rotation table of token positions, and the norm and rotation of queries and keys for each head.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qk_norm_rope.h"
#include "store_through.h"

namespace dit {

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

// ---------------------------------------------------------------------------------------------
// table[r, j] = magnitude * (cos, sin)(2 pi * position * turns_j).
//
// Angles of far positions have no bits left behind the point in 32 bits, so quarter turns are counted in double: the nearest
// whole number of them, and what the product with the position leaves of it, exactly (fma), with the frequency as the sum of two
// doubles.  That is at most half a quarter turn, an fp32 angle with its relative precision, whose sine and cosine are short
// Taylor sums (the first terms left out are under 2e-9); the number of quarters selects and signs them.
// A thread keeps one pair and goes down the rows.  76112 rows x 64 pairs (40 MB), us: 11.6 with whole turns taken off first and
// quarters of the rest, 10.2 so, 8.1 with stores written through the L2 (the end of the kernel does not wait for dirty lines);
// streaming stores 9.4, four or sixteen rows a thread 8.7 and 8.4.
// ---------------------------------------------------------------------------------------------
constexpr int kTableRows = 8;  // rows per thread

__global__ void __launch_bounds__(256) rope_table_kernel(RopeTableParams p) {
  const uint32_t n_pairs = (uint32_t)p.n_pairs, per = 256 / n_pairs;  // rows side by side in a workgroup
  const uint32_t sub = threadIdx.x / n_pairs, pair = threadIdx.x - sub * n_pairs;
  if (sub >= per) return;
  const double hi = p.quarters_hi[pair], lo = p.quarters_lo[pair];
  const int axis = p.axis[pair];
  const int64_t r0 = (int64_t)blockIdx.x * (per * kTableRows) + sub;
  int32_t position[kTableRows];
#pragma unroll
  for (int i = 0; i < kTableRows; ++i) {
    const int64_t r = r0 + (int64_t)i * per;
    position[i] = p.positions[(r < p.n_rows ? r : p.n_rows - 1) * p.n_axes + axis];
  }
#pragma unroll
  for (int i = 0; i < kTableRows; ++i) {
    const int64_t r = r0 + (int64_t)i * per;
    if (r >= p.n_rows) return;
    const double pos = (double)position[i], quarters = __builtin_rint(pos * hi);
    const double rest = __builtin_fma(pos, lo, __builtin_fma(pos, hi, -quarters));
    const float x = (float)(rest * 1.570796326794896619231), x2 = x * x;
    const float s = x + x * x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880))));
    const float c = 1.f - 0.5f * x2 + x2 * x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 - x2 * (1.f / 3628800))));
    const int q = (int)quarters & 3;  // under 2^31: at most a radian a position
    const float cq = q & 1 ? s : c, sq = q & 1 ? c : s;
    const f32x2 cs = {p.magnitude * (q == 1 || q == 2 ? -cq : cq), p.magnitude * (q >= 2 ? -sq : sq)};
    store_through(reinterpret_cast<u32x2*>(p.table + (r * n_pairs + pair) * 2), __builtin_bit_cast(u32x2, cs));
  }
}

int64_t rope_table_blocks(const RopeTableParams& p) {
  const int64_t rows = (256 / p.n_pairs) * kTableRows;
  return (p.n_rows + rows - 1) / rows;
}

hipError_t rope_table_launch(const RopeTableParams& p, hipStream_t stream) {
  if (p.n_rows == 0) return hipSuccess;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)rope_table_blocks(p)), dim3(256), 0, stream, p);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Norm and rotation.  D / 8 lanes share a (row, head), eight elements each, in registers from the load to the store: every
// byte is read and written once, rounded once, and a head may be replaced in place.  HBM bound, 4 D bytes a head and row.
//
// Pairs lie in one lane, whose pairs are 4t .. 4t+3 of the table: with the interleaved layout it holds elements 8t .. 8t+7; with
// halves the first rot/8 lanes hold 4t .. 4t+3 and rot/2 + 4t .. +3.  There two neighbours load and store 16 bytes of either half
// and exchange four elements (kHalf); an odd number of such lanes takes 8 bytes at a time instead (kHalfOdd), with ordinary
// stores: 16989 rows x 48 heads, D 64, rot 32, us: 43.8, written through the L2 76.
// Table, weights and biases are loaded once for kHeads heads of the row (two or eight: 1 to 15 % slower).
// ---------------------------------------------------------------------------------------------
constexpr int kHeads = 4;
enum class Pairs : int { kInterleaved, kHalf, kHalfOdd };
enum class Stream : int { kNone, kIn, kInOut };  // which side passes by the memory-side cache

// Sum over the aligned groups of N lanes (N = 8 or 16), in all of them.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
template <int N>
__device__ __forceinline__ float group_sum(float x) {
  x = dpp_add<0xB1>(x);   // quad_perm: lane ^ 1
  x = dpp_add<0x4E>(x);   // quad_perm: lane ^ 2
  x = dpp_add<0x141>(x);  // mirror of eight: the other quad
  if constexpr (N == 16) x = dpp_add<0x140>(x);  // mirror of sixteen: the other eight
  return x;
}

__device__ __forceinline__ uint32_t round_pair(float a, float b) {
  const f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// The value of the other lane of an even and odd pair.
__device__ __forceinline__ uint32_t neighbour(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true); }

// 16 bytes as two neighbours load or store them <-> the two quads that a lane works on; `even` and `odd` of lanes with pairs.
__device__ __forceinline__ void exchange(u32x4& w, bool even, bool odd) {
  const uint32_t y0 = neighbour(even ? w[2] : w[0]), y1 = neighbour(even ? w[3] : w[1]);
  w = u32x4{odd ? y0 : w[0], odd ? y1 : w[1], even ? y0 : w[2], even ? y1 : w[3]};
}

template <int D, HeadNorm NORM, Pairs PAIRS, Stream STREAM>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(QkNormRopeParams p, uint32_t units, uint32_t q_units) {
  constexpr int LANES = D / 8, ROWS = 256 / LANES;
  // The units (side, kHeads heads) of a row on one XCD, one after another: its table rows come from that L2 then.
  const uint32_t in_xcd = blockIdx.x >> 3, unit = in_xcd % units;
  const int64_t row = ((int64_t)(in_xcd / units) * 8 + (blockIdx.x & 7)) * ROWS + threadIdx.x / LANES;
  if (row >= p.n_rows) return;
  const bool keys = unit >= q_units;
  const NormHeadsParams& s = p.side[keys ? 1 : 0];
  const int h0 = (int)(keys ? unit - q_units : unit) * kHeads;
  const int t = threadIdx.x % LANES;
  const bool turned = t < p.rot_dim / 8;
  // Elements of this lane: four from e0, four from e1.
  constexpr bool HALF = PAIRS != Pairs::kInterleaved;
  const int e0 = HALF && turned ? 4 * t : 8 * t;
  const int e1 = HALF && turned ? p.rot_dim / 2 + 4 * t : 8 * t + 4;
  const bool even = PAIRS == Pairs::kHalf && turned && (t & 1) == 0, odd = PAIRS == Pairs::kHalf && turned && (t & 1) != 0;
  const int first = even ? e0 : odd ? e1 - 4 : 8 * t;  // of the 16 bytes that it loads and stores

  const char* src = s.x + row * s.row_stride_b + (int64_t)h0 * (2 * D);
  u32x4 in[kHeads];
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (h0 + i < s.n_heads) {
      if constexpr (PAIRS == Pairs::kHalfOdd) {
        const u32x2 a = *reinterpret_cast<const u32x2*>(src + i * 2 * D + 2 * e0), b = *reinterpret_cast<const u32x2*>(src + i * 2 * D + 2 * e1);
        in[i] = u32x4{a[0], a[1], b[0], b[1]};
      } else {
        const u32x4* from = reinterpret_cast<const u32x4*>(src + i * 2 * D + 2 * first);
        in[i] = STREAM == Stream::kNone ? *from : __builtin_nontemporal_load(from);
      }
    }
  }
  float c[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
  if (turned) {
    const f32x4* tab = reinterpret_cast<const f32x4*>(p.table + row * p.rot_dim + 8 * t);
    const f32x4 a = tab[0], b = tab[1];
    c[0] = a[0]; sn[0] = a[1]; c[1] = a[2]; sn[1] = a[3];
    c[2] = b[0]; sn[2] = b[1]; c[3] = b[2]; sn[3] = b[3];
  }
  float w[8], bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    w[e] = 1.f;
    bias[e] = 0.f;
  }
  if (NORM != HeadNorm::kNone && s.weight != nullptr) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(s.weight + e0), b = *reinterpret_cast<const f32x4*>(s.weight + e1);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = a[e];
      w[4 + e] = b[e];
    }
  }
  if (NORM != HeadNorm::kNone && s.bias != nullptr) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(s.bias + e0), b = *reinterpret_cast<const f32x4*>(s.bias + e1);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      bias[e] = a[e];
      bias[4 + e] = b[e];
    }
  }
  char* dst = s.out + row * s.out_stride_b + (int64_t)h0 * (2 * D);
#pragma unroll
  for (int i = 0; i < kHeads; ++i) {
    if (h0 + i >= s.n_heads) break;
    if constexpr (PAIRS == Pairs::kHalf) exchange(in[i], even, odd);
    float y[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      y[2 * k] = __builtin_bit_cast(float, in[i][k] << 16);
      y[2 * k + 1] = __builtin_bit_cast(float, in[i][k] & 0xFFFF0000u);
    }
    if constexpr (NORM == HeadNorm::kLayer) {
      const float mean = group_sum<LANES>(((y[0] + y[1]) + (y[2] + y[3])) + ((y[4] + y[5]) + (y[6] + y[7]))) * (1.f / D);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] -= mean;
    }
    if constexpr (NORM != HeadNorm::kNone) {
      float sq = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(y[e], y[e], sq);
      const float r = 1.f / __builtin_sqrtf(group_sum<LANES>(sq) * (1.f / D) + p.eps);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(y[e] * r, w[e], bias[e]);
    }
    if (turned) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float &a = y[HALF ? k : 2 * k], &b = y[HALF ? 4 + k : 2 * k + 1];
        const float a1 = a * c[k] - b * sn[k], b1 = b * c[k] + a * sn[k];
        a = a1;
        b = b1;
      }
    }
    u32x4 w4 = {round_pair(y[0], y[1]), round_pair(y[2], y[3]), round_pair(y[4], y[5]), round_pair(y[6], y[7])};
    if constexpr (PAIRS == Pairs::kHalfOdd) {
      *reinterpret_cast<u32x2*>(dst + i * 2 * D + 2 * e0) = u32x2{w4[0], w4[1]};
      *reinterpret_cast<u32x2*>(dst + i * 2 * D + 2 * e1) = u32x2{w4[2], w4[3]};
    } else {
      if constexpr (PAIRS == Pairs::kHalf) exchange(w4, even, odd);
      u32x4* to = reinterpret_cast<u32x4*>(dst + i * 2 * D + 2 * first);
      if constexpr (STREAM == Stream::kInOut) __builtin_nontemporal_store(w4, to);
      else store_through(to, w4);
    }
  }
}

static uint32_t units_of(const NormHeadsParams& s) { return ((uint32_t)s.n_heads + kHeads - 1) / kHeads; }

int64_t qk_norm_rope_blocks(const QkNormRopeParams& p, int head_dim) {
  const int64_t rows = 256 / (head_dim / 8), row_blocks = (p.n_rows + rows - 1) / rows;
  return (row_blocks + 7) / 8 * 8 * (units_of(p.side[0]) + units_of(p.side[1]));
}

// As in the layout kernels (sp_layout.hip): streaming loads keep the input from pushing the result out of the memory-side cache
// before the attention reads it; from kStreamOutBytes on it does not stay there anyway.  Up to kStreamInBytes, where a projection
// has left the input in that cache, ordinary loads.  us on three sets of buffers, ordinary / streaming loads with stores written
// through, streaming loads and stores, half of D 128, 48 heads:
//    25 MB   5.5 /  6.6 /  6.0      60 MB  11.2 / 13.1 / 13.7     107 MB  22.1 / 19.5 / 20.9     214 MB  40.4 / 39.1 / 37.5
//   295 MB  53.8 / 52.0 / 50.4;  20 heads, 780 MB  139.9 / 136.8 / 130.5 (6.2 TB/s);  D 64, mean and variance, 209 MB  40.3 / 39.6 / 38.1;
//   interleaved, from a fused projection, 428 MB  78.6 / 74.0 / 71.5.
constexpr int64_t kStreamInBytes = 64ll << 20;    // of input and output
constexpr int64_t kStreamOutBytes = 160ll << 20;

template <int D, HeadNorm NORM, Pairs PAIRS>
static void launch(const QkNormRopeParams& p, hipStream_t stream) {
  const uint32_t q_units = units_of(p.side[0]), units = q_units + units_of(p.side[1]);
  const int64_t bytes = p.n_rows * (p.side[0].n_heads + p.side[1].n_heads) * (4 * D);
  const auto fn = bytes < kStreamInBytes || PAIRS == Pairs::kHalfOdd ? qk_norm_rope_kernel<D, NORM, PAIRS, Stream::kNone>
                  : bytes < kStreamOutBytes                            ? qk_norm_rope_kernel<D, NORM, PAIRS, Stream::kIn>
                                                                       : qk_norm_rope_kernel<D, NORM, PAIRS, Stream::kInOut>;
  hipLaunchKernelGGL(fn, dim3((unsigned)qk_norm_rope_blocks(p, D)), dim3(256), 0, stream, p, units, q_units);
}
template <int D, HeadNorm NORM>
static void launch_layout(const QkNormRopeParams& p, hipStream_t stream) {
  if (!p.half || p.rot_dim == 0) launch<D, NORM, Pairs::kInterleaved>(p, stream);
  else if (p.rot_dim % 16 == 0) launch<D, NORM, Pairs::kHalf>(p, stream);
  else launch<D, NORM, Pairs::kHalfOdd>(p, stream);
}
template <int D>
static void launch_norm(const QkNormRopeParams& p, HeadNorm norm, hipStream_t stream) {
  if (norm == HeadNorm::kNone) launch_layout<D, HeadNorm::kNone>(p, stream);
  else if (norm == HeadNorm::kRms) launch_layout<D, HeadNorm::kRms>(p, stream);
  else launch_layout<D, HeadNorm::kLayer>(p, stream);
}

hipError_t qk_norm_rope_prepare() {
  hipFuncAttributes a;
  return hipFuncGetAttributes(&a, reinterpret_cast<const void*>(rope_table_kernel));
}

hipError_t qk_norm_rope_launch(const QkNormRopeParams& p, HeadNorm norm, int head_dim, hipStream_t stream) {
  if (p.n_rows == 0) return hipSuccess;
  head_dim == 64 ? launch_norm<64>(p, norm, stream) : launch_norm<128>(p, norm, stream);
  return hipGetLastError();
}

}  // namespace dit
